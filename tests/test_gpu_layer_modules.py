"""The layer operators' modules where their callers are awkward: tensors at any address, checkpointing, inference before training, a hook that compresses."""
import pytest
import torch
from torch.utils.checkpoint import checkpoint

import paper_2208_04187_amd as pkg

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_takes_dense_tensors_at_any_address(dtype):
    gen = torch.Generator().manual_seed(1)
    n = 2 * 37 * 4 * 24
    room = [torch.randn(8 + n, generator=gen).to(dtype).cuda() for _ in range(4)]
    for off in (1, 3, 16 // room[0].element_size() - 1):
        at = [r[off: off + n].view(2, 37, 4, 24) for r in room]
        got = [t.detach().requires_grad_() for t in at[:3]]
        want = [t.clone().requires_grad_() for t in at[:3]]
        a, b = pkg.division_token_attention(*got, causal=True), pkg.division_token_attention(*want, causal=True)
        assert got[0].data_ptr() % 16 and torch.equal(a, b)
        assert all(torch.equal(p, q) for p, q in zip(torch.autograd.grad(a, got, at[3]), torch.autograd.grad(b, want, at[3].clone())))
