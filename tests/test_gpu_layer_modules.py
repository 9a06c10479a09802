"""The layer operators' modules where their callers are awkward: tensors at any address, checkpointing, inference before training, a hook that compresses."""
import pytest
import torch
from torch.utils.checkpoint import checkpoint

import paper_2208_04187_amd as pkg

from .test_gpu_autograd import oracle_saved_tensors
from .test_gpu_layers import Layer, _inputs

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


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("reentrant", [False, True])
def test_a_checkpointed_layer_has_the_gradients_of_a_plain_one(reentrant, dtype):
    """Both dropout modules with seeds from torch's generator; attention, rotation and table are computed again as they were"""
    grads = []
    ids, positions, g = _inputs(2, 33, 40, 64, 3)
    for again in (False, True):
        torch.manual_seed(1)
        m = Layer(40, 64, 4, 2, dtype=dtype)
        m.drop, other = pkg.DivisionResidualDropout(0.25, seed=None), pkg.DivisionDropout(0.5, seed=None)
        x = g.to(dtype).cuda().requires_grad_()

        def block(t):
            return other(m(ids.cuda(), positions.cuda()) * t).tanh()
        torch.manual_seed(2)
        out = checkpoint(block, x, use_reentrant=reentrant) if again else block(x)
        (out.float() ** 2).sum().backward()
        grads.append([out.detach(), x.grad, *(p.grad for p in m.parameters())])
    assert all(torch.equal(a, b) for a, b in zip(*grads)) and (grads[0][0] == 0).any()


def test_numbered_dropout_raises_where_it_would_drop_others():
    x = torch.randn(64, 64, device="cuda", requires_grad=True)
    for d in (pkg.DivisionResidualDropout(0.5, seed=3), pkg.DivisionDropout(0.5, seed=3)):
        for reentrant in (False, True):
            y = checkpoint(lambda t: d(t.sin()).exp(), x, use_reentrant=reentrant)
            with pytest.raises(RuntimeError, match="seed=None"):
                y.sum().backward()
        y = d(x)
        y.sum().backward()                           # and goes on as before


def test_a_rotation_that_began_in_inference_mode_trains():
    q, k = (torch.randn(2, 9, n, 32, device="cuda") for n in (4, 2))
    at = torch.arange(18, device="cuda").view(2, 9)
    m, fresh = pkg.DivisionHeadNormRotation(32, device="cuda"), pkg.DivisionHeadNormRotation(32, device="cuda")
    with torch.inference_mode():
        first = [t.clone() for t in m(q, k, at)]
    grads = []
    for n in (m, fresh):
        leaves = [t.clone().requires_grad_() for t in (q, k)]
        a, b = n(*leaves, at)
        assert torch.equal(a, first[0]) and torch.equal(b, first[1])
        grads.append(torch.autograd.grad((a * a * a).sum() + b.sum(), [*leaves, *n.parameters()]))
    assert all(torch.equal(a, b) for a, b in zip(*grads))


@pytest.mark.parametrize("pairs", ["halves", "next"])
@pytest.mark.parametrize("b", [2, 8])
@pytest.mark.parametrize("apart", [False, True])
def test_a_layers_gradients_under_a_hook_that_compresses(apart, b, pairs):
    """Equal to those of the same layer whose cached maps are the oracle's reconstructions.  Queries and keys of projections of their own are cached as maps; parts of one projection's output, as
    all that attention caches, exactly"""
    ids, positions, g = _inputs(3, 37, 50, 96, 2)
    lengths = torch.tensor([37, 20, 35], dtype=torch.int32, device="cuda")
    grads, hooks = [], []
    for make in (lambda: pkg.division_saved_tensors(B=8, b=b, seed=1, min_elements=1), lambda: oracle_saved_tensors(8, b, 1, min_elements=1), None):
        torch.manual_seed(1)
        m = Layer(50, 96, 6, 2, pairs)
        if apart:
            parts = torch.nn.ModuleList(torch.nn.Linear(96, n, bias=False, device="cuda") for n in (96, 32, 32))

            def forward(ids, positions, lengths, m=m, parts=parts):
                x = m.embed(ids)
                q, k, v = (p(x).unflatten(2, (-1, m.f)) for p in parts)
                a = pkg.division_token_attention(*m.rotate(q, k, positions), v, causal=True, lengths=lengths)
                return m.drop(m.out(a.flatten(2)), x)
        else:
            parts, forward = torch.nn.ModuleList(), m
        args = (ids.cuda(), positions.cuda(), lengths)
        if make is None:
            out = forward(*args)
        else:
            hooks.append(make())
            with hooks[-1]:
                out = forward(*args)
        out.backward(g.cuda())
        grads.append([p.grad for p in (*m.parameters(), *parts.parameters()) if p.grad is not None])
    assert hooks[0].cached_maps == hooks[1].maps
    if not apart:
        assert hooks[0].cached_maps == 0 and all(torch.equal(a, p) for a, p in zip(grads[0], grads[2]))
        return
    assert hooks[0].cached_maps >= 2 and hooks[0].cached_bytes < hooks[0].original_bytes
    # one build of the same kernels on the same bits; the projections are a library's, whose sums may take another order: 96 and 111 products of a half unit each
    for a, r in zip(grads[0], grads[1]):
        assert (a.double() - r.double()).norm() <= 128 * 2.0 ** -24 * r.double().norm()
    assert any(not torch.equal(a, p) for a, p in zip(grads[0], grads[2]))
