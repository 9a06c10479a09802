"""Forms of the layer operators' kernels that only larger calls take: many sequences of few queries in fp32, and tensors beyond the caches."""
import pytest
import torch

import paper_2208_04187_amd as pkg

from .test_gpu_attention import _check, _inputs

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
CACHED = 2 ** 28


@pytest.mark.parametrize("size", [(40, 1, 130, 8, 8, 24), (20, 1, 700, 8, 4, 64), (20, 3, 700, 8, 4, 128), (90, 2, 70, 9, 3, 72), (70, 1, 520, 20, 4, 128)])
def test_few_queries_of_many_sequences(size):
    """At most 32 columns a key head and more than 256 workgroups, whole and in parts of the keys"""
    B, Sq, Sk = size[:3]
    x = _inputs(*size, F32, seed=31)
    _check(*x)
    _check(*x, causal=True, window=Sk // 2, lengths=[Sk - 13 * b % (Sk + 5) for b in range(B)])


def _rotation_inputs(dtype, T, heads, D, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    q, k = (torch.randn(T, n, D, generator=gen, device="cuda").to(dtype) for n in heads)
    w = [torch.rand(D, generator=gen, device="cuda") + 0.5 for _ in range(2)]
    return q, k, w, torch.tensor([10000.0 ** (-p / D) for p in range(0, D, 2)], dtype=torch.float64, device="cuda"), torch.randint(0, 100000, (T,), generator=gen, device="cuda")


@pytest.mark.parametrize("pairs", ["halves", "next"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D", [32, 64, 128, 256, 512])
def test_rotation_beyond_the_caches(D, dtype, pairs):
    """A token's results are its own: the same bits as in two calls that stay within the caches"""
    heads = (32, 8)
    T = CACHED // (2 * sum(heads) * D * dtype.itemsize) + 77
    q, k, w, f, at = _rotation_inputs(dtype, T, heads, D, 1)
    halves = [slice(0, T // 3), slice(T // 3, 2 * T // 3), slice(2 * T // 3, T)]
    whole = pkg.division_head_norm_rotate(q, k, *w, f, at, pairs=pairs)
    parts = [pkg.division_head_norm_rotate(q[s], k[s], *w, f, at[s], pairs=pairs) for s in halves]
    for a, b in zip(whole, zip(*parts)):
        assert torch.equal(a, torch.cat(b))
    gq, gk = whole.k.repeat(1, 4, 1), whole.q[:, :8].contiguous()
    back = pkg.division_head_norm_rotate_backward(gq, gk, q, k, *w, f, at, whole.q_rstd, whole.k_rstd, pairs=pairs)
    parts = [pkg.division_head_norm_rotate_backward(gq[s], gk[s], q[s], k[s], *w, f, at[s], whole.q_rstd[s], whole.k_rstd[s], pairs=pairs) for s in halves]
    for a, b in zip(back[:2], zip(*parts)):
        assert torch.equal(a, torch.cat(b))
    # the weights' gradients are sums over all tokens: of whole numbers, whose sums stay below 2^24 and are exact in any order
    at.zero_()
    for t in (q, k):
        t.copy_(torch.where(t > 0, 1.0, -1.0))
    for t in (gq, gk):
        t.copy_(t.float().clamp(-3, 3).round())
    one = [torch.ones(t.shape[:2], device="cuda") for t in (q, k)]
    back = pkg.division_head_norm_rotate_backward(gq, gk, q, k, *w, f, at, *one, pairs=pairs)
    for got, g, x in zip(back[2:], (gq, gk), (q, k)):
        assert torch.equal(got, (g.double() * x.double()).sum((0, 1)).float())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D", [2048, 2047])
def test_rows_of_the_table_beyond_the_caches(D, dtype):
    T = CACHED // (D * dtype.itemsize) + 99
    gen = torch.Generator(device="cuda").manual_seed(2)
    table, ids = torch.randn(999, D, generator=gen, device="cuda").to(dtype), torch.randint(0, 999, (T,), generator=gen, device="cuda")
    ids[5], ids[T - 1], ids[T - 2] = -100, 999, -7
    got = pkg.division_embedding(ids, table, 0.3)
    want = (table.float() * torch.tensor(0.3, device="cuda")).to(dtype)[ids.clamp(0, 998)]
    want[5] = 0
    assert torch.equal(got[:-2], want[:-2]) and got[-2:].isnan().all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_dropout_with_a_residual_beyond_the_caches(dtype):
    n = CACHED // (3 * dtype.itemsize) + 4099
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, r = (torch.randn(n, generator=gen, device="cuda").to(dtype) for _ in range(2))
    kept = pkg.division_dropout_forward(torch.ones(n, device="cuda"), 0.3, 5)[0] != 0
    by = torch.tensor(1.0 / 0.7, dtype=F32, device="cuda")
    for at in (0, 1):                                # the second begins off 16 bytes
        m = n - at
        got = pkg.division_dropout_add(x[at:], 0.3, 5, residual=r[at:])
        assert torch.equal(got, (torch.where(kept[:m], x[at:].float() * by, 0.0) + r[at:].float()).to(dtype))
