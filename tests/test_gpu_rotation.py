"""The norms of queries and keys with the rotation, and their backward pass, against the definition in 64 bits.

Bounds.  EPS is half a unit in the last place of binary32.  The sum of a head's D squares is at most eight products a lane one after the other, four such runs for heads that are no whole vectors, and a tree of six steps; the root halves
its error.  Cosines and sines are off by a few EPS of 1: the turn is rounded to 24 bits (pi EPS of the angle), the function by 2 EPS more.  A turned element is off by that of both of its
pair's.  A weight's gradient is a sum of n terms in some order, off by n EPS of their magnitudes.  Results in bfloat16 are what some number within the bound rounds to."""
import ctypes
import math

import pytest
import torch

import paper_2208_04187_amd as pkg

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16
# tokens, heads, key heads, features, rotated
SIZES = [(1, 1, 1, 2, 2), (1, 4, 2, 64, 64), (3, 5, 1, 6, 2), (2, 8, 2, 128, 128), (7, 3, 3, 80, 40), (5, 2, 1, 256, 64), (3, 1, 1, 512, 512), (4, 6, 2, 96, 90), (2, 3, 2, 130, 130), (9, 2, 2, 48, 0),
         (70, 40, 8, 64, 32), (5, 2, 1, 510, 512 - 8), (1100, 3, 1, 16, 16), (4100, 2, 1, 32, 24), (33, 33, 7, 8, 8)]


def _within(got, want, bound):
    lo, hi = want - bound, want + bound
    if got.dtype == BF16:                           # rounding keeps the order
        lo, hi = lo.float().bfloat16().double(), hi.float().bfloat16().double()
    got = got.double().cpu()
    bad = ~((lo <= got) & (got <= hi))
    assert not bad.any(), (int(bad.sum()), ((got - want).abs() - bound).max().item())


def _inputs(T, H, G, D, R, dtype, seed=0, first=0):
    gen = torch.Generator().manual_seed(1000 * T + D + R + seed)
    q, k, gq, gk = ((torch.randn(T, n, D, generator=gen) * (0.1 + 1.9 * torch.rand(D, generator=gen))).to(dtype) for n in (H, G, H, G))
    wq, wk = (torch.rand(D, generator=gen) + 0.5 for _ in range(2))
    freq = 10000.0 ** (-torch.arange(0, R, 2, dtype=torch.float64) / max(R, 1))
    at = torch.randint(0, 5000, (T,), generator=gen) + first
    return q, k, gq, gk, wq, wk, freq, at


def _turned(x, freq, at, pairs, back=False):
    """x's first elements turned, and how large the pairs are"""
    R = 2 * len(freq)
    a, b = (x[..., 0:R:2], x[..., 1:R:2]) if pairs == "next" else (x[..., :R // 2], x[..., R // 2:R])
    angle = at.double()[:, None, None] * freq * (-1 if back else 1)
    y, size = x.clone(), x.abs()
    one, two = a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()
    both = a.abs() + b.abs()
    if pairs == "next":
        y[..., 0:R:2], y[..., 1:R:2], size[..., 0:R:2], size[..., 1:R:2] = one, two, both, both
    else:
        y[..., :R // 2], y[..., R // 2:R], size[..., :R // 2], size[..., R // 2:R] = one, two, both, both
    return y, size


def _check(x, g, w, rstd, y, dx, dw, freq, at, pairs, eps):
    T, H, D = x.shape
    steps = 4 * 8 + 6 + 8
    xd = x.double()
    want = 1.0 / torch.sqrt((xd * xd).mean(2) + eps)
    _within(rstd, want, want * steps * EPS)
    wd = w.double()
    yd, size = _turned(xd * want[..., None] * wd, freq, at, pairs)
    _within(y, yd, size * (steps + 16) * EPS + 1e-37)
    r = rstd.double().cpu()[..., None]              # backward from what was written
    gd, gsize = _turned(g.double(), freq, at, pairs, back=True)
    u = xd * r
    along = (gd * wd * u).mean(2, keepdim=True)
    large = (gsize * wd.abs() * u.abs()).mean(2, keepdim=True)
    _within(dx, r * (gd * wd - u * along), r * (gsize * wd.abs() + u.abs() * large) * (steps + 32) * EPS + 1e-37)
    _within(dw, (gd * u).sum((0, 1)), (gsize * u.abs()).sum((0, 1)) * (T * H + 64) * EPS)


@pytest.mark.parametrize("pairs", ["halves", "next"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", SIZES)
def test_matches_the_definition(size, dtype, pairs):
    q, k, gq, gk, wq, wk, freq, at = _inputs(*size, dtype)
    for weight_type, eps in ((F32, 1e-6), (BF16, 0.5)):
        w = [t.to(weight_type) for t in (wq, wk)]
        dev = [t.cuda() for t in (q, k, *w, freq, at)]
        r = pkg.division_head_norm_rotate(*dev, eps, pairs=pairs)
        b = pkg.division_head_norm_rotate_backward(gq.cuda(), gk.cuda(), *dev, r.q_rstd, r.k_rstd, pairs=pairs)
        torch.cuda.synchronize()
        assert b[2].dtype == weight_type and r.q.dtype == dtype and b[0].dtype == dtype
        _check(q, gq, w[0], r.q_rstd, r.q, b[0], b[2], freq, at, pairs, eps)
        _check(k, gk, w[1], r.k_rstd, r.k, b[1], b[3], freq, at, pairs, eps)
    # the queries alone
    alone = pkg.division_head_norm_rotate(dev[0], None, dev[2], None, dev[4], dev[5], eps, pairs=pairs)
    assert torch.equal(alone.q, r.q) and torch.equal(alone.q_rstd, r.q_rstd) and alone.k is None and alone.k_rstd is None
    dq, dk, dwq, dwk = pkg.division_head_norm_rotate_backward(gq.cuda(), None, dev[0], None, dev[2], None, dev[4], dev[5], r.q_rstd, None, pairs=pairs)
    assert torch.equal(dq, b[0]) and dk is None and dwk is None
    _within(dwq, b[2].double().cpu(), b[2].double().cpu().abs() * 2.0 ** -8 + gq.double().abs().sum((0, 1)) * 1e-4)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_far_positions_turn_as_exactly_as_near_ones(dtype):
    q, k, gq, gk, wq, wk, freq, _ = _inputs(6, 2, 1, 64, 64, dtype)
    at = torch.tensor([2 ** 20 + 1, 2 ** 24 + 3, 2 ** 31 - 1, -5, -(2 ** 20) - 7, 123456789])
    dev = [t.cuda() for t in (q, k, wq, wk, freq, at)]
    r = pkg.division_head_norm_rotate(*dev)
    b = pkg.division_head_norm_rotate_backward(gq.cuda(), gk.cuda(), *dev, r.q_rstd, r.k_rstd)
    _check(q, gq, wq, r.q_rstd, r.q, b[0], b[2], freq, at, "halves", 1e-6)
    _check(k, gk, wk, r.k_rstd, r.k, b[1], b[3], freq, at, "halves", 1e-6)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D,R", [(64, 64), (40, 18)])
def test_strides_and_shapes(D, R, dtype):
    gen = torch.Generator().manual_seed(3)
    H, G = 6, 2
    x = torch.randn(3, 7, (H + 2 * G) * D + 1, generator=gen).to(dtype).cuda()
    freq = (10.0 ** -torch.arange(R // 2, dtype=torch.float64)).cuda()
    at = torch.randint(0, 99, (3, 7), generator=gen).cuda()
    wq, wk = torch.rand(D, generator=gen).cuda(), torch.rand(D, generator=gen).cuda()
    q, k = x[..., 1:1 + H * D].unflatten(2, (H, D)), x[..., 1 + H * D:1 + (H + G) * D].unflatten(2, (G, D))
    g = torch.randn(3, 7, H + G, D + 8, generator=gen).to(dtype).cuda()
    gq, gk = g[:, :, :H, :D], g[:, :, H:, 8:]
    for qq, kk, a, b, p in ((q, k, gq, gk, at), (q[1], k[1], gq[1], gk[1], at[1].contiguous()), (q[0, 0], k[0, 0], gq[0, 0], gk[0, 0], at[0, 0].clone()),
                            (q[:1, :1].expand(3, 7, H, D), k[:, :, :1].expand(3, 7, G, D), gq, gk, at), (q[:, ::2], k[:, ::2], gq[:, ::2], gk[:, ::2], at[:, ::2].contiguous())):
        if qq.dim() == 4 and qq.stride(0) != qq.stride(1) * qq.shape[1]:
            with pytest.raises(ValueError, match="rows of one stride"):
                pkg.division_head_norm_rotate(qq, kk, wq, wk, freq, p)
            qq, kk, a, b = (t[:1] for t in (qq, kk, a, b))
            p = p[:1]
        dense = [t.contiguous() for t in (qq, kk)]
        m, n = pkg.division_head_norm_rotate(qq, kk, wq, wk, freq, p), pkg.division_head_norm_rotate(*dense, wq, wk, freq, p)
        assert all(torch.equal(s, t) and s.shape == t.shape for s, t in zip(m, n)) and m.q.shape == qq.shape and m.q_rstd.shape == qq.shape[:-1]
        u = pkg.division_head_norm_rotate_backward(a, b, qq, kk, wq, wk, freq, p, m.q_rstd, m.k_rstd)
        v = pkg.division_head_norm_rotate_backward(a.contiguous(), b.contiguous(), *dense, wq, wk, freq, p, m.q_rstd, m.k_rstd)
        assert all(torch.equal(s, t) for s, t in zip(u, v))


def test_in_place_and_beside_the_outputs():
    """The library's own entries: outputs over the inputs' memory, nothing written beside them"""
    from paper_2208_04187_amd import layer_operators as ops
    q, k, gq, gk, wq, wk, freq, at = (t.cuda() for t in _inputs(33, 6, 2, 48, 40, BF16))
    L, st, guard = pkg.lib(), torch.cuda.current_stream().cuda_stream, 64
    r = pkg.division_head_norm_rotate(q, k, wq, wk, freq, at)
    want = pkg.division_head_norm_rotate_backward(gq, gk, q, k, wq, wk, freq, at, r.q_rstd, r.k_rstd)

    def room(t):
        x = torch.full((t.numel() + 2 * guard,), 77.0, dtype=t.dtype, device="cuda")
        x[guard:-guard] = t.reshape(-1)
        return x, x[guard:-guard].view(t.shape)
    (wholeq, q1), (wholek, k1), (whole_gq, g1), (whole_gk, g2) = room(q), room(k), room(gq), room(gk)
    d, _ = ops._rotation(q1, k1, wq, wk, freq, at, 1e-6, "halves")
    d.y[0], d.y[1] = q1.data_ptr(), k1.data_ptr()
    assert L.division_head_norm_rotate(ctypes.byref(d), st) == 0                  # without rstd
    assert torch.equal(q1, r.q) and torch.equal(k1, r.k)
    d, _ = ops._rotation(q, k, wq, wk, freq, at, 0.0, "halves")
    b = ops._RotateBackDesc()
    need = L.division_head_norm_rotate_backward_workspace(33, 48)
    ws = torch.full((need // 4 + 2 * guard,), 77.0, device="cuda")
    for i, (g, rstd, w) in enumerate(((g1, r.q_rstd, wq), (g2, r.k_rstd, wk))):
        b.grad_y[i], b.rstd[i], b.grad_x[i], b.token_strides[i], b.head_strides[i] = g.data_ptr(), rstd.data_ptr(), g.data_ptr(), g.stride(0), g.stride(1)
    dws = [torch.empty_like(w) for w in (wq, wk)]
    b.grad_weight[0], b.grad_weight[1], b.workspace, b.workspace_bytes = dws[0].data_ptr(), dws[1].data_ptr(), ws[guard:].data_ptr(), need
    assert L.division_head_norm_rotate_backward(ctypes.byref(d), ctypes.byref(b), st) == 0
    torch.cuda.synchronize()
    assert torch.equal(g1, want[0]) and torch.equal(g2, want[1]) and torch.equal(dws[0], want[2]) and torch.equal(dws[1], want[3])
    assert all((x[:guard] == 77).all() and (x[-guard:] == 77).all() for x in (wholeq, wholek, whole_gq, whole_gk, ws))


def test_rows_that_are_not_finite_stay_alone_and_no_tokens():
    q, k, gq, gk, wq, wk, freq, at = (t.cuda() for t in _inputs(5, 3, 2, 64, 64, F32))
    want = pkg.division_head_norm_rotate(q, k, wq, wk, freq, at)
    q[2, 1, 7], k[3, 0, 2] = math.nan, math.inf
    got = pkg.division_head_norm_rotate(q, k, wq, wk, freq, at)
    keep = torch.ones(5, 3, dtype=torch.bool, device="cuda")
    keep[2, 1] = False
    assert torch.equal(got.q[keep], want.q[keep]) and got.q[2, 1].isnan().all()
    none = pkg.division_head_norm_rotate(q[:0], k[:0], wq, wk, freq, at[:0])
    assert none.q.shape == (0, 3, 64) and none.k_rstd.shape == (0, 2)
    dq, dk, dwq, dwk = pkg.division_head_norm_rotate_backward(gq[:0], gk[:0], q[:0], k[:0], wq, wk, freq, at[:0], none.q_rstd, none.k_rstd)
    assert dq.shape == (0, 3, 64) and not dwq.any() and not dwk.any()
    zero = pkg.division_head_norm_rotate(torch.zeros_like(q), torch.zeros_like(k), wq, wk, freq, at, 0.0)
    assert zero.q_rstd.isinf().all() and zero.q.isnan().all()                     # 0 / 0, as the definition has it


def test_gradients_against_differences():
    q, k, gq, gk, wq, wk, freq, at = _inputs(9, 2, 1, 20, 12, F32)
    dev = [t.cuda() for t in (q, k, wq, wk, freq, at)]
    r = pkg.division_head_norm_rotate(*dev, 1e-3)
    dq, _, dw, _ = pkg.division_head_norm_rotate_backward(gq.cuda(), gk.cuda(), *dev, r.q_rstd, r.k_rstd)

    def value(x, w):
        return (_turned(x * torch.rsqrt((x * x).mean(2, keepdim=True) + 1e-3) * w, freq, at, "halves")[0] * gq.double()).sum()
    gen = torch.Generator().manual_seed(4)
    x, w, step = q.double(), wq.double(), 1e-5
    for got, way, move in ((dq, torch.randn(x.shape, generator=gen, dtype=torch.float64), 0), (dw, torch.randn(w.shape, generator=gen, dtype=torch.float64), 1)):
        up, down = (value(x + s * step * way, w) if move == 0 else value(x, w + s * step * way) for s in (1, -1))
        parts = got.double().cpu() * way
        assert abs(parts.sum() - (up - down) / (2 * step)) <= 1e-5 * parts.abs().sum()


def test_the_same_bits_on_another_stream_and_in_graphs():
    q, k, gq, gk, wq, wk, freq, at = (t.cuda() for t in _inputs(5000, 4, 2, 64, 64, BF16))

    def calls():
        r = pkg.division_head_norm_rotate(q, k, wq, wk, freq, at)
        return (*r, *pkg.division_head_norm_rotate_backward(gq, gk, q, k, wq, wk, freq, at, r.q_rstd, r.k_rstd))
    want = calls()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    r = pkg.division_head_norm_rotate(q, k, wq, wk, freq, at, stream=side)
    got = (*r, *pkg.division_head_norm_rotate_backward(gq, gk, q, k, wq, wk, freq, at, r.q_rstd, r.k_rstd, stream=side))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    with torch.cuda.stream(side):
        calls()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            outs = calls()
    for n in range(3):
        q.mul_(1.25)
        at.add_(n + 3)
        want = calls()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), n
