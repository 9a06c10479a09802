"""Attention and its backward pass against the definition in 64 bits.

Bounds.  EPS is half a unit in the last place of binary32, HALF that of a probability (or a score's gradient) as a factor of the second products: 2^-8 in bfloat16, EPS in fp32.
A score is a sum of D products, off by at most (D + 8) EPS of the sum of their magnitudes; a weight exp(z - m) by that and a few EPS of its exponent, relatively; a weighted mean of n values
by the weights' error twice (weight and sum), HALF once and (n + 64) EPS for the sums.  The same, step by step, backward.  A number below TINY, the smallest normal of binary32 and of bfloat16, may
be 0 (the machine's exponential and matrix products take no smaller ones): a weight, a score's gradient, a factor or a sum is off by TINY more.  Results in bfloat16 are what some number within the
bound rounds to."""
import ctypes
import math

import pytest
import torch

import paper_2208_04187_amd as pkg
from paper_2208_04187_amd import layer_operators as ops

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24
TINY = 2.0 ** -126
F32, BF16 = torch.float32, torch.bfloat16


def _within(got, want, bound, what=""):
    want, bound = want.cpu(), bound.cpu()
    lo, hi = want - bound, want + bound
    if got.dtype == BF16:                           # rounding keeps the order
        lo, hi = lo.float().bfloat16().double(), hi.float().bfloat16().double()
    got = got.double().cpu()
    bad = ~((lo <= got) & (got <= hi))
    assert not bad.any(), (what, int(bad.sum()), ((got - want).abs() - bound).nan_to_num(math.inf).max().item())


def _inputs(B, Sq, Sk, H, G, D, dtype, seed=0, by=1.2):
    gen = torch.Generator().manual_seed(seed + 1000 * Sq + Sk + D)
    return tuple((torch.randn(s, generator=gen) * by).to(dtype) for s in ((B, Sq, H, D), (B, Sk, G, D), (B, Sk, G, D), (B, Sq, H, D)))


def _seen(B, Sq, Sk, causal, window, lengths, starts):
    seen = torch.zeros(B, Sq, Sk, dtype=torch.bool)
    j = torch.arange(Sk)
    for b in range(B):
        n = Sk if lengths is None else max(0, min(Sk, lengths[b]))
        for i in range(Sq):
            at = i + (Sk - Sq if starts is None else starts[b])
            s = j < n
            if causal:
                s = s & (j <= at)
            if window:
                s = s & ((j - at).abs() < window)
            seen[b, i] = s
    return seen


def _definition(q, k, v, g, seen, scale, half, lse=None, out=None):
    """(values, bounds) of out, lse, dq, dk and dv; the gradients from lse and out as they were written, if given"""
    B, Sq, H, D = q.shape
    Sk, G = k.shape[1:3]
    R = H // G
    Q, K, V, DO = (t.double().transpose(1, 2) for t in (q, k.repeat_interleave(R, 2), v.repeat_interleave(R, 2), g))       # [B, H, S, D]
    hidden = ~seen[:, None]
    kt, vt = K.transpose(2, 3), V.transpose(2, 3)
    z = (Q @ kt * scale).masked_fill(hidden, -math.inf)
    size = (Q.abs() @ kt.abs() * scale).masked_fill(hidden, 0.0)
    want_lse = torch.logsumexp(z, 3) if Sk else torch.full((B, H, Sq), -math.inf, dtype=torch.float64)
    empty = want_lse == -math.inf
    p = torch.exp(z - torch.where(empty, 0.0, want_lse)[..., None])
    off = ((D + 8) * size + 8 * torch.where(hidden, 0.0, z).abs()) * EPS
    worst = off.amax(3, keepdim=True) if Sk else off.sum(3, keepdim=True)
    e_p = off + worst + 16 * EPS
    o = p @ V
    b_o = (2 * e_p * p) @ V.abs() + (half + (Sk + 64) * EPS) * (p @ V.abs()) + TINY * (V.abs().sum(2, keepdim=True) + 1)
    b_lse = torch.where(empty, 0.0, worst.squeeze(3) + (Sk + 64) * EPS + 4 * EPS * want_lse.abs())
    got = {"out": (o.transpose(1, 2), b_o.transpose(1, 2)), "lse": (torch.where(empty, -math.inf, want_lse), b_lse)}
    if lse is None:
        return got
    L = lse.double().cpu()
    p = torch.where(hidden, 0.0, torch.exp(torch.where(hidden, 0.0, z) - torch.where(empty, 0.0, L)[..., None]))
    O = out.double().cpu().transpose(1, 2)
    d = DO @ vt - (DO * O).sum(3, keepdim=True)
    ds = p * d
    e_p = off + 16 * EPS + 4 * EPS * torch.where(empty, 0.0, L).abs()[..., None]
    b_p = p * e_p
    b_ds = p * (e_p * d.abs() + (D + 8) * EPS * (DO.abs() @ vt.abs() + (DO * O).abs().sum(3, keepdim=True))) + 4 * EPS * ds.abs()
    seeing = (~hidden).double()
    b_p, b_ds = b_p + half * p + TINY * seeing, b_ds + half * (ds.abs() + b_ds) + TINY * seeing * (d.abs() + 1)
    n, m = (Sk + 64) * EPS, (Sq * R + 64) * EPS
    group = lambda t: t.unflatten(1, (G, R)).sum(2).transpose(1, 2)                                                       # noqa: E731
    got["dq"] = ((ds @ K * scale).transpose(1, 2), ((b_ds + n * ds.abs()) @ K.abs() * scale).transpose(1, 2) + TINY)
    dst, pt = ds.transpose(2, 3), p.transpose(2, 3)
    got["dk"] = (group(dst @ Q * scale), group((b_ds.transpose(2, 3) + m * dst.abs()) @ Q.abs() * scale) + TINY)
    got["dv"] = (group(pt @ DO), group((b_p.transpose(2, 3) + m * pt) @ DO.abs()) + TINY)
    return got


def _check(q, k, v, g, causal=False, window=0, lengths=None, starts=None, scale=None):
    B, Sq, H, D = q.shape
    half = 2.0 ** -8 if q.dtype == BF16 else EPS
    dev = [t.cuda() for t in (q, k, v, g)]
    kw = dict(causal=causal, window=window, scale=scale, **{n: None if t is None else torch.tensor(t, dtype=torch.int32, device="cuda") for n, t in (("lengths", lengths), ("starts", starts))})
    a = pkg.division_attention(*dev[:3], **kw)
    grads = pkg.division_attention_backward(dev[3], *dev[:3], a.out, a.lse, **kw)
    torch.cuda.synchronize()
    seen = _seen(B, Sq, k.shape[1], causal, window, lengths, starts)
    want = _definition(q, k, v, g, seen, 1.0 / math.sqrt(D) if scale is None else scale, half, a.lse, a.out)
    assert torch.equal(a.lse.cpu() == -math.inf, want["lse"][0] == -math.inf)
    some = want["lse"][0] > -math.inf
    _within(a.lse.cpu()[some], want["lse"][0][some], want["lse"][1][some], "lse")
    for name, got in zip(("out", "dq", "dk", "dv"), (a.out, *grads)):
        assert got.dtype == q.dtype
        _within(got, *want[name], name)
    empty = ~seen.any(2)
    assert not a.out.cpu()[empty].any() and not grads[0].cpu()[empty].any()
    unseen = ~seen.any(1)
    assert not grads[1].cpu()[unseen].any() and not grads[2].cpu()[unseen].any()
    return a, grads


# batch, queries, keys, heads, key heads, features
SIZES = [(1, 1, 1, 1, 1, 8), (2, 1, 1, 4, 2, 64), (1, 2, 2, 1, 1, 128), (2, 31, 31, 2, 1, 64), (1, 32, 32, 3, 3, 40), (2, 33, 33, 4, 2, 128), (1, 63, 65, 2, 2, 64), (2, 65, 64, 6, 2, 72),
         (1, 129, 129, 2, 1, 128), (1, 200, 77, 5, 1, 16), (1, 77, 200, 5, 1, 96), (1, 1, 300, 8, 2, 128), (2, 1, 1000, 32, 1, 64), (1, 1, 33, 33, 1, 24), (1, 6, 515, 5, 1, 128),
         (2, 7, 515, 10, 2, 64), (1, 1, 500, 4, 1, 96), (2, 2, 70, 6, 3, 88), (1, 8, 700, 8, 2, 104), (1, 300, 1, 2, 1, 64), (1, 1, 4097, 4, 2, 128), (1, 257, 600, 2, 2, 120)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", SIZES)
def test_matches_the_definition(size, dtype):
    x = _inputs(*size, dtype)
    _check(*x)
    _check(*x, causal=True)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", [(3, 33, 33, 4, 2, 64), (3, 70, 130, 2, 1, 128), (3, 1, 200, 8, 2, 128), (4, 3, 90, 12, 4, 72), (3, 130, 40, 2, 2, 64)])
def test_masks(size, dtype):
    x = _inputs(*size, dtype, seed=1)
    B, Sq, Sk = size[:3]
    lengths = [Sk // 2 + 1, 0, Sk, 1][:B]
    for kw in (dict(window=1), dict(window=1, causal=True), dict(window=7), dict(window=40, causal=True), dict(window=2 ** 62), dict(window=2 ** 40, causal=True)):
        _check(*x, **kw)
        _check(*x, **kw, lengths=lengths)
    for causal in (False, True):
        _check(*x, causal=causal, lengths=lengths)
        _check(*x, causal=causal, lengths=[Sk + 5, -3, 2 ** 31 - 1, -2 ** 31][:B])
        _check(*x, causal=causal, lengths=lengths, starts=[n - Sq for n in lengths], window=9 if causal else 0)
        _check(*x, causal=causal, starts=[-5, Sk + 3, 0, -Sq][:B], window=11)
    # positions at the ends of what 32 bits hold: everything or nothing lies before them
    _check(*x, causal=True, starts=[2 ** 31 - 1, -2 ** 31, 7, 0][:B])
    _check(*x, causal=True, starts=[2 ** 31 - 1, -2 ** 31, 7, 0][:B], window=2 ** 31)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", [(1, 1100, 70, 4, 2, 64), (2, 700, 130, 6, 2, 128), (1, 300, 33, 40, 1, 24), (3, 520, 520, 2, 1, 96)])
def test_many_queries_of_few_keys_heads(size, dtype):
    """Whose columns are cut into parts that are added up"""
    x = _inputs(*size, dtype, seed=12)
    B, Sq, Sk = size[:3]
    lengths = [Sk // 2 + 1, 0, Sk - 1][:B]
    _check(*x)
    _check(*x, causal=True, lengths=lengths)
    _check(*x, causal=True, window=40, starts=[Sk - 9, 3, -Sq // 2][:B])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D", [24, 64, 72, 128])
def test_many_workgroups(D, dtype):
    """Whole blocks of 128 queries for all CUs, without parts of the keys, and as few as that a block of 32 pays"""
    _check(*_inputs(16, 130, 140, 16, 16, D, dtype), causal=True)
    _check(*_inputs(16, 130, 140, 16, 8, D, dtype), window=50, lengths=[140 - 9 * b for b in range(16)])
    _check(*_inputs(3, 200, 600, 16, 8, D, dtype), causal=True, lengths=[600, 77, 0])


@pytest.mark.parametrize("D", [40, 64, 96, 128])
def test_gradients_of_few_workgroups(D):
    """Blocks of 64 whose tiles four groups of wavefronts share, in parts and not; many keys of few queries, many queries of few keys"""
    _check(*_inputs(2, 700, 700, 2, 2, D, BF16), causal=True, lengths=[700, 333])
    _check(*_inputs(1, 70, 1900, 4, 2, D, BF16), causal=True, window=900)
    _check(*_inputs(1, 1030, 130, 8, 2, D, BF16))
    _check(*_inputs(1, 1300, 130, 8, 2, D, BF16), window=100)


@pytest.mark.parametrize("size", [(1, 200, 2500, 2, 1, 64), (2, 70, 2100, 4, 2, 128), (1, 300, 2300, 3, 3, 96)])
def test_parts_of_long_sequences(size):
    _check(*_inputs(*size, BF16), causal=True)
    _check(*_inputs(*size, BF16), window=700, lengths=[2000, 100][:size[0]])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scales_and_large_scores(dtype):
    x = _inputs(2, 40, 70, 4, 2, 64, dtype, seed=2)
    _check(*x, scale=1.0)
    _check(*x, scale=1e-30)
    q, k, v, g = _inputs(1, 40, 200, 2, 2, 64, dtype, seed=3, by=8.0)
    _check(q, k, v, g, causal=True)
    # scores that rise from key to key, by more than any factor that is carried along
    k = (torch.arange(200).view(1, 200, 1, 1) * 0.25 * torch.ones(1, 200, 2, 64)).to(dtype)
    _check(q.abs(), k, v, g, causal=True)
    _check(q.abs(), -k, v, g)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", [(3, 50, 50, 4, 2, 64), (3, 1, 150, 8, 2, 128), (3, 140, 200, 2, 2, 72)])
def test_what_lies_behind_a_sequence_is_not_looked_at(size, dtype):
    q, k, v, g = (t.cuda() for t in _inputs(*size, dtype, seed=4))
    Sk = size[2]
    for lengths in ([Sk // 3, 0, Sk - 1], [1, Sk, 33]):
        n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        behind = (torch.arange(Sk, device="cuda") >= n[:, None])[..., None, None]
        got = []
        for word in (0.0, math.nan, math.inf, -math.inf, torch.finfo(dtype).min):
            kk, vv = k.masked_fill(behind, word), v.masked_fill(behind, word)
            for kw in (dict(lengths=n), dict(lengths=n, causal=True, window=20)):
                a = pkg.division_attention(q, kk, vv, **kw)
                got.append((*a, *pkg.division_attention_backward(g, q, kk, vv, a.out, a.lse, **kw)))
        for k1, row in enumerate(got[2:]):
            assert all(torch.equal(p, r) for p, r in zip(row, got[k1 % 2])), k1
        assert all(t.isfinite().all() for row in got for t in (row[0], *row[2:]))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", [(2, 50, 300, 4, 2, 64), (2, 1, 300, 8, 2, 128), (2, 5, 300, 4, 4, 40), (2, 140, 300, 2, 2, 96)])
def test_what_no_query_sees_is_not_looked_at(size, dtype):
    """A cache behind the position that a sequence has come to, or before its window, holds anything"""
    q, k, v, g = (t.cuda() for t in _inputs(*size, dtype, seed=14))
    B, Sq, Sk = size[:3]
    starts = [37, 101]
    for kw in (dict(causal=True), dict(causal=True, window=21), dict(window=21), dict(window=70, lengths=[90, 300])):
        seen = _seen(B, Sq, Sk, kw.get("causal", False), kw.get("window", 0), kw.get("lengths"), starts)
        none = ~seen.any(1).cuda()[..., None, None]
        assert none.any(1).all()
        kw = {**kw, "starts": torch.tensor(starts, dtype=torch.int32, device="cuda")}
        if "lengths" in kw:
            kw["lengths"] = torch.tensor(kw["lengths"], dtype=torch.int32, device="cuda")
        got = []
        for word in (0.0, math.nan, math.inf, torch.finfo(dtype).min):
            kk, vv = k.masked_fill(none, word), v.masked_fill(none, word)
            a = pkg.division_attention(q, kk, vv, **kw)
            got.append((*a, *pkg.division_attention_backward(g, q, kk, vv, a.out, a.lse, **kw)))
        for row in got[1:]:
            assert all(torch.equal(p, r) for p, r in zip(row, got[0]))
        assert all(t.isfinite().all() for t in (got[0][0], *got[0][2:]))


def test_nan_and_infinity_reach_those_who_see_them():
    q, k, v, g = (t.cuda() for t in _inputs(1, 70, 70, 2, 2, 64, F32, seed=5))
    for t, place in ((q, 0), (k, 1), (v, 2)):
        bad = [x.clone() for x in (q, k, v)]
        bad[place][0, 40, 1, 3] = math.nan
        out, lse = pkg.division_attention(*bad, causal=True)
        assert out[0, :, 0].isfinite().all() and not out[0, 40, 1].isfinite().all()
        if place == 0:
            assert out[0, :40, 1].isfinite().all() and out[0, 41:, 1].isfinite().all()
    k[0, 5] = math.inf
    assert not pkg.division_attention(q, k, v).out.isfinite().any(-1).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strides(dtype):
    gen = torch.Generator().manual_seed(6)
    B, S, H, G, D = 2, 75, 6, 2, 40
    per = 8 if dtype == BF16 else 4
    x = torch.randn(B, S, (H + 2 * G) * D + 3 * per, generator=gen).to(dtype).cuda()
    q, k, v = x[..., per: per + H * D].unflatten(2, (H, D)), x[..., per + H * D: per + (H + G) * D].unflatten(2, (G, D)), x[..., -G * D:].unflatten(2, (G, D))
    g = torch.randn(B, H, S, D, generator=gen).to(dtype).cuda().transpose(1, 2)
    other = torch.randn(S, G, B, D, generator=gen).to(dtype).cuda().permute(2, 0, 1, 3)
    far = torch.empty(H * (1 << 24), dtype=dtype, device="cuda").as_strided((B, S, H, D), (S * D, D, 1 << 24, 1))      # heads 32 or 64 MB apart, tokens next to one another
    far.copy_(q)
    for qq, kk, vv, gg in ((q, k, v, g), (q, other, v, g), (far, far[:, :, :G], v, far), (q[:1].expand(B, S, H, D), k[:, :, :1].expand(B, S, G, D), v, g[:, :1].expand(B, S, H, D)), (q[:, 5:], k[:, 3:60], v[:, 10:67], g[:, 5:])):
        dense = [t.contiguous() for t in (qq, kk, vv, gg)]
        a, b = pkg.division_attention(qq, kk, vv, causal=True), pkg.division_attention(*dense[:3], causal=True)
        assert torch.equal(a.out, b.out) and torch.equal(a.lse, b.lse) and a.out.is_contiguous()
        for p, r in zip(pkg.division_attention_backward(gg, qq, kk, vv, a.out, a.lse, causal=True), pkg.division_attention_backward(dense[3], *dense[:3], a.out, a.lse, causal=True)):
            assert torch.equal(p, r)


def test_offsets_beyond_32_bits():
    """A cache whose tokens lie 128 KB apart, and whose sequences begin behind 4 GB"""
    B, Sk, G, D, apart = 2, 36000, 2, 64, 65536
    room = torch.empty((Sk + Sk // 2 + 1) * apart, dtype=BF16, device="cuda")
    assert room.numel() * 2 > 2 ** 32
    gen = torch.Generator(device="cuda").manual_seed(7)
    k = room.as_strided((B, Sk, G, D), (Sk * apart // 2, apart, D, 1))            # the second sequence begins in the middle of the first one's room
    v = room[G * D:].as_strided((B, Sk, G, D), (Sk * apart // 2, apart, D, 1))
    fresh = [torch.randn((B, Sk, G, D), generator=gen, device="cuda").bfloat16() for _ in range(2)]
    keep = Sk // 2
    for t, f in ((k, fresh[0]), (v, fresh[1])):
        t[1, :keep].copy_(f[1, :keep])                                            # sequence 1's tokens are sequence 0's later ones
        t[0, :keep].copy_(f[0, :keep])
    n = torch.tensor([keep, keep], dtype=torch.int32, device="cuda")
    q = torch.randn((B, 2, 4, D), generator=gen, device="cuda").bfloat16()
    for s in (2, 40):
        q = torch.randn((B, s, 4, D), generator=gen, device="cuda").bfloat16()
        a, b = pkg.division_attention(q, k, v, lengths=n), pkg.division_attention(q, k.contiguous(), v.contiguous(), lengths=n)
        assert torch.equal(a.out, b.out) and torch.equal(a.lse, b.lse)
        for p, r in zip(pkg.division_attention_backward(q, q, k, v, a.out, a.lse, lengths=n), pkg.division_attention_backward(q, q, k.contiguous(), v.contiguous(), a.out, a.lse, lengths=n)):
            assert torch.equal(p, r)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_nothing_is_written_beside_the_outputs(dtype):
    B, Sq, Sk, H, G, D = 2, 37, 53, 6, 2, 24
    q, k, v, g = (t.cuda() for t in _inputs(B, Sq, Sk, H, G, D, dtype, seed=8))
    lengths = torch.tensor([11, 53], dtype=torch.int32, device="cuda")
    for sq in (37, 2):
        q1, g1 = q[:, :sq].contiguous(), g[:, :sq].contiguous()
        d = ops._attention(q1, k, v, None, True, 0, lengths, None)
        L = pkg.lib()
        guard = 4096

        def room(shape, t):
            x = torch.full((math.prod(shape) + 2 * guard,), 77.0, dtype=t, device="cuda")
            return x, x[guard: guard + math.prod(shape)]
        whole, parts = zip(*[room(s, t) for s, t in (((B, sq, H, D), dtype), ((B, H, sq), F32), ((B, sq, H, D), dtype), ((B, Sk, G, D), dtype), ((B, Sk, G, D), dtype))])
        need, back = L.division_attention_workspace(ctypes.byref(d)), L.division_attention_backward_workspace(ctypes.byref(d))
        ws = torch.full((max(need, back) // 4 + 2 * guard,), 77.0, device="cuda")
        st = torch.cuda.current_stream().cuda_stream
        assert L.division_attend(ctypes.byref(d), parts[0].data_ptr(), parts[1].data_ptr(), ws[guard:].data_ptr(), need, st) == 0
        torch.cuda.synchronize()
        assert (ws[:guard] == 77).all() and (ws[guard + need // 4:] == 77).all()
        b = ops._AttentionBackDesc(g1.data_ptr(), parts[0].data_ptr(), parts[1].data_ptr(), (ctypes.c_int64 * 3)(*g1.stride()[:3]), parts[2].data_ptr(), parts[3].data_ptr(), parts[4].data_ptr(),
                                   ws[guard:].data_ptr(), back)
        assert L.division_attention_backward(ctypes.byref(d), ctypes.byref(b), st) == 0
        torch.cuda.synchronize()
        assert (ws[:guard] == 77).all() and (ws[guard + back // 4:] == 77).all()
        for x in whole:
            assert (x[:guard] == 77).all() and (x[-guard:] == 77).all()
        a = pkg.division_attention(q1, k, v, causal=True, lengths=lengths)
        want = (a.out, a.lse, *pkg.division_attention_backward(g1, q1, k, v, a.out, a.lse, causal=True, lengths=lengths))
        assert all(torch.equal(p, w.view(-1)) for p, w in zip(parts, want))


def test_calls_without_rows():
    q, k = torch.zeros(2, 5, 4, 64, device="cuda"), torch.ones(2, 7, 2, 64, device="cuda")
    a = pkg.division_attention(q, k[:, :0], k[:, :0])
    assert not a.out.any() and (a.lse == -math.inf).all()
    dq, dk, dv = pkg.division_attention_backward(q, q, k[:, :0], k[:, :0], a.out, a.lse)
    assert not dq.any() and dk.shape == (2, 0, 2, 64)
    a = pkg.division_attention(q[:, :0], k, k)
    assert a.out.shape == (2, 0, 4, 64) and a.lse.shape == (2, 4, 0)
    _, dk, dv = pkg.division_attention_backward(q[:, :0], q[:, :0], k, k, a.out, a.lse)
    assert dk.shape == k.shape and not dk.any() and not dv.any()
    assert pkg.division_attention(q[:0], k[:0], k[:0]).out.shape == (0, 5, 4, 64)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gradients_against_differences(dtype):
    """The derivative along a direction, by differences of the definition in 64 bits: their step's square is some 1e-8 of it"""
    size = (2, 20, 27, 4, 2, 16)
    q, k, v, g = _inputs(*size, dtype, seed=9, by=0.7)
    lengths = [27, 9]
    seen = _seen(2, 20, 27, True, 0, lengths, None)
    a, grads = _check(q, k, v, g, causal=True, lengths=lengths)

    def value(x, y, w):
        return (_definition(x, y, w, g, seen, 0.25, 0.0)["out"][0] * g.double()).sum()
    gen = torch.Generator().manual_seed(10)
    xs = [t.double() for t in (q, k, v)]
    for i, got in enumerate(grads):
        way = torch.randn(xs[i].shape, generator=gen, dtype=torch.float64)
        step = 1e-4
        up, down = ([x + s * step * way if n == i else x for n, x in enumerate(xs)] for s in (1, -1))
        slope = (value(*up) - value(*down)) / (2 * step)
        parts = got.double().cpu() * way
        # each entry of a bfloat16 gradient is off by a few times 2^-8 of the terms that make it up, all in all far less than of the sum of magnitudes
        assert abs(parts.sum() - slope) <= (2.0 ** -7 if dtype == BF16 else 1e-5) * parts.abs().sum()


def _calls(q, k, v, g, kw):
    a = pkg.division_attention(q, k, v, **kw)
    return (*a, *pkg.division_attention_backward(g, q, k, v, a.out, a.lse, **kw))


@pytest.mark.parametrize("sq", [1, 150])
def test_the_same_bits_on_other_streams_and_in_graphs(sq):
    q, k, v, g = (t.cuda() for t in _inputs(2, sq, 700, 8, 2, 128, BF16, seed=11))
    kw = dict(causal=True, lengths=torch.tensor([700, 600], dtype=torch.int32, device="cuda"))
    want = _calls(q, k, v, g, kw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a = pkg.division_attention(q, k, v, **kw, stream=side)
    got = (*a, *pkg.division_attention_backward(g, q, k, v, a.out, a.lse, **kw, stream=side.cuda_stream))
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(p, r) for p, r in zip(got, want))
    with torch.cuda.stream(side):
        _calls(q, k, v, g, kw)
        graphs, outs = [], []
        torch.cuda.synchronize()
        for _ in range(2):                          # two graphs that may be replayed in any order
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                outs.append(_calls(q, k, v, g, kw))
            graphs.append(graph)
    for n in range(3):
        with torch.no_grad():
            q.add_(0.25)
            kw["lengths"].sub_(17)
        want = _calls(q, k, v, g, kw)
        for graph in graphs[:: 1 if n % 2 else -1]:
            graph.replay()
        torch.cuda.synchronize()
        for row in outs:
            assert all(torch.equal(p, r) for p, r in zip(row, want)), n


def test_refusals_on_the_device():
    q, k = torch.zeros(2, 5, 4, 64, device="cuda"), torch.zeros(2, 7, 2, 64, device="cuda")
    n = torch.zeros(2, dtype=torch.int32, device="cuda")
    a = pkg.division_attention(q, k, k)
    for call in (lambda: pkg.division_attention(q[..., ::2], k[..., ::2], k[..., ::2]), lambda: pkg.division_attention(q, k, k[:, :6]), lambda: pkg.division_attention(q, k[:1], k[:1]),
                 lambda: pkg.division_attention(q, k[:, :, :0], k[:, :, :0]), lambda: pkg.division_attention(q[:, :, :3], k, k), lambda: pkg.division_attention(q, k, k, lengths=n[:1]),
                 lambda: pkg.division_attention(q, k, k, lengths=n.cpu()), lambda: pkg.division_attention(q, k, k, window=-1), lambda: pkg.division_attention(q[0], k[0], k[0]),
                 lambda: pkg.division_attention_backward(q[:, :4], q, k, k, a.out, a.lse), lambda: pkg.division_attention_backward(q, q, k, k, a.out[:, :4], a.lse),
                 lambda: pkg.division_attention_backward(q, q, k, k, a.out, a.lse[:1])):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: pkg.division_attention(q, k.bfloat16(), k), lambda: pkg.division_attention(q.double(), k.double(), k.double()), lambda: pkg.division_attention(q, k, k, starts=n.long()),
                 lambda: pkg.division_attention(q.half(), k.half(), k.half())):
        with pytest.raises(TypeError):
            call()
    wide = torch.zeros(2, 5, 4, 136, device="cuda")
    for call in (lambda: pkg.division_attention(wide, wide, wide), lambda: pkg.division_attention(wide[..., :7], wide[..., :7], wide[..., :7]), lambda: pkg.division_attention(q, k, k, scale=0.0),
                 lambda: pkg.division_attention(q, k, k, scale=-1.0), lambda: pkg.division_attention(q, k, k, scale=math.inf), lambda: pkg.division_attention(wide[..., 1:65], wide[..., 1:65], wide[..., 1:65]),
                 lambda: pkg.division_attention(torch.zeros(2, 5, 4, 66, device="cuda")[..., :64], k, k)):
        with pytest.raises(pkg.DivisionError):
            call()
