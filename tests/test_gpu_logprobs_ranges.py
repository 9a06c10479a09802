"""Log probabilities where logits are large, share an offset, or are masked with finite numbers, against the definition in 64 bits.

Bounds.  EPS is half a unit in the last place of binary32.  e^d of d = z - max <= 0 is off by (2 |d| + 3) EPS of itself; its exponent is taken against the maximum's own,
whose rounding r EPS, r up to 2^30 log2 e, is put back later: `back` is that in e's powers, and costs EPS of itself in every term and in the logarithm.  A thread adds up to V / 64
terms and joins in twenty steps more."""
import math

import pytest
import torch

import paper_2208_04187_amd as pkg

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24
INF = math.inf
TYPES = [torch.float32, torch.bfloat16]


def _definition(z, ids):
    """lse, logp, entropy, ln S, mean |d|, the maximum"""
    z = z.double().cpu()
    most = z.amax(1)
    d = z - most[:, None]
    e = d.exp()
    S, U = e.sum(1), -(e * d.clamp(min=-1e30)).sum(1)
    logp = d.gather(1, ids.cpu()[:, None])[:, 0] - S.log()
    return most + S.log(), logp, S.log() + U / S, S.log(), U / S, most


def _bounds(V, mean, most):
    back = most.abs().clamp(max=2.0 ** 30) * EPS
    return (V / 64 + 30 + 2 * mean + 4 * back) * EPS, back


def _near(got, want, bound, what):
    got = got.double().cpu()
    same = got == want.float().double()
    bad = ~(same | ((got - want).abs() <= bound))
    assert not bad.any(), (what, int(bad.sum()), got[bad][:4], want[bad][:4])


def _order(z, top):
    z = torch.where(z.isnan(), -INF, z.float().cpu())
    return z.sort(dim=1, descending=True, stable=True).indices[:, :top]


def _check(z, ids, got, top):
    lse, logp, H, ln, mean, most = _definition(z, ids)
    off, back = _bounds(z.shape[1], mean, most)
    _near(got.lse, lse, off + 2 * EPS * lse.abs(), "lse")
    _near(got.logp, logp, off + 2 * EPS * (lse.abs() + logp.abs()), "logp")
    _near(got.entropy, H, (off + 10 * EPS) * (1 + H + 3 * mean) + 2 * EPS * H + 4 * EPS * back, "entropy")
    if top:
        want = _order(z, top)
        assert torch.equal(got.top_ids.cpu(), want)
        d = z.cpu().double().gather(1, want) - lse[:, None]
        _near(got.top_logp, d, (off + 2 * EPS * lse.abs())[:, None] + 2 * EPS * d.abs(), "top")


LARGE = [1e9, 2.0 ** 30 - 64, 2.0 ** 30, 3e9, 1e10, 1e12, 1e20, 1e30]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V", [(1, 40), (3, 3000), (1, 70001), (1300, 300), (1030, 9001)])
def test_rows_of_one_large_number_are_uniform(T, V, dtype):
    values = torch.tensor([s * v for v in LARGE for s in (-1.0, 1.0)]).to(dtype)
    for lo in range(0, len(values), T):
        rows = values[lo:lo + T]
        z = rows[:, None].expand(len(rows), V).repeat(-(-T // len(rows)), 1)[:T].contiguous()
        ids = (torch.arange(T) * 7) % V
        got = pkg.division_log_probs(z.cuda(), ids.cuda(), top=min(V, 20))
        _check(z, ids, got, min(V, 20))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V", [(2, 40), (1, 3000), (1, 131072), (5, 70001), (1300, 500), (1030, 9001)])
def test_finite_masks_leave_the_rest_what_it_is(T, V, dtype):
    """A mask of a large negative number is -inf to all that is not masked: whole threads', whole shares' columns of it"""
    gen = torch.Generator().manual_seed(V)
    z = (torch.randn(T, V, generator=gen) * 3).to(dtype)
    ids = torch.randint(0, max(1, V // 20), (T,), generator=gen)
    c = torch.arange(V)
    for masked in (c >= max(1, V // 20), (c < V - max(1, V // 20)), c % 2 == 1):
        at = torch.where(masked[ids], (~masked).nonzero()[0], ids)
        hard = pkg.division_log_probs(z.masked_fill(masked, -INF).cuda(), at.cuda(), top=2)
        for m in (-1e9, -1e10, -1e12, -1e20, -1e30, torch.finfo(dtype).min):
            soft = z.masked_fill(masked, m)
            got = pkg.division_log_probs(soft.cuda(), at.cuda(), top=2)
            _check(soft, at, got, 2)
            for a, b in ((got.lse, hard.lse), (got.logp, hard.logp), (got.entropy, hard.entropy)):
                # a term that is zero either way: the same bits
                assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", TYPES)
def test_large_logits_of_many_sizes(dtype):
    gen = torch.Generator().manual_seed(4)
    for V in (50, 5000, 40000):
        z = torch.randn(24, V, generator=gen)
        for t in range(24):
            z[t] *= 10.0 ** (t * 1.5)
        z[0, ::3] = 2.0 ** 30
        z[1, ::3] = 2.0 ** 30
        z[1, 1::3] = 2.0 ** 30 - 64
        z[2] = 2.0 ** 30 - 64
        z[2, ::5] = 2.0 ** 30 - 128
        z[3] = -2.0 ** 30
        z[3, ::5] = -2.0 ** 30 + 64
        z = z.to(dtype)
        ids = torch.randint(0, V, (24,), generator=gen)
        for rows in (slice(None), slice(1, 2), slice(2, 3), slice(20, 21)):
            _check(z[rows], ids[rows], pkg.division_log_probs(z[rows].cuda(), ids[rows].cuda(), top=9), 9)


def _check_offsets(z, ids, got, top):
    """As _check, by bounds that do not grow with lse"""
    lse, logp, H, ln, mean, most = _definition(z, ids)
    off, back = _bounds(z.shape[1], mean, most)
    # the difference from the maximum, ln S, what is put back, and their difference: each rounded once
    near = off + 2 * EPS * (ln + back)
    d = z.double().cpu() - most[:, None]
    _near(got.logp, logp, near + 2 * EPS * (d.gather(1, ids.cpu()[:, None])[:, 0].abs() + logp.abs()), "logp")
    if top:
        want = _order(z, top)
        d = d.gather(1, want)
        _near(got.top_logp, d - ln[:, None], near[:, None] + 2 * EPS * (d.abs() + (d - ln[:, None]).abs()), "top")


def _confident(T, V, gen):
    """Rows with one token of nearly all probability: log probabilities of -1e-4 to -1e-1"""
    z = torch.randn(T, V, generator=gen)
    ids = torch.randint(0, V, (T,), generator=gen)
    z.scatter_(1, ids[:, None], math.log(V) + 3 + 6 * torch.rand(T, 1, generator=gen))
    return z, ids


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V", [(1, 1000), (3, 40), (2, 70001), (1300, 300), (1030, 9001)])
def test_log_probabilities_do_not_lose_digits_to_a_common_offset(T, V, dtype):
    gen = torch.Generator().manual_seed(T + V)
    z, ids = _confident(T, V, gen)
    for offset in (0.0, 300.0, -3e3, 1e4, 1e5):
        moved = (z + offset).to(dtype)
        top = min(V, 8)
        _check_offsets(moved, ids, pkg.division_log_probs(moved.cuda(), ids.cuda(), top=top), top)


def _gradient(z, ids, g, gh=None):
    """The gradient of the logits with respect to the definition itself, and its bound: p is off as e^d and as S are, the entropy as in _check"""
    lse, _, H, ln, mean, most = _definition(z, ids)
    off, back = _bounds(z.shape[1], mean, most)
    d = z.double().cpu() - most[:, None] - ln[:, None]
    p, g = d.exp(), g.double()[:, None]
    one = torch.zeros_like(p).scatter_(1, ids[:, None], 1.0)
    lost = (2 * d.abs() + 12) * EPS + (off + 2 * EPS * (ln + back))[:, None]
    if gh is None:
        return g * one - p * g, p * g.abs() * lost + 1e-37
    gh = gh.double()[:, None]
    per, size = g + gh * (d + H[:, None]), g.abs() + gh.abs() * (d.abs() + H[:, None].abs())
    wrong = (off + 10 * EPS) * (1 + H + 3 * mean) + 2 * EPS * H + 4 * EPS * back
    return g * one - p * per, p * (size * lost + gh.abs() * (wrong + off + 2 * EPS * (ln + back))[:, None]) + 1e-37


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V", [(1, 1000), (3, 40), (2, 70001), (1300, 300), (1030, 9001)])
def test_gradients_do_not_lose_digits_to_a_common_offset(T, V, dtype):
    gen = torch.Generator().manual_seed(T + V + 1)
    z, ids = _confident(T, V, gen)
    g, gh = torch.randn(T, generator=gen), torch.randn(T, generator=gen)
    for offset in (0.0, -3e3, 1e4, 1e5, 1e10, -1e30):
        moved = (z + offset).to(dtype)
        zc, ic = moved.cuda(), ids.cuda()
        low = torch.empty(T, device="cuda")
        f = pkg.division_log_probs(zc, ic, lse_low=low)
        lse, _, _, ln, mean, most = _definition(moved, ids)
        off, back = _bounds(V, mean, most)
        _near(f.lse.double() + low.double(), lse, off + 4 * EPS * (ln + back) + lse.abs() * 2.0 ** -46, "both words")
        for entropy in (False, True):
            want, bound = _gradient(moved, ids, g, gh if entropy else None)
            kw = dict(entropy=f.entropy, grad_entropy=gh.cuda()) if entropy else {}
            got = pkg.division_log_probs_backward(zc, ic, f.lse, g.cuda(), lse_low=low, **kw)
            lo, hi = want - bound - 2 * EPS * want.abs(), want + bound + 2 * EPS * want.abs()
            if dtype == torch.bfloat16:
                lo, hi = lo.float().bfloat16().double(), hi.float().bfloat16().double()
            r = got.double().cpu()
            bad = ~((lo <= r) & (r <= hi))
            assert not bad.any(), (offset, entropy, int(bad.sum()), r[bad][:4], want[bad][:4])
            # under autograd the second word comes along
            leaf = zc.clone().requires_grad_()
            t = pkg.division_token_log_probs(leaf, ic)
            ((t.logp * g.cuda()).sum() + ((t.entropy * gh.cuda()).sum() if entropy else 0.0)).backward()
            assert torch.equal(leaf.grad, got)


def test_the_second_word_of_lse_is_zero_where_there_is_none():
    z = torch.randn(6, 3000, generator=torch.Generator().manual_seed(1))
    z[0] = -INF
    z[1, 5] = INF
    z[2, 5] = float("nan")
    ids = torch.arange(6)
    for rows in (z, z.repeat(300, 1)):
        low = torch.full((len(rows),), 7.0, device="cuda")
        f = pkg.division_log_probs(rows.cuda(), ids.repeat(len(rows) // 6).cuda(), lse_low=low)
        assert f.lse[0] == -INF and low[0] == 0 and f.lse[1].isnan() and f.lse[2].isnan() and (low[3:6].abs() <= EPS * f.lse[3:6].abs()).all()
        back = pkg.division_log_probs_backward(rows[:6].cuda(), ids.cuda(), f.lse[:6], torch.ones(6).cuda(), lse_low=low[:6])
        assert not back[0].any() and back[1:3].isnan().all() and torch.isfinite(back[3:]).all()


def test_second_words_of_other_types_and_shapes_are_refused():
    z, ids = torch.randn(4, 100, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    f = pkg.division_log_probs(z, ids)
    for low, err in ((torch.empty(4, dtype=torch.float64, device="cuda"), TypeError), (torch.empty(3, device="cuda"), ValueError), (torch.empty(4), ValueError),
                     (torch.empty(8, device="cuda")[::2], ValueError)):
        with pytest.raises(err):
            pkg.division_log_probs(z, ids, lse_low=low)
        with pytest.raises(err):
            pkg.division_log_probs_backward(z, ids, f.lse, f.logp, lse_low=low)


def test_the_second_word_through_both_sides_of_the_binding():
    from paper_2208_04187_amd import binding
    z, ids = torch.randn(3, 5, 3000, device="cuda") + 500, torch.randint(0, 3000, (3, 5), device="cuda")
    binding._load_fast()
    results = []
    for fast in (binding._fast, binding._NothingFast()):
        was, binding._fast = binding._fast, fast
        try:
            low = torch.empty(3, 5, device="cuda")
            f = pkg.division_log_probs(z, ids, top=2, lse_low=low)
            results.append([*f, low, pkg.division_log_probs_backward(z, ids, f.lse, f.logp, entropy=f.entropy, grad_entropy=f.logp, lse_low=low)])
        finally:
            binding._fast = was
    assert all(torch.equal(a, b) for a, b in zip(*results)) and results[0][-2].any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V", [(1100, 20001), (1, 20001), (1, 131072), (1300, 8000), (1300, 4000), (1300, 30)])
def test_nan_counts_as_minus_infinity_among_many_of_them(T, V, dtype):
    """More tokens that cannot be than fit beside one another, NaN before them, and fewer finite logits than alternatives"""
    z = torch.full((T, V), -INF)
    z[:, :8] = float("nan")
    z[:, V - 3] = 1.0
    if T > 1:
        z[1] = -INF
        z[1, 9:17] = float("nan")
        z[2, 100 % V:] = float("nan")
        z[3] = float("nan")
    z = z.to(dtype)
    ids = torch.zeros(T, dtype=torch.int64)
    for top in (5, 20, 30):
        got = pkg.division_log_probs(z.cuda(), ids.cuda(), top=top)
        assert torch.equal(got.top_ids[:5].cpu(), _order(z[:5], top)) and (got.top_ids[4:] == got.top_ids[-1]).all()
