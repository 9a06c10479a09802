"""Clipping at the ends of the range, and what autograd is told of it."""
import math

import pytest
import torch

import paper_2208_04187_amd as pkg

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24


def _norm64(grads):
    return math.sqrt(math.fsum(float((g.double().cpu() ** 2).sum()) for g in grads))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [3, 9000, 40000])
def test_a_small_factor_under_a_large_limit(n, dtype):
    """The factor vanishes from binary32's normal range, its products with the largest elements do not: every element is within the limit"""
    for largest in (1e32, 1e36, 3e38):
        g = torch.full((n,), 1e25).to(dtype)
        g[0], g[n // 2] = largest, -largest / 3
        g = g.cuda()
        grads = [g, torch.full((5,), 2.0, device="cuda")]
        norm = _norm64(grads)
        for limit in (1e-30, 1e-3, 3.9, 4.0, 100.0, 1e7):
            c = min(1.0, limit / (norm + 1e-6))
            for out_type in (None, torch.float32, torch.bfloat16):
                mine = [t.clone() for t in grads]
                out = None if out_type is None else [torch.full_like(t, 7.0, dtype=out_type) for t in grads]
                pkg.division_clip_grads(mine, limit, out=out)
                for a, b in zip(mine if out is None else out, grads):
                    want, r = b.double() * c, a.double()
                    # the factor, the product and the end of the range
                    lo, hi = want - 4 * EPS * want.abs() - 2.0 ** -149, want + 4 * EPS * want.abs() + 2.0 ** -149
                    if a.dtype == torch.bfloat16:
                        lo, hi = lo.float().bfloat16().double(), hi.float().bfloat16().double()
                    assert ((lo <= r) & (r <= hi)).all(), (largest, limit, out_type)


def test_no_limit():
    """An infinite limit: finite gradients stay, an infinite norm makes the factor 0 as under any other limit"""
    for many in (1, 300):
        g = [torch.randn(70, device="cuda") for _ in range(many)] + [torch.randn(9, device="cuda").bfloat16()]
        keep = [t.clone() for t in g]
        assert math.isfinite(pkg.division_clip_grads(g, math.inf).item()) and all(torch.equal(a, b) for a, b in zip(g, keep))
        g[0][3] = math.inf
        assert pkg.division_clip_grads(g, math.inf).item() == math.inf
        assert g[0][3].isnan() and not g[0][:3].any() and not g[0][4:].any() and not any(t.any() for t in g[1:])
        keep[0][3] = float("nan")
        assert pkg.division_clip_grads(keep, math.inf).isnan() and all(t.isnan().all() for t in keep)
