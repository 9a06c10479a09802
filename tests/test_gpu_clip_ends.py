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


def _general(call):
    """The call without the binding's native side"""
    from paper_2208_04187_amd import binding
    binding._load_fast()
    fast, binding._fast = binding._fast, binding._NothingFast()
    try:
        return call()
    finally:
        binding._fast = fast


def test_autograd_is_told_of_what_is_written_over():
    def moved(tensors, call):
        was = [t._version for t in tensors]
        call()
        return [t._version > v for t, v in zip(tensors, was)]
    for how in (lambda call: call(), _general):
        g, out = [torch.randn(40, device="cuda"), torch.randn(3, 5, device="cuda")], [torch.empty(40, device="cuda"), torch.empty(3, 5, device="cuda")]
        assert moved(g + out, lambda: how(lambda: pkg.division_clip_grads(g, 0.1))) == [True, True, False, False]
        assert moved(g + out, lambda: how(lambda: pkg.division_clip_grads(g, 0.1, out=out))) == [False, False, True, True]
        assert moved(g, lambda: how(lambda: pkg.division_grad_norm(g))) == [False, False]
    x, w, ids = torch.randn(4, 64, device="cuda"), torch.ones(64, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    n, f = pkg.division_rms_norm(x, w, code="int8"), pkg.division_log_probs(x, ids)
    out = torch.empty_like(x)
    assert moved([x, out], lambda: pkg.division_read_codes(n.codes, n.scales, out=out)) == [False, True]
    assert moved([x, out], lambda: pkg.division_rms_norm_backward(x, x, w, n.rstd, out=out)) == [False, True]
    assert moved([x, out], lambda: pkg.division_log_probs_backward(x, ids, f.lse, f.logp, out=out)) == [False, True]
    # who saved the logits is told that they are gone
    leaf = torch.randn(4, 64, device="cuda", requires_grad=True)
    z = leaf * 1.0
    square = (z * z).sum()
    pkg.division_log_probs_backward(z.detach(), ids, f.lse, f.logp, out=z.detach())
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        square.backward()


def test_tensors_without_versions_are_clipped_too():
    with torch.inference_mode():
        g = [torch.randn(40, device="cuda"), torch.randn(7, device="cuda")]
        out = [torch.empty_like(t) for t in g]
    keep = [t.clone() for t in g]
    for how in (lambda call: call(), _general):
        how(lambda: pkg.division_clip_grads(g, 0.5, out=out))
        assert all(not torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(g, out, keep))
    pkg.division_clip_grads(g, 0.5)
    assert all(torch.equal(a, b) for a, b in zip(g, out))
