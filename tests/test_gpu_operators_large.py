"""Tensors of more than 2^31 elements, whose byte offsets pass 32 bits several times: the last rows give what they give by themselves."""
import pytest
import torch

import paper_2208_04187_amd as pkg

pytestmark = pytest.mark.gpu


def _tiled(rows, columns, dtype, seed):
    """Rows that repeat every 997, so that a wrong offset is a wrong row"""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    part = torch.randn(997, columns, device="cuda", generator=gen).to(dtype)
    return part.repeat(rows // 997 + 1, 1)[:rows]


def test_norm_of_many_rows():
    T, D = 530001, 4100
    x, r = _tiled(T, D, torch.bfloat16, 1), _tiled(T, D, torch.bfloat16, 2)
    w = torch.rand(D, device="cuda") + 0.5
    n = pkg.division_rms_norm(x, w, residual=r, code="int8", group=128)
    values = pkg.division_read_codes(n.codes, n.scales)
    dx, _ = pkg.division_rms_norm_backward(r, n.sum, w, n.rstd, grad_sum=x)
    for s in (slice(T - 5, T), slice(T // 2, T // 2 + 3), slice(0, 2)):
        part = pkg.division_rms_norm(x[s], w, residual=r[s], code="int8", group=128)
        assert all(torch.equal(a, b[s]) for a, b in zip(part, n))
        assert torch.equal(values[s], pkg.division_read_codes(part.codes, part.scales))
        assert torch.equal(dx[s], pkg.division_rms_norm_backward(r[s], part.sum, w, part.rstd, grad_sum=x[s])[0])


def test_log_probs_of_many_rows():
    T, V = 36001, 60011
    z = _tiled(T, V, torch.bfloat16, 3)
    ids = (torch.arange(T, device="cuda") * 7919) % V
    g = torch.rand(T, device="cuda")
    f = pkg.division_log_probs(z, ids, top=3)
    dz = pkg.division_log_probs_backward(z, ids, f.lse, g)
    for s in (slice(T - 3, T), slice(T // 2, T // 2 + 2), slice(0, 1)):
        rows = z[s].double()
        assert ((torch.logsumexp(rows, 1) - f.lse[s]).abs() < 1e-4).all()
        assert ((rows.gather(1, ids[s, None])[:, 0] - torch.logsumexp(rows, 1) - f.logp[s]).abs() < 1e-4).all()
        assert torch.equal(rows.float().sort(dim=1, descending=True, stable=True).indices[:, :3], f.top_ids[s])
        assert torch.equal(dz[s], pkg.division_log_probs_backward(z[s], ids[s], f.lse[s], g[s]))


def test_gradients_of_many_elements():
    n = (1 << 31) + 12345
    a = torch.full((n,), 0.5, dtype=torch.bfloat16, device="cuda")
    a[-1], a[n // 2] = 1000.0, -3008.0                 # both are bfloat16's
    b = torch.full((77,), 2.0, device="cuda")
    want = ((n - 2) * 0.25 + 1e6 + 3008.0 ** 2 + 77 * 4.0) ** 0.5
    norm = pkg.division_clip_grads([a, b], want / 2)
    # the sum is binary64's, the norm is rounded to binary32; the factor is one half less 10^-6 / norm, from a limit rounded to binary32
    assert abs(norm.item() - want) <= 2 * 2.0 ** -24 * want
    assert a[-1] == 500.0 and a[n // 2] == -1504.0 and ((b - 1.0).abs() <= 1e-6 / want + 4 * 2.0 ** -24).all()
    assert (a[-1000:-1] == 0.25).all() and (a[: 1 << 20] == 0.25).all() and (a[(1 << 31) - 5000:(1 << 31) + 5000] == 0.25).all()
