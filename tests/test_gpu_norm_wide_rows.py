"""Rows beyond the registers mean what shorter ones do: the row's scale comes from the norm's output itself."""
import pytest
import torch

import paper_2208_04187_amd as pkg

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_rows_scale_is_that_of_its_output_under_extreme_weights(dtype, code):
    """s * weight leaves binary32 here where s * rstd * weight does not"""
    top = 127.0 if code == "int8" else 448.0
    gen = torch.Generator().manual_seed(1)
    for D in (8000, 40000):
        x = torch.randn(3, D, generator=gen)
        for size, weight in ((1e16, 1e24), (1e-15, 1e-27), (1.0, 1.0)):
            s, w = (x * size).to(dtype), torch.rand(D, generator=gen) * weight + weight
            # eps 0: the output is of the weight's size, whatever the input's
            n = pkg.division_rms_norm(s.cuda(), w.cuda(), 0.0, code=code)
            sd = s.double()
            y = sd / sd.square().mean(1, keepdim=True).sqrt() * w.double()
            most = y.abs().amax(1)
            scales = n.scales.double().cpu().view(-1)
            # the row's sum: up to D / 256 products a thread and a tree of ten steps, of which the root leaves half; eight operations more
            slack = (D / 512 + 20) * EPS
            assert ((scales - most / top).abs() <= slack * most / top).all(), (D, size, scales, most / top)
            values = pkg.division_read_codes(n.codes, n.scales, torch.float32).double().cpu()
            half = 0.5 * scales[:, None] if code == "int8" else torch.maximum(y.abs() * 2.0 ** -4, scales[:, None] * 2.0 ** -10)
            assert ((values - y).abs() <= half + slack * most[:, None]).all()


@pytest.mark.parametrize("T,D", [(2101, 16392), (2101, 20007)])
def test_a_rows_scale_does_not_depend_on_how_many_rows_there_are(T, D):
    """bfloat16 with a residual: rows of up to 32768 columns stay in registers where the call is beyond the caches, and do not where it is within them"""
    gen = torch.Generator(device="cuda").manual_seed(D)
    x, r = (torch.randn(T, D, device="cuda", generator=gen).bfloat16() for _ in range(2))
    w = torch.rand(D, device="cuda", generator=gen) + 0.5
    for code in ("int8", "e4m3"):
        big = pkg.division_rms_norm(x, w, residual=r, code=code)
        for s in (slice(0, 300), slice(T - 300, T)):
            part = pkg.division_rms_norm(x[s], w, residual=r[s], code=code)
            for a, b in zip(part, big):
                assert torch.equal(a.view(torch.int8), b[s].view(torch.int8))
