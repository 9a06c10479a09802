"""Dropout without a stored mask drops what the form with a stored mask drops, and adds the rest to the residual stream: a product and a sum in binary32, each rounded, equal to torch's."""
import math

import pytest
import torch

import paper_2208_04187_amd as pkg

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def _kept(n, p, seed):
    return pkg.division_dropout_forward(torch.ones(n, device="cuda"), p, seed)[0] != 0


def _want(x, r, p, kept):
    by = torch.tensor(1.0 / (1.0 - p) if p < 1.0 else 0.0, dtype=F32, device="cuda")
    y = torch.where(kept.view(x.shape), x.float() * by, 0.0)
    return (y if r is None else y + r.float()).to(x.dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [1, 2, 3, 7, 8, 9, 31, 63, 64, 1000, 4095, 4096, 4097, 100003, 2 ** 21 + 5])
def test_drops_what_the_stored_mask_drops(n, dtype):
    gen = torch.Generator().manual_seed(n)
    x, r = torch.randn(n + 1, generator=gen).to(dtype).cuda(), torch.randn(n + 1, generator=gen).to(dtype).cuda()
    for p, seed in ((0.1, 7), (0.5, 2 ** 63 + 12345), (0.0, 3), (1.0, 4), (0.999, -5), (1e-9, 6), (0.3, 2 ** 32)):
        kept = _kept(n, p, seed)
        for a, b in ((x[:n], r[:n]), (x[1:], r[1:])):          # the second starts at any element
            for res in (None, b):
                got = pkg.division_dropout_add(a, p, seed, residual=res)
                assert torch.equal(got, _want(a, res, p, kept)), (p, seed, res is None)
        at = torch.tensor([seed if seed < 2 ** 63 else seed - 2 ** 64], device="cuda")
        assert torch.equal(pkg.division_dropout_add(x[:n], p, at, residual=r[:n]), _want(x[:n], r[:n], p, kept))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_dropped_elements_may_hold_anything(dtype):
    n, p, seed = 5000, 0.4, 11
    kept = _kept(n, p, seed)
    x, r = torch.ones(n, dtype=dtype, device="cuda"), torch.arange(n, device="cuda").to(dtype)
    want = pkg.division_dropout_add(x, p, seed, residual=r)
    for word in (math.nan, math.inf, -math.inf, torch.finfo(dtype).max):
        assert torch.equal(pkg.division_dropout_add(x.masked_fill(~kept, word), p, seed, residual=r), want)
    assert not pkg.division_dropout_add(x.fill_(math.nan), 1.0, seed).any()


def test_in_place_shapes_and_streams():
    gen = torch.Generator().manual_seed(5)
    x, r = torch.randn(3, 5, 77, generator=gen).cuda(), torch.randn(3, 5, 77, generator=gen).cuda()
    want = pkg.division_dropout_add(x, 0.3, 9, residual=r)
    assert want.shape == x.shape
    a, b = x.clone(), r.clone()
    version = a._version
    assert pkg.division_dropout_add(a, 0.3, 9, residual=r, out=a) is a and torch.equal(a, want) and a._version > version
    assert torch.equal(pkg.division_dropout_add(x, 0.3, 9, residual=b, out=b), want) and torch.equal(b, want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = pkg.division_dropout_add(x, 0.3, 9, residual=r, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    assert pkg.division_dropout_add(x[:0], 0.3, 9).shape == (0, 5, 77)
    room = torch.full((x.numel() + 128,), 77.0, device="cuda")
    pkg.division_dropout_add(x, 0.3, 9, out=room[64:-64].view(x.shape))
    assert (room[:64] == 77).all() and (room[-64:] == 77).all()


def test_a_graph_drops_other_elements_when_its_seed_is_another():
    x, seed = torch.randn(10000, device="cuda"), torch.tensor([1], device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        pkg.division_dropout_add(x, 0.5, seed)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = pkg.division_dropout_add(x, 0.5, seed)
    seen = []
    for n in range(3):
        seed.add_(5)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, pkg.division_dropout_add(x, 0.5, 6 + 5 * n))
        seen.append(out != 0)
    assert not torch.equal(seen[0], seen[1]) and not torch.equal(seen[1], seen[2])


def test_beyond_32_bits():
    """Elements of the second stretch of 2^32 have words of their own"""
    n = 2 ** 32 + 4096
    x = torch.ones(n, dtype=BF16, device="cuda")
    got = pkg.division_dropout_add(x, 0.25, 3, out=x)
    y, mask = pkg.division_dropout_forward(torch.ones(n, dtype=BF16, device="cuda"), 0.25, 3)
    for a in (0, 2 ** 32 - 4096, 2 ** 32):
        assert torch.equal(got[a:a + 4096] != 0, y[a:a + 4096] != 0)
    assert not torch.equal(got[:4096], got[2 ** 32:])


def test_refusals_on_the_device():
    x = torch.zeros(4, 6, device="cuda")
    for call in (lambda: pkg.division_dropout_add(x.t(), 0.1, 1), lambda: pkg.division_dropout_add(x, 0.1, 1, residual=x[0]), lambda: pkg.division_dropout_add(x, 0.1, torch.zeros(2, dtype=torch.int64, device="cuda")),
                 lambda: pkg.division_dropout_add(x, 0.1, torch.zeros(1, dtype=torch.int64)), lambda: pkg.division_dropout_add(x, 0.1, 1, out=x[:2])):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: pkg.division_dropout_add(x.double(), 0.1, 1), lambda: pkg.division_dropout_add(x, 0.1, 1, residual=x.bfloat16()),
                 lambda: pkg.division_dropout_add(x, 0.1, torch.zeros(1, dtype=torch.int32, device="cuda"))):
        with pytest.raises(TypeError):
            call()
    for p in (-0.1, 1.1, math.nan):
        with pytest.raises(pkg.DivisionError):
            pkg.division_dropout_add(x, p, 1)
