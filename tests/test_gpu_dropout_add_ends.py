"""Dropout without a stored mask at the largest size that it takes, 2^35 elements: fp32 and bfloat16 keep the same ones, whose words are those of their numbers alone."""
import pytest
import torch

import paper_2208_04187_amd as pkg

from .pyref import rand16

pytestmark = pytest.mark.gpu


def test_the_largest_size():
    n, p, seed = 2 ** 35, 0.25, 3
    places = (0, 2 ** 32 - 4096, 2 ** 34 - 4096, 2 ** 34, 2 ** 35 - 2 ** 32, 2 ** 35 - 4096)
    torch.cuda.empty_cache()
    kept = {}
    for dtype in (torch.bfloat16, torch.float32):
        x = torch.ones(n, dtype=dtype, device="cuda")                              # 64 and 128 GB
        assert pkg.division_dropout_add(x, p, seed, out=x) is x
        parts = [x[a: a + 4096].float().cpu() for a in places]
        del x
        torch.cuda.empty_cache()
        by = torch.tensor(1.0 / (1.0 - p), dtype=dtype).float()
        assert all(((t == 0) | (t == by)).all() for t in parts)
        kept[dtype] = [t != 0 for t in parts]
    assert all(torch.equal(a, b) for a, b in zip(*kept.values()))
    for a, t in zip(places, kept[torch.float32]):
        words = [rand16(seed ^ 0xD509A5B3C2E1F047, i >> 32, i & (2 ** 32 - 1)) for i in range(a, a + 4096)]
        assert t.tolist() == [w >= 16384 for w in words]                           # p * 2^16
