"""Attention over keys in parts whose number times that of the columns is no multiple of four, against the definition in 64 bits."""
import pytest
import torch

from .test_attention_sizes_host import ODD_PARTS
from .test_gpu_attention import _check, _inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("size", ODD_PARTS)
def test_parts_of_any_number(size, dtype):
    x = _inputs(*size, dtype, seed=21)
    _check(*x)
    _check(*x, causal=True, lengths=[size[2] - 7, 30, 0][:size[0]])
