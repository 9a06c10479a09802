"""The entries with lse's second word refuse what those without it refuse, and a word that is not aligned (no GPU needed)."""
import ctypes

import pytest

import paper_2208_04187_amd as pkg
from paper_2208_04187_amd import operators as ops

EINVAL, EALIGN = 1, 3
FORWARD = dict(logits=4096, ids=4096, stride=64, T=4096, V=64, ignore_index=-100, dt=0, top=0, logp=4096, entropy=None, lse=4096, top_logp=None, top_ids=None, workspace=None,
               workspace_bytes=0)
BACK = dict(logits=4096, ids=4096, lse=4096, entropy=None, grad_logp=4096, grad_entropy=None, stride=64, grad_stride=64, T=4, V=64, ignore_index=-100, dt=0, grad_logits=4096)


@pytest.mark.parametrize("low,change,code", [(2, {}, EALIGN), (4, dict(lse=None), EINVAL), (None, dict(lse=None), EINVAL), (4, dict(V=0), EINVAL), (2, dict(T=0), 0), (None, dict(T=0), 0)])
def test_entries_with_the_second_word_refuse(low, change, code):
    L = pkg.lib()
    a, b = ops._LogitsDesc(*{**FORWARD, **change}.values()), ops._LogitsBackDesc(*{**BACK, **change}.values())
    assert L.division_log_probs_low(ctypes.byref(a), low, None) == code and L.division_log_probs_backward_low(ctypes.byref(b), low, None) == code
    if low != 2:
        assert L.division_log_probs(ctypes.byref(a), None) == code and L.division_log_probs_backward(ctypes.byref(b), None) == code
    assert L.division_log_probs_low(None, low, None) == EINVAL and L.division_log_probs_backward_low(None, low, None) == EINVAL
