"""Sizes of attention that no launch has room for are refused, whatever the number of queries and keys (no GPU needed)."""
import ctypes

import pytest

import paper_2208_04187_amd as pkg

from .test_layer_operators_host import ERANGE, _attend, _attention, _attention_back

# products of sequences and key heads that 32 bits take for none, for a negative number, for a few, and the first that is too many
GROUPS = [(1 << 20, 4096), (1 << 21, 4096), (1 << 19, 4096), ((1 << 20) + 1, 4096), (1 << 24, 256), (1 << 13, 2048), (1 << 24, 1)]


@pytest.mark.parametrize("B,G", GROUPS)
@pytest.mark.parametrize("Sq,Sk", [(1, 1), (0, 1), (1, 0)])
def test_sequences_times_key_heads(B, G, Sq, Sk):
    size = dict(B=B, H=G, G=G, D=8, Sq=Sq, Sk=Sk)
    assert _attend(**size) == ERANGE and _attention_back(dict(**size, workspace_bytes=1 << 62)) == ERANGE
    d = _attention(**size)
    assert pkg.lib().division_attention_workspace(ctypes.byref(d)) == 0 and pkg.lib().division_attention_backward_workspace(ctypes.byref(d)) == 0


def test_no_queries_and_no_keys_are_no_work():
    for B, G in GROUPS:
        size = dict(B=B, H=G, G=G, D=8, Sq=0, Sk=0)
        assert _attend(**size) == 0 and _attention_back(dict(**size, workspace_bytes=1 << 62)) == 0


# batch, queries, keys, heads, key heads, features: parts times columns that are no multiple of four
ODD_PARTS = [(1, 1, 300, 3, 3, 64), (1, 1, 300, 1, 1, 8), (1, 3, 900, 3, 1, 40), (3, 1, 1100, 7, 7, 128), (1, 1, 4097, 5, 1, 72), (1, 1, 16400, 1, 1, 128), (1, 5, 2100, 3, 3, 24)]


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("size", ODD_PARTS)
def test_parts_lie_on_16_bytes(size, dt):
    """Each part's lse, and behind them rows of values in vectors of 16 bytes"""
    B, Sq, Sk, H, G, D = size
    need = pkg.lib().division_attention_workspace(ctypes.byref(_attention(B=B, Sq=Sq, Sk=Sk, H=H, G=G, D=D, dt=dt)))
    rows = need // (4 * (D + 1))                # the room for the lse is less than a row's
    assert rows > 1 and rows % (B * Sq * H) == 0 and need == (rows * 4 + 15) // 16 * 16 + rows * D * 4
