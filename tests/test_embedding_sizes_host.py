"""Tables and tokens that no launch has room for are refused (no GPU needed)."""
import pytest

from .test_layer_operators_host import ERANGE, _embed, _embed_back


@pytest.mark.parametrize("T,D,dt", [(1 << 22, 4096, 0), ((1 << 22) - 1, 4097, 0), (1 << 24, 2048, 1), ((1 << 31) - 1, 9, 0)])
def test_rows_of_too_many_pieces(T, D, dt):
    size = 4 if dt == 0 else 8
    assert T * -(-D // size) > 2 ** 32 - 256 and _embed(T=T, D=D, V=7, dt=dt) == ERANGE


@pytest.mark.parametrize("change", [dict(V=1 << 30, D=1), dict(V=(1 << 31) - 1, D=1), dict(V=1 << 28, D=600), dict(V=1 << 20, D=1 << 19)])
def test_gradients_of_too_many_rows(change):
    assert _embed_back(**{**change, "grad_stride": change["D"], "workspace_bytes": 1 << 60}) == ERANGE
