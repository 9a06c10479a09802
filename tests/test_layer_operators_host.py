"""The operators of a token model's layers refuse what they cannot take, before anything is launched (no GPU needed)."""
import ctypes
import math

import pytest
import torch

import paper_2208_04187_amd as pkg
from paper_2208_04187_amd import layer_operators as ops

EINVAL, ESIZE, EALIGN, ERANGE = 1, 2, 3, 4
S = (ctypes.c_int64 * 3)


def _attention(**kw):
    d = dict(q=4096, k=4096, v=4096, q_strides=(64, 64, 64), k_strides=(64, 64, 64), v_strides=(64, 64, 64), B=2, Sq=5, Sk=7, H=4, G=2, D=64, dt=1, scale=0.125, causal=0, window=0, lengths=None, starts=None)
    d.update(kw)
    return ops._AttentionDesc(*[S(*v) if isinstance(v, tuple) else v for v in d.values()])


def _attend(desc=None, out=4096, lse=4096, workspace=None, workspace_bytes=0, **kw):
    d = _attention(**kw) if desc is None else desc
    return pkg.lib().division_attend(ctypes.byref(d), out, lse, workspace, workspace_bytes, None)


BAD = [(dict(dt=2), EINVAL), (dict(dt=7), EINVAL), (dict(B=-1), EINVAL), (dict(Sq=-1), EINVAL), (dict(Sk=-1), EINVAL), (dict(H=0), EINVAL), (dict(G=0), EINVAL), (dict(H=3), EINVAL), (dict(D=0), EINVAL),
       (dict(D=136), EINVAL), (dict(D=60), EINVAL), (dict(D=4), EINVAL), (dict(window=-1), EINVAL), (dict(causal=2), EINVAL), (dict(scale=0.0), EINVAL), (dict(scale=-1.0), EINVAL),
       (dict(scale=math.inf), EINVAL), (dict(scale=math.nan), EINVAL), (dict(q=None), EINVAL), (dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(q=4104), EALIGN), (dict(k=4104), EALIGN),
       (dict(v=4104), EALIGN), (dict(q_strides=(4, 64, 64)), EALIGN), (dict(k_strides=(64, 4, 64)), EALIGN), (dict(v_strides=(64, 64, 4)), EALIGN), (dict(q_strides=(-8, 64, 64)), EINVAL),
       (dict(k_strides=(64, -8, 64)), EINVAL), (dict(q_strides=(64, 1 << 23, 64)), ERANGE), (dict(k_strides=(64, 64, (1 << 29) + 8)), ERANGE), (dict(q_strides=(64, 64, (1 << 28) + 8)), ERANGE), (dict(scale=3e38), EINVAL), (dict(v_strides=(1 << 40, 64, 64)), ERANGE), (dict(lengths=2), EALIGN),
       (dict(starts=6), EALIGN), (dict(Sk=(1 << 29) + 1), ERANGE), (dict(Sq=(1 << 29) + 1), ERANGE), (dict(H=8194, G=2), ERANGE), (dict(Sq=1 << 29, H=8), ERANGE), (dict(B=(1 << 24) + 1), ERANGE)]


@pytest.mark.parametrize("change,code", BAD + [(dict(out=None), EINVAL), (dict(lse=None), EINVAL), (dict(out=8), EALIGN), (dict(lse=2), EALIGN), (dict(B=0, q=None), 0), (dict(Sq=0, q=None), 0),
                                               (dict(B=1 << 20, Sq=1 << 15), ERANGE)])
def test_attention_refuses(change, code):
    assert _attend(**change) == code


def test_attention_workspaces():
    L = pkg.lib()
    assert L.division_attend(None, 4096, 4096, None, 0, None) == EINVAL and L.division_attention_workspace(None) == 0 and L.division_attention_backward_workspace(None) == 0
    for kw in (dict(D=7), dict(B=0), dict(Sq=0)):
        assert L.division_attention_workspace(ctypes.byref(_attention(**kw))) == 0
    long = _attention(Sq=1, Sk=8192, B=1)
    need = L.division_attention_workspace(ctypes.byref(long))
    assert need > 0 and need % (4 * 65 * 4) == 0                                  # parts of each head's 64 values and its lse
    assert _attend(long) == EINVAL and _attend(long, workspace=4096, workspace_bytes=need - 1) == ESIZE and _attend(long, workspace=4100, workspace_bytes=need) == EALIGN
    assert L.division_attention_workspace(ctypes.byref(_attention(B=64, Sq=4096, Sk=4096))) == 0
    assert L.division_attention_backward_workspace(ctypes.byref(_attention())) == 2 * 5 * 4 * 8


def _attention_back(change):
    d = dict(grad_out=4096, out=4096, lse=4096, grad_out_strides=(64, 64, 64), grad_q=4096, grad_k=4096, grad_v=4096, workspace=4096, workspace_bytes=1 << 30)
    fields = {k: v for k, v in change.items() if k in d}
    b = ops._AttentionBackDesc(*[S(*v) if isinstance(v, tuple) else v for v in {**d, **fields}.values()])
    return pkg.lib().division_attention_backward(ctypes.byref(_attention(**{k: v for k, v in change.items() if k not in d})), ctypes.byref(b), None)


@pytest.mark.parametrize("change,code", BAD + [*[({k: None}, EINVAL) for k in ("grad_out", "out", "lse", "grad_q", "grad_k", "grad_v", "workspace")], *[({k: 8}, EALIGN) for k in ("grad_out", "out", "grad_q", "grad_k", "grad_v", "workspace")],
                                               (dict(lse=2), EALIGN), (dict(grad_out_strides=(64, 4, 64)), EALIGN), (dict(grad_out_strides=(64, 64, -8)), EINVAL),
                                               (dict(workspace_bytes=2 * 5 * 4 * 8 - 1), ESIZE), (dict(B=0, grad_out=None), 0),
                                               # without queries the keys' gradients are zeros, and the keys as they have to be; more workgroups of keys than a launch has
                                               (dict(Sq=0, Sk=(1 << 29) + 1), ERANGE), (dict(Sq=0, k_strides=(64, 1 << 23, 64)), ERANGE), (dict(Sq=0, v_strides=(64, 4, 64)), EALIGN),
                                               (dict(B=1 << 20, Sq=1, Sk=1 << 15, G=1, workspace_bytes=1 << 50), ERANGE)])
def test_attention_backward_refuses(change, code):
    assert _attention_back(change) == code


P, T2 = ctypes.c_void_p * 2, ctypes.c_int64 * 2


def _rotate_desc(**kw):
    d = dict(x=(4096, 8192), weight=(4096, 4096), token_strides=(256, 128), head_strides=(64, 64), heads=(4, 2), weight_dt=(0, 0), T=5, D=64, rotated=32, dt=0, next=0, eps=1e-6, frequencies=4096,
             positions=4096, y=(4096, 4096), rstd=(4096, None))
    d.update(kw)
    kinds = dict(x=P, weight=P, token_strides=T2, head_strides=T2, heads=T2, weight_dt=ctypes.c_int * 2, y=P, rstd=P)
    return ops._RotateDesc(*[kinds[k](*v) if k in kinds else v for k, v in d.items()])


SIDES = [(dict(x=(None, 64)), EINVAL), (dict(x=(64, None)), EINVAL), (dict(weight=(None, 64)), EINVAL), (dict(weight=(64, None)), EINVAL), (dict(dt=2), EINVAL), (dict(weight_dt=(0, 2)), EINVAL),
         (dict(T=-1), EINVAL), (dict(D=0), EINVAL), (dict(D=63, rotated=0), EINVAL), (dict(D=514), EINVAL), (dict(rotated=66), EINVAL), (dict(rotated=31), EINVAL), (dict(rotated=-2), EINVAL),
         (dict(next=2), EINVAL), (dict(eps=-1.0), EINVAL), (dict(eps=math.nan), EINVAL), (dict(heads=(0, 2)), EINVAL), (dict(heads=(4, -1)), EINVAL), (dict(token_strides=(-1, 0)), EINVAL),
         (dict(head_strides=(0, -1)), EINVAL), (dict(frequencies=None), EINVAL), (dict(positions=None), EINVAL), (dict(frequencies=4), EALIGN), (dict(positions=4), EALIGN), (dict(x=(2, 64)), EALIGN),
         (dict(weight=(64, 2)), EALIGN), (dict(T=1 << 31), ERANGE), (dict(heads=(4097, 2)), ERANGE), (dict(token_strides=(1 << 40, 0)), ERANGE)]


@pytest.mark.parametrize("change,code", SIDES + [(dict(y=(None, 64)), EINVAL), (dict(y=(64, 2)), EALIGN), (dict(rstd=(2, None)), EALIGN), (dict(T=0, x=(None, None)), 0)])
def test_rotation_refuses(change, code):
    assert pkg.lib().division_head_norm_rotate(ctypes.byref(_rotate_desc(**change)), None) == code


@pytest.mark.parametrize("change,code", SIDES + [*[({k: v}, EINVAL) for k in ("grad_y", "grad_rstd", "grad_x", "grad_weight") for v in ((None, 64), (64, None))], (dict(grad_y=(2, 64)), EALIGN),
                                                 (dict(grad_rstd=(64, 2)), EALIGN), (dict(grad_x=(2, 64)), EALIGN), (dict(grad_weight=(2, 64)), EALIGN), (dict(grad_token=(-1, 0)), EINVAL),
                                                 (dict(grad_head=(0, 1 << 40)), ERANGE), (dict(workspace=None), EINVAL), (dict(workspace=4), EALIGN), (dict(workspace_bytes=64), ESIZE)])
def test_rotation_backward_refuses(change, code):
    d = dict(grad_y=(4096, 4096), grad_rstd=(4096, 4096), grad_token=(256, 128), grad_head=(64, 64), grad_x=(4096, 4096), grad_weight=(4096, 4096), workspace=4096, workspace_bytes=1 << 20)
    own = {**d, **{k: v for k, v in change.items() if k in d}}
    kinds = dict(grad_y=P, grad_rstd=P, grad_token=T2, grad_head=T2, grad_x=P, grad_weight=P)
    b = ops._RotateBackDesc(*[kinds[k](*v) if k in kinds else v for k, v in own.items()])
    assert pkg.lib().division_head_norm_rotate_backward(ctypes.byref(_rotate_desc(**{k: v for k, v in change.items() if k not in d})), ctypes.byref(b), None) == code


def _embed(ids=4096, T=4, table=4096, V=5, D=8, dt=0, scale=1.0, ignore=-100, out=4096):
    return pkg.lib().division_embedding(ids, T, table, V, D, dt, scale, ignore, out, None)


@pytest.mark.parametrize("change,code", [(dict(ids=None), EINVAL), (dict(table=None), EINVAL), (dict(out=None), EINVAL), (dict(dt=2), EINVAL), (dict(T=-1), EINVAL), (dict(V=0), EINVAL), (dict(D=0), EINVAL),
                                         (dict(ids=4), EALIGN), (dict(table=2), EALIGN), (dict(out=2), EALIGN), (dict(out=1, dt=1), EALIGN), (dict(T=1 << 31), ERANGE), (dict(V=1 << 31), ERANGE),
                                         (dict(T=1 << 30, D=1 << 12), ERANGE), (dict(T=0, ids=None), 0)])
def test_embedding_refuses(change, code):
    assert _embed(**change) == code


def _embed_back(**kw):
    d = dict(grad=4096, ids=4096, grad_stride=8, T=4, V=5, D=8, ignore_index=-100, dt=0, table_dt=0, scale=1.0, add=0, grad_table=4096, workspace=4096, workspace_bytes=1 << 20)
    return pkg.lib().division_embedding_backward(ctypes.byref(ops._EmbeddingBackDesc(*{**d, **kw}.values())), None)


@pytest.mark.parametrize("change,code", [*[({k: None}, EINVAL) for k in ("grad", "ids", "grad_table", "workspace")], (dict(dt=2), EINVAL), (dict(table_dt=3), EINVAL), (dict(T=-1), EINVAL), (dict(V=0), EINVAL),
                                         (dict(D=0), EINVAL), (dict(grad_stride=-1), EINVAL), (dict(add=2), EINVAL), (dict(grad=2), EALIGN), (dict(ids=4), EALIGN), (dict(grad_table=2), EALIGN),
                                         (dict(workspace=8), EALIGN), (dict(workspace_bytes=47), ESIZE), (dict(grad_stride=1 << 40), ERANGE), (dict(V=1 << 31), ERANGE)])
def test_embedding_backward_refuses(change, code):
    assert _embed_back(**change) == code


def _dropout(x=4096, residual=None, n=10, dt=0, p=0.5, seed=1, at=None, y=4096):
    return pkg.lib().division_dropout_add(x, residual, n, dt, p, seed, at, y, None)


@pytest.mark.parametrize("change,code", [(dict(x=None), EINVAL), (dict(y=None), EINVAL), (dict(n=-1), EINVAL), (dict(dt=2), EINVAL), (dict(p=-0.1), EINVAL), (dict(p=1.1), EINVAL), (dict(p=math.nan), EINVAL),
                                         (dict(x=2), EALIGN), (dict(residual=2), EALIGN), (dict(y=2), EALIGN), (dict(y=1, dt=1), EALIGN), (dict(at=4), EALIGN), (dict(n=(1 << 35) + 1), ERANGE), (dict(n=0, x=None), 0)])
def test_dropout_refuses(change, code):
    assert _dropout(**change) == code


def test_null_descriptors_and_workspaces():
    L = pkg.lib()
    assert L.division_head_norm_rotate(None, None) == EINVAL and L.division_head_norm_rotate_backward(None, None, None) == EINVAL and L.division_embedding_backward(None, None) == EINVAL
    assert L.division_attention_backward(None, None, None) == EINVAL
    assert L.division_head_norm_rotate_backward_workspace(0, 64) == 0 and L.division_head_norm_rotate_backward_workspace(4, 514) == 0 and L.division_head_norm_rotate_backward_workspace(4, 64) > 0
    assert L.division_embedding_backward_workspace(-1, 5, 8) == 0 and L.division_embedding_backward_workspace(0, 5, 8) >= 24 and L.division_embedding_backward_workspace(4, 1 << 31, 8) == 0


def test_tensors_of_the_host_and_wrong_arguments_are_refused():
    x, ids = torch.zeros(2, 3, 4, 16), torch.zeros(3, dtype=torch.int64)
    w, f = torch.ones(16), torch.ones(8, dtype=torch.float64)
    lse = torch.zeros(2, 4, 3)
    for call in (lambda: pkg.division_attention(x, x, x), lambda: pkg.division_attention_backward(x, x, x, x, x, lse), lambda: pkg.division_head_norm_rotate(x, x, w, w, f, ids),
                 lambda: pkg.division_head_norm_rotate(x, x, w, w, f, ids, pairs="other"), lambda: pkg.division_head_norm_rotate(x, x, w, None, f, ids), lambda: pkg.division_head_norm_rotate(x, None, w, w, f, ids),
                 lambda: pkg.division_head_norm_rotate_backward(x, x, x, x, w, w, f, ids, lse, lse), lambda: pkg.division_embedding(ids, x[0, 0]), lambda: pkg.division_embedding_backward(x[0, :, 0], ids, 5),
                 lambda: pkg.division_dropout_add(x, 0.1, 1), lambda: pkg.division_token_attention(x, x, x), lambda: pkg.DivisionResidualDropout(1.5), lambda: pkg.DivisionResidualDropout(math.nan),
                 lambda: pkg.DivisionHeadNormRotation(16, rotated=18), lambda: pkg.DivisionHeadNormRotation(16, rotated=3), lambda: pkg.DivisionHeadNormRotation(16, pairs="both")):
        with pytest.raises(ValueError):
            call()
