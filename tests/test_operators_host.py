"""The operators of a token model's step refuse what they cannot take, before anything is launched (no GPU needed)."""
import ctypes

import pytest
import torch

import paper_2208_04187_amd as pkg
from paper_2208_04187_amd import operators as ops

EINVAL, ESIZE, EALIGN, ERANGE = 1, 2, 3, 4


def _norm(**kw):
    d = dict(x=4096, residual=None, weight=8192, x_stride=64, residual_stride=64, T=4, D=64, dt=0, weight_dt=0, eps=1e-6, sum=None, y=16384, rstd=None, code=0, group=0,
             codes=None, scales=None)
    return pkg.lib().division_rms_norm(ctypes.byref(ops._NormDesc(*{**d, **kw}.values())), None)


@pytest.mark.parametrize("change,code", [
    (dict(x=None), EINVAL), (dict(weight=None), EINVAL), (dict(dt=2), EINVAL), (dict(dt=7), EINVAL), (dict(weight_dt=2), EINVAL), (dict(eps=-1.0), EINVAL),
    (dict(eps=float("nan")), EINVAL), (dict(D=0), EINVAL), (dict(T=-1), EINVAL), (dict(x_stride=-1), EINVAL), (dict(residual=64), EINVAL), (dict(code=3), EINVAL),
    (dict(code=1, codes=64), EINVAL), (dict(code=1, scales=64), EINVAL), (dict(code=1, codes=64, scales=64, group=16), EINVAL), (dict(x=4098), EALIGN), (dict(y=4097, dt=1), EALIGN),
    (dict(weight=4098), EALIGN), (dict(weight=4097, weight_dt=1), EALIGN), (dict(rstd=4098), EALIGN), (dict(code=1, codes=1, scales=2), EALIGN),
    (dict(T=1 << 31), ERANGE), (dict(D=1 << 31), ERANGE), (dict(T=1 << 20, D=(1 << 20) + 1), ERANGE), (dict(x_stride=1 << 40), ERANGE), (dict(T=0, x=None), 0)])
def test_norm_refuses(change, code):
    assert _norm(**change) == code


def _back(**kw):
    d = dict(grad_y=4096, sum=8192, grad_sum=None, weight=4096, rstd=4096, grad_y_stride=64, sum_stride=64, grad_sum_stride=64, T=4, D=64, dt=0, weight_dt=0, grad_x=4096,
             grad_weight=4096, workspace=4096, workspace_bytes=1 << 30)
    return pkg.lib().division_rms_norm_backward(ctypes.byref(ops._NormBackDesc(*{**d, **kw}.values())), None)


@pytest.mark.parametrize("change,code", [
    *[({k: None}, EINVAL) for k in ("grad_y", "sum", "weight", "rstd", "grad_x", "grad_weight", "workspace")], (dict(dt=2), EINVAL), (dict(weight_dt=5), EINVAL),
    (dict(D=0), EINVAL), (dict(T=-2), EINVAL), (dict(grad_y_stride=-1), EINVAL), (dict(sum_stride=-1), EINVAL), (dict(grad_sum=64, grad_sum_stride=-1), EINVAL),
    (dict(grad_y=2), EALIGN), (dict(sum=2), EALIGN), (dict(grad_sum=2), EALIGN), (dict(grad_x=2), EALIGN), (dict(weight=2), EALIGN), (dict(grad_weight=2), EALIGN),
    (dict(rstd=2), EALIGN), (dict(workspace=2), EALIGN), (dict(workspace_bytes=255), ESIZE), (dict(T=1 << 31), ERANGE), (dict(sum_stride=1 << 40), ERANGE)])
def test_norm_backward_refuses(change, code):
    assert _back(**change) == code


def test_null_descriptors_and_workspaces():
    L = pkg.lib()
    assert L.division_rms_norm(None, None) == EINVAL and L.division_rms_norm_backward(None, None) == EINVAL
    assert L.division_rms_norm_backward_workspace(0, 64) == 0 and L.division_rms_norm_backward_workspace(4, 0) == 0
    assert L.division_rms_norm_backward_workspace(4, 64) >= 64 * 4


def _read(codes=64, scales=64, T=4, D=64, code=1, group=0, dt=0, out=64):
    return pkg.lib().division_read_codes(codes, scales, T, D, code, group, dt, out, None)


@pytest.mark.parametrize("change,code", [(dict(codes=None), EINVAL), (dict(scales=None), EINVAL), (dict(out=None), EINVAL), (dict(code=0), EINVAL), (dict(code=3), EINVAL),
                                         (dict(group=48), EINVAL), (dict(dt=2), EINVAL), (dict(D=0), EINVAL), (dict(T=-1), EINVAL), (dict(scales=2), EALIGN),
                                         (dict(out=2), EALIGN), (dict(out=1, dt=1), EALIGN), (dict(T=1 << 31), ERANGE), (dict(T=0, codes=None), 0)])
def test_read_codes_refuses(change, code):
    assert _read(**change) == code


def test_tensors_of_the_host_and_wrong_arguments_are_refused():
    x, w = torch.zeros(2, 64), torch.ones(64)
    for call in (lambda: pkg.division_rms_norm(x, w), lambda: pkg.division_rms_norm(x, w, code="int4"), lambda: pkg.division_rms_norm(x, w, code="int8", group=48),
                 lambda: pkg.division_read_codes(torch.zeros(2, 64, dtype=torch.int8), torch.zeros(2)),
                 lambda: pkg.division_rms_norm_backward(x, x, w, torch.zeros(2)), lambda: pkg.division_rms_norm(torch.zeros(()), w)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        pkg.division_read_codes(torch.zeros(2, 64), torch.zeros(2))


def _logits(**kw):
    d = dict(logits=4096, ids=4096, stride=64, T=4096, V=64, ignore_index=-100, dt=0, top=0, logp=4096, entropy=None, lse=4096, top_logp=None, top_ids=None, workspace=None,
             workspace_bytes=0)
    return pkg.lib().division_log_probs(ctypes.byref(ops._LogitsDesc(*{**d, **kw}.values())), None)


@pytest.mark.parametrize("change,code", [
    *[({k: None}, EINVAL) for k in ("logits", "ids", "logp", "lse")], (dict(dt=2), EINVAL), (dict(V=0), EINVAL), (dict(T=-1), EINVAL), (dict(stride=-1), EINVAL), (dict(top=-1), EINVAL),
    (dict(top=65, V=100), EINVAL), (dict(top=64, V=63), EINVAL), (dict(top=2, top_logp=4096), EINVAL), (dict(top=2, top_ids=4096), EINVAL), (dict(T=1, V=1 << 20), EINVAL),
    (dict(T=1, V=1 << 20, workspace=4096, workspace_bytes=11), ESIZE), (dict(T=1, V=1 << 20, workspace=4100, workspace_bytes=1 << 20), EALIGN), (dict(logits=2), EALIGN),
    (dict(logits=1, dt=1), EALIGN), (dict(ids=4), EALIGN), (dict(logp=2), EALIGN), (dict(lse=2), EALIGN), (dict(entropy=2), EALIGN), (dict(top=2, top_logp=2, top_ids=8), EALIGN),
    (dict(top=2, top_logp=4, top_ids=4), EALIGN), (dict(T=1 << 31), ERANGE), (dict(V=1 << 31), ERANGE), (dict(stride=1 << 39), ERANGE), (dict(T=0, logits=None), 0)])
def test_log_probs_refuses(change, code):
    assert _logits(**change) == code


def _logits_back(**kw):
    d = dict(logits=4096, ids=4096, lse=4096, entropy=None, grad_logp=4096, grad_entropy=None, stride=64, grad_stride=64, T=4, V=64, ignore_index=-100, dt=0, grad_logits=4096)
    return pkg.lib().division_log_probs_backward(ctypes.byref(ops._LogitsBackDesc(*{**d, **kw}.values())), None)


@pytest.mark.parametrize("change,code", [
    *[({k: None}, EINVAL) for k in ("logits", "ids", "lse", "grad_logp", "grad_logits")], (dict(grad_entropy=64), EINVAL), (dict(dt=2), EINVAL), (dict(V=0), EINVAL),
    (dict(T=-1), EINVAL), (dict(stride=-1), EINVAL), (dict(grad_stride=63), EINVAL), (dict(grad_stride=-1), EINVAL), *[({k: 2}, EALIGN) for k in ("logits", "lse", "grad_logp", "grad_logits")],
    (dict(ids=4), EALIGN), (dict(grad_entropy=2, entropy=4), EALIGN), (dict(grad_entropy=4, entropy=2), EALIGN), (dict(grad_stride=1 << 39), ERANGE), (dict(T=0, logits=None), 0)])
def test_log_probs_backward_refuses(change, code):
    assert _logits_back(**change) == code


def test_log_probs_workspace():
    L = pkg.lib()
    assert L.division_log_probs_workspace(1 << 20, 64, 0) == 0 and L.division_log_probs_workspace(1, 64, 65) == 0 and L.division_log_probs_workspace(1, 0, 0) == 0
    assert 0 < L.division_log_probs_workspace(1, 1 << 17, 0) < L.division_log_probs_workspace(1, 1 << 17, 20)
    with pytest.raises(ValueError):
        pkg.division_log_probs(torch.zeros(2, 64), torch.zeros(2, dtype=torch.int64))
    assert L.division_log_probs(None, None) == EINVAL and L.division_log_probs_backward(None, None) == EINVAL


def _clip(grads=((4096, 4096, 10, 0, 0),), count=None, limit=1.0, clip=1, norm=4096, workspace=4096, workspace_bytes=1 << 30, entry=True):
    d = (ops._GradientDesc * max(1, len(grads)))(*[ops._GradientDesc(*g) for g in grads])
    n = len(grads) if count is None else count
    return pkg.lib().division_clip_grads(n, d if entry else None, limit, clip, norm, workspace, workspace_bytes, None)


@pytest.mark.parametrize("change,code", [
    (dict(count=-1), EINVAL), (dict(entry=False), EINVAL), (dict(norm=None), EINVAL), (dict(workspace=None), EINVAL), (dict(limit=-1.0), EINVAL), (dict(limit=float("nan")), EINVAL),
    (dict(grads=((None, 64, 10, 0, 0),)), EINVAL), (dict(grads=((64, None, 10, 0, 0),)), EINVAL), (dict(grads=((64, 64, -1, 0, 0),)), EINVAL), (dict(grads=((64, 64, 1, 2, 0),)), EINVAL),
    (dict(grads=((64, 64, 1, 0, 2),)), EINVAL), (dict(grads=((64, 64, 1, 0, 0), (66, 64, 1, 0, 0))), EALIGN), (dict(grads=((64, 66, 1, 0, 0),)), EALIGN), (dict(grads=((65, 64, 1, 1, 0),)), EALIGN),
    (dict(grads=((64, 64, (1 << 40) + 1, 0, 0),)), ERANGE), (dict(norm=2), EALIGN), (dict(workspace=8), EALIGN), (dict(workspace_bytes=23), ESIZE)])
def test_clipping_refuses(change, code):
    assert _clip(**change) == code


def test_clipping_into_its_own_memory_keeps_the_type():
    assert _clip(grads=((4096, 4096, 10, 1, 0),)) == EINVAL and _clip(grads=((4096, 4096, 10, 0, 1),)) == EINVAL


def test_gradient_workspace():
    L = pkg.lib()
    d = (ops._GradientDesc * 2)(ops._GradientDesc(64, None, 10, 0, 0), ops._GradientDesc(None, None, 0, 0, 0))
    assert L.division_grad_norm_workspace(2, d) == 24 and L.division_grad_norm_workspace(0, None) == 16 and L.division_grad_norm_workspace(-1, None) == 0
    for call in (lambda: pkg.division_grad_norm([torch.zeros(3)]), lambda: pkg.division_clip_grads([torch.zeros(3)], 1.0), lambda: pkg.division_clip_grads([torch.zeros(3)], -1.0)):
        with pytest.raises(ValueError):
            call()
