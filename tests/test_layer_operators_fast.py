"""The native side of the binding serves plain calls of the layer operators with the results of the general ones and leaves it all others."""
import ctypes

import pytest
import torch

import paper_2208_04187_amd as pkg
from paper_2208_04187_amd import binding


def test_native_side_knows_the_operators_and_leaves_host_tensors_alone():
    fast = binding._load_fast()
    x, ids = torch.zeros(1, 2, 3, 16), torch.zeros(2, dtype=torch.int64)
    assert fast.attention(x, x, x, None, False, 0, None, None) is None and fast.attention_backward(x, x, x, None, False, 0, None, None, x, x, x) is None
    assert fast.head_norm_rotate(x, None, x, None, x, ids, 1e-6, False) is None and fast.head_norm_rotate_backward(x, None, x, None, x, ids, 1e-6, False, x, None, x, None) is None
    assert fast.embedding(ids, x, 1.0, -100) is None and fast.embedding_backward(x, ids, 5, 1.0, -100) is None and fast.dropout_add(x, 0.5, 1, None) is None
    assert fast.attention() is None and fast.dropout_add(None, 0.5, 1, None) is None


@pytest.mark.parametrize("entries,sizes", [(10, None), (12, None), (11, [1, 2, 3, 4, 5]), (11, [])])
def test_native_side_of_other_operators_is_not_used(monkeypatch, entries, sizes):
    fast = binding._load_fast()
    sizes = [ctypes.sizeof(d) for d in binding.LAYER_DESCS] if sizes is None else sizes
    with pytest.raises(ValueError, match="another set"):
        fast.bind_layers([1] * entries, sizes)
    bind = fast.bind_layers
    monkeypatch.setattr(fast, "bind_layers", lambda *args: bind([1] * entries, sizes))
    monkeypatch.setattr(binding, "_fast", None)
    with pytest.warns(RuntimeWarning, match="another set"):
        assert isinstance(binding._load_fast(), binding._NothingFast)
    monkeypatch.undo()
    assert binding._load_fast() is fast


class _General:
    """The binding without its native side"""

    def __enter__(self):
        binding._load_fast()
        self.fast, binding._fast = binding._fast, binding._NothingFast()

    def __exit__(self, *exc):
        binding._fast = self.fast


def _equal(a, b):
    if a is None or b is None:
        return a is b
    if isinstance(a, (list, tuple)):
        return type(a) is type(b) and len(a) == len(b) and all(_equal(p, q) for p, q in zip(a, b))
    return a.shape == b.shape and a.dtype == b.dtype and a.device == b.device and a.stride() == b.stride() and torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_plain_calls_give_what_the_general_ones_give(dtype):
    gen = torch.Generator().manual_seed(3)
    x = torch.randn(2, 9, 8 * 16, generator=gen).to(dtype).cuda()
    q, k, v = (t.unflatten(2, (-1, 16)) for t in x.split([64, 32, 32], 2))
    n = torch.tensor([9, 4], dtype=torch.int32, device="cuda")
    w, par = torch.rand(16, generator=gen).cuda(), torch.nn.Parameter(torch.rand(16, generator=gen).bfloat16().cuda())
    f, at = torch.rand(6, generator=gen).double().cuda(), torch.arange(18, device="cuda").view(2, 9)
    a = pkg.division_attention(q, k, v, causal=True, lengths=n)
    r = pkg.division_head_norm_rotate(q, k, w, par, f, at)
    g = torch.randn(2, 9, 4, 16, generator=gen).to(dtype).cuda()
    table, ids = torch.nn.Parameter(x.detach().view(18, 128)), torch.randint(0, 18, (5, 3), generator=gen).cuda()
    grad = torch.randn(5, 3, 40, generator=gen).to(dtype).cuda()
    native = binding._load_fast()
    plain = [lambda: pkg.division_attention(q, k, v), lambda: pkg.division_attention(q, k, v, 0.5, True, 3, n, n), lambda: pkg.division_attention(q[:1, :1], k[:1], v[:1]),
             lambda: pkg.division_attention_backward(g, q, k, v, a.out, a.lse, causal=True, lengths=n), lambda: pkg.division_head_norm_rotate(q, k, w, par, f, at),
             lambda: pkg.division_head_norm_rotate(q, None, w, None, f, at, 0.5, pairs="next"), lambda: pkg.division_head_norm_rotate(q[1, 2], k[1, 2], par, w, f, at[1, 2].clone()),
             lambda: pkg.division_head_norm_rotate_backward(g, k, q, k, w, par, f, at, r.q_rstd, r.k_rstd), lambda: pkg.division_head_norm_rotate_backward(g, None, q, None, w, None, f, at, r.q_rstd, None, pairs="next"),
             lambda: pkg.division_embedding(ids, table, 0.5), lambda: pkg.division_embedding(ids[0, 0].clone(), table, 1.0, 4), lambda: pkg.division_embedding_backward(grad, ids, 18, 2.0),
             lambda: pkg.division_embedding_backward(grad, ids, 18, 1.0, 7), lambda: pkg.division_dropout_add(g, 0.25, 7), lambda: pkg.division_dropout_add(g, 0.25, -7, residual=g),
             lambda: pkg.division_dropout_add(g, 0.5, 2 ** 64 - 1, residual=g)]
    for i, call in enumerate(plain):
        served = []

        class Watched:
            def __getattr__(self, name):
                def entry(*args):
                    served.append(getattr(native, name)(*args))
                    return served[-1]
                return entry
        binding._fast = Watched()
        try:
            got = call()
        finally:
            binding._fast = native
        assert len(served) == 1 and served[0] is not None, i
        with _General():
            want = call()
        torch.cuda.synchronize()
        assert _equal(got, want), i


@pytest.mark.gpu
def test_other_calls_are_the_general_ones_still():
    q, n = torch.randn(2, 5, 4, 16, device="cuda"), torch.tensor([5, 5], dtype=torch.int32, device="cuda")
    w, f, at, ids = torch.ones(16, device="cuda"), torch.ones(8, dtype=torch.float64, device="cuda"), torch.zeros(2, 5, dtype=torch.int64, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    for call, err in ((lambda: pkg.division_attention(q, q.bfloat16(), q), TypeError), (lambda: pkg.division_attention(q, q[:, :, :3], q[:, :, :3]), ValueError), (lambda: pkg.division_attention(q, q, q, lengths=n[:1]), ValueError),
                      (lambda: pkg.division_attention(q, q, q, window=-1), ValueError), (lambda: pkg.division_attention(q.double(), q.double(), q.double()), TypeError), (lambda: pkg.division_attention(q, q, q, 0.0), pkg.DivisionError),
                      (lambda: pkg.division_head_norm_rotate(q, q, w[:8], w, f, at), ValueError), (lambda: pkg.division_head_norm_rotate(q, q, w, w, f.float(), at), TypeError),
                      (lambda: pkg.division_head_norm_rotate(q, q, w, w, f, at[0]), ValueError), (lambda: pkg.division_head_norm_rotate(q, q, w, w, f, at, -1.0), pkg.DivisionError),
                      (lambda: pkg.division_head_norm_rotate(q, q, w, w, torch.ones(9, dtype=torch.float64, device="cuda"), at), pkg.DivisionError), (lambda: pkg.division_embedding(ids.int(), q[0, 0]), TypeError),
                      (lambda: pkg.division_embedding_backward(q[0, 0], ids, 0), pkg.DivisionError), (lambda: pkg.division_dropout_add(q, 2.0, 1), pkg.DivisionError),
                      (lambda: pkg.division_dropout_add(q, 0.5, 1, residual=q[0]), ValueError)):
        with pytest.raises(err) as native:
            call()
        with _General(), pytest.raises(err) as general:
            call()
        assert type(native.value) is type(general.value) and str(native.value) == str(general.value)
