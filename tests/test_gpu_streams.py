"""Calls on a stream of their own: what they write is memory of that stream, not what the current stream has given back and may still be using.

Shown by the addresses alone, between waits for the device: a block that the current stream has just given back, of the very size that the call asks for, is what the allocator would hand
out to the current stream."""
import pytest
import torch

import paper_2208_04187_amd as pkg

pytestmark = pytest.mark.gpu


def _tensors(got):
    return [t for t in (got if isinstance(got, (list, tuple)) else [got]) if t is not None]


def _place(t):
    s = t.untyped_storage()
    return s.data_ptr(), s.data_ptr() + max(s.nbytes(), 1)


def _apart(call, inputs=()):
    """call(stream): the same results on a stream of its own and on the current one, in memory that the current stream has not had"""
    want = [t.clone() for t in _tensors(call(None))]
    spare = _tensors(call(None))
    torch.cuda.synchronize()
    own = [_place(t) for t in spare if not any(t is i for i in inputs)]
    del spare
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        got = _tensors(call(stream))
        torch.cuda.synchronize()
        for t in got:
            a, b = _place(t)
            assert any(t is i for i in inputs) or all(b <= p or q <= a for p, q in own)
        assert len(got) == len(want) and all(torch.equal(a.reshape(-1).view(torch.uint8), b.reshape(-1).view(torch.uint8)) for a, b in zip(got, want))
        # given back while the current stream has them in use: not the side stream's next memory
        made = [t for t in got if not any(t is i for i in inputs) and t.numel()]
        places = [_place(t) for t in made]
        torch.cuda._sleep(2 ** 26)
        kept = [t.clone() for t in made]
        sizes = [t.untyped_storage().nbytes() for t in made]
        del got, made, t
        with torch.cuda.stream(side):
            again = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes]
        assert not set(_place(t)[0] for t in again) & set(p for p, _ in places)
        torch.cuda.synchronize()
        del again, kept


def _layer_calls():
    gen = torch.Generator().manual_seed(1)
    q, k = torch.randn(2, 300, 8, 64, generator=gen).cuda(), torch.randn(2, 300, 2, 64, generator=gen).cuda()
    a = pkg.division_attention(q, k, k, causal=True)
    w, f, at = torch.rand(64, generator=gen).cuda(), torch.rand(32, generator=gen).double().cuda(), torch.arange(600, device="cuda").view(2, 300)
    r = pkg.division_head_norm_rotate(q, k, w, w, f, at)
    ids, table = torch.randint(0, 500, (600,), generator=gen).cuda(), torch.randn(500, 1000, generator=gen).cuda()
    rows = torch.randn(600, 1000, generator=gen).cuda()
    held, summed = torch.empty_like(rows), torch.zeros(500, 1000, device="cuda")
    return {"attention": lambda s: pkg.division_attention(q, k, k, causal=True, stream=s), "attention_token": lambda s: pkg.division_attention(q[:, :1], k, k, stream=s),
            "attention_backward": lambda s: pkg.division_attention_backward(q, q, k, k, a.out, a.lse, causal=True, stream=s),
            "rotate": lambda s: pkg.division_head_norm_rotate(q, k, w, w, f, at, stream=s),
            "rotate_backward": lambda s: pkg.division_head_norm_rotate_backward(q, k, q, k, w, w, f, at, r.q_rstd, r.k_rstd, stream=s),
            "embedding": lambda s: pkg.division_embedding(ids, table, stream=s), "embedding_backward": lambda s: pkg.division_embedding_backward(rows, ids, 500, stream=s),
            "embedding_backward_out": lambda s: pkg.division_embedding_backward(rows, ids, 500, out=summed, stream=s), "dropout_add": lambda s: pkg.division_dropout_add(rows, 0.5, 3, stream=s),
            "dropout_add_out": lambda s: pkg.division_dropout_add(rows, 0.5, 3, out=held, stream=s)}, (held, summed)


@pytest.mark.parametrize("name", ["attention", "attention_token", "attention_backward", "rotate", "rotate_backward", "embedding", "embedding_backward", "embedding_backward_out", "dropout_add",
                                  "dropout_add_out"])
def test_layer_operators(name):
    calls, inputs = _layer_calls()
    torch.cuda.synchronize()
    _apart(calls[name], inputs)


def _step_calls():
    gen = torch.Generator().manual_seed(2)
    x, r, w = torch.randn(700, 500, generator=gen).cuda(), torch.randn(700, 500, generator=gen).cuda(), torch.rand(500, generator=gen).cuda()
    n = pkg.division_rms_norm(x, w, residual=r, code="int8")
    logits, ids = torch.randn(64, 20000, generator=gen).cuda(), torch.randint(0, 20000, (64,), generator=gen).cuda()
    f = pkg.division_log_probs(logits, ids)
    grads = [torch.randn(1000, 300, generator=gen).cuda(), torch.randn(77, generator=gen).cuda()]
    held = torch.empty_like(x)
    return {"rms_norm": lambda s: pkg.division_rms_norm(x, w, residual=r, code="e4m3", group=128, stream=s)[:4], "read_codes": lambda s: pkg.division_read_codes(n.codes, n.scales, torch.float32, stream=s),
            "rms_norm_backward": lambda s: pkg.division_rms_norm_backward(r, x, w, n.rstd, stream=s), "rms_norm_backward_out": lambda s: pkg.division_rms_norm_backward(r, x, w, n.rstd, out=held, stream=s),
            "log_probs": lambda s: pkg.division_log_probs(logits, ids, top=5, stream=s), "log_probs_backward": lambda s: pkg.division_log_probs_backward(logits, ids, f.lse, f.lse, stream=s),
            "grad_norm": lambda s: pkg.division_grad_norm(grads, stream=s)}, (held,)


@pytest.mark.parametrize("name", ["rms_norm", "read_codes", "rms_norm_backward", "rms_norm_backward_out", "log_probs", "log_probs_backward", "grad_norm"])
def test_step_operators(name):
    calls, inputs = _step_calls()
    torch.cuda.synchronize()
    _apart(calls[name], inputs)


def _codec_calls():
    gen = torch.Generator().manual_seed(3)
    x = torch.randn(4, 16, 32, 32, generator=gen).cuda()
    deep = torch.randn(2, 8, 4, 16, 16, generator=gen).cuda()
    packed, packed3 = pkg.division_compress(x, 8, 2, 1), pkg.division_compress_3d(deep, 8, 2, 1)
    (_, kept), (_, at) = pkg.division_dropout_forward(x, 0.5, 1), pkg.division_maxpool_forward(x, 2)
    small = torch.randn(4, 16, 16, 16, generator=gen).cuda()
    return {"compress": lambda s: pkg.division_compress(x, 8, 2, 1, stream=s), "decompress": lambda s: pkg.division_decompress(packed, x.shape, 8, 2, stream=s),
            "compress_3d": lambda s: pkg.division_compress_3d(deep, 8, 2, 1, stream=s), "decompress_3d": lambda s: pkg.division_decompress_3d(packed3, deep.shape, 8, 2, stream=s),
            "compress_maps": lambda s: pkg.division_compress_maps([x, small], 8, 2, [1, 2], stream=s), "decompress_maps": lambda s: pkg.division_decompress_maps([packed, packed], [x.shape] * 2, 8, 2, stream=s),
            "compress_batch": lambda s: pkg.division_compress_batch([x, x], 8, 2, [1, 2], stream=s), "decompress_batch": lambda s: pkg.division_decompress_batch([packed, packed], x.shape, 8, 2, stream=s),
            "relu_forward": lambda s: pkg.division_relu_forward(x, stream=s), "relu_compress": lambda s: pkg.division_relu_compress(x, 8, 2, 1, stream=s),
            "dropout_forward": lambda s: pkg.division_dropout_forward(x, 0.5, 1, stream=s), "mask_backward": lambda s: pkg.division_mask_backward(kept, x, stream=s),
            "maxpool_forward": lambda s: pkg.division_maxpool_forward(x, 2, stream=s), "maxpool_backward": lambda s: pkg.division_maxpool_backward(at, small, x.shape, 2, stream=s)}


@pytest.mark.parametrize("name", ["compress", "decompress", "compress_3d", "decompress_3d", "compress_maps", "decompress_maps", "compress_batch", "decompress_batch", "relu_forward", "relu_compress",
                                  "dropout_forward", "mask_backward", "maxpool_forward", "maxpool_backward"])
def test_codec_and_masks(name):
    calls = _codec_calls()
    torch.cuda.synchronize()
    _apart(calls[name])


def test_the_default_stream_by_its_handle_and_the_current_one_by_name():
    calls = {**_layer_calls()[0], **_step_calls()[0], **_codec_calls()}
    torch.cuda.synchronize()
    for name, call in calls.items():
        want = [t.clone() for t in _tensors(call(None))]
        assert torch.cuda.default_stream().cuda_stream == 0
        for stream in (0, torch.cuda.default_stream(), torch.cuda.current_stream()):
            got = _tensors(call(stream))
            torch.cuda.synchronize()
            assert all(torch.equal(a.reshape(-1).view(torch.uint8), b.reshape(-1).view(torch.uint8)) for a, b in zip(got, want)), name


def test_a_fork_within_a_graph():
    """Calls on another stream that a captured one waits for, replayed between eager work"""
    gen = torch.Generator().manual_seed(4)
    q, k = torch.randn(2, 60, 4, 64, generator=gen).cuda(), torch.randn(2, 900, 2, 64, generator=gen).cuda()
    w, x = torch.rand(64, generator=gen).cuda(), torch.randn(300, 64, generator=gen).cuda()

    def step(side=None):
        current = torch.cuda.current_stream()
        if side is not None:
            side.wait_stream(current)
        a = pkg.division_attention(q, k, k, causal=True, stream=side)
        back = pkg.division_attention_backward(q, q, k, k, a.out, a.lse, causal=True, stream=side)
        n = pkg.division_rms_norm(x, w, stream=side)
        b = pkg.division_rms_norm_backward(x, x, w, n.rstd, stream=side)
        d = pkg.division_dropout_add(n.y, 0.5, 3, residual=x, stream=side)
        y = x * 2
        if side is not None:
            current.wait_stream(side)
        return (*a, *back, n.y, *b, d, y)
    main, side = torch.cuda.Stream(), torch.cuda.Stream()
    main.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(main):
        step(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=main):
            outs = step(side)
    for _ in range(3):
        for t in (q, k, x):
            t.mul_(0.9).add_(0.01)
        want = step()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
