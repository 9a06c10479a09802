"""The operators of a token model's layers under autograd and together: gradients against torch's in 64 bits, the saved-tensor hook, graphs, the example."""
import math
import os
import sys

import pytest
import torch
import torch.nn.functional as F

import paper_2208_04187_amd as pkg

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24


def _close(a, b, rel):
    a, b = a.double().cpu(), b.double().cpu()
    assert a.shape == b.shape and ((a - b).norm() <= rel * b.norm()), ((a - b).norm() / b.norm()).item()


class Layer(torch.nn.Module):
    """Embedding, attention with normed and turned heads, dropout, addition: every operator once"""

    def __init__(self, vocabulary, width, heads, key_heads, pairs="halves", dtype=None, p=0.25):
        super().__init__()
        self.f, self.heads, self.key_heads = width // heads, heads, key_heads
        self.embed = pkg.DivisionEmbedding(vocabulary, width, scale=2.0, ignore_index=1, device="cuda", dtype=dtype)
        self.project = torch.nn.Linear(width, (heads + 2 * key_heads) * self.f, bias=False, device="cuda", dtype=dtype)
        self.rotate = pkg.DivisionHeadNormRotation(self.f, rotated=self.f // 2, pairs=pairs, device="cuda", dtype=dtype)
        self.out = torch.nn.Linear(width, width, bias=False, device="cuda", dtype=dtype)
        self.drop = pkg.DivisionResidualDropout(p, seed=5)

    def forward(self, ids, positions, lengths=None, window=0):
        x = self.embed(ids)
        q, k, v = (t.unflatten(2, (-1, self.f)) for t in self.project(x).split([self.heads * self.f, self.key_heads * self.f, self.key_heads * self.f], 2))
        q, k = self.rotate(q, k, positions)
        a = pkg.division_token_attention(q, k, v, causal=True, lengths=lengths, window=window)
        return self.drop(self.out(a.flatten(2)), x)


def _reference(m, ids, positions, lengths, window, kept):
    """The same in 64 bits, from the definitions"""
    w = {n: t.detach().double().cpu().requires_grad_() for n, t in m.named_parameters()}
    B, S = ids.shape
    x = torch.where((ids == 1)[..., None], 0.0, w["embed.weight"][ids] * 2.0)
    q, k, v = (t.unflatten(2, (-1, m.f)) for t in (x @ w["project.weight"].t()).split([m.heads * m.f, m.key_heads * m.f, m.key_heads * m.f], 2))
    R = m.f // 2
    angle = positions.double()[..., None, None] * torch.tensor([10000.0 ** (-p / R) for p in range(0, R, 2)], dtype=torch.float64)

    def rotate(t, weight):
        t = t * torch.rsqrt((t * t).mean(-1, keepdim=True) + 1e-6) * weight
        a, b = (t[..., 0:R:2], t[..., 1:R:2]) if m.rotate.pairs == "next" else (t[..., :R // 2], t[..., R // 2:R])
        one, two = a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()
        return torch.cat([torch.stack([one, two], -1).flatten(-2) if m.rotate.pairs == "next" else torch.cat([one, two], -1), t[..., R:]], -1)
    q, k = rotate(q, w["rotate.q_weight"]), rotate(k, w["rotate.k_weight"])
    k, v = (t.repeat_interleave(m.heads // m.key_heads, 2) for t in (k, v))
    z = torch.einsum("bihd,bjhd->bhij", q, k) / math.sqrt(m.f)
    far = torch.arange(S)[:, None] - torch.arange(S)
    hidden = ((far < 0) | ((far >= window) if window else torch.zeros_like(far, dtype=torch.bool)))[None, None] | (torch.arange(S) >= lengths[:, None, None, None])
    p = torch.softmax(z.masked_fill(hidden, -math.inf), 3).masked_fill(hidden.all(3, keepdim=True), 0.0)
    a = torch.einsum("bhij,bjhd->bihd", p, v).flatten(2) @ w["out.weight"].t()
    return x + torch.where(kept.view(a.shape), a / (1.0 - m.drop.p), 0.0), w


def _inputs(B, S, vocabulary, width, seed):
    gen = torch.Generator().manual_seed(seed)
    ids = (torch.rand(B, S, generator=gen) ** 3 * vocabulary).long()
    ids[:, 3] = 1
    return ids, torch.arange(S).repeat(B, 1) + torch.randint(0, 100, (B, 1), generator=gen), torch.randn(B, S, width, generator=gen)


@pytest.mark.parametrize("pairs", ["halves", "next"])
@pytest.mark.parametrize("hook", [False, True])
@pytest.mark.parametrize("window", [0, 9])
def test_a_layer_has_torchs_gradients(pairs, hook, window):
    torch.manual_seed(1)
    m = Layer(50, 96, 6, 2, pairs)
    ids, positions, g = _inputs(3, 37, 50, 96, 2)
    lengths = torch.tensor([37, 20, 35])
    kept = pkg.division_dropout_forward(torch.ones(g.numel(), device="cuda"), 0.25, 6)[0].cpu() != 0        # the module's first call
    args = (ids.cuda(), positions.cuda(), lengths.int().cuda(), window)
    if hook:
        # tensors of three dimensions are compressed here, others' operators' too: with 8 bits a map's error is far from a missing or wrong one's
        with pkg.division_saved_tensors(B=8, b=8, seed=1, min_elements=1 << 30):
            out = m(*args)
    else:
        out = m(*args)
    out.backward(g.cuda())
    want, w = _reference(m, ids, positions, lengths, window, kept)
    want.backward(g.double())
    # six layers of sums of up to some hundred products each; the norm of a tensor sees their roundings' mean, not their sum
    _close(out, want.detach(), 512 * EPS)
    for name, t in m.named_parameters():
        _close(t.grad, w[name].grad, 512 * EPS)


def test_attention_caches_exact_tensors_under_the_hook_and_shares_a_projections_output():
    gen = torch.Generator().manual_seed(3)
    x = torch.randn(2, 64, 4 * 32 + 2 * 2 * 32, generator=gen).cuda()

    def run():
        t = x.clone().requires_grad_()
        q, k, v = (p.unflatten(2, (-1, 32)) for p in t.split([128, 64, 64], 2))
        out = pkg.division_token_attention(q, k, v, causal=True)
        return t, out
    t, out = run()
    out.sum().backward()
    with pkg.division_saved_tensors(B=8, b=1, seed=0, min_elements=1) as hook:
        u, again = run()
    assert hook.cached_maps == 0
    again.sum().backward()
    assert torch.equal(again, out) and torch.equal(u.grad, t.grad)
    q = torch.randn(2, 64, 4, 32, generator=gen).cuda().requires_grad_()            # tensors of their own
    k = torch.randn(2, 64, 2, 32, generator=gen).cuda().requires_grad_()
    with pkg.division_saved_tensors(B=8, b=1, seed=0, min_elements=1) as hook:
        again = pkg.division_token_attention(q * 1.0, k * 1.0, k * 1.0)
    held = hook.cached_maps
    again.sum().backward()
    want = torch.autograd.grad(pkg.division_token_attention(q * 1.0, k * 1.0, k * 1.0).sum(), (q, k))
    assert held == 0 and torch.equal(q.grad, want[0]) and torch.equal(k.grad, want[1])


def test_the_rotations_statistic_stays_exact_under_the_hook():
    gen = torch.Generator().manual_seed(4)
    m = pkg.DivisionHeadNormRotation(32, device="cuda")
    at = torch.arange(64, device="cuda").repeat(2, 1)
    seen = []
    q, k = (torch.randn(2, 64, n, 32, generator=gen).cuda().requires_grad_() for n in (4, 2))
    with torch.autograd.graph.saved_tensors_hooks(lambda t: (seen.append(t.dim()), t)[1], lambda t: t):
        a, b = m(q * 1.0, k * 1.0, at)
    assert sorted(seen).count(3) == 2                                              # the maps, as tokens x features; the rest vectors and matrices
    with pkg.division_saved_tensors(B=8, b=8, seed=0, min_elements=1) as hook:
        a, b = m(q * 1.0, k * 1.0, at)
    assert hook.cached_maps == 2
    (a.sum() + (b * b).sum()).backward()
    want = torch.autograd.grad([s.sum() if n == 0 else (s * s).sum() for n, s in enumerate(m(q, k, at))], (q, k))
    # maps of 8 bits: a step is a 255th of a plane's range, some 7 of a standard deviation; seen by the norm half a percent of the gradient or so
    _close(q.grad, want[0], 0.05)
    # the squares of a normed row add up to a constant, so that this gradient is the difference of two equal terms, rstd * 2 b each but for the turn, which keeps their norm: the maps' error is of these
    rstd = torch.rsqrt((k.detach() ** 2).mean(-1, keepdim=True) + 1e-6)
    assert (k.grad - want[1]).norm() <= 0.05 * (2 * b.detach() * rstd).norm()


def test_partial_uses():
    m = pkg.DivisionHeadNormRotation(16, device="cuda")
    q, k, at = torch.randn(5, 3, 16, device="cuda", requires_grad=True), torch.randn(5, 1, 16, device="cuda", requires_grad=True), torch.arange(5, device="cuda")
    a, b = m(q, k, at)
    (2 * a.sum()).backward()
    assert k.grad is None and m.k_weight.grad is None and q.grad is not None
    a, b = m(q, k, at)
    both = torch.autograd.grad(2 * a.sum() + 0 * b.sum(), (q, m.q_weight))
    _close(q.grad, both[0], 4 * EPS)
    q.grad = m.q_weight.grad = None
    m(q, k, at)[1].sum().backward()
    assert q.grad is None and m.q_weight.grad is None and k.grad is not None and m.k_weight.grad is not None
    assert m.to(torch.bfloat16).frequencies(q.device).dtype == torch.float64
    with pytest.raises(ValueError):
        pkg.DivisionHeadNormRotation(15)
    x = torch.randn(4, 6, device="cuda", requires_grad=True)
    d = pkg.DivisionResidualDropout(0.5, seed=3)
    kept = pkg.division_dropout_forward(torch.ones(24, device="cuda"), 0.5, 4)[0].view(4, 6)
    y = d(x)
    y.sum().backward()
    assert torch.equal(x.grad, kept * 2) and torch.equal(y, (x * 2 * kept).detach())
    assert not torch.equal(d(x) != 0, y != 0) and d.calls == 2
    d.eval()
    assert d(x) is x and torch.equal(d(x, x), x + x) and d.calls == 2
    e = pkg.DivisionEmbedding(7, 4, device="cuda")
    e(torch.tensor([[1, 2], [2, -100]], device="cuda")).sum().backward()
    assert torch.equal(e.weight.grad[:, 0].cpu(), torch.tensor([0.0, 1, 2, 0, 0, 0, 0]))


def test_rows_that_attention_does_not_take_as_they_lie_are_copied():
    gen = torch.Generator().manual_seed(5)
    x = torch.randn(2, 9, 4 * 8 + 1, generator=gen).bfloat16().cuda().requires_grad_()
    q = x[..., 1:].unflatten(2, (4, 8))                                            # rows start at any element
    out = pkg.division_token_attention(q, q, q, causal=True)
    got = torch.autograd.grad((out * out).sum(), x)[0]
    y = x.detach()[..., 1:].contiguous().requires_grad_()
    p = y.unflatten(2, (4, 8))
    out = pkg.division_token_attention(p, p, p, causal=True)
    assert torch.equal(got[..., 1:], torch.autograd.grad((out * out).sum(), y)[0]) and not got[..., 0].any()


def test_rows_farther_apart_than_attention_takes_are_copied():
    """Tokens 9 MB apart, as in a batch of thousands whose first dimension is the tokens; heads 300 MB apart"""
    gen = torch.Generator().manual_seed(6)
    x = torch.randn(2, 5, 4, 16, generator=gen).bfloat16().cuda()
    dense = [x.clone().requires_grad_() for _ in range(2)]
    want = torch.autograd.grad(pkg.division_token_attention(dense[0], dense[1], dense[1], causal=True).float().square().sum(), dense)
    for tokens, heads in ((9 << 19, 16), (16, 150 << 20)):
        far = [torch.empty(2 * 80 + 5 * tokens + 4 * heads, dtype=torch.bfloat16, device="cuda").as_strided(x.shape, (80, tokens, heads, 1)).copy_(x).requires_grad_() for _ in range(2)]
        out = pkg.division_token_attention(far[0], far[1], far[1], causal=True)
        assert all(torch.equal(g, w) for g, w in zip(torch.autograd.grad(out.float().square().sum(), far), want))
        del far, out


def test_second_derivatives_raise():
    x = torch.randn(1, 4, 2, 16, device="cuda", requires_grad=True)
    e = pkg.DivisionEmbedding(7, 4, device="cuda")
    m = pkg.DivisionHeadNormRotation(16, device="cuda")
    d = pkg.DivisionResidualDropout(0.5)
    for out, of in ((pkg.division_token_attention(x, x, x), x), (m(x, x, torch.zeros(1, 4, dtype=torch.int64, device="cuda"))[0], x), (e(torch.tensor([1, 2], device="cuda")), e.weight), (d(x), x)):
        (g,) = torch.autograd.grad(out.sum(), of, create_graph=True)
        with pytest.raises(RuntimeError, match="first derivatives only"):
            g.sum().backward()


def test_a_layers_step_in_a_graph():
    """Forward and backward captured together, replayed with other tokens between eager work on tensors of their own"""
    torch.manual_seed(6)
    m = Layer(40, 64, 4, 2, p=0.0)
    ids, positions, g = _inputs(2, 24, 40, 64, 7)
    ids, positions, g = ids.cuda(), positions.cuda(), g.cuda()
    lengths = torch.tensor([24, 15], dtype=torch.int32, device="cuda")
    params = list(m.parameters())

    def step():
        out = m(ids, positions, lengths)
        return (out, *torch.autograd.grad(out, params, g))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            outs = step()
    torch.cuda.current_stream().wait_stream(side)
    for n in range(3):
        ids.add_(1).remainder_(40)
        lengths.sub_(2)
        g.mul_(0.9)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.detach().clone() for t in outs]
        want = step()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            _close(a, b.detach(), 1e-6)             # the projections are a library's, which may take another order


def test_example_model_with_attention():
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import token_model
    net, losses, norms, (cached, original) = token_model.train(steps=6, heads=4, width=64, hidden=128, layers=2)
    assert losses.isfinite().all() and norms.isfinite().all() and 0 < cached < original
    tokens, seen = token_model.follow(net, 5, 9)
    assert len(tokens) == 10 and len(seen) == 9 and net.training
    # token by token with a cache, and all at once without one: products of other shapes round otherwise, and bfloat16's steps are 2^-8
    net.eval()
    with torch.no_grad():
        whole = net(torch.tensor([tokens[:-1]], device="cuda"))[0].float()
        cache, one = net.cache(1, 9), []
        for k in range(9):
            one.append(net(torch.tensor([[tokens[k]]], device="cuda"), cache, k)[0, 0].float())
    _close(torch.stack(one), whole, 2.0 ** -5)


def test_example_models_gradients():
    """The example's model in fp32 against itself with torch's own operators in the place of attention, rotation and embedding"""
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import token_model
    torch.manual_seed(8)
    net = token_model.TokenModel(31, width=64, hidden=96, layers=2, dtype=torch.float32, heads=4, dropout=0.0)
    tokens = torch.randint(0, 31, (3, 21), device="cuda")

    def loss():
        return -pkg.division_token_log_probs(net(tokens[:, :-1]), tokens[:, 1:].contiguous()).logp.mean()
    got = torch.autograd.grad(loss(), list(net.parameters()))

    def plain(a, x, residual, positions, cache=None):
        h, stream = a.project(x, residual)
        q, k, v = (p.unflatten(2, (-1, a.features)) for p in h.split(a.parts, 2))
        angle = positions.double()[..., None, None] * a.rotate.frequencies(x.device)
        cos, sin = angle.cos().float(), angle.sin().float()

        def rotate(t, w):
            t = t * torch.rsqrt((t * t).mean(-1, keepdim=True) + 1e-6) * w
            one, two = t.chunk(2, -1)
            return torch.cat([one * cos - two * sin, one * sin + two * cos], -1)
        q, k = rotate(q, a.rotate.q_weight), rotate(k, a.rotate.k_weight)
        k, v = (t.repeat_interleave(a.heads // a.key_heads, 2) for t in (k, v))
        z = torch.einsum("bihd,bjhd->bhij", q, k) / math.sqrt(a.features)
        z = z.masked_fill(torch.ones(z.shape[2:], dtype=torch.bool, device=z.device).triu(1), -math.inf)
        return a.out(torch.einsum("bhij,bjhd->bihd", torch.softmax(z, 3), v).flatten(2)), stream
    for a in net.attention:
        a.forward = lambda *args, a=a: plain(a, *args)
    net.embed.forward = lambda ids: F.embedding(ids, net.embed.weight)
    want = torch.autograd.grad(loss(), list(net.parameters()))
    # the layers' inputs are cached in 8 bits on both sides, where a rounding apart in front of them may be a code apart behind: a 127th of an element now and then
    for p, a, b in zip(net.parameters(), got, want):
        _close(a, b, 0.01)
