"""The operators under autograd and together: gradients against torch's in 64 bits, the example's training run, the saved-tensor hook."""
import math
import os
import sys

import pytest
import torch
import torch.nn.functional as F

import paper_2208_04187_amd as pkg

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24


def _norm64(s, w, eps=1e-6):
    return s * torch.rsqrt((s * s).mean(-1, keepdim=True) + eps) * w


def _close(a, b, rel):
    a, b = a.double().cpu(), b.double().cpu()
    assert a.shape == b.shape and ((a - b).norm() <= rel * b.norm()), ((a - b).norm() / b.norm()).item()


@pytest.mark.parametrize("residual", [False, True])
def test_norm_module_has_torchs_gradients(residual):
    gen = torch.Generator().manual_seed(1)
    x, r, gy, gs = (torch.randn(3, 5, 200, generator=gen) for _ in range(4))
    m = pkg.DivisionRMSNorm(200, device="cuda")
    with torch.no_grad():
        m.weight.copy_(torch.rand(200, generator=gen) + 0.5)
    xc, rc = x.cuda().requires_grad_(), r.cuda().requires_grad_()
    y, s = m(xc, rc if residual else None)
    assert residual or s is xc
    (y * gy.cuda()).sum().add((s * gs.cuda()).sum()).backward()
    xd, rd, wd = x.double().requires_grad_(), r.double().requires_grad_(), m.weight.detach().double().cpu().requires_grad_()
    sd = xd + rd if residual else xd
    (_norm64(sd, wd) * gy.double()).sum().add((sd * gs.double()).sum()).backward()
    # some sixty roundings of a row's sums, seen through the norm of a tensor
    _close(xc.grad, xd.grad, 64 * EPS)
    _close(m.weight.grad, wd.grad, 64 * EPS)
    if residual:
        _close(rc.grad, rd.grad, 64 * EPS)
        xc.grad = rc.grad = None
        m(xc, rc)[1].sum().backward()             # only the stream goes on
        assert torch.equal(xc.grad, torch.ones_like(xc)) and torch.equal(rc.grad, xc.grad)
        xc.grad = None
        m(xc, rc)[0].sum().backward()             # only the norm, with a gradient that is one number broadcast
        _close(xc.grad, torch.autograd.grad(_norm64(xd + rd, wd).sum(), xd)[0], 256 * EPS)


@pytest.mark.parametrize("code,group,half", [("int8", 0, 0.5 / 127), ("e4m3", 64, 2.0 ** -4)])
def test_norm_linear_has_the_gradients_of_its_cached_input(code, group, half):
    gen = torch.Generator().manual_seed(2)
    x, r = torch.randn(4, 6, 192, generator=gen), torch.randn(4, 6, 192, generator=gen)
    m = pkg.DivisionNormLinear(192, 96, bias=True, code=code, group=group, device="cuda")
    xc, rc = x.cuda().requires_grad_(), r.cuda().requires_grad_()
    out, s = m(xc, rc)
    g = torch.randn(4, 6, 96, generator=gen).cuda()
    (out * g).sum().add(s.sum()).backward()
    xd, rd = x.double().requires_grad_(), r.double().requires_grad_()
    w, b, nw = (p.detach().double().cpu().requires_grad_() for p in (m.linear.weight, m.linear.bias, m.norm.weight))
    y = _norm64(xd + rd, nw)
    want = F.linear(y, w, b)
    (want * g.double().cpu()).sum().add((xd + rd).sum()).backward()
    # the layer itself and its input's gradient are fp32's own (products of 192 terms); the weight's gradient comes from codes: the exact formula over their values
    _close(out, want.detach(), 256 * EPS)
    for a, e in ((xc.grad, xd.grad), (rc.grad, rd.grad), (m.norm.weight.grad, nw.grad), (m.linear.bias.grad, b.grad)):
        _close(a, e, 256 * EPS)
    n = pkg.division_rms_norm(xc.detach(), m.norm.weight.detach(), residual=rc.detach(), code=code, group=group)
    values = pkg.division_read_codes(n.codes, n.scales, torch.float32).double().cpu()
    _close(m.linear.weight.grad, g.double().cpu().view(-1, 96).t() @ values.view(-1, 192), 256 * EPS)
    # a value is half a step off at most, of the largest of its group
    assert ((values - y.detach()).abs() <= half * 1.001 * y.detach().abs().amax(-1, keepdim=True)).all()


def test_log_probs_have_torchs_gradients():
    gen = torch.Generator().manual_seed(3)
    z, ids = torch.randn(3, 4, 301, generator=gen) * 2, torch.randint(0, 301, (3, 4), generator=gen)
    ids[1, 2] = -100
    g, gh = torch.randn(3, 4, generator=gen), torch.randn(3, 4, generator=gen)
    zd = z.double().requires_grad_()
    p = torch.log_softmax(zd, -1)
    logp = p.gather(-1, ids.clamp(min=0)[..., None])[..., 0] * (ids != -100)
    H = -(p.exp() * p).sum(-1)
    for use in ((g, None), (None, gh), (g, gh)):
        want = torch.autograd.grad(sum((v * t.double()).sum() for v, t in zip((logp, H), use) if t is not None), zd, retain_graph=True)[0]
        for overwrite in (False, True):
            leaf = z.cuda().requires_grad_()
            zc = leaf * 1.0
            f = pkg.division_token_log_probs(zc, ids.cuda(), top=5, overwrite=overwrite)
            assert not f.top_logp.requires_grad and not f.lse.requires_grad and f.top_ids.shape == (3, 4, 5)
            sum((v * t.cuda()).sum() for v, t in zip((f.logp, f.entropy), use) if t is not None).backward()
            # two roundings of an exponent of at most twenty, and those of a sum
            _close(leaf.grad, want, 64 * EPS)
            assert torch.equal(zc.detach(), leaf.detach()) != overwrite
    zc = leaf.detach().clone().requires_grad_() * 1.0
    f = pkg.division_token_log_probs(zc, ids.cuda(), overwrite=True)
    f.logp.sum().backward(retain_graph=True)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        f.logp.sum().backward()
    # broadcast gradients, and logits that are a slice
    wide = torch.randn(3, 4, 400, generator=gen).cuda().requires_grad_()
    pkg.division_token_log_probs(wide[..., 3:304], ids.cuda()).logp.mean().backward()
    assert not wide.grad[..., :3].any() and not wide.grad[..., 304:].any() and torch.isfinite(wide.grad).all() and wide.grad.any()


def test_saved_tensor_hook_compresses_the_stream_and_keeps_the_logits():
    gen = torch.Generator().manual_seed(4)
    x, r = (torch.randn(8, 64, 256, generator=gen).cuda() for _ in range(2))
    m = pkg.DivisionRMSNorm(256, device="cuda")
    head = torch.nn.Linear(256, 512, bias=False, device="cuda")
    ids = torch.randint(0, 512, (8, 64), generator=gen).cuda()
    grads = []
    for hook in (False, True):
        xc, rc = x.clone().requires_grad_() * 1.0, r.clone().requires_grad_()
        xc.retain_grad()
        with (pkg.division_saved_tensors(B=8, b=8, seed=1) if hook else torch.autograd.graph.saved_tensors_hooks(lambda t: t, lambda t: t)) as cache:
            y, s = m(xc, rc)
            z = head(y)
            z.retain_grad()
            logp = pkg.division_token_log_probs(z, ids).logp
        logp.sum().backward()
        grads.append((xc.grad, z.grad))
        if hook:
            assert cache.cached_maps >= 1 and cache.cached_bytes < cache.original_bytes
    assert torch.equal(grads[0][1], grads[1][1])                # the logits are kept as they are
    # 8-bit codes of the stream: half a percent of its range
    _close(grads[1][0], grads[0][0], 0.02)
    assert not torch.equal(grads[0][0], grads[1][0])


def test_example_trains_and_follows_its_tokens():
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import token_model
    for code, group in (("int8", 0), ("e4m3", 64)):
        net, losses, norms, (cached, original) = token_model.train(steps=120, code=code, group=group)
        assert torch.isfinite(losses).all() and torch.isfinite(norms).all() and (norms > 0).all()
        assert losses[0] > 4.0 and losses[-10:].mean() < 0.9 and 0 < cached < original / 2
        tokens, seen = token_model.follow(net, 5, 4)
        for a, b, (top_ids, top_logp, entropy) in zip(tokens, tokens[1:], seen):
            assert b in ((3 * a + 1) % 97, (5 * a + 2) % 97) and set(top_ids[:2]) == {(3 * a + 1) % 97, (5 * a + 2) % 97}
            assert abs(top_logp[0] + math.log(2)) < 0.5 and top_ids[0] == b and 0.3 < entropy < 1.5
