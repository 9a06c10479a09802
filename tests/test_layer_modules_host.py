"""The layer operators' modules with stand-ins for the kernels: what they do around them (no GPU needed)."""
import pytest
import torch
from torch.utils.checkpoint import checkpoint

import paper_2208_04187_amd as pkg
from paper_2208_04187_amd import autograd, layer_modules


def _drop(x, p, seed, residual=None):
    kept = torch.rand(x.shape, generator=torch.Generator().manual_seed(seed % 2 ** 63)) >= p
    y = torch.where(kept, x / (1 - p), 0.0)
    return y if residual is None else y + residual


@pytest.fixture
def stand_in(monkeypatch):
    monkeypatch.setattr(layer_modules, "division_dropout_add", _drop)


def _model(seed):
    torch.manual_seed(1)
    return torch.nn.Linear(16, 16), pkg.DivisionResidualDropout(0.5, seed=seed), torch.nn.Linear(16, 16)


def _step(parts, x, wrap):
    """One step behind one seed of torch's: the loss, and all gradients"""
    first, drop, last = parts
    x = x.clone().requires_grad_()
    torch.manual_seed(2)
    y = wrap(lambda t: last(drop(first(t), t)).tanh(), x)
    loss = (y * y).sum()
    return loss, torch.autograd.grad(loss, [x, *first.parameters(), *last.parameters()])


@pytest.mark.parametrize("reentrant", [False, True])
def test_a_checkpointed_forward_drops_the_same_again(stand_in, reentrant):
    x = torch.randn(8, 16, generator=torch.Generator().manual_seed(3))
    want = _step(_model(None), x, lambda f, t: f(t))

    def step():
        parts = _model(None)
        leaf = x.clone().requires_grad_()
        torch.manual_seed(2)
        y = checkpoint(lambda t: parts[2](parts[1](parts[0](t), t)).tanh(), leaf, use_reentrant=reentrant)
        loss = (y * y).sum()
        loss.backward()
        return loss, (leaf.grad, *(p.grad for m in (parts[0], parts[2]) for p in m.parameters()))
    got = step()
    assert torch.equal(got[0], want[0]) and all(torch.equal(a, b) for a, b in zip(got[1], want[1]))


@pytest.mark.parametrize("reentrant", [False, True])
def test_a_numbered_call_is_not_made_again_in_the_backward_pass(stand_in, reentrant):
    """Its number would be another, and its mask not the one that made the loss"""
    first, drop, last = _model(5)
    x = torch.randn(8, 16, generator=torch.Generator().manual_seed(3)).requires_grad_()
    y = checkpoint(lambda t: last(drop(first(t), t)).tanh(), x, use_reentrant=reentrant)
    with pytest.raises(RuntimeError, match="seed=None"):
        y.sum().backward()
    assert drop.calls == 1


def test_calls_have_their_numbers_and_drawn_seeds_are_torchs(stand_in):
    x, r = torch.ones(64), torch.zeros(64)
    drop = pkg.DivisionResidualDropout(0.5, seed=7)
    assert torch.equal(drop(x, r), _drop(x, 0.5, 8, r)) and torch.equal(drop(x), _drop(x, 0.5, 9)) and drop.calls == 2
    drop = pkg.DivisionResidualDropout(0.5, seed=None)
    torch.manual_seed(4)
    a, b = drop(x), drop(x)
    torch.manual_seed(4)
    assert torch.equal(drop(x), a) and torch.equal(drop(x), b) and not torch.equal(a, b)
    state = torch.get_rng_state()
    drop.eval()
    assert drop(x) is x and torch.equal(torch.get_rng_state(), state)


@pytest.fixture
def mask_stand_in(monkeypatch):
    monkeypatch.setattr(autograd, "division_dropout_forward", lambda x, p, seed: (_drop(x, p, seed) * (1 - p), _drop(torch.ones_like(x), p, seed) != 0))
    monkeypatch.setattr(autograd, "division_mask_backward", lambda mask, grad: torch.where(mask, grad, 0.0))


@pytest.mark.parametrize("reentrant", [False, True])
def test_dropout_with_a_stored_mask_under_checkpointing(mask_stand_in, reentrant):
    x = torch.randn(8, 16, generator=torch.Generator().manual_seed(3))
    grads = []
    for run in (lambda f, t: f(t), lambda f, t: checkpoint(f, t, use_reentrant=reentrant)):
        torch.manual_seed(1)
        net = torch.nn.Sequential(torch.nn.Linear(16, 16), pkg.DivisionDropout(0.5, seed=None), torch.nn.Linear(16, 16), torch.nn.Tanh())
        leaf = x.clone().requires_grad_()
        torch.manual_seed(2)
        (run(net, leaf) ** 2).sum().backward()
        grads.append([leaf.grad, *(p.grad for p in net.parameters())])
    assert all(torch.equal(a, b) for a, b in zip(*grads))
    drop = pkg.DivisionDropout(0.5, seed=5)
    leaf = x.clone().requires_grad_()
    y = checkpoint(lambda t: drop(t.sin()).exp(), leaf, use_reentrant=reentrant)
    with pytest.raises(RuntimeError, match="seed=None"):
        y.sum().backward()
    assert drop.calls == 1
    drop = pkg.DivisionDropout(0.5, seed=5)
    for n in (6, 7):
        assert torch.equal(drop(x), autograd.division_dropout_forward(x, 0.5, n)[0])


class _Save(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, f):
        ctx.save_for_backward(f)
        return x * 1.0

    @staticmethod
    def backward(ctx, g):
        return g * ctx.saved_tensors[0].sum(), None


def test_a_rotation_that_began_in_inference_mode_trains():
    m = pkg.DivisionHeadNormRotation(16, rotated=8)
    cpu = torch.device("cpu")
    with torch.inference_mode():
        first = m.frequencies(cpu)
    assert not first.is_inference() and m.frequencies(cpu) is first
    assert torch.equal(first, torch.tensor([10000.0 ** (-p / 8) for p in (0, 2, 4, 6)], dtype=torch.float64))
    x = torch.ones(3, dtype=torch.float64, requires_grad=True)
    _Save.apply(x, first).sum().backward()
    assert torch.equal(x.grad, first.sum().expand(3))


class _Attended:
    def __init__(self, q):
        self.out, self.lse = torch.zeros(q.shape, dtype=q.dtype), torch.zeros(q.shape[0], q.shape[2], q.shape[1])


def test_attention_under_autograd_copies_dense_rows_that_start_off_16_bytes(monkeypatch):
    """A dense tensor is its own contiguous()"""
    seen = []

    def attend(q, k, v, *rest):
        seen.extend((q, k, v))
        return _Attended(q)

    def backward(grad_out, q, k, v, *rest):
        seen.extend((grad_out, q, k, v))
        return torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    monkeypatch.setattr(layer_modules, "division_attention", attend)
    monkeypatch.setattr(layer_modules, "division_attention_backward", backward)
    for dtype in (torch.float32, torch.bfloat16):
        room = torch.randn(8 + 2 * 5 * 4 * 16).to(dtype)
        for off in range(1, 16 // room.element_size()):
            x = room[off: off + 2 * 5 * 4 * 16].view(2, 5, 4, 16).requires_grad_()
            assert x.is_contiguous() and x.data_ptr() % 16
            seen.clear()
            out = pkg.division_token_attention(x, x, x)
            out.backward(x.detach())
            assert len(seen) == 7 and all(t.data_ptr() % 16 == 0 and torch.equal(t, x) for t in seen)


def test_attention_under_autograd_refuses_other_than_four_dimensions():
    for shape in ((4,), (3, 16), (2, 3, 16), (1, 2, 3, 4, 16)):
        x = torch.zeros(shape, requires_grad=True)
        with pytest.raises(ValueError, match="batch, tokens, heads, features"):
            pkg.division_token_attention(x, x, x)
