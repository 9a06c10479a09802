"""A small token model trained under a compressed cache, and then asked for tokens one by one.

    python examples/token_model.py [steps]

Every step runs the package's operators together: norms with the residual's addition whose outputs are cached in 8 bits, Relu with a 1-bit
mask, all other maps compressed by the saved-tensor hook, the log probabilities of the next tokens with a small entropy term, their gradient over the logits'
own memory, and the clipping of all gradients into fp32 buffers that the update reads.  The data are synthetic: a token is followed by one of two
others, so the best loss is ln 2 = 0.69.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2208_04187_amd as dv  # noqa: E402


class Block(torch.nn.Module):
    def __init__(self, width, hidden, code, group, dtype):
        super().__init__()
        self.up = dv.DivisionNormLinear(width, hidden, code=code, group=group, device="cuda", dtype=dtype)
        self.relu = dv.DivisionReLU()
        self.down = torch.nn.Linear(hidden, width, bias=False, device="cuda", dtype=dtype)

    def forward(self, x, residual):
        h, stream = self.up(x, residual)
        return self.down(self.relu(h)), stream


class TokenModel(torch.nn.Module):
    def __init__(self, vocabulary, width=128, hidden=256, layers=3, code="int8", group=0, dtype=torch.bfloat16):
        super().__init__()
        self.embed = torch.nn.Embedding(vocabulary, width, device="cuda", dtype=dtype)
        self.blocks = torch.nn.ModuleList([Block(width, hidden, code, group, dtype) for _ in range(layers)])
        self.norm = dv.DivisionRMSNorm(width, device="cuda", dtype=dtype)
        self.head = torch.nn.Linear(width, vocabulary, bias=False, device="cuda", dtype=dtype)

    def forward(self, tokens):
        x, stream = self.embed(tokens), None
        for block in self.blocks:
            x, stream = block(x, stream)
        return self.head(self.norm(x, stream)[0])


def sample(vocabulary, batch, length, gen):
    """Token t is followed by 3 t + 1 or 5 t + 2"""
    t = torch.randint(0, vocabulary, (batch,), generator=gen, device="cuda")
    got = [t]
    for _ in range(length):
        up = torch.rand(batch, generator=gen, device="cuda") < 0.5
        t = torch.where(up, 3 * t + 1, 5 * t + 2) % vocabulary
        got.append(t)
    return torch.stack(got, 1)


def train(steps=150, vocabulary=97, batch=32, length=64, lr=0.01, max_norm=0.5, seed=0, **model):
    torch.manual_seed(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    net = TokenModel(vocabulary, **model)
    params = list(net.parameters())
    # fp32 weights and gradients of the update; the model's own are what it computes with
    master = [p.detach().float().requires_grad_() for p in params]
    for m in master:
        m.grad = torch.zeros_like(m)
    adam = torch.optim.Adam(master, lr=lr)
    losses, norms, cached = [], [], (0, 0)
    for step in range(steps):
        tokens = sample(vocabulary, batch, length, gen)
        with dv.division_saved_tensors(B=8, b=4, seed=step * 1000) as hook:
            logits = net(tokens[:, :-1])
            f = dv.division_token_log_probs(logits, tokens[:, 1:].contiguous(), overwrite=True)
            loss = -f.logp.mean() - 1e-3 * f.entropy.mean()
        loss.backward()
        norms.append(dv.division_clip_grads([p.grad for p in params], max_norm, out=[m.grad for m in master]))
        adam.step()
        with torch.no_grad():
            for p, m in zip(params, master):
                p.copy_(m)
                p.grad = None
        losses.append(-f.logp.detach().mean())
        cached = (hook.cached_bytes, hook.original_bytes)
    return net, torch.stack(losses), torch.stack(norms), cached


@torch.no_grad()
def follow(net, token, count, top=4):
    """`count` tokens after `token`, one at a time, each the most probable one; with the alternatives of every step"""
    tokens, seen = torch.tensor([[token]], device="cuda"), []
    for _ in range(count):
        logits = net(tokens[:, -1:])[:, -1]
        best = logits.float().argmax(1)
        f = dv.division_log_probs(logits, best, top=top)
        seen.append((f.top_ids[0].tolist(), [round(v, 3) for v in f.top_logp[0].tolist()], round(f.entropy.item(), 3)))
        tokens = torch.cat([tokens, best[:, None]], 1)
    return tokens[0].tolist(), seen


if __name__ == "__main__":
    net, losses, norms, (cached, original) = train(int(sys.argv[1]) if len(sys.argv) > 1 else 150)
    for k in range(0, len(losses), max(1, len(losses) // 10)):
        print(f"step {k:4d}  loss {losses[k].item():.3f}  gradient norm {norms[k].item():.3f}")
    print(f"last loss {losses[-1].item():.3f} (best possible 0.693); maps of a step cached in {cached} bytes instead of {original}")
    tokens, seen = follow(net, 5, 4)
    print("tokens", tokens)
    for ids, logps, entropy in seen:
        print("  alternatives", ids, logps, "entropy", entropy)
