"""Timed cases of the operators of a token model's training step that are no matrix products: the root-mean-square
norm with the residual's addition and its 8-bit output, the log probabilities of given tokens with their gradient,
and the global norm of all gradients with clipping.

run() is one pass through one operator: the framework's where `own` is true, else its plain form in torch, in 32 bits,
rounded once at the end.  exact() is the definition in 64 bits, on the same inputs.
"""
import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
TOP_CODE = {"int8": 127.0, "e4m3": 448.0}       # the value of the largest code
TINY = 2.0 ** -90                               # a group whose largest value is smaller is held as zeros
EPS = 1e-6                                      # of the norm, and beside the norm of all gradients
IGNORE = -100

# parameters of the networks whose activation maps the benchmark caches (weights and the two vectors of each batch norm)
CIFAR_RESNET18 = ("64x3x3x3*1 64*2 64x64x3x3*4 64*8 128x64x3x3*1 128x128x3x3*3 128x64x1x1*1 128*10 256x128x3x3*1 256x256x3x3*3"
                  " 256x128x1x1*1 256*10 512x256x3x3*1 512x512x3x3*3 512x256x1x1*1 512*10 10x512*1 10*1")
IMAGENET_RESNET50 = ("64x3x7x7*1 64*14 64x64x1x1*1 64x256x1x1*2 64x64x3x3*3 256x64x1x1*4 256*8 128x256x1x1*1 128x512x1x1*3 128x128x3x3*4"
                     " 512x128x1x1*4 512x256x1x1*1 128*16 512*10 256x512x1x1*1 256x1024x1x1*5 256x256x3x3*6 1024x256x1x1*6"
                     " 1024x512x1x1*1 256*24 1024*14 512x1024x1x1*1 512x2048x1x1*2 512x512x3x3*3 2048x512x1x1*3 2048x1024x1x1*1"
                     " 512*12 2048*8 1000x2048*1 1000*1")
TOKEN_MODEL = "32768x1024*1 1024x1024*96 4096x1024*24 1024x4096*24 1024*49"


def listed():
    return [
        # decoding: one token's residual stream, only the 8-bit input of the next product is wanted
        {"name": "norm_one_token", "kind": "norm", "T": 1, "D": 4096, "dtype": "bf16", "residual": True, "code": "int8", "group": 0, "y": False},
        # a training step of a large model: the output goes on in 16 bits and is cached in 8, a scale for 128 columns
        {"name": "norm_tokens_e4m3", "kind": "norm", "T": 16384, "D": 4096, "dtype": "bf16", "residual": True, "code": "e4m3", "group": 128, "y": True},
        # odd sizes in 32 bits, the first norm of a model (no residual yet, nothing cached in 8 bits)
        {"name": "norm_odd_f32", "kind": "norm", "T": 1999, "D": 1155, "dtype": "f32", "residual": False, "code": "", "group": 0, "y": True},
        # the backward pass at T5-base's width, batch 32 of 512 tokens; the residual stream brings a gradient of its own
        {"name": "norm_back_tokens", "kind": "norm_back", "T": 16384, "D": 768, "dtype": "bf16", "residual": True},
        # a wide odd model in 32 bits
        {"name": "norm_back_odd_f32", "kind": "norm_back", "T": 8191, "D": 2561, "dtype": "f32", "residual": False},
        # decoding: the chosen token's log probability, the entropy and twenty alternatives
        {"name": "logp_one_token", "kind": "logp", "T": 1, "V": 131072, "dtype": "bf16", "top": 20, "masked": 0.0, "ignored": 0.0},
        # scoring answers: an odd vocabulary whose last entries are no tokens, five alternatives each
        {"name": "logp_score", "kind": "logp", "T": 2048, "V": 50021, "dtype": "bf16", "top": 5, "masked": 0.05, "ignored": 0.25},
        # the gradient of a training step's loss over a large vocabulary, with an entropy term
        {"name": "logp_back_large", "kind": "logp_back", "T": 4096, "V": 131072, "dtype": "bf16", "masked": 0.0, "ignored": 0.1, "entropy": True},
        # the same in 32 bits over an odd vocabulary, without the entropy term
        {"name": "logp_back_odd_f32", "kind": "logp_back", "T": 513, "V": 32003, "dtype": "f32", "masked": 0.05, "ignored": 0.1, "entropy": False},
        # ResNet-18 on CIFAR: 62 gradients, views of one bucket, within the limit (most steps of a run are)
        {"name": "clip_cifar_resnet18", "kind": "clip", "sizes": CIFAR_RESNET18, "dtype": "f32", "into": "same", "over": 0.5},
        # ResNet-50 in mixed precision: 161 gradients in 16 bits, clipped into the optimizer's 32-bit buffer
        {"name": "clip_resnet50", "kind": "clip", "sizes": IMAGENET_RESNET50, "dtype": "bf16", "into": "f32", "over": 3.0},
        # a token model of 24 layers in mixed precision
        {"name": "clip_token_model", "kind": "clip", "sizes": TOKEN_MODEL, "dtype": "bf16", "into": "f32", "over": 20.0},
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A width: one of a model, or any."""
    return rng.choice([lo * 2 ** k for k in range(1 + int(math.log2(hi / lo)))]) if rng.random() < 0.4 else _spread(rng, lo, hi)


def draw(rng):
    kind = rng.choice(["norm", "norm", "norm_back", "logp", "logp", "logp_back", "clip"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind in ("norm", "norm_back"):
        D = _width(rng, 64, 8192)
        T = _spread(rng, 1, max(1, min(16384, 2 ** 26 // D)))
        if kind == "norm_back":
            return {"kind": kind, "T": T, "D": D, "dtype": dtype, "residual": rng.random() < 0.6}
        code = rng.choice(["", "int8", "e4m3"]) if dtype == "bf16" else ""
        return {"kind": kind, "T": T, "D": D, "dtype": dtype, "residual": rng.random() < 0.7, "code": code,
                "group": rng.choice([0, 32, 64, 128]) if code else 0, "y": not code or rng.random() < 0.7}
    if kind in ("logp", "logp_back"):
        V = _width(rng, 1024, 131072)
        T = _spread(rng, 1, max(1, min(4096, 2 ** (28 if dtype == "bf16" else 27) // V)))
        c = {"kind": kind, "T": T, "V": V, "dtype": dtype, "masked": rng.choice([0.0, 0.05, 0.5, 0.95]), "ignored": rng.choice([0.0, 0.1, 0.25])}
        return {**c, "top": rng.choice([0, 1, 5, 20])} if kind == "logp" else {**c, "entropy": rng.random() < 0.5}
    items = []
    for _ in range(rng.randint(1, 5)):              # groups of tensors, from biases to embeddings
        n = _spread(rng, 1, 2 ** 24)
        items.append("%d*%d" % (n, rng.randint(1, max(1, min(80, 2 ** 26 // n)))))
    return {"kind": "clip", "sizes": " ".join(items), "dtype": dtype, "into": rng.choice(["f32", "f32", "same"]), "over": 0.5}


def _shapes(case):
    got = []
    for item in case["sizes"].split():
        dims, count = item.split("*")
        got += [tuple(int(v) for v in dims.split("x"))] * int(count)
    return got


def _views(flat, shapes):
    return [v.view(s) for v, s in zip(flat.split([math.prod(s) for s in shapes]), shapes)]


def _stream(T, D, gen):
    """The residual stream of a token model: features of different scales."""
    gain = torch.rand(D, generator=gen, device=DEV) * 1.9 + 0.1
    return torch.randn(T, D, generator=gen, device=DEV) * gain


def _logits(case, gen):
    z = torch.randn(case["T"], case["V"], generator=gen, device=DEV).mul_(2.5)
    ids = torch.randint(0, case["V"], (case["T"],), generator=gen, device=DEV)
    kept = max(1, int(case["V"] * (1.0 - case["masked"])))
    ids %= kept
    z.scatter_add_(1, ids.unsqueeze(1), torch.rand(case["T"], 1, generator=gen, device=DEV) * 12.0)
    z[:, kept:] = -math.inf
    ids[torch.rand(case["T"], generator=gen, device=DEV) < case["ignored"]] = IGNORE
    return z.to(DTYPES[case["dtype"]]), ids


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    dt, s = DTYPES[case["dtype"]], {"case": case}
    if case["kind"] in ("norm", "norm_back"):
        T, D = case["T"], case["D"]
        s["weight"] = torch.rand(D, generator=gen, device=DEV) + 0.5
        s["x"] = _stream(T, D, gen).to(dt)
        s["r"] = _stream(T, D, gen).to(dt) if case["residual"] else None
        if case["kind"] == "norm_back":             # x is the stored sum here, r the gradient that the residual stream brings
            s["grad"] = (torch.randn(T, D, generator=gen, device=DEV) * 0.1).to(dt)
            s["rstd"] = torch.rsqrt(s["x"].float().square().mean(1) + EPS)
    elif case["kind"] in ("logp", "logp_back"):
        s["z"], s["ids"] = _logits(case, gen)
        if case["kind"] == "logp_back":             # what the forward pass left, and the gradients of its results
            lse, entropy = [], []
            for z in s["z"].split(256):
                p = torch.log_softmax(z.double(), 1)
                lse.append(torch.logsumexp(z.double(), 1))
                entropy.append(-(p.exp() * p.clamp(min=-1e4)).sum(1))
            s["lse"], s["entropy"] = torch.cat(lse).float(), torch.cat(entropy).float()
            s["g"] = -torch.rand(case["T"], generator=gen, device=DEV) - 0.5
            s["gh"] = -0.01 * torch.ones(case["T"], device=DEV) if case["entropy"] else None
    else:
        shapes = _shapes(case)
        flat = torch.randn(sum(math.prod(v) for v in shapes), generator=gen, device=DEV).mul_(0.02).to(dt)
        norm = flat.float().norm().item()
        s["limit"] = norm / case["over"]
        if case["into"] == "same":
            s["flat"], s["grads"], s["into"] = flat, _views(flat, shapes), None
        else:
            s["grads"] = [v.clone() for v in _views(flat, shapes)]
            s["flat"] = torch.zeros(flat.numel(), device=DEV)
            s["into"] = _views(s["flat"], shapes)
    return s


# ---------------------------------------------------------------- the framework's operators

def _run_own(s):
    import paper_2208_04187_amd as pkg
    case, kind = s["case"], s["case"]["kind"]
    if kind == "norm":
        n = pkg.division_rms_norm(s["x"], s["weight"], EPS, residual=s["r"], code=case["code"] or None, group=case["group"], want_y=case["y"])
        values = pkg.division_read_codes(n.codes, n.scales, s["x"].dtype) if case["code"] else None
        return {"y": n.y, "sum": n.sum if case["residual"] else None, "rstd": n.rstd, "scales": n.scales, "values": values}
    if kind == "norm_back":
        dx, dw = pkg.division_rms_norm_backward(s["grad"], s["x"], s["weight"], s["rstd"], grad_sum=s["r"])
        return {"dx": dx, "dw": dw}
    if kind == "logp":
        p = pkg.division_log_probs(s["z"], s["ids"], top=case["top"], ignore_index=IGNORE)
        return {"logp": p.logp, "entropy": p.entropy, "lse": p.lse, "top": p.top_logp, "top_ids": p.top_ids}
    if kind == "logp_back":
        return pkg.division_log_probs_backward(s["z"], s["ids"], s["lse"], s["g"], entropy=s["entropy"], grad_entropy=s["gh"], ignore_index=IGNORE)
    norm = pkg.division_clip_grads(s["grads"], s["limit"], out=s["into"])
    return {"norm": norm, "grads": s["flat"]}


# ---------------------------------------------------------------- their plain forms

def _codes(y, code, group):
    """y's groups as the values that codes of 8 bits stand for, and the scales"""
    T, D = y.shape
    g = group or D
    n = -(-D // g)
    v = torch.cat([y, y.new_zeros(T, n * g - D)], 1).view(T, n, g) if n * g > D else y.reshape(T, n, g)
    most = v.abs().amax(2)
    dead = most < TINY
    scale = torch.where(dead, 0.0, most / TOP_CODE[code])
    inverse = torch.where(dead, 0.0, TOP_CODE[code] / most).unsqueeze(2)
    q = (v * inverse).round() if code == "int8" else (v * inverse).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).float()
    return (q * scale.unsqueeze(2)).view(T, n * g)[:, :D], scale


def run(s):
    if own:
        return _run_own(s)
    case, kind = s["case"], s["case"]["kind"]
    if kind == "norm":
        x = s["x"].float()
        v = x + s["r"].float() if s["r"] is not None else x
        rstd = torch.rsqrt(v.square().mean(1) + EPS)
        y = v * rstd.unsqueeze(1) * s["weight"]
        values, scales = _codes(y, case["code"], case["group"]) if case["code"] else (None, None)
        dt = s["x"].dtype
        return {"y": y.to(dt) if case["y"] else None, "sum": v.to(dt) if case["residual"] else None, "rstd": rstd, "scales": scales,
                "values": values.to(dt) if case["code"] else None}
    if kind == "norm_back":
        x, dy, rstd = s["x"].float(), s["grad"].float(), s["rstd"].unsqueeze(1)
        unit = x * rstd
        g = dy * s["weight"]
        dx = rstd * (g - unit * (g * unit).mean(1, keepdim=True))
        if s["r"] is not None:
            dx = dx + s["r"].float()
        return {"dx": dx.to(s["x"].dtype), "dw": (dy * unit).sum(0)}
    if kind == "logp":
        z = s["z"].float()
        most = z.amax(1, keepdim=True)
        most = torch.where(most == -math.inf, 0.0, most)
        d = z - most
        e = d.exp()
        total = e.sum(1)
        moment = (e * d.clamp(min=-1e4)).sum(1)
        log_total = total.log()
        lse = most.squeeze(1) + log_total
        empty = total == 0
        entropy = torch.where(empty, 0.0, log_total - moment / total)
        ids = s["ids"].clamp(min=0).unsqueeze(1)
        logp = torch.where(empty, -math.inf, z.gather(1, ids).squeeze(1) - lse)
        logp = torch.where(s["ids"] == IGNORE, 0.0, logp)
        top = top_ids = None
        if case["top"]:                             # by value, equal ones by the lower index: both in one whole number
            bits = (z + 0.0).view(torch.int32).long()
            order = torch.where(bits < 0, -2147483648 - bits, bits)
            at = (order << 32) + (z.shape[1] - 1 - torch.arange(z.shape[1], device=z.device))
            top_ids = z.shape[1] - 1 - (at.topk(case["top"], 1).values & 0xFFFFFFFF)
            top = torch.where(empty.unsqueeze(1), -math.inf, z.gather(1, top_ids) - lse.unsqueeze(1))
        return {"logp": logp, "entropy": entropy, "lse": lse, "top": top, "top_ids": top_ids}
    if kind == "logp_back":
        logp = s["z"].float() - s["lse"].unsqueeze(1)
        p = logp.exp()
        g = torch.where(s["ids"] == IGNORE, 0.0, s["g"]).unsqueeze(1)
        dz = -g * p
        if s["gh"] is not None:
            dz = dz - s["gh"].unsqueeze(1) * p * (logp.clamp(min=-1e4) + s["entropy"].unsqueeze(1))
        return dz.scatter_add_(1, s["ids"].clamp(min=0).unsqueeze(1), g).to(s["z"].dtype)
    norm = torch.stack([g.float().square().sum() for g in s["grads"]]).sum().sqrt()
    c = (s["limit"] / (norm + EPS)).clamp(max=1.0)
    into = s["into"] if s["into"] is not None else s["grads"]
    [o.copy_(g.float() * c) for o, g in zip(into, s["grads"])]
    return {"norm": norm, "grads": s["flat"]}


def work(case):
    e, kind = 2 if case["dtype"] == "bf16" else 4, case["kind"]
    if kind in ("norm", "norm_back"):
        T, D = case["T"], case["D"]
        if kind == "norm_back":                     # the sum, one or two gradients in, one out; the weight and its gradient
            return {"bytes": T * D * e * (4 if case["residual"] else 3) + 4 * T + 8 * D, "flops": 12 * T * D}
        b = T * D * e * (1 + 2 * case["residual"] + case["y"]) + 4 * T + 4 * D
        if case["code"]:                            # codes and scales out, in again, and their values out
            b += T * D * (2 + e) + 8 * T * -(-D // (case["group"] or D))
        return {"bytes": b, "flops": 10 * T * D}
    if kind in ("logp", "logp_back"):
        n = case["T"] * case["V"]
        if kind == "logp":
            return {"bytes": n * e + case["T"] * (20 + 12 * case["top"]), "flops": 6 * n}
        return {"bytes": 2 * n * e + 24 * case["T"], "flops": 8 * n}
    n = sum(math.prod(v) for v in _shapes(case))
    if case["over"] <= 1.0 and case["into"] == "same":
        return {"bytes": n * e, "flops": 2 * n}     # within the limit nothing is changed
    return {"bytes": n * (e + (4 if case["into"] == "f32" else e)), "flops": 3 * n}


# ---------------------------------------------------------------- the definitions in 64 bits

def _nearest_e4m3(v):
    """The nearest number with three bits behind the leading one, steps of 2^-9 at the least, ties to even"""
    _, power = torch.frexp(v)
    step = torch.pow(2.0, (power - 4).clamp(min=-9).double())
    return torch.round(v / step) * step


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind == "norm":
        v = s["x"].double()
        if case["residual"]:
            v = v + s["r"].double()
        rstd = 1.0 / torch.sqrt((v * v).sum(1) / case["D"] + EPS)
        y = torch.einsum("td,t,d->td", v, rstd, s["weight"].double())
        values, scales = None, None
        if case["code"]:
            parts = [(p, p.abs().max(1).values / TOP_CODE[case["code"]]) for p in y.split(case["group"] or case["D"], 1)]
            q = [p / torch.where(a == 0, 1.0, a).unsqueeze(1) for p, a in parts]
            q = [torch.round(p) if case["code"] == "int8" else _nearest_e4m3(p) for p in q]
            values = torch.cat([p * a.unsqueeze(1) for p, (_, a) in zip(q, parts)], 1)
            scales = torch.stack([a for _, a in parts], 1)
        return {"y": y if case["y"] else None, "sum": v if case["residual"] else None, "rstd": rstd, "scales": scales, "values": values}
    if kind == "norm_back":
        x, dy, w, rstd = s["x"].double(), s["grad"].double(), s["weight"].double(), s["rstd"].double()
        along = ((dy * w) * x).sum(1) * rstd ** 3 / case["D"]
        dx = (dy * w) * rstd[:, None] - x * along[:, None]
        return {"dx": dx + s["r"].double() if case["residual"] else dx, "dw": torch.mv((dy * x).t().contiguous(), rstd)}
    if kind == "logp":
        out = {"logp": [], "entropy": [], "lse": [], "top": []}
        for z, ids in zip(s["z"].split(256), s["ids"].split(256)):
            p = torch.log_softmax(z.double(), 1)
            out["lse"].append(torch.logsumexp(z.double(), 1))
            out["entropy"].append(-torch.special.xlogy(p.exp(), p.exp()).sum(1))
            out["logp"].append(torch.where(ids < 0, 0.0, p.gather(1, ids.clamp(min=0)[:, None])[:, 0]))
            out["top"].append(p.sort(1, descending=True).values[:, : case["top"]])
        got = {k: torch.cat(v) for k, v in out.items()}
        return {**got, "top": got["top"] if case["top"] else None, "top_ids": None}
    if kind == "logp_back":
        out = []
        for z, ids, lse, h, g, k in zip(*(s[v].split(256) for v in ("z", "ids", "lse", "entropy", "g")), torch.arange(case["T"], device=DEV).split(256)):
            logp = z.double() - lse.double()[:, None]
            p, g = torch.exp(logp), torch.where(ids < 0, 0.0, g.double())
            one = torch.zeros_like(p).scatter_(1, ids.clamp(min=0)[:, None], 1.0)
            dz = g[:, None] * (one - p)
            if case["entropy"]:
                dz -= s["gh"][k].double()[:, None] * (torch.special.xlogy(p, p) + p * h.double()[:, None])
            out.append(dz)
        return torch.cat(out)
    total = math.fsum(torch.dot(v, v).item() for v in (g.double().view(-1) for g in s["grads"]))
    c = min(1.0, s["limit"] / (math.sqrt(total) + EPS))
    return {"norm": torch.tensor(math.sqrt(total), dtype=torch.float64), "grads": torch.cat([g.double().view(-1) for g in s["grads"]]) * c}
