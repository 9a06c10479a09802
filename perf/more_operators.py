"""Timed cases of the operators of a token model's layers beside its products and norms: attention and its backward pass,
the norms of queries and keys with the position rotation, the embedding lookup and its gradient, and dropout without a
stored mask.

run() is one pass through one operator: the framework's where `own` is true, else its plain form in torch, in 32 bits,
rounded once at the end.  exact() is the definition in 64 bits, on the same inputs.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6                                          # of the norms
IGNORE = -100                                       # a token that is none (padding)
BASE = 10000.0                                      # of the rotation's frequencies


def listed():
    return [
        # decoding: one token of one sequence against its cache
        {"name": "attend_one_token", "kind": "attend", "B": 1, "H": 32, "G": 8, "D": 128, "Sq": 1, "Sk": 4097, "dtype": "bf16", "causal": True, "window": 0, "ragged": False},
        # decoding: a token each of many sequences, of all lengths up to that of their caches, which hold few heads
        {"name": "attend_cache", "kind": "attend", "B": 32, "H": 32, "G": 4, "D": 128, "Sq": 1, "Sk": 8192, "dtype": "bf16", "causal": False, "window": 0, "ragged": True},
        # a training step of a large model: queries, keys and values are parts of one projection's output
        {"name": "attend_causal", "kind": "attend", "B": 2, "H": 32, "G": 8, "D": 128, "Sq": 4096, "Sk": 4096, "dtype": "bf16", "causal": True, "window": 0, "ragged": False},
        # odd sizes in 32 bits, a padded batch
        {"name": "attend_odd_f32", "kind": "attend", "B": 3, "H": 6, "G": 2, "D": 72, "Sq": 777, "Sk": 777, "dtype": "f32", "causal": True, "window": 0, "ragged": True},
        # the backward pass of the training step above
        {"name": "attend_back_causal", "kind": "attend_back", "B": 2, "H": 32, "G": 8, "D": 128, "Sq": 4096, "Sk": 4096, "dtype": "bf16", "causal": True, "window": 0, "ragged": False},
        # the backward pass in 32 bits over an odd length, every token sees those near it
        {"name": "attend_back_near_f32", "kind": "attend_back", "B": 2, "H": 12, "G": 12, "D": 64, "Sq": 1531, "Sk": 1531, "dtype": "f32", "causal": False, "window": 256, "ragged": False},
        # norms and rotation in front of that attention
        {"name": "rotate_tokens", "kind": "rotate", "B": 4, "S": 4096, "H": 32, "G": 8, "D": 128, "R": 128, "dtype": "bf16", "pairs": "halves", "first": 0},
        {"name": "rotate_back_tokens", "kind": "rotate_back", "B": 4, "S": 4096, "H": 32, "G": 8, "D": 128, "R": 128, "dtype": "bf16", "pairs": "halves", "first": 0},
        # rows of a table of odd sizes in 32 bits
        {"name": "embed_odd_f32", "kind": "embed", "T": 2999, "V": 50021, "D": 1155, "dtype": "f32", "ignored": 0.05, "add": False},
        # the gradient of a token model's table, tokens as uneven as those of a text are
        {"name": "embed_back_tokens", "kind": "embed_back", "T": 16384, "V": 32768, "D": 1024, "dtype": "bf16", "ignored": 0.05, "add": False},
        # dropout of a layer's output and its addition to the residual stream
        {"name": "dropout_tokens", "kind": "dropout", "T": 16384, "D": 4096, "dtype": "bf16", "p": 0.1, "residual": True},
        # the gradient of one of odd sizes in 32 bits
        {"name": "dropout_odd_f32", "kind": "dropout", "T": 1999, "D": 1155, "dtype": "f32", "p": 0.25, "residual": False},
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "attend_back", "attend_back", "rotate", "rotate_back", "embed", "embed_back", "embed_back", "dropout"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind in ("attend", "attend_back"):
        D = rng.choice([64, 128, 128, 8 * rng.randint(1, 16)])
        G = rng.choice([1, 2, 3, 4, 8])
        H = G * rng.choice([1, 1, 2, 4, 5, 8])
        B = _spread(rng, 1, 32)
        most = 2 ** (30 if dtype == "bf16" else 27) // (B * H)             # pairs of tokens
        c = {"kind": kind, "B": B, "H": H, "G": G, "D": D, "dtype": dtype, "window": rng.choice([0, 0, _spread(rng, 1, 1024)]), "ragged": rng.random() < 0.4}
        if kind == "attend" and rng.random() < 0.5:                        # few tokens against a cache
            Sq = rng.choice([1, 1, rng.randint(2, 40)])
            return {**c, "Sq": Sq, "Sk": _spread(rng, 1, max(2, min(32768, most // Sq, 2 ** 29 // (B * G * D)))), "causal": rng.random() < 0.7}
        S = _spread(rng, 1, min(4096, math.isqrt(most)))
        return {**c, "Sq": S, "Sk": S if rng.random() < 0.7 else _spread(rng, 1, min(4096, max(1, most // S))), "causal": rng.random() < 0.6}
    if kind in ("rotate", "rotate_back"):
        D = rng.choice([64, 128, 256, 2 * rng.randint(2, 128)])
        R = D if rng.random() < 0.6 else 2 * rng.randint(1, D // 2)
        G = rng.randint(1, 8)
        H = G * rng.randint(1, 8)
        B = _spread(rng, 1, 8)
        return {"kind": kind, "B": B, "S": _spread(rng, 1, max(1, min(4096, 2 ** 26 // (B * (H + G) * D)))), "H": H, "G": G, "D": D, "R": R, "dtype": dtype,
                "pairs": rng.choice(["halves", "halves", "next"]), "first": rng.choice([0, rng.randint(0, 2 ** 20)])}
    if kind in ("embed", "embed_back"):
        V = _spread(rng, 32, 131072)
        D = rng.choice([64, 256, 1024, 4096, _spread(rng, 1, 4096)])
        D = min(D, 2 ** 28 // V)
        return {"kind": kind, "T": _spread(rng, 1, min(16384, 2 ** 26 // D)), "V": V, "D": D, "dtype": dtype, "ignored": rng.choice([0.0, 0.05, 0.5]),
                "add": kind == "embed_back" and rng.random() < 0.3}
    D = _spread(rng, 1, 8192)
    return {"kind": kind, "T": _spread(rng, 1, max(1, min(16384, 2 ** 26 // D))), "D": D, "dtype": dtype, "p": rng.choice([0.1, 0.5, rng.random()]),
            "residual": rng.random() < 0.6}


def _lengths(case):
    """Keys that each sequence of a padded batch has; the last of three and more has none"""
    n = [1 + int((case["Sk"] - 1) * ((b + 1) * 0.6180339887 % 1.0)) for b in range(case["B"])]
    return n[:-1] + [0] if len(n) > 2 else n


def _normal(shape, gen, dtype, by=1.0):
    return (torch.randn(shape, generator=gen, device=DEV) * by).to(dtype)


def _parts(x, B, S, sizes, D):
    """Heads that lie one behind the other in the rows of x"""
    return [p.view(B, S, h, D) for p, h in zip(x.split([h * D for h in sizes], 2), sizes)]


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    dt, kind, s = DTYPES[case["dtype"]], case["kind"], {"case": case}
    if kind in ("attend", "attend_back"):
        B, H, G, D, Sq, Sk = (case[k] for k in ("B", "H", "G", "D", "Sq", "Sk"))
        if Sq == Sk:
            s["q"], s["k"], s["v"] = _parts(_normal((B, Sq, (H + 2 * G) * D), gen, dt, 1.2), B, Sq, (H, G, G), D)
        else:                                       # a cache with room for more
            s["q"] = _normal((B, Sq, H, D), gen, dt, 1.2)
            s["k"], s["v"] = (_normal((B, Sk + 32, G, D), gen, dt, 1.2)[:, :Sk] for _ in range(2))
        s["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device=DEV) if case["ragged"] else None
        s["starts"] = s["lengths"] - Sq if case["ragged"] and Sq != Sk else None        # tokens at a sequence's end
        if kind == "attend_back":                   # what the forward pass left, and the output's gradient
            s["grad"] = _normal((B, Sq, H, D), gen, dt)
            s["out"], s["lse"] = _attend(s)
    elif kind in ("rotate", "rotate_back"):
        B, S, H, G, D = (case[k] for k in ("B", "S", "H", "G", "D"))
        gain = torch.rand((H + 2 * G) * D, generator=gen, device=DEV) * 1.9 + 0.1
        x = (torch.randn(B, S, (H + 2 * G) * D, generator=gen, device=DEV) * gain).to(dt)
        s["q"], s["k"], _ = _parts(x, B, S, (H, G, G), D)
        s["wq"], s["wk"] = (torch.rand(D, generator=gen, device=DEV) + 0.5 for _ in range(2))
        s["freq"] = BASE ** (-torch.arange(0, case["R"], 2, dtype=torch.float64, device=DEV) / case["R"])
        s["at"] = case["first"] + torch.arange(S, device=DEV).repeat(B, 1)
        if kind == "rotate_back":
            s["gq"], s["gk"] = _normal((B, S, H, D), gen, dt, 0.1), _normal((B, S, G, D), gen, dt, 0.1)
            s["rq"], s["rk"] = (torch.rsqrt(v.float().square().mean(3) + EPS) for v in (s["q"], s["k"]))
    elif kind in ("embed", "embed_back"):
        T, V, D = case["T"], case["V"], case["D"]
        # few tokens are frequent, many are rare
        ids = (torch.rand(T, generator=gen, device=DEV, dtype=torch.float64) ** 4 * V).long().clamp(max=V - 1)
        s["ids"] = torch.randperm(V, generator=gen, device=DEV)[ids]
        s["ids"][torch.rand(T, generator=gen, device=DEV) < case["ignored"]] = IGNORE
        s["scale"] = math.sqrt(D)
        if kind == "embed":
            s["table"] = _normal((V, D), gen, dt, 0.02)
        else:
            s["grad"] = _normal((T, D), gen, dt, 0.1)
            # a gradient that is there already, as a table has it that is the last layer's weight too
            s["before"] = _normal((V, D), gen, dt, 0.1) if case["add"] else None
    else:
        s["x"] = _normal((case["T"], case["D"]), gen, dt)
        s["r"] = _normal((case["T"], case["D"]), gen, dt) if case["residual"] else None
        s["seed"] = int(torch.randint(0, 2 ** 62, (1,), generator=gen, device=DEV).item())
    return s


# ---------------------------------------------------------------- the framework's operators

def _run_own(s):
    import paper_2208_04187_amd as pkg
    case, kind = s["case"], s["case"]["kind"]
    if kind == "attend":
        a = pkg.division_attention(s["q"], s["k"], s["v"], causal=case["causal"], window=case["window"], lengths=s["lengths"], starts=s["starts"])
        return {"out": a.out, "lse": a.lse}
    if kind == "attend_back":
        dq, dk, dv = pkg.division_attention_backward(s["grad"], s["q"], s["k"], s["v"], s["out"], s["lse"], causal=case["causal"], window=case["window"],
                                                     lengths=s["lengths"], starts=s["starts"])
        return {"dq": dq, "dk": dk, "dv": dv}
    if kind == "rotate":
        r = pkg.division_head_norm_rotate(s["q"], s["k"], s["wq"], s["wk"], s["freq"], s["at"], EPS, pairs=case["pairs"])
        return {"q": r.q, "k": r.k, "rq": r.q_rstd, "rk": r.k_rstd}
    if kind == "rotate_back":
        dq, dk, dwq, dwk = pkg.division_head_norm_rotate_backward(s["gq"], s["gk"], s["q"], s["k"], s["wq"], s["wk"], s["freq"], s["at"], s["rq"], s["rk"],
                                                                  pairs=case["pairs"])
        return {"dq": dq, "dk": dk, "dwq": dwq, "dwk": dwk}
    if kind == "embed":
        return pkg.division_embedding(s["ids"], s["table"], s["scale"], ignore_index=IGNORE)
    if kind == "embed_back":
        if case["add"]:
            return pkg.division_embedding_backward(s["grad"], s["ids"], case["V"], s["scale"], ignore_index=IGNORE, out=s["before"].clone(), add=True)
        return pkg.division_embedding_backward(s["grad"], s["ids"], case["V"], s["scale"], ignore_index=IGNORE)
    return pkg.division_dropout_add(s["x"], case["p"], s["seed"], residual=s["r"])


# ---------------------------------------------------------------- their plain forms

def _visible(s):
    """[B or 1, Sq, Sk]: whether a query sees a key"""
    case = s["case"]
    at = torch.arange(case["Sq"], device=DEV) + (s["starts"][:, None] if s["starts"] is not None else case["Sk"] - case["Sq"])
    at, j = at.view(-1, case["Sq"], 1), torch.arange(case["Sk"], device=DEV)
    seen = (j <= at) if case["causal"] else torch.ones_like(j <= at)
    if case["window"]:
        seen &= (at - j).abs() < case["window"]
    if s["lengths"] is not None:
        seen = seen & (j < s["lengths"][:, None, None])
    return seen


def _by_head(x, groups):
    """[B, S, H, D] as [B * groups, H / groups * S, D]"""
    B, S, H, D = x.shape
    return x.float().view(B, S, groups, H // groups, D).permute(0, 2, 3, 1, 4).reshape(B * groups, H // groups * S, D)


def _of_heads(x, like):
    B, S, H, D = like.shape
    return x.view(B, H, S, D).transpose(1, 2).to(like.dtype).contiguous()


def _scores(s):
    case = s["case"]
    B, H, G, Sq, Sk = (case[k] for k in ("B", "H", "G", "Sq", "Sk"))
    z = torch.bmm(_by_head(s["q"], G), _by_head(s["k"], G).transpose(1, 2).contiguous()).mul_(1.0 / math.sqrt(case["D"]))
    return z.view(B, H, Sq, Sk), _visible(s).unsqueeze(1)


def _attend(s):
    case = s["case"]
    B, H, G, Sq, Sk = (case[k] for k in ("B", "H", "G", "Sq", "Sk"))
    z, seen = _scores(s)
    z = z.masked_fill_(~seen, -math.inf)
    most = z.amax(3, keepdim=True)
    most = torch.where(most == -math.inf, 0.0, most)
    e = z.sub_(most).exp_()
    total = e.sum(3, keepdim=True)
    o = torch.bmm(e.view(B * G, H // G * Sq, Sk), _by_head(s["v"], G)).view(B, H, Sq, -1) / torch.where(total == 0, 1.0, total)
    return o.transpose(1, 2).to(s["q"].dtype).contiguous(), (most + total.log()).squeeze(3)


def _attend_back(s):
    case = s["case"]
    B, H, G, Sq, Sk, D = (case[k] for k in ("B", "H", "G", "Sq", "Sk", "D"))
    z, seen = _scores(s)
    p = z.sub_(s["lse"].unsqueeze(3)).exp_().masked_fill_(~seen, 0.0).view(B * G, H // G * Sq, Sk)
    grad = _by_head(s["grad"], G)
    dv = torch.bmm(p.transpose(1, 2), grad)
    dp = torch.bmm(grad, _by_head(s["v"], G).transpose(1, 2).contiguous())
    ds = dp.sub_((grad * _by_head(s["out"], G)).sum(2, keepdim=True)).mul_(p).mul_(1.0 / math.sqrt(D))
    dq = torch.bmm(ds, _by_head(s["k"], G))
    dk = torch.bmm(ds.transpose(1, 2), _by_head(s["q"], G))
    return {"dq": _of_heads(dq, s["q"]), "dk": _of_heads(dk, s["k"]), "dv": _of_heads(dv, s["v"])}


def _turns(s):
    """cosine and sine of every token's angles, the angles in 64 bits"""
    angle = s["at"].double()[:, :, None, None] * s["freq"]
    return angle.cos().float(), angle.sin().float()


def _apart(x, R, pairs):
    """the two sides of the rotated pairs"""
    return (x[..., 0:R:2], x[..., 1:R:2]) if pairs == "next" else (x[..., : R // 2], x[..., R // 2: R])


def _together(a, b, rest, pairs):
    return torch.cat([torch.stack([a, b], -1).flatten(-2) if pairs == "next" else torch.cat([a, b], -1), rest], -1)


def _rotate(x, w, s):
    case, (cos, sin) = s["case"], _turns(s)
    R, x32 = case["R"], x.float()
    rstd = torch.rsqrt(x32.square().mean(3) + EPS)
    y = x32 * rstd.unsqueeze(3) * w
    a, b = _apart(y, R, case["pairs"])
    return _together(a * cos - b * sin, a * sin + b * cos, y[..., R:], case["pairs"]).to(x.dtype), rstd


def _rotate_back(g, x, w, rstd, s):
    case, (cos, sin) = s["case"], _turns(s)
    R, g32 = case["R"], g.float()
    a, b = _apart(g32, R, case["pairs"])
    g32 = _together(a * cos + b * sin, b * cos - a * sin, g32[..., R:], case["pairs"])
    unit, gw = x.float() * rstd.unsqueeze(3), g32 * w
    dx = rstd.unsqueeze(3) * (gw - unit * (gw * unit).mean(3, keepdim=True))
    return dx.to(x.dtype), (g32 * unit).sum((0, 1, 2))


def _mix(x):
    """the codec's finaliser of 32 bits"""
    x = (x ^ (x >> 16)) * 0x7FEB352D & 0xFFFFFFFF
    x = (x ^ (x >> 15)) * 0x846CA68B & 0xFFFFFFFF
    return x ^ (x >> 16)


def _keys(seed):
    """of the first 2^32 elements of a seed's stream"""
    seed = (seed ^ 0xD509A5B3C2E1F047) & (2 ** 64 - 1)
    k1 = _mix(_mix((seed & 0xFFFFFFFF) ^ 0x243F6A88))
    return k1, _mix((k1 + _mix((seed >> 32) ^ 0x85A308D3)) & 0xFFFFFFFF)


def _threshold(p):
    return min(65536, int(float(np.float32(p)) * 65536.0 + 0.5))


def _kept(n, p, seed):
    """whether each of n elements is kept: two have the halves of a word of 32 bits"""
    k1, k2 = _keys(seed)
    x = (torch.arange((n + 1) // 2, device=DEV) * 0x9E3779B9 + k1) & 0xFFFFFFFF
    x = (x ^ (x >> 16)) * 0x7FEB352D & 0xFFFFFFFF
    x = (x ^ (x >> 15) ^ k2) * 0x846CA68B & 0xFFFFFFFF
    x = x ^ (x >> 16)
    return torch.stack([x & 0xFFFF, x >> 16], 1).view(-1)[:n] >= _threshold(p)


def run(s):
    if own:
        return _run_own(s)
    case, kind = s["case"], s["case"]["kind"]
    if kind == "attend":
        out, lse = _attend(s)
        return {"out": out, "lse": lse}
    if kind == "attend_back":
        return _attend_back(s)
    if kind == "rotate":
        (q, rq), (k, rk) = _rotate(s["q"], s["wq"], s), _rotate(s["k"], s["wk"], s)
        return {"q": q, "k": k, "rq": rq, "rk": rk}
    if kind == "rotate_back":
        (dq, dwq), (dk, dwk) = _rotate_back(s["gq"], s["q"], s["wq"], s["rq"], s), _rotate_back(s["gk"], s["k"], s["wk"], s["rk"], s)
        return {"dq": dq, "dk": dk, "dwq": dwq, "dwk": dwk}
    if kind == "embed":
        rows = s["table"][s["ids"].clamp(min=0)].float() * s["scale"]
        return rows.masked_fill_((s["ids"] == IGNORE).unsqueeze(1), 0.0).to(s["table"].dtype)
    if kind == "embed_back":
        keep = s["ids"] != IGNORE
        total = torch.zeros((case["V"], case["D"]), device=DEV)
        total.index_add_(0, s["ids"][keep], s["grad"][keep].float() * s["scale"])
        return (total if s["before"] is None else total + s["before"].float()).to(s["grad"].dtype)
    x = s["x"].float() * (1.0 / (1.0 - case["p"]))
    x = torch.where(_kept(x.numel(), case["p"], s["seed"]).view(x.shape), x, 0.0)
    return (x if s["r"] is None else x + s["r"].float()).to(s["x"].dtype)


def _pairs(case):
    """how many pairs of a query and a key of one head see each other, and how many keys have a query that sees them, over the batch"""
    Sq, Sk = case["Sq"], case["Sk"]
    n = np.array(_lengths(case) if case["ragged"] else [Sk] * case["B"])[:, None]
    at = np.arange(Sq)[None, :] + (n - Sq if case["ragged"] and Sq != Sk else Sk - Sq)
    lo = np.maximum(0, at - case["window"] + 1) if case["window"] else np.zeros_like(at)
    hi = np.minimum(n, at + 1 if case["causal"] else at + case["window"] if case["window"] else n)
    seen = np.maximum(0, hi - lo)
    some = seen > 0                                 # queries move on by one: what they see together has no gaps
    first, last = np.where(some, lo, Sk).min(1), np.where(some, hi, 0).max(1)
    return int(seen.sum()), int(np.maximum(0, last - first).sum())


def work(case):
    e, kind = 2 if case["dtype"] == "bf16" else 4, case["kind"]
    if kind in ("attend", "attend_back"):
        B, H, G, D, Sq, Sk = (case[k] for k in ("B", "H", "G", "D", "Sq", "Sk"))
        pairs, keys = _pairs(case)
        if kind == "attend":                        # queries and outputs, keys and values that are seen; two products
            return {"bytes": 2 * B * Sq * H * D * e + 4 * B * Sq * H + 2 * keys * G * D * e, "flops": 4 * pairs * H * D + 5 * pairs * H}
        # queries, outputs and their gradients, keys, values and theirs; five products
        return {"bytes": 4 * B * Sq * H * D * e + 4 * B * Sq * H + 2 * (keys + B * Sk) * G * D * e, "flops": 10 * pairs * H * D + 8 * pairs * H}
    if kind in ("rotate", "rotate_back"):
        T, heads, D = case["B"] * case["S"], case["H"] + case["G"], case["D"]
        return {"bytes": T * heads * D * e * (2 if kind == "rotate" else 3) + 4 * T * heads + 8 * T + 8 * D, "flops": T * heads * D * (8 if kind == "rotate" else 14)}
    if kind == "embed":                             # every row out, each row of the table that is used in (at most)
        return {"bytes": case["T"] * (8 + case["D"] * e) + min(case["T"], case["V"]) * case["D"] * e, "flops": case["T"] * case["D"]}
    if kind == "embed_back":
        rows = 2 * min(case["T"], case["V"]) if case["add"] else case["V"]
        # with "add" the caller's copy too, which the pass makes before it
        return {"bytes": case["T"] * (8 + case["D"] * e) + rows * case["D"] * e + (2 * case["V"] * case["D"] * e if case["add"] else 0), "flops": 2 * case["T"] * case["D"]}
    n = case["T"] * case["D"]
    return {"bytes": n * e * (3 if case["residual"] else 2), "flops": n * (3 if case["residual"] else 2)}


# ---------------------------------------------------------------- the definitions in 64 bits

def _attend64(s, back):
    """one sequence and one head of the keys at a time"""
    case = s["case"]
    B, H, G, D, Sq, Sk = (case[k] for k in ("B", "H", "G", "D", "Sq", "Sk"))
    R, f64 = H // G, dict(dtype=torch.float64, device=DEV)
    out, lse = torch.zeros(B, Sq, H, D, **f64), torch.full((B, H, Sq), -math.inf, **f64)
    dq, dk, dv = torch.zeros(B, Sq, H, D, **f64), torch.zeros(B, Sk, G, D, **f64), torch.zeros(B, Sk, G, D, **f64)
    for b in range(B):
        n = int(s["lengths"][b]) if s["lengths"] is not None else Sk
        start = int(s["starts"][b]) if s["starts"] is not None else Sk - Sq
        far = torch.arange(Sk, device=DEV)[None, :] - (torch.arange(Sq, device=DEV)[:, None] + start)    # how far behind the query a key lies
        hidden = (torch.arange(Sk, device=DEV) >= n)[None, :] | ((far > 0) & case["causal"])
        if case["window"]:
            hidden = hidden | (far >= case["window"]) | (far <= -case["window"])
        some = ~hidden.all(1)
        for h in range(H):
            g = h // R
            q, k, v = s["q"][b, :, h].double(), s["k"][b, :, g].double(), s["v"][b, :, g].double()
            z = torch.mm(q, k.t().contiguous()) / math.sqrt(D)
            z[hidden] = -math.inf
            if back:
                w = torch.where(hidden, 0.0, torch.exp(z - s["lse"][b, h].double()[:, None]))
                o, go = s["out"][b, :, h].double(), s["grad"][b, :, h].double()
                dv[b, :, g] += torch.mm(w.t().contiguous(), go)
                d = w * (torch.mm(go, v.t().contiguous()) - torch.einsum("id,id->i", go, o)[:, None]) / math.sqrt(D)
                dq[b, :, h] = torch.mm(d, k)
                dk[b, :, g] += torch.mm(d.t().contiguous(), q)
            else:
                lse[b, h] = torch.logsumexp(z, 1)
                out[b, some, h] = torch.mm(torch.softmax(z[some], 1), v)
    return {"dq": dq, "dk": dk, "dv": dv} if back else {"out": out, "lse": lse}


def _angles64(s, inverse):
    """the tokens' rotations as complex numbers"""
    turn = s["at"].double()[..., None] * s["freq"]
    return torch.polar(torch.ones_like(turn), -turn if inverse else turn)[:, :, None, :]


def _rotated64(x, s, inverse):
    R = s["case"]["R"]
    order = torch.arange(R, device=DEV)
    if s["case"]["pairs"] == "halves":
        order = order.view(2, R // 2).t().reshape(-1)       # the partners next to each other
    z = torch.view_as_complex(x[..., order].unflatten(-1, (R // 2, 2)).contiguous()) * _angles64(s, inverse)
    y = x.clone()
    y[..., order] = torch.view_as_real(z).flatten(-2)
    return y


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind in ("attend", "attend_back"):
        return _attend64(s, kind == "attend_back")
    if kind == "rotate":
        got = {}
        for n, w in (("q", "wq"), ("k", "wk")):
            x = s[n].double()
            got["r" + n] = 1.0 / torch.sqrt(torch.linalg.vector_norm(x, dim=3) ** 2 / case["D"] + EPS)
            got[n] = _rotated64(torch.einsum("bshd,bsh,d->bshd", x, got["r" + n], s[w].double()), s, False)
        return {k: got[k] for k in ("q", "k", "rq", "rk")}
    if kind == "rotate_back":
        got = {}
        for n in ("q", "k"):
            x, r, w = s[n].double(), s["r" + n].double(), s["w" + n].double()
            g = _rotated64(s["g" + n].double(), s, True)
            along = torch.einsum("bshd,bshd,d->bsh", g, x, w) * r ** 3 / case["D"]
            got["d" + n] = g * w * r[..., None] - x * along[..., None]
            got["dw" + n] = torch.einsum("bshd,bshd,bsh->d", g, x, r)
        return {k: got[k] for k in ("dq", "dk", "dwq", "dwk")}
    if kind == "embed":
        got = torch.zeros(case["T"], case["D"], dtype=torch.float64, device=DEV)
        used = s["ids"] >= 0
        got[used] = torch.index_select(s["table"], 0, s["ids"][used]).double() * s["scale"]
        return got
    if kind == "embed_back":
        ids, order = torch.sort(s["ids"], stable=True)      # each token's run of the sorted rows: differences of the running sum would lose digits
        rows, inverse = torch.unique_consecutive(ids, return_inverse=True)
        total = torch.zeros(len(rows), case["D"], dtype=torch.float64, device=DEV).index_add_(0, inverse, s["grad"][order].double())
        got = torch.zeros(case["V"], case["D"], dtype=torch.float64, device=DEV) if s["before"] is None else s["before"].double()
        got[rows[rows >= 0]] += total[rows >= 0] * s["scale"]
        return got
    # the stream once more, in whole numbers of 32 bits on the host
    x = s["x"].double()
    k1, k2 = (np.uint32(k) for k in _keys(s["seed"]))
    with np.errstate(over="ignore"):
        w = np.arange((x.numel() + 1) // 2, dtype=np.uint32) * np.uint32(0x9E3779B9) + k1
        w ^= w >> np.uint32(16)
        w *= np.uint32(0x7FEB352D)
        w ^= (w >> np.uint32(15)) ^ k2
        w *= np.uint32(0x846CA68B)
        w ^= w >> np.uint32(16)
    kept = torch.from_numpy(w.view(np.uint16)[: x.numel()].astype(np.int32) >= _threshold(case["p"])).to(DEV).view(x.shape)
    got = torch.where(kept, x / (1.0 - case["p"]), 0.0)
    return got if s["r"] is None else got + s["r"].double()
