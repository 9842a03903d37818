"""Performance cases of the operators of a transformer layer: what running and timing a model's layers takes.

The planner's input is a profile: the forward and backward time of every layer on 1..M GPUs.  These operators are
what those layers are made of, and a GPU's share of a layer is the same operators with fewer columns or heads.
A case is a dict of plain values; "op" says which operator it is:
  linear     y = act(x W^T + b) + r, and its gradients
  attention  o = softmax(cap tanh(s q.k / cap) - slope |i - j|) v over a range of keys per query, and its gradients
  norm       x' = alpha x + gate * dropout(post(z)), h = pre(x'): the norms around a block, and their gradients
  dropout    y = x * keep / (1 - p), keep from a counter-based generator (its backward pass is the same call)
Sizes are those of the planning configurations: a microbatch is 4096 tokens (boundary bytes / hidden width), widths
2048, 4096 and 12288, up to 8 GPUs a layer; small and odd ones beside them.
"""
import math
from types import SimpleNamespace

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}


def listed():
    return [
        # A handful of tokens through a square projection (attention's output, hidden width 2048): the weights have to
        # be read and hardly anything else counts.
        dict(name="linear-16-tokens", op="linear", T=16, K=2048, N=2048, act="none", residual=True, type="bf16", train=False),
        # Odd numbers of tokens and columns: a ragged last microbatch, a vocabulary-like width; rows of no alignment.
        dict(name="linear-odd", op="linear", T=1021, K=1030, N=2061, act="silu", residual=True, type="fp16", train=True),
        # First feed-forward product of the 175B-shaped model on 8 GPUs, one GPU's 6144 of 49152 columns, one microbatch,
        # forward and backward.
        dict(name="linear-ff-12288-of-8", op="linear", T=4096, K=12288, N=6144, act="gelu_tanh", residual=False, type="bf16", train=True),
        # One short sequence, few heads: the launch and a few steps.
        dict(name="attention-short", op="attention", B=1, S=128, H=16, G=16, D=64, mask="causal", docs=1, slopes=False, cap=0.0,
             type="bf16", train=False),
        # 1.3B-shaped: two sequences of 2048 packed with documents of odd lengths, the last tokens padding that sees nothing.
        dict(name="attention-documents", op="attention", B=2, S=2048, H=16, G=16, D=128, mask="document", docs=5, slopes=False,
             cap=0.0, type="bf16", train=True),
        # An odd length, a prefix that is seen whole, shared key heads, distance bias and capped scores, a head of 80.
        dict(name="attention-prefix-odd", op="attention", B=2, S=1531, H=8, G=2, D=80, mask="prefix", docs=1, slopes=True, cap=30.0,
             type="fp16", train=True),
        # 175B-shaped on 8 GPUs: 12 of 96 heads, one sequence of 4096, causal.
        dict(name="attention-12-of-96-heads", op="attention", B=1, S=4096, H=12, G=12, D=128, mask="causal", docs=1, slopes=False,
             cap=0.0, type="bf16", train=True),
        # Norm before the block of a few tokens, after the residual sum: latency.
        dict(name="norm-64-tokens", op="norm", T=64, C=2048, pre="layer", post="none", gate="none", alpha=1.0, p=0.0, type="bf16", train=False),
        # Norms on both sides, a gate per sequence, a scaled residual; odd width, 32 bits.
        dict(name="norm-gate-odd", op="norm", T=2001, C=2051, pre="rms", post="rms", gate="group", alpha=0.5, p=0.0, type="fp32", train=True),
        # 175B-shaped: residual dropout, sum and norm of a microbatch, forward and backward.
        dict(name="norm-dropout-12288", op="norm", T=4096, C=12288, pre="layer", post="none", gate="none", alpha=1.0, p=0.1, type="bf16", train=True),
        # Dropout of a few tokens' embeddings: latency.
        dict(name="dropout-16-tokens", op="dropout", n=16 * 2048, p=0.1, type="fp16"),
        # Dropout of the embeddings' sum, 6.7B-shaped microbatch, an element past the end of a row of eight.
        dict(name="dropout-embedding", op="dropout", n=4096 * 4096 + 1, p=0.1, type="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["linear", "linear", "attention", "attention", "norm", "dropout"])
    kind = rng.choice(["bf16", "bf16", "fp16"])
    if op == "linear":
        T, K, N = _log(rng, 1, 4096), _log(rng, 64, 12288), _log(rng, 64, 12288)
        if rng.random() < 0.6:  # widths of models are mostly multiples of 64
            K, N = max(64, K // 64 * 64), max(64, N // 64 * 64)
        while T * K * N > 4096 * 12288 * 6144:
            N = max(64, N // 2)
        return _not_3072(dict(op="linear", T=T, K=K, N=N, act=rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"]),
                              residual=rng.random() < 0.5, type=kind, train=rng.random() < 0.6))
    if op == "attention":
        S, D = _log(rng, 1, 4096), rng.choice([64, 64, 128, 128, 80, 96, 32, 40])
        B = max(1, min(8, _log(rng, 1, 4096) // S))
        G = rng.choice([1, 2, 4, 8])
        return _not_3072(dict(op="attention", B=B, S=S, H=G * rng.choice([1, 1, 2, 4]) if G < 8 else G, G=G, D=D,
                              mask=rng.choice(["causal", "causal", "full", "document", "prefix"]), docs=rng.randint(1, 6),
                              slopes=rng.random() < 0.3, cap=rng.choice([0.0, 0.0, 20.0, 50.0]), type=kind, train=rng.random() < 0.6))
    if op == "norm":
        T, C = _log(rng, 1, 8192), _log(rng, 64, 12288)
        if rng.random() < 0.6:
            C = max(64, C // 64 * 64)
        while T * C > 4096 * 12288:
            T //= 2
        post = rng.choice(["none", "none", "rms", "layer"])
        return _not_3072(dict(op="norm", T=T, C=C, pre=rng.choice(["layer", "rms"]), post=post, gate=rng.choice(["none", "channel", "group"]),
                              alpha=rng.choice([1.0, 0.5]), p=rng.choice([0.0, 0.1]), type=rng.choice(["bf16", "fp16", "fp32"]),
                              train=rng.random() < 0.6))
    return dict(op="dropout", n=_log(rng, 1, 4096 * 12288), p=rng.choice([0.05, 0.1, 0.2, 0.5]), type=rng.choice(["bf16", "fp16", "fp32"]))


def _not_3072(case):
    """No size of 3072: no configuration of this repository has it."""
    return {k: 3008 if type(v) is int and v == 3072 else v for k, v in case.items()}


# ---- masks: a range of keys for every query ------------------------------------------------------------
def key_ranges(c):
    """(begin, end) per sequence and query, as int32 arrays [B, S], or None where the mask is causal or full."""
    if c["mask"] in ("causal", "full"):
        return None
    S, b = c["S"], np.arange(c["B"])[:, None]
    i = np.arange(S)
    if c["mask"] == "prefix":
        end = np.maximum(i + 1, S * (b + 1) // (2 * c["B"] + 1))
        return np.zeros_like(end, dtype=np.int32), end.astype(np.int32)
    used = S - S * b // 32 - S // 64  # what is behind the last document is padding
    cuts = used * (3 * np.arange(c["docs"]) + b % 2) // (3 * c["docs"])  # where documents begin, the first one aside
    cuts[:, 0] = 0
    of = (cuts[:, :, None] <= i).sum(1) - 1
    seen = i < used
    return np.where(seen, np.take_along_axis(cuts, of, 1), 0).astype(np.int32), np.where(seen, i + 1, 0).astype(np.int32)


def _pairs(c):
    r = key_ranges(c)
    if r is None:
        return c["B"] * (c["S"] ** 2 if c["mask"] == "full" else c["S"] * (c["S"] + 1) // 2)
    return int((r[1].astype(np.int64) - r[0]).clip(0).sum())


# ---- inputs ----------------------------------------------------------------------------------------------
def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = TYPES[c["type"]]
    normal = lambda *shape, std=1.0, mean=0.0: (torch.randn(*shape, generator=g, device="cuda") * std + mean).to(t)  # noqa: E731
    s = SimpleNamespace(case=c)
    if c["op"] == "linear":
        s.x = normal(c["T"], c["K"])
        s.w = normal(c["N"], c["K"], std=c["K"] ** -0.5)
        s.b = normal(c["N"], std=0.1)
        s.r = normal(c["T"], c["N"]) if c["residual"] else None
        s.dy = normal(c["T"], c["N"]) if c["train"] else None
    elif c["op"] == "attention":
        B, S, H, G, D = (c[k] for k in "BSHGD")
        s.qkv = normal(B, S, (H + 2 * G) * D)
        s.do = normal(B, S, H, D) if c["train"] else None
        s.scale = D ** -0.5
        s.slopes = torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], device="cuda") if c["slopes"] else None
        r = key_ranges(c)
        s.begin, s.end = (torch.from_numpy(a).cuda() for a in r) if r is not None else (None, None)
    elif c["op"] == "norm":
        T, C = c["T"], c["C"]
        s.z, s.x = normal(T, C), normal(T, C, std=2.0, mean=0.1)
        s.w, s.b = normal(C, std=0.1, mean=1.0), normal(C, std=0.1) if c["pre"] == "layer" else None
        s.pw = normal(C, std=0.1, mean=1.0) if c["post"] != "none" else None
        s.pb = normal(C, std=0.1) if c["post"] == "layer" else None
        s.groups = {"none": 0, "channel": 1, "group": next(n for n in (4, 3, 2, 1) if T % n == 0)}[c["gate"]]
        s.gate = normal(s.groups, C, std=0.5) if s.groups else None
        s.dxp, s.dh = (normal(T, C), normal(T, C)) if c["train"] else (None, None)
        s.seed, s.offset = seed * 7919 + 12345, (seed * 977) % 100003
    else:
        s.x = normal(c["n"])
        s.seed, s.offset = seed * 7919 + 54321, (seed * 977) % 100003
    return s


def split_qkv(c, t):
    """The q, k and v heads in a tensor whose last axis holds all of them: [B, S, heads, D] views."""
    B, S, H, G, D = (c[k] for k in "BSHGD")
    t = t.view(B, S, H + 2 * G, D)
    return t[:, :, :H], t[:, :, H:H + G], t[:, :, H + G:]


# ---- the plain forms: elementary operations in 32 bits --------------------------------------------------
def _golden(x):
    """A 64-bit constant as the signed number that torch takes."""
    return x - (1 << 64) if x >= 1 << 63 else x


GOLDEN, MIX1, MIX2 = 0x9E3779B97F4A7C15, 0xBF58476D1CE4E5B9, 0x94D049BB133111EB


def _mix(z):
    """The output function of SplitMix64 on a tensor of 64-bit words (products wrap)."""
    z = (z ^ ((z >> 30) & ((1 << 34) - 1))) * _golden(MIX1)
    z = (z ^ ((z >> 27) & ((1 << 37) - 1))) * _golden(MIX2)
    return z ^ ((z >> 31) & ((1 << 33) - 1))


def _keep(n, p, seed, offset):
    """keep / (1 - p) of elements 0 .. n-1, 32 bits: 16 of the 64 bits of word (offset + i) // 4 against round(65536 p)."""
    threshold = int(p * 65536 + 0.5)
    at = torch.arange(offset // 4, (offset + n + 3) // 4, device="cuda", dtype=torch.int64)
    key = _mix(torch.tensor(_golden(seed & ((1 << 64) - 1)), device="cuda"))
    word = _mix(key + (at + 1) * _golden(GOLDEN))
    parts = torch.stack([(word >> k) & 0xFFFF for k in (0, 16, 32, 48)], dim=1).reshape(-1)[offset % 4: offset % 4 + n]
    return (parts >= threshold).float() * (65536.0 / (65536 - threshold))


def _act(z, act):
    """act(z) and its derivative."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        on = (z > 0).float()
        return z * on, on
    if act == "silu":
        e = 1 / (1 + torch.exp(-z))
        return z * e, e * (1 + z * (1 - e))
    if act == "gelu":
        e = 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
        return z * e, e + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    k = math.sqrt(2 / math.pi)
    t = torch.tanh(k * (z + 0.044715 * z * z * z))
    return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * k * (1 + 3 * 0.044715 * z * z)


def _plain_linear(s):
    c, t = s.case, s.x.dtype
    x, w = s.x.float(), s.w.float()
    y, slope = _act(x @ w.t() + s.b.float(), c["act"])
    if s.r is not None:
        y = y + s.r.float()
    if not c["train"]:
        return {"y": y.to(t)}
    dz = s.dy.float() * slope
    return {"y": y.to(t), "dx": (dz @ w).to(t), "dw": (dz.t() @ x).to(t), "db": dz.sum(0).to(t)}


def _plain_attention(s):
    c, t = s.case, s.qkv.dtype
    B, S, H, G, D = (c[k] for k in "BSHGD")
    q, k, v = (a.float().transpose(1, 2).contiguous() for a in split_qkv(c, s.qkv))
    q = q.view(B, G, H // G, S, D)
    k, v = k.unsqueeze(2), v.unsqueeze(2)
    raw = torch.matmul(q, k.transpose(3, 4).contiguous()) * s.scale
    th = torch.tanh(raw / c["cap"]) if c["cap"] else None
    score = c["cap"] * th if c["cap"] else raw
    i, j = torch.arange(S, device="cuda").view(S, 1), torch.arange(S, device="cuda")
    if s.slopes is not None:
        score = score - s.slopes.view(1, G, H // G, 1, 1) * (i - j).abs()
    if s.begin is not None:
        seen = (j >= s.begin.view(B, 1, 1, S, 1)) & (j < s.end.view(B, 1, 1, S, 1))
    else:
        seen = (j <= i if c["mask"] == "causal" else j >= 0).expand(S, S)
    top = torch.where(seen, score, -math.inf).amax(-1, keepdim=True)
    e = torch.where(seen, torch.exp(score - torch.where(top == -math.inf, 0.0, top)), 0.0)
    total = e.sum(-1, keepdim=True)
    P = e / torch.where(total == 0, 1.0, total)
    o = torch.matmul(P, v.expand(B, G, H // G, S, D).contiguous())
    out = {"o": o.reshape(B, H, S, D).transpose(1, 2).contiguous().to(t)}
    if not c["train"]:
        return out
    do = s.do.float().transpose(1, 2).reshape(B, G, H // G, S, D)
    dP = torch.matmul(do, v.transpose(3, 4).contiguous())
    dS = P * (dP - (do * o).sum(-1, keepdim=True))
    if c["cap"]:
        dS = dS * (1 - th * th)
    dS = dS * s.scale
    dq = torch.matmul(dS, k.expand(B, G, H // G, S, D).contiguous()).reshape(B, H, S, D)
    dk = torch.matmul(dS.transpose(3, 4).contiguous(), q).sum(2)
    dv = torch.matmul(P.transpose(3, 4).contiguous(), do).sum(2)
    out["dqkv"] = torch.cat([a.transpose(1, 2) for a in (dq, dk, dv)], dim=2).reshape(B, S, -1).to(t)
    return out


def _norm(x, kind, eps=1e-5):
    """(x - mean) / deviation, and 1 / deviation."""
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    return x * r, r


def _norm_back(d, xhat, r, kind):
    d = d - xhat * (d * xhat).mean(-1, keepdim=True) - (d.mean(-1, keepdim=True) if kind == "layer" else 0)
    return d * r


def _plain_norm(s):
    c, t = s.case, s.x.dtype
    T, C = c["T"], c["C"]
    f = lambda a: None if a is None else a.float()  # noqa: E731
    w, b, pw, pb, gate = f(s.w), f(s.b), f(s.pw), f(s.pb), f(s.gate)
    group = torch.arange(T, device="cuda") // (T // s.groups) if s.groups else None
    u = s.z.float()
    if c["post"] != "none":
        zhat, zr = _norm(u, c["post"])
        u = zhat * pw + (pb if pb is not None else 0)
    keep = _keep(T * C, c["p"], s.seed, s.offset).view(T, C) if c["p"] else 1.0
    u = u * keep
    xp = c["alpha"] * s.x.float() + (u * gate[group] if s.groups else u)
    hat, r = _norm(xp, c["pre"])
    out = {"xp": xp.to(t), "h": (hat * w + (b if b is not None else 0)).to(t)}
    if not c["train"]:
        return out
    dh = s.dh.float()
    d = s.dxp.float() + _norm_back(dh * w, hat, r, c["pre"])
    out |= {"dx": (c["alpha"] * d).to(t), "dw": (dh * hat).sum(0).to(t)}
    if b is not None:
        out["db"] = dh.sum(0).to(t)
    du = d
    if s.groups:
        out["dgate"] = (d * u).view(s.groups, -1, C).sum(1).to(t)
        du = d * gate[group]
    du = du * keep
    if c["post"] != "none":
        out["dpost_w"] = (du * zhat).sum(0).to(t)
        if pb is not None:
            out["dpost_b"] = du.sum(0).to(t)
        du = _norm_back(du * pw, zhat, zr, c["post"])
    out["dz"] = du.to(t)
    return out


def run(s):
    return (_own if own else _plain)(s)


def _plain(s):
    op = s.case["op"]
    if op == "dropout":
        return (s.x.float() * _keep(s.case["n"], s.case["p"], s.seed, s.offset)).to(s.x.dtype)
    return {"linear": _plain_linear, "attention": _plain_attention, "norm": _plain_norm}[op](s)


# ---- the framework's operators ---------------------------------------------------------------------------
def _own(s):
    import paper_2309_08125_amd as P

    c = s.case
    if c["op"] == "linear":
        if not c["train"]:
            return {"y": P.linear(s.x, s.w, s.b, act=c["act"], residual=s.r)}
        y, z = P.linear(s.x, s.w, s.b, act=c["act"], residual=s.r, keep=True)
        dx, dw, db = P.linear_backward(s.dy, s.x, s.w, z, act=c["act"])
        return {"y": y, "dx": dx, "dw": dw, "db": db}
    if c["op"] == "attention":
        q, k, v = split_qkv(c, s.qkv)
        kind = dict(scale=s.scale, causal=c["mask"] == "causal", key_begin=s.begin, key_end=s.end, slopes=s.slopes, cap=c["cap"])
        o, lse = P.attention(q, k, v, **kind)
        if not c["train"]:
            return {"o": o}
        dqkv = torch.empty_like(s.qkv)
        P.attention_backward(s.do, q, k, v, o, lse, out=split_qkv(c, dqkv), **kind)
        return {"o": o, "dqkv": dqkv}
    if c["op"] == "norm":
        kind = dict(weight=s.w, bias=s.b, pre=c["pre"], post=c["post"], post_weight=s.pw, post_bias=s.pb, gate=s.gate,
                    alpha=c["alpha"], p=c["p"], seed=s.seed, offset=s.offset)
        xp, h, saved = P.residual_norm(s.x, s.z, **kind)
        out = {"xp": xp, "h": h}
        if c["train"]:
            d = P.residual_norm_backward(s.dxp, s.dh, xp, s.z, saved, **kind)
            names = {"x": "dx", "z": "dz", "weight": "dw", "bias": "db", "post_weight": "dpost_w", "post_bias": "dpost_b", "gate": "dgate"}
            out |= {names[n]: a for n, a in d.items() if a is not None}
        return out
    return P.dropout(s.x, c["p"], s.seed, s.offset)


# ---- what a pass cannot do without ------------------------------------------------------------------------
def work(case):
    c, e = case, BYTES[case["type"]]
    if c["op"] == "linear":
        T, K, N = c["T"], c["K"], c["N"]
        values = T * K + N * K + N + T * N * (2 if c["residual"] else 1)
        if c["train"]:
            values += T * N + T * K + N * K + N
        return {"bytes": e * values, "flops": (6 if c["train"] else 2) * T * K * N}
    if c["op"] == "attention":
        B, S, H, G, D = (c[k] for k in "BSHGD")
        values = B * S * D * (2 * H + 2 * G)
        if c["train"]:
            values += B * S * D * (2 * H + 2 * G)
        return {"bytes": e * values, "flops": (14 if c["train"] else 4) * D * H * _pairs(c)}
    if c["op"] == "norm":
        n = c["T"] * c["C"]
        return {"bytes": e * (n * (8 if c["train"] else 4) + 2 * c["C"]), "flops": (25 if c["train"] else 10) * n}
    return {"bytes": 2 * e * c["n"], "flops": 2 * c["n"]}


# ---- the definitions in 64 bits, by differentiation instead of written-out gradients ---------------------
def _keep64(n, p, seed, offset):
    """The kept elements from 64-bit unsigned words on the host."""
    threshold = int(p * 65536 + 0.5)

    def mix(z):
        z = (z ^ (z >> np.uint64(30))) * np.uint64(MIX1)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(MIX2)
        return z ^ (z >> np.uint64(31))

    with np.errstate(over="ignore"):
        i = np.arange(offset // 4, (offset + n - 1) // 4 + 1, dtype=np.uint64)
        words = mix(mix(np.full(1, seed & ((1 << 64) - 1), np.uint64)) + (i + np.uint64(1)) * np.uint64(GOLDEN))
    got = words.astype("<u8").view("<u2")[offset % 4: offset % 4 + n]
    return torch.from_numpy((got >= threshold).astype(np.float64)).cuda() / (1 - threshold / 65536)


def _norm64(x, kind, w, b):
    mean = x.mean(-1, keepdim=True) if kind == "layer" else 0.0
    y = (x - mean) / ((x - mean).pow(2).mean(-1, keepdim=True) + 1e-5).sqrt() * w
    return y if b is None else y + b


def exact(case, seed):
    s, c = prepare(case, seed), case
    d = lambda a: None if a is None else a.double().requires_grad_()  # noqa: E731
    if c["op"] == "dropout":
        return s.x.double() * _keep64(c["n"], c["p"], s.seed, s.offset)
    if c["op"] == "linear":
        x, w, b = d(s.x), d(s.w), d(s.b)
        z = torch.addmm(b, x, w.t())
        y = {"none": lambda v: v, "relu": lambda v: v.clamp(min=0), "silu": lambda v: v * v.sigmoid(),
             "gelu": lambda v: v * 0.5 * torch.special.erfc(-v / math.sqrt(2)),
             "gelu_tanh": lambda v: v * torch.sigmoid(math.sqrt(8 / math.pi) * (v + 0.044715 * v ** 3))}[c["act"]](z)
        out = {"y": (y if s.r is None else y + s.r.double()).detach()}
        if c["train"]:
            out |= dict(zip(("dx", "dw", "db"), torch.autograd.grad(y, (x, w, b), s.dy.double())))
        return out
    if c["op"] == "attention":
        B, S, H, G, D = (c[k] for k in "BSHGD")
        qkv = d(s.qkv)
        outs, grads = [], []
        i = torch.arange(S, device="cuda")
        for n in range(B):  # a sequence and a head at a time: memory
            begin = s.begin[n] if s.begin is not None else torch.zeros_like(i)
            end = s.end[n] if s.end is not None else (i + 1 if c["mask"] == "causal" else torch.full_like(i, S))
            hidden = (i[None] < begin[:, None]) | (i[None] >= end[:, None])
            lone = hidden.all(1, keepdim=True)
            heads = []
            for h in range(H):
                at = qkv[n].view(S, -1, D)
                q, k, v = at[:, h], at[:, H + h // (H // G)], at[:, H + G + h // (H // G)]
                a = q @ k.t() * s.scale
                if c["cap"]:
                    a = c["cap"] * (a / c["cap"]).tanh()
                if s.slopes is not None:
                    a = a - s.slopes[h].double() * (i[:, None] - i).abs()
                o = (a.masked_fill(hidden, -1e300).softmax(-1).masked_fill(lone, 0.0)) @ v
                heads.append(o.detach())
                if c["train"]:
                    grads.append(torch.autograd.grad(o, qkv, s.do[n, :, h].double())[0] if not grads else
                                 grads.pop().add_(torch.autograd.grad(o, qkv, s.do[n, :, h].double())[0]))
            outs.append(torch.stack(heads, 1))
        return {"o": torch.stack(outs)} | ({"dqkv": grads[0]} if c["train"] else {})
    T, C = c["T"], c["C"]
    x, z, w, b, pw, pb, gate = (d(a) for a in (s.x, s.z, s.w, s.b, s.pw, s.pb, s.gate))
    u = z if c["post"] == "none" else _norm64(z, c["post"], pw, pb)
    if c["p"]:
        u = u * _keep64(T * C, c["p"], s.seed, s.offset).view(T, C)
    if s.groups:
        u = u * gate[torch.arange(T, device="cuda").div(T // s.groups, rounding_mode="floor")]
    xp = x * c["alpha"] + u
    h = _norm64(xp, c["pre"], w, b)
    out = {"xp": xp.detach(), "h": h.detach()}
    if c["train"]:
        names = {"dx": x, "dz": z, "dw": w, "db": b, "dpost_w": pw, "dpost_b": pb, "dgate": gate}
        names = {n: a for n, a in names.items() if a is not None}
        out |= dict(zip(names, torch.autograd.grad((xp, h), list(names.values()), (s.dxp.double(), s.dh.double()))))
    return out
