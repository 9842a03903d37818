"""Plain 64-bit forms of the operators of a transformer layer, and bounds on what their kernels may differ by.

The bounds follow from the kernels' roundings: U is the unit roundoff of the type (results, and the matrix instructions' operands that a
kernel forms itself, are rounded to it), EPS stands for sums, exponentials and statistics in 32 bits (some thousand terms of 2^-24 each)."""
import numpy as np
import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 1e-30, torch.float16: 2.0 ** -24, torch.float32: 1e-30}  # float16 has subnormal results
EPS = 1e-4


def within(got, want, bound, name=""):
    got = got.double()
    assert got.shape == want.shape, name
    bad = ~((got - want).abs() <= bound)
    assert not bool(bad.any()), (f"{name}: {int(bad.sum())} of {bad.numel()} values outside their bounds; the worst is off by "
                                 f"{((got - want).abs() / bound.clamp(min=1e-300)).nan_to_num(1e9).max().item():.3g} times the bound")


def act(z, kind):
    return {"none": lambda v: v, "relu": lambda v: v.clamp(min=0), "silu": lambda v: v * torch.sigmoid(v),
            "gelu": lambda v: 0.5 * v * (1 + torch.erf(v * 0.5 ** 0.5)),
            "gelu_tanh": lambda v: 0.5 * v * (1 + torch.tanh((2 / np.pi) ** 0.5 * (v + 0.044715 * v ** 3)))}[kind](z)


def mix(z):
    z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
    z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
    return z ^ (z >> np.uint64(31))


def keep(n, p, seed, offset):
    """keep / (1 - p) of n elements, float64 on the host."""
    threshold = int(p * 65536 + 0.5)
    with np.errstate(over="ignore"):
        at = np.uint64(offset) + np.arange(n, dtype=np.uint64)
        word = mix(mix(np.array([seed], dtype=np.uint64)) + ((at >> np.uint64(2)) + np.uint64(1)) * np.uint64(0x9E3779B97F4A7C15))
    part = (word >> ((at & np.uint64(3)) * np.uint64(16))) & np.uint64(0xFFFF)
    return torch.from_numpy((part >= threshold) * (65536.0 / (65536 - threshold)))


def seen(B, Sq, Sk, causal, begin, end, device):
    i, j = torch.arange(Sq, device=device)[:, None], torch.arange(Sk, device=device)
    m = torch.ones(B, 1, Sq, Sk, dtype=torch.bool, device=device)
    if causal:
        m = m & (j <= i + Sk - Sq)
    if begin is not None:
        m = m & (j >= begin[:, None, :, None])
    if end is not None:
        m = m & (j < end[:, None, :, None])
    return m


def attention(q, k, v, m, scale, slopes, cap):
    """(o, P) in float64 from float64 inputs; rows that see nothing are 0."""
    B, Sq, H, D = q.shape
    Sk, G = k.shape[1:3]
    k, v = k.repeat_interleave(H // G, 2), v.repeat_interleave(H // G, 2)
    s = q.transpose(1, 2) @ k.transpose(1, 2).transpose(2, 3) * scale
    if cap:
        s = cap * torch.tanh(s / cap)
    if slopes is not None:
        i, j = torch.arange(Sq, device=q.device)[:, None], torch.arange(Sk, device=q.device)
        s = s - slopes.double()[None, :, None, None] * (i + Sk - Sq - j).abs()
    p = s.masked_fill(~m, -1e300).softmax(-1) * m if Sk else s
    return (p @ v.transpose(1, 2)).transpose(1, 2), p


def norm(x, kind, eps):
    """(x - mean) / deviation"""
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    return x / ((x * x).mean(-1, keepdim=True) + eps).sqrt()


def residual_norm(x, z, w, b, pre, post, pw, pb, gate, alpha, eps, kept):
    """(xp, h) on rows [T, C]"""
    xp = alpha * x
    if z is not None:
        u = z
        if post != "none":
            u = norm(u, post, eps) * (1 if pw is None else pw) + (0 if pb is None else pb)
        if kept is not None:
            u = u * kept
        if gate is not None:
            u = u * gate.reshape(-1, x.shape[1]).repeat_interleave(x.shape[0] // (gate.numel() // x.shape[1]), 0)
        xp = xp + u
    return xp, norm(xp, pre, eps) * (1 if w is None else w) + (0 if b is None else b)
