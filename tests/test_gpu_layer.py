"""The operators of a transformer layer against their plain 64-bit forms: values, gradients (against the formula's by differentiation and
against differences), strides, empty masks, streams, graphs, refusals."""
import numpy as np
import pytest
import torch

import layer_oracle as O
from layer_oracle import EPS, TINY, U, within

pytestmark = pytest.mark.gpu
HALF = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def P():
    import paper_2309_08125_amd as pkg

    assert torch.cuda.is_available()
    pkg.load()
    return pkg


@pytest.fixture(autouse=True)
def tell(request):
    print("case", request.node.name, flush=True)
    torch.manual_seed(len(request.node.name))
    yield
    torch.cuda.synchronize()


def rand(*shape, t=torch.bfloat16, std=1.0, mean=0.0):
    return (torch.randn(*shape, device="cuda") * std + mean).to(t)


def strided(t, pad=5, at=1):
    """The same values as a view of wider rows that start `at` elements in."""
    wide = torch.full((*t.shape[:-1], t.shape[-1] + pad), 7.0, dtype=t.dtype, device=t.device)
    view = wide[..., at: at + t.shape[-1]]
    view.copy_(t)
    return view


def d64(*ts):
    return [None if t is None else t.double().requires_grad_() for t in ts]


# ---- linear ------------------------------------------------------------------------------------------------
def linear_case(P, T, N, K, act, t, bias=True, residual=True, view=lambda a: a, need=("x", "w", "b")):
    u, tiny = U[t], TINY[t]
    x, w, b, r, dy = view(rand(T, K, t=t)), view(rand(N, K, t=t, std=K ** -0.5)), rand(N, t=t), view(rand(T, N, t=t)), view(rand(T, N, t=t))
    y, z = P.linear(x, w, b if bias else None, act=act, residual=r if residual else None, keep=True)
    assert (z is None) == (act == "none")
    X, W, B = d64(x, w, b if bias else torch.zeros_like(b))
    Z = X @ W.t() + B
    A = O.act(Z, act)
    sums = x.double().abs() @ w.double().abs().t() + b.double().abs()
    within(y, (A + r.double() if residual else A).detach(), u * (A + (r.double() if residual else 0)).abs().detach() + EPS * (sums + r.double().abs()) + tiny, "y")
    dx, dw, db = P.linear_backward(dy, x, w, z, act=act, need=need)
    want = torch.autograd.grad(A, (X, W, B), dy.double())
    slope = torch.autograd.grad(O.act(Z, act).sum(), Z)[0]
    # dz is formed from z rounded (|act''| <= 1.2) and rounded itself, where there is an activation
    dz = (dy.double() * slope).abs()
    off = EPS * dy.double().abs() + (0 if act == "none" else u * dz + 1.2 * u * dy.double().abs() * Z.abs().detach() + tiny)
    if act == "relu":  # a jump of the slope where z rounds to the other side of 0: nothing else
        off = off + dy.double().abs() * (Z.abs().detach() <= EPS * sums)
    for name, got, val, bound in (("dx", dx, want[0], (off + EPS * dz) @ w.double().abs()), ("dw", dw, want[1], (off + EPS * dz).t() @ x.double().abs()),
                                  ("db", db, want[2], (off + EPS * dz).sum(0))):
        if got is None:
            assert name[1] not in need
        else:
            within(got, val, bound + u * val.abs() + tiny, name)


@pytest.mark.parametrize("t", HALF)
@pytest.mark.parametrize("T,N,K", [(1, 1, 1), (1, 64, 8), (3, 7, 5), (16, 2048, 256), (64, 64, 64), (65, 63, 72), (130, 520, 1000), (1, 1000, 2048), (700, 130, 33)])
def test_linear_sizes(P, T, N, K, t):
    linear_case(P, T, N, K, "none", t)
    linear_case(P, T, N, K, "gelu_tanh", t)


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
def test_linear_activations(P, act):
    for t in HALF:
        linear_case(P, 100, 72, 136, act, t)
        linear_case(P, 100, 72, 136, act, t, bias=False, residual=False)


@pytest.mark.parametrize("T,N,K", [(2048, 4096, 512), (1500, 1600, 192), (4000, 4104, 72)])
def test_linear_large_tiles(P, T, N, K):
    linear_case(P, T, N, K, "silu", torch.bfloat16)


def test_linear_strides_and_parts(P):
    for at in (0, 1):
        linear_case(P, 90, 48, 40, "gelu", torch.float16, view=lambda a: strided(a, 8, at))
    linear_case(P, 90, 48, 40, "gelu", torch.bfloat16, need=("x",))
    linear_case(P, 90, 48, 40, "none", torch.bfloat16, need=("w",))
    linear_case(P, 90, 48, 40, "none", torch.bfloat16, need=("b",))


def test_linear_without_tokens(P):
    x, w = rand(0, 24), rand(16, 24)
    assert P.linear(x, w).shape == (0, 16)
    dx, dw, db = P.linear_backward(rand(0, 16), x, w)
    assert dx.shape == (0, 24) and not dw.any() and not db.any()


def test_linear_of_several_axes_and_poison_beside(P):
    x, w = rand(3, 5, 40), rand(24, 40)
    y = P.linear(x, w)
    assert y.shape == (3, 5, 24) and torch.equal(y.view(15, 24), P.linear(x.view(15, 40), w))
    # what lies beside the operands' rows does not enter: rows of 72 in wider rows of infinities, a ragged last step of k
    wide = torch.full((70, 104), float("inf"), device="cuda", dtype=torch.bfloat16)
    wide[:, :72] = rand(70, 72)
    w = rand(24, 72)
    got, want = P.linear(wide[:, :72], w), P.linear(wide[:, :72].contiguous(), w)
    assert torch.equal(got, want) and torch.isfinite(got).all()
    dy = rand(70, 24)
    assert all(torch.equal(a, b) for a, b in zip(P.linear_backward(dy, wide[:, :72], w), P.linear_backward(dy, wide[:, :72].contiguous(), w)))


def test_linear_gradient_against_differences(P):
    T, N, K, t = 33, 40, 24, torch.float16
    x, w, b, dy = rand(T, K, t=t), rand(N, K, t=t, std=0.2), rand(N, t=t), rand(T, N, t=t)
    for act in ("gelu", "gelu_tanh", "silu"):
        _, z = P.linear(x, w, b, act=act, keep=True)
        grads = P.linear_backward(dy, x, w, z, act=act)
        loss = lambda X, W, B: (O.act(X @ W.t() + B, act) * dy.double()).sum()  # noqa: B023, E731
        base = [a.double() for a in (x, w, b)]
        for i, g in enumerate(grads):
            d, h = torch.randn_like(base[i]), 1e-4
            plus, minus = ([a + s * h * d if k == i else a for k, a in enumerate(base)] for s in (1, -1))
            diff = (loss(*plus) - loss(*minus)) / (2 * h)
            # each gradient has the error of two roundings of 16-bit values (z, dz) and its own
            assert abs((g.double() * d).sum() - diff) <= 4 * U[t] * g.double().norm() * d.norm() + 1e-5


# ---- attention ---------------------------------------------------------------------------------------------
def attention_case(P, B, Sq, Sk, H, G, D, t, causal=False, begin=None, end=None, slopes=False, cap=0.0, scale=None, view=lambda a: a, std=1.0):
    u, tiny = U[t], TINY[t]
    q, k, v, do = view(rand(B, Sq, H, D, t=t, std=std)), view(rand(B, Sk, G, D, t=t, std=std)), view(rand(B, Sk, G, D, t=t)), view(rand(B, Sq, H, D, t=t))
    sl = torch.tensor([2.0 ** -(1 + h) for h in range(H)], device="cuda") if slopes else None
    kind = dict(scale=scale, causal=causal, key_begin=begin, key_end=end, slopes=sl, cap=cap)
    o, lse = P.attention(q, k, v, **kind)
    out = tuple(torch.full_like(a, 3.0) for a in (q, k, v))
    assert all(a is b for a, b in zip(P.attention_backward(do, q, k, v, o, lse, out=out, **kind), out))
    scale = D ** -0.5 if scale is None else scale
    m = O.seen(B, Sq, Sk, causal, begin, end, "cuda")
    Q, K, V = d64(q, k, v)
    want, p = O.attention(Q, K, V, m, scale, sl, cap)
    grads = torch.autograd.grad(want, (Q, K, V), do.double()) if Sq and Sk else [torch.zeros_like(a) for a in (Q, K, V)]
    p, want = p.detach(), want.detach()
    rows = lambda a: a.double().abs().repeat_interleave(H // a.shape[2], 2).transpose(1, 2)  # noqa: E731
    # p is rounded to the type before its product with v, and so is the result; 32 bits between
    off_o = u * want.abs() + 2 * (u + EPS) * (p @ rows(v)).transpose(1, 2) + tiny
    within(o, want, off_o, "o")
    # ds = p (dp - delta): rounded; p and dp to 32 bits; delta from o as it is returned
    dp = do.double().transpose(1, 2) @ v.double().repeat_interleave(H // G, 2).transpose(1, 2).transpose(2, 3)
    big = rows(do) @ rows(v).transpose(2, 3) + (rows(do) * rows(o)).sum(-1, keepdim=True)
    ds = (p * (dp - (do.double() * want).sum(-1).transpose(1, 2)[..., None])).abs()
    off = u * ds + p * ((rows(do) * off_o.transpose(1, 2)).sum(-1, keepdim=True) + 2 * EPS * big) + (tiny if t == torch.float16 else 0) * m
    group = lambda a: a.view(B, G, H // G, *a.shape[2:]).sum(2).transpose(1, 2)  # noqa: E731
    bounds = (scale * (off @ rows(k)).transpose(1, 2), group(scale * (off.transpose(2, 3) @ rows(q))),
              group(((u + EPS) * p + (tiny if t == torch.float16 else 0) * m).transpose(2, 3) @ rows(do)))
    for name, got, val, bound in zip(("dq", "dk", "dv"), out, grads, bounds):
        within(got, val, bound + u * val.abs() + tiny, name)
    lone = ~m.any(-1).expand(B, H, Sq)
    assert not o.transpose(1, 2)[lone].any() and (lse[lone] == -float("inf")).all() and torch.isfinite(lse[~lone]).all()


@pytest.mark.parametrize("t", HALF)
@pytest.mark.parametrize("D", [1, 8, 33, 64, 80, 96, 128])
def test_attention_widths(P, D, t):
    attention_case(P, 2, 70, 70, 4, 2, D, t, causal=True)


@pytest.mark.parametrize("Sq,Sk", [(1, 1), (1, 63), (1, 1000), (2, 129), (31, 32), (64, 64), (65, 127), (129, 256), (200, 70), (128, 1), (333, 500)])
@pytest.mark.parametrize("causal", [False, True])
def test_attention_lengths(P, Sq, Sk, causal):
    attention_case(P, 1, Sq, Sk, 2, 1, 64, torch.bfloat16, causal=causal)
    attention_case(P, 1, Sq, Sk, 2, 2, 128, torch.float16, causal=causal)


@pytest.mark.parametrize("H,G", [(1, 1), (8, 8), (8, 2), (6, 3), (5, 1)])
def test_attention_shared_heads(P, H, G):
    attention_case(P, 2, 150, 150, H, G, 64, torch.bfloat16, causal=True)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("slopes,cap", [(True, 0.0), (False, 20.0), (True, 5.0)])
def test_attention_scores(P, slopes, cap, D):
    attention_case(P, 1, 190, 190, 3, 3, D, torch.float16, causal=True, slopes=slopes, cap=cap)
    attention_case(P, 2, 100, 140, 2, 1, D, torch.bfloat16, slopes=slopes, cap=cap, scale=0.3)


def test_attention_documents_and_prefixes(P):
    begin, end = P.document_ranges([[100, 3, 0, 250], [400], [1] * 40, []], 400)
    for D in (64, 128):
        attention_case(P, 4, 400, 400, 4, 2, D, torch.bfloat16, begin=begin, end=end)
    begin, end = P.prefix_ranges([0, 1, 200, 300], 300)
    attention_case(P, 4, 300, 300, 2, 2, 64, torch.float16, begin=begin, end=end)


@pytest.mark.parametrize("D", [64, 128])
def test_attention_any_ranges(P, D):
    """Windows, ranges out of bounds and empty ones, in no order at all."""
    g = np.random.Generator(np.random.PCG64(5))
    B, S, Sk = 2, 260, 300
    begin = torch.from_numpy(g.integers(-20, Sk + 20, size=(B, S)).astype(np.int32)).cuda()
    end = begin + torch.from_numpy(g.integers(-3, 90, size=(B, S)).astype(np.int32)).cuda()
    attention_case(P, B, S, Sk, 2, 1, D, torch.bfloat16, begin=begin, end=end)
    attention_case(P, B, S, Sk, 2, 1, D, torch.float16, begin=begin)
    attention_case(P, B, S, Sk, 2, 1, D, torch.float16, end=end, causal=True)
    nothing = torch.zeros_like(begin)
    attention_case(P, B, S, Sk, 2, 1, D, torch.bfloat16, end=nothing)


def test_attention_large_scores(P):
    attention_case(P, 1, 200, 200, 2, 2, 64, torch.bfloat16, std=4.0, scale=0.5)  # scores of hundreds


def test_attention_strides(P):
    for t in HALF:
        attention_case(P, 2, 75, 75, 4, 2, 40, t, causal=True, view=lambda a: strided(a, 8, 0))  # loads as they are
        attention_case(P, 2, 75, 75, 4, 2, 40, t, causal=True, view=lambda a: strided(a, 3, 1))  # packed
        attention_case(P, 2, 75, 75, 4, 2, 40, t, causal=True, view=lambda a: a.transpose(1, 2).contiguous().transpose(1, 2))


def test_attention_without_rows(P):
    q, k = rand(2, 0, 4, 32), rand(2, 5, 4, 32)
    o, lse = P.attention(q, k, k)
    dq, dk, dv = P.attention_backward(o, q, k, k, o, lse)
    assert o.shape == q.shape and not dk.any() and not dv.any()
    q, k = rand(2, 5, 4, 32), rand(2, 0, 4, 32)
    o, lse = P.attention(q, k, k)
    dq, dk, dv = P.attention_backward(q, q, k, k, o, lse)
    assert not o.any() and (lse == -float("inf")).all() and not dq.any() and dk.shape == k.shape


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("poison", [float("nan"), float("inf"), -float("inf")])
def test_attention_padding_that_holds_anything(P, poison, D):
    """Tokens behind the last document are seen by none and see nothing: whatever they hold changes nothing."""
    B, S, H, used = 2, 200, 2, [130, 67]
    begin, end = P.document_ranges([[100, 30], [67]], S)
    q, k, v, do = (rand(B, S, H, D) for _ in range(4))
    results = []
    for value in (0.0, poison):
        for a in (q, k, v, do):
            for b in range(B):
                a[b, used[b]:] = value
        o, lse = P.attention(q, k, v, key_begin=begin, key_end=end)
        results.append((o, lse, *P.attention_backward(do, q, k, v, o, lse, key_begin=begin, key_end=end)))
    assert all(torch.equal(a, b) for a, b in zip(*results)) and all(torch.isfinite(a).all() for a in results[1][2:])


def test_attention_gradient_against_differences(P):
    B, S, H, G, D, t = 1, 40, 4, 2, 16, torch.float16
    q, k, v, do = rand(B, S, H, D, t=t), rand(B, S, G, D, t=t), rand(B, S, G, D, t=t), rand(B, S, H, D, t=t)
    sl = torch.tensor([0.5, 0.25, 0.1, 0.05], device="cuda")
    kind = dict(causal=True, slopes=sl, cap=4.0)
    o, lse = P.attention(q, k, v, **kind)
    grads = P.attention_backward(do, q, k, v, o, lse, **kind)
    m = O.seen(B, S, S, True, None, None, "cuda")
    loss = lambda a: (O.attention(*a, m, D ** -0.5, sl, 4.0)[0] * do.double()).sum()  # noqa: E731
    base = [a.double() for a in (q, k, v)]
    for i, g in enumerate(grads):
        d, h = torch.randn_like(base[i]), 1e-4
        plus, minus = ([a + s * h * d if n == i else a for n, a in enumerate(base)] for s in (1, -1))
        diff = (loss(plus) - loss(minus)) / (2 * h)
        # roundings of p or ds, of o within delta, and of the result
        assert abs((g.double() * d).sum() - diff) <= 6 * U[t] * g.double().norm() * d.norm() + 1e-5


def test_attention_long_keys(P):
    """One query over 70 000 keys whose rows lie far apart: offsets pass 32 bits."""
    Sk, D = 70000, 64
    wide = torch.empty(Sk, 1, 32768, dtype=torch.bfloat16, device="cuda")
    kv = wide[None, :, :, 32768 - 2 * D:]
    kv.copy_(rand(1, Sk, 1, 2 * D))
    k, v, q = kv[..., :D], kv[..., D:], rand(1, 1, 1, D)
    o, _ = P.attention(q, k, v)
    o2, _ = P.attention(q, k.contiguous(), v.contiguous())
    assert torch.equal(o, o2)
    want, p = O.attention(q.double(), k.double(), v.double(), O.seen(1, 1, Sk, False, None, None, "cuda"), D ** -0.5, None, 0.0)
    within(o, want, U[q.dtype] * want.abs() + 2 * (U[q.dtype] + EPS) * (p @ v.double().abs().transpose(1, 2)).transpose(1, 2), "o")


# ---- norms -------------------------------------------------------------------------------------------------
def norm_case(P, T, C, t, pre="layer", post="none", gates=0, alpha=1.0, p=0.0, weights=True, z=True, dxp=True, view=lambda a: a, eps=1e-5):
    u = U[t]
    x, zz = view(rand(T, C, t=t, std=2.0, mean=0.3)), view(rand(T, C, t=t)) if z else None
    vec = lambda on: rand(C, t=t, mean=1.0, std=0.2) if on and weights else None  # noqa: E731
    w, b, pw, pb = vec(True), vec(pre == "layer"), vec(post != "none"), vec(post == "layer")
    gate = rand(gates, C, t=t) if gates else None
    kind = dict(weight=w, bias=b, pre=pre, post=post, post_weight=pw, post_bias=pb, gate=gate, alpha=alpha, p=p, seed=99, offset=5, eps=eps)
    xp, h, saved = P.residual_norm(x, zz, **kind)
    kept = O.keep(T * C, p, 99, 5).view(T, C).cuda() if p else None
    ins = d64(x, zz, w, b, pw, pb, gate)
    X, Z, W, B, PW, PB, GT = ins
    wxp, wh = O.residual_norm(X, Z, W, B, pre, post, PW, PB, GT, alpha, eps, kept)
    within(xp, wxp.detach(), u * wxp.detach().abs() + 1e-5 * (1 + wxp.detach().abs()), "xp")
    within(h, wh.detach(), u * wh.detach().abs() + 1e-4 * (1 + wh.detach().abs()), "h")
    if not z:
        assert xp is x
    dh, dx = view(rand(T, C, t=t)), view(rand(T, C, t=t)) if dxp else None
    got = P.residual_norm_backward(dx, dh, xp, zz, saved, **kind)
    names = ("x", "z", "weight", "bias", "post_weight", "post_bias", "gate")
    use = [(n, a) for n, a in zip(names, ins) if a is not None]
    # the backward pass's input is x' as the forward pass returned it: its value there (narrow rows of nearly equal values have gradients
    # that turn with the rounding of x')
    leaf = xp.double().requires_grad_()
    lh = O.residual_norm(leaf, None, W, B, pre, post, None, None, None, 1.0, eps, None)[1]
    front = {n: torch.autograd.grad(lh, a, dh.double(), retain_graph=True)[0] for n, a in (("xp", leaf), ("weight", W), ("bias", B)) if a is not None}
    d = front["xp"] + (dx.double() if dxp else 0)
    behind = [(n, a) for n, a in use if n not in front]
    front |= dict(zip([n for n, _ in behind], torch.autograd.grad(wxp, [a for _, a in behind], d)))
    want = [front[n] for n, _ in use]
    assert all(got[n] is None for n, a in zip(names, ins) if a is None)
    # results are rounded once, the rest is 32 bits.  2-norms: 4 U and 32-bit sums
    for (n, _), g in zip(use, want):
        err = (got[n].double() - g).norm()
        assert got[n].shape == g.shape and err <= (4 * u + 2e-5) * g.norm() + 1e-6, (n, float(err), float(g.norm()))


@pytest.mark.parametrize("t", HALF + [torch.float32])
@pytest.mark.parametrize("C", [2, 7, 64, 100, 512, 513, 1000, 2048, 2051, 4096, 5000, 8192, 12288, 16384])
def test_norm_widths(P, C, t):
    norm_case(P, 37, C, t)
    norm_case(P, 37, C, t, pre="rms", post="layer", gates=1, alpha=0.5, p=0.25)


@pytest.mark.parametrize("pre", ["layer", "rms"])
@pytest.mark.parametrize("post", ["none", "layer", "rms"])
@pytest.mark.parametrize("gates", [0, 1, 3])
def test_norm_kinds(P, pre, post, gates):
    for t, p in ((torch.float32, 0.0), (torch.bfloat16, 0.1)):
        norm_case(P, 60, 200, t, pre=pre, post=post, gates=gates, p=p)
        norm_case(P, 60, 200, t, pre=pre, post=post, gates=gates, p=p, weights=False, alpha=0.7)


@pytest.mark.parametrize("T", [1, 2, 5, 511, 513, 3000])
def test_norm_rows(P, T):
    norm_case(P, T, 264, torch.float32)
    norm_case(P, T, 264, torch.float32, post="rms", gates=T)  # a gate per row: past 512 of them a workgroup has whole gates


def test_norm_alone_strides_and_no_gradient_of_the_stream(P):
    norm_case(P, 30, 136, torch.bfloat16, z=False)
    norm_case(P, 30, 136, torch.float32, z=False, dxp=False)
    norm_case(P, 30, 136, torch.float16, view=lambda a: strided(a, 8, 0))
    norm_case(P, 30, 136, torch.float16, view=lambda a: strided(a, 3, 1), p=0.5)


def test_norm_without_rows(P):
    x, w = rand(0, 64), rand(64)
    xp, h, saved = P.residual_norm(x, x, weight=w)
    d = P.residual_norm_backward(x, x, xp, x, saved, weight=w)
    assert h.shape == (0, 64) and d["x"].shape == (0, 64) and not d["weight"].any()


def test_norm_gradient_against_differences(P):
    T, C = 12, 48
    x, z, w, b, pw, gate = rand(T, C, t=torch.float32), rand(T, C, t=torch.float32), *(rand(C, t=torch.float32) for _ in range(3)), rand(2, C, t=torch.float32)
    kind = dict(weight=w, bias=b, post="rms", post_weight=pw, gate=gate, alpha=0.5, p=0.25, seed=3)
    xp, h, saved = P.residual_norm(x, z, **kind)
    dxp, dh = rand(T, C, t=torch.float32), rand(T, C, t=torch.float32)
    got = P.residual_norm_backward(dxp, dh, xp, z, saved, **kind)
    kept = O.keep(T * C, 0.25, 3, 0).view(T, C).cuda()

    def loss(a):
        xp, h = O.residual_norm(a["x"], a["z"], a["weight"], a["bias"], "layer", "rms", a["post_weight"], None, a["gate"], 0.5, 1e-5, kept)
        return (xp * dxp.double()).sum() + (h * dh.double()).sum()

    base = {n: a.double() for n, a in dict(x=x, z=z, weight=w, bias=b, post_weight=pw, gate=gate).items()}
    for n, a in base.items():
        d = torch.randn_like(a)
        diff = (loss({**base, n: a + 1e-5 * d}) - loss({**base, n: a - 1e-5 * d})) / 2e-5
        assert abs((got[n].double() * d).sum() - diff) <= 1e-5 * got[n].double().norm() * d.norm() + 1e-5, n


def test_norm_of_large_means(P):
    """The deviation is taken from the mean: a mean of 1000 with a spread of 1 keeps its digits."""
    x = rand(20, 1000, t=torch.float32, mean=1000.0)
    _, h, _ = P.residual_norm(x)
    want = O.norm(x.double(), "layer", 1e-5)
    within(h, want, 2e-4 * torch.ones_like(want), "h")  # 1000 * 2^-24 a value and three times that in the mean, over a deviation of 1


# ---- dropout -----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("t", HALF + [torch.float32])
@pytest.mark.parametrize("n,offset", [(1, 0), (7, 1), (8, 2), (1000, 3), (4096, 4), (100003, (1 << 32) + 5), (2048 * 4096 + 3, 0)])
def test_dropout(P, n, offset, t):
    x = rand(n, t=t)
    for p in (0.0, 0.1, 0.5):
        y = P.dropout(x, p, 1234567, offset)
        want = x.double() * O.keep(n, p, 1234567, offset).cuda()
        within(y, want, 2 * U[t] * want.abs() + TINY[t] * (want != 0), "y")  # the scale and the product are rounded
        assert torch.equal(y == 0, want == 0) or p == 0
    assert torch.equal(P.dropout(x, 0.0, 1), x)
    again = x.clone()
    assert P.dropout(again, 0.5, 1234567, offset, out=again) is again and torch.equal(again, P.dropout(x, 0.5, 1234567, offset))


def test_dropout_share_and_the_norms_mask(P):
    n = 1 << 20
    ones = torch.ones(n, device="cuda")
    for p in (0.1, 0.5):
        kept = (P.dropout(ones, p, 42) != 0).float().mean().item()
        assert abs(kept - (1 - p)) < 6 * (p * (1 - p) / n) ** 0.5  # six deviations of a fair draw
    # the norm's dropout is this one, element by element of its rows, odd widths included
    T, C = 50, 333
    x, z = torch.zeros(T, C, device="cuda"), rand(T, C, t=torch.float32)
    xp, _, _ = P.residual_norm(x, z, p=0.3, seed=8, offset=77)
    assert torch.equal(xp, P.dropout(z, 0.3, 8, 77))


# ---- streams, graphs, order, refusals ---------------------------------------------------------------------
def layer_pass(P, x, w1, b1, w2, nw, nb, begin, end, dy):
    """One of everything, forward and backward."""
    B, S, C = x.shape
    _, h, s0 = P.residual_norm(x, weight=nw, bias=nb)
    q = h.view(B, S, 4, C // 4)
    o, lse = P.attention(q, q, q, key_begin=begin, key_end=end)
    a, za = P.linear(o.view(B, S, C), w1, b1, act="gelu_tanh", keep=True)
    z = P.linear(a, w2)
    xp, y, s1 = P.residual_norm(x, z, weight=nw, bias=nb, p=0.1, seed=5)
    d = P.residual_norm_backward(None, dy, xp, z, s1, weight=nw, bias=nb, p=0.1, seed=5)
    da, dw2, _ = P.linear_backward(d["z"], a, w2, need=("x", "w"))
    do, dw1, db1 = P.linear_backward(da, o.view(B, S, C), w1, za, act="gelu_tanh")
    dq, dk, dv = P.attention_backward(do.view(q.shape), q, q, q, o, lse, key_begin=begin, key_end=end)
    g = P.residual_norm_backward(d["x"], (dq + dk + dv).view(B, S, C), x, None, s0, weight=nw, bias=nb)
    return y, g["x"], g["weight"], dw1, db1, dw2, d["weight"], P.dropout(y, 0.2, 9)


def layer_inputs(P, B=2, S=130, C=256):
    begin, end = P.document_ranges([[70, 50], [S]], S)
    return (rand(B, S, C), rand(512, C, std=C ** -0.5), rand(512), rand(C, 512, std=512 ** -0.5), rand(C, mean=1.0), rand(C), begin, end, rand(B, S, C))


def test_other_streams_and_every_run_alike(P):
    args = layer_inputs(P)
    want = layer_pass(P, *args)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = [layer_pass(P, *args) for _ in range(3)]
    side.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, want))


def test_captured_in_a_graph(P):
    args = layer_inputs(P)
    layer_pass(P, *args)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer_pass(P, *args)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer_pass(P, *args)
    for k in range(4):
        args[0].copy_(rand(*args[0].shape))
        want = [a.clone() for a in layer_pass(P, *args)]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), k


def test_refusals(P):
    x, w = rand(8, 16), rand(4, 16)
    bad = [lambda: P.linear(x, rand(4, 15)), lambda: P.linear(x.float(), w.float()), lambda: P.linear(x, w.half()), lambda: P.linear(x.cpu(), w.cpu()),
           lambda: P.linear(x, w, act="tanh"), lambda: P.linear(x, w, rand(5)), lambda: P.linear(x, w, residual=rand(7, 4)),
           lambda: P.linear(x.t().contiguous().t(), w), lambda: P.linear_backward(rand(8, 4), x, w, act="gelu"), lambda: P.linear_backward(rand(7, 4), x, w),
           lambda: P.linear_backward(rand(8, 4), x, w, need=("q",)), lambda: P.dropout(x, 1.0, 1), lambda: P.dropout(x[:, ::2], 0.1, 1),
           lambda: P.dropout(x, 0.1, 1, out=rand(8, 15)), lambda: P.residual_norm(x, rand(8, 15)), lambda: P.residual_norm(x, pre="none"),
           lambda: P.residual_norm(x, p=0.1), lambda: P.residual_norm(x, x, post_weight=rand(16)), lambda: P.residual_norm(x, x, gate=rand(3, 16)),
           lambda: P.residual_norm(x, x, weight=rand(15)), lambda: P.residual_norm(rand(2, 16385))]
    q, k = rand(1, 8, 4, 16), rand(1, 8, 3, 16)
    i32 = torch.zeros(1, 8, dtype=torch.int32, device="cuda")
    bad += [lambda: P.attention(q, k, k), lambda: P.attention(q, q, q[:, :7]), lambda: P.attention(q, q, q, scale=0), lambda: P.attention(q, q, q, cap=-1.0),
            lambda: P.attention(q, q, q, key_begin=i32.long()), lambda: P.attention(q, q, q, key_end=i32[:, :7]), lambda: P.attention(q, q, q, slopes=torch.ones(3, device="cuda")),
            lambda: P.attention(rand(1, 8, 4, 129), rand(1, 8, 4, 129), rand(1, 8, 4, 129)), lambda: P.attention(q.float(), q.float(), q.float()),
            lambda: P.attention(q.transpose(2, 3), q.transpose(2, 3), q.transpose(2, 3))]
    for n, call in enumerate(bad):
        with pytest.raises((ValueError, RuntimeError)):
            call()
            pytest.fail(f"call {n} was not refused")
