"""The operators of a transformer layer where values are extreme, masked or missing."""
import pytest
import torch

from layer_oracle import TINY, U, within
from test_gpu_layer import HALF, P, attention_case, linear_case, norm_case, rand, tell  # noqa: F401
from test_layer_sizes import LARGE

pytestmark = pytest.mark.gpu


def ranges(B, S, spans):
    """key_begin, key_end [B, S] from (first query, behind the last, first key, behind the last); the others see nothing."""
    begin, end = torch.zeros(2, B, S, dtype=torch.int32)
    for q0, q1, k0, k1 in spans:
        begin[:, q0:q1], end[:, q0:q1] = k0, k1
    return begin.cuda(), end.cuda()


# ---- attention: keys between the ranges of a tile's queries ---------------------------------------------------
PADDED = [(0, 40, 0, 40), (64, 100, 64, 100), (128, 190, 128, 190), (192, 193, 192, 193), (256, 300, 256, 300)]  # documents, each padded to 64s
SCATTERED = [(0, 1, 3, 4), (1, 2, 290, 300), (2, 5, 70, 71), (5, 130, 128, 160), (130, 300, 0, 300)]  # holes of any size; a tile that sees all
LONE = [(17, 18, 100, 101), (200, 201, 63, 65)]  # hardly anything seen at all


@pytest.mark.parametrize("spans", [PADDED, SCATTERED, LONE])
@pytest.mark.parametrize("D", [64, 80, 128])
@pytest.mark.parametrize("poison", [float("nan"), float("inf"), -float("inf")])
def test_attention_keys_that_no_query_of_a_tile_sees(P, poison, D, spans):
    B, S, H, G = 2, 300, 4, 2
    begin, end = ranges(B, S, spans)
    if spans is SCATTERED:  # the second tile's queries see everything: the first's alone
        begin[:, 128:], end[:, 128:] = 0, 0
    seen = torch.zeros(S, dtype=torch.bool, device="cuda")
    for b, e in zip(begin[0].tolist(), end[0].tolist()):
        seen[b:e] = True
    sees = (end > begin)[0]
    for t in HALF:
        q, do = rand(B, S, H, D, t=t), rand(B, S, H, D, t=t)
        k, v = rand(B, S, G, D, t=t), rand(B, S, G, D, t=t)
        results = []
        for value in (0.0, poison):
            for a in (k, v):
                a[:, ~seen] = value
            for a in (q, do):
                a[:, ~sees] = value
            for kind in ({}, dict(causal=True, slopes=torch.full((H,), 0.1, device="cuda"), cap=9.0)):
                o, lse = P.attention(q, k, v, key_begin=begin, key_end=end, **kind)
                results.append((o, lse, *P.attention_backward(do, q, k, v, o, lse, key_begin=begin, key_end=end, **kind)))
        for clean, dirty in zip(results[:2], results[2:]):
            assert all(torch.equal(a, b) for a, b in zip(clean, dirty)) and all(torch.isfinite(a).all() for a in (dirty[0], *dirty[2:]))
            assert not dirty[3][:, ~seen].any() and not dirty[4][:, ~seen].any() and not dirty[0][:, ~sees].any() and not dirty[2][:, ~sees].any()


@pytest.mark.parametrize("spans", [PADDED, SCATTERED, LONE])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_ranges_with_holes(P, D, spans):
    begin, end = ranges(1, 300, spans)
    attention_case(P, 1, 300, 300, 4, 2, D, torch.bfloat16, begin=begin, end=end)
    attention_case(P, 1, 300, 300, 2, 2, D, torch.float16, begin=begin, causal=True, slopes=True)


# ---- NaN in, NaN out ----------------------------------------------------------------------------------------
@pytest.mark.parametrize("t", HALF + [torch.float32])
@pytest.mark.parametrize("C", [64, 1000, 9000])
def test_norm_gradients_of_a_row_that_holds_a_nan(P, C, t):
    """xhat of the row is NaN in every column: so are the weights' gradients, which add it up; other rows do not see it."""
    T, bad = 5, 2
    x, z, w, pw, dh = rand(T, C, t=t), rand(T, C, t=t), rand(C, t=t, mean=1.0), rand(C, t=t, mean=1.0), rand(T, C, t=t)
    for pre in ("rms", "layer"):
        kind = dict(weight=w, pre=pre)
        _, _, saved = P.residual_norm(x, **kind)
        clean = P.residual_norm_backward(None, dh, x, None, saved, **kind)
        y = x.clone()
        y[bad, C // 3] = float("nan")
        _, h, saved = P.residual_norm(y, **kind)
        d = P.residual_norm_backward(None, dh, y, None, saved, **kind)
        assert torch.isnan(h[bad]).all() and torch.isnan(d["x"][bad]).all() and torch.isnan(d["weight"]).all()
        rest = [i for i in range(T) if i != bad]
        assert torch.equal(d["x"][rest], clean["x"][rest])
    for post in ("rms", "layer"):  # the norm behind the block alone: the stream stays finite
        kind = dict(weight=w, post=post, post_weight=pw)
        xp, _, saved = P.residual_norm(x, z, **kind)
        y = z.clone()
        y[bad, C // 3] = float("nan")
        d = P.residual_norm_backward(None, dh, xp, y, saved, **kind)
        assert torch.isnan(d["post_weight"]).all() and torch.isnan(d["z"][bad]).all() and torch.isfinite(d["weight"]).all()


@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
def test_linear_gradients_of_a_nan(P, act):
    x, w, z, dy = rand(3, 16), rand(24, 16), rand(3, 24), rand(3, 24)
    z[1, 5] = float("nan")
    dx, dw, db = P.linear_backward(dy, x, w, z, act=act)
    assert torch.isnan(dx[1]).all() and torch.isfinite(dx[[0, 2]]).all()
    assert torch.isnan(dw[5]).all() and torch.isnan(db[5]) and int(torch.isnan(db).sum()) == 1


# ---- activations where z is large ---------------------------------------------------------------------------
@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("t", HALF)
def test_slope_where_it_is_constant(P, act, t):
    """1 above, 0 below, as far as z goes: float16 stores a z beyond 65504 as an infinity."""
    big = torch.tensor([200.0, 60000.0, float("inf")] + ([1e13, 1e20, 3e38] if t == torch.bfloat16 else []), device="cuda").to(t)
    z = torch.cat([big, -big])[None]
    dy, x, w = torch.full_like(z, 3.0), rand(1, 8, t=t), rand(z.shape[1], 8, t=t)
    assert P.linear_backward(dy, x, w, z, act=act)[2].tolist() == [3.0] * len(big) + [0.0] * len(big)


@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
def test_linear_whose_z_passes_float16(P, act):
    x, w = rand(4, 16, t=torch.float16), rand(24, 16, t=torch.float16)
    x[:, 0], w[:, 0] = 1000.0, torch.where(torch.arange(24) % 2 == 0, -100.0, 0.0).cuda()
    y, z = P.linear(x, w, act=act, keep=True)
    assert torch.isinf(z[:, ::2]).all() and not y[:, ::2].any()
    dy = rand(4, 24, t=torch.float16)
    for got in P.linear_backward(dy, x, w, z, act=act):
        assert torch.isfinite(got).all()


@pytest.mark.parametrize("t", HALF)
def test_gelu_keeps_its_digits(P, t):
    """Values and slopes relative to themselves, far into the tail: products of one term, so that z is exact."""
    z = torch.cat([torch.linspace(-6, 6, 777), torch.linspace(-12, -6, 100) if t == torch.bfloat16 else torch.zeros(0)]).cuda().to(t)
    one = torch.ones(1, 1, device="cuda", dtype=t)
    y = P.linear(z[:, None], one, act="gelu")[:, 0]
    Z = z.double()
    phi = 0.5 * torch.special.erfc(-Z * 0.5 ** 0.5)
    # the argument's rounding: 2 a^2 2^-23 of erfc(a), a <= 8.5; the rest a few units of 2^-23
    within(y, Z * phi, (U[t] + 1e-4) * (Z * phi).abs() + TINY[t], "y")
    slope = P.linear_backward(torch.ones_like(z)[None], one, z[:, None], z[None], act="gelu")[2]
    bell = Z * torch.exp(-0.5 * Z * Z) / (2 * torch.pi) ** 0.5
    within(slope, phi + bell, U[t] * (phi + bell).abs() + 1e-4 * (phi + bell.abs()) + TINY[t], "slope")


# ---- sizes that reach every launch --------------------------------------------------------------------------
@pytest.mark.parametrize("t", HALF)
@pytest.mark.parametrize("T,N,K", LARGE)
def test_linear_tiles(P, T, N, K, t):
    linear_case(P, T, N, K, "silu" if t == torch.bfloat16 else "none", t)


@pytest.mark.parametrize("H,D", [(16, 64), (24, 128), (16, 80)])
@pytest.mark.parametrize("Sq,Sk", [(130, 130), (20, 130), (33, 200), (200, 33)])
def test_attention_heads_that_share_keys_in_one_workgroup(P, H, D, Sq, Sk):
    """From 256 workgroups of keys on, one goes through all heads that share them: teams on different heads where a head has one tile."""
    B, G = 32, 8
    assert B * G * -(-Sk // 128) >= 256 and H > G
    attention_case(P, B, Sq, Sk, H, G, D, torch.bfloat16, causal=True)
    attention_case(P, B, Sq, Sk, H, G, D, torch.float16, slopes=True, cap=7.0)
    begin, end = ranges(B, Sq, [(0, 9, 0, 9), (12, 17, 5, 30)] + ([(40, 130, 20, 130), (150, 200, 0, 33)] if Sq > 33 else []))
    attention_case(P, B, Sq, Sk, H, G, D, torch.bfloat16, begin=begin, end=end)


@pytest.mark.parametrize("T,C", [(8300, 130), (8200, 1000), (2100, 1500), (2100, 4000), (900, 4500), (900, 8200), (800, 12296)])
def test_norm_of_more_rows_than_workgroups(P, T, C):
    for t in HALF + [torch.float32]:
        norm_case(P, T, C, t)
        norm_case(P, T, C, t, pre="rms", post="layer", gates=2, alpha=0.5, p=0.25)
    norm_case(P, T, C, torch.bfloat16, post="rms", gates=T // 2)


def test_linear_of_long_rows(P):
    """Rows of 2^24 - 8 values: offsets within a tile up to the buffer's end, all three products."""
    T, N, K, t = 3, 64, (1 << 24) - 8, torch.bfloat16
    x, w, dy = rand(T, K, t=t), rand(N, K, t=t), rand(T, N, t=t)
    y = P.linear(x, w)
    dx, dw, _ = P.linear_backward(dy, x, w, need=("x", "w"))
    want = torch.zeros(T, N, device="cuda", dtype=torch.float64)
    for k in range(0, K, 1 << 20):
        xs, ws = x[:, k: k + (1 << 20)].double(), w[:, k: k + (1 << 20)].double()
        want += xs @ ws.t()
        for got, val, terms in ((dx, dy.double() @ ws, N), (dw, dy.double().t() @ xs, T)):
            within(got[:, k: k + (1 << 20)], val, U[t] * val.abs() + 1e-5 * terms, "dx" if got is dx else "dw")
    # 32-bit sums of n = 2^24 terms of deviation 1 in 32 parts: partial sums of some 1000 are rounded by 3e-5, n / 32 times a part, at random
    within(y, want, U[t] * want.abs() + 1.0, "y")


def test_attention_of_expanded_inputs(P):
    """Keys and values that all sequences (or heads) share through strides of 0: results and gradients are those of their copies."""
    B, S, H, D = 3, 150, 4, 64
    for t, one in ((torch.bfloat16, (1, S, 2, D)), (torch.float16, (B, S, 1, D))):
        q, do, k, v = rand(B, S, H, D, t=t), rand(B, S, H, D, t=t), rand(*one, t=t).expand(B, S, 2, D), rand(*one, t=t).expand(B, S, 2, D)
        results = []
        for a, b in ((k, v), (k.contiguous(), v.contiguous())):
            o, lse = P.attention(q, a, b, causal=True)
            results.append((o, lse, *P.attention_backward(do, q, a, b, o, lse, causal=True)))
        assert all(torch.equal(a, b) for a, b in zip(*results))
        with pytest.raises(RuntimeError):
            P.attention_backward(do, q, k, v, *results[0][:2], causal=True, out=(torch.empty_like(q), k.clone().expand(B, S, 2, D), torch.empty(one, dtype=t, device="cuda").expand(B, S, 2, D)))
