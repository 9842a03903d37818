"""The operators of a layer with experts against their plain 64-bit forms: choices and ties, values, gradients (against the formula's by
differentiation and against differences), rows that are nobody's, strides, numbers out of range, streams, graphs, refusals."""
import math

import pytest
import torch

import expert_oracle as X
import layer_oracle as O
from layer_oracle import EPS, TINY, U, within

pytestmark = pytest.mark.gpu
HALF = [torch.bfloat16, torch.float16]
ALL = HALF + [torch.float32]


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


# ---- routing -----------------------------------------------------------------------------------------------
def route_case(P, logits, k, score="softmax", bias=None, groups=1, keep=1, best=2, renormalize=True, scale=1.0):
    T = logits.shape[0]
    kind = dict(score=score, renormalize=renormalize, scale=scale)
    experts, w = P.route(logits, k, bias=bias, groups=groups, keep_groups=keep, group_best=best, **kind)
    l = logits.double().cpu()  # noqa: E741
    want = X.choose(l, k, score, None if bias is None else bias.double().cpu(), groups, keep, best)
    assert experts.dtype == torch.int32 and torch.equal(experts.cpu().long(), want)
    leaf = l.clone().requires_grad_()
    v = X.weights(leaf, want, score, renormalize, scale)
    # two exponentials of arguments rounded to 32 bits (|l| 2^-24 each, at most 60 2^-24 where the score is not lost), a sum, a division
    within(w.cpu(), v.detach(), 1e-5 * v.detach().abs() + 1e-30, "weights")
    dw = rand(T, k, t=torch.float32)
    d = P.route_backward(dw, logits, experts, **kind)
    if not T:
        return
    g = torch.autograd.grad(v, leaf, dw.double().cpu())[0]
    g = torch.where(l == -math.inf, 0.0, g)
    # differences of products of such scores, each with the sizes of what is subtracted
    s = X.scores(l, score)
    most = (torch.gather(s, 1, want) * dw.double().cpu().abs()).sum(1, keepdim=True) if not renormalize and score == "softmax" else None
    p = X.weights(l, want, score, renormalize, 1.0) if renormalize else None
    size = torch.zeros_like(l)
    if most is not None:
        size = s * most + torch.zeros_like(l).scatter_(1, want, torch.gather(s, 1, want) * dw.double().cpu().abs())
    elif renormalize:
        size.scatter_(1, want, p * (dw.double().cpu().abs() + (p * dw.double().cpu().abs()).sum(1, keepdim=True)))
    else:
        size.scatter_(1, want, torch.gather(s * (1 - s), 1, want) * dw.double().cpu().abs())
    t = logits.dtype
    within(d.cpu(), g, U[t] * g.abs() + 2e-5 * abs(scale) * size + TINY[t], "dlogits")


@pytest.mark.parametrize("t", ALL)
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 8, 2), (3, 5, 5), (70, 60, 5), (33, 64, 8), (9, 255, 7), (5, 1024, 64), (130, 130, 1), (0, 8, 2)])
def test_route_sizes(P, T, E, k, t):
    for score in ("softmax", "sigmoid"):
        for renormalize in (True, False):
            route_case(P, rand(T, E, t=t, std=2.0), k, score, renormalize=renormalize, scale=1.0 if renormalize else 2.5)


@pytest.mark.parametrize("groups,per,keep,k", [(2, 2, 1, 2), (4, 8, 2, 6), (8, 32, 4, 8), (3, 5, 2, 4), (5, 15, 5, 20), (64, 16, 3, 9), (33, 31, 7, 12), (6, 1, 4, 3)])
def test_route_groups_and_bias(P, groups, per, keep, k):
    E = groups * per
    for t in ALL:
        for score in ("softmax", "sigmoid"):
            for best in (1, 2):
                bias = rand(E, t=torch.float32, std=0.2)
                route_case(P, rand(20, E, t=t), k, score, bias, groups, keep, best, scale=2.5)
                route_case(P, rand(20, E, t=t), k, score, None, groups, keep, best, renormalize=False)
    route_case(P, rand(20, E, t=torch.float32), min(k, E), "sigmoid", rand(E, t=torch.float32))


def test_route_ties_go_to_the_first(P):
    for t in ALL:
        for groups, keep in ((1, 1), (4, 2)):
            for score in ("softmax", "sigmoid"):
                l = torch.randint(0, 3, (64, 32), device="cuda").to(t)  # noqa: E741  many equal ones, sums of equal ones too
                route_case(P, l, 6, score, None, groups, keep)
                route_case(P, l, 6, score, torch.zeros(32, device="cuda"), groups, keep)
        zero = torch.zeros(4, 16, device="cuda", dtype=t)
        zero[:, ::2] = -0.0
        assert P.route(zero, 3)[0].tolist() == [[0, 1, 2]] * 4


def test_route_closed_experts_and_lowest_values(P):
    for t in ALL:
        l = rand(40, 24, t=t)  # noqa: E741
        l[torch.rand(40, 24, device="cuda") < 0.4] = -math.inf
        l[5], l[6, :23], l[7, 1:] = -math.inf, -math.inf, torch.finfo(t).min  # none, the last, one and lowest values
        l[8] = torch.finfo(t).min
        l[9, 3:] = -math.inf
        for score in ("softmax", "sigmoid"):
            for renormalize in (True, False):
                route_case(P, l, 4, score, renormalize=renormalize)
                route_case(P, l, 4, score, rand(24, t=torch.float32), renormalize=renormalize)
                route_case(P, l, 4, score, None, 4, 2, renormalize=renormalize)
        experts, w = P.route(l, 4)
        assert experts[5].tolist() == [0, 1, 2, 3] and not w[5].any()
        only = bool(l[6, 23] > -math.inf)  # the draw above may have closed it too
        assert experts[6].tolist() == ([23, 0, 1, 2] if only else [0, 1, 2, 3]) and w[6].tolist() == [float(only), 0, 0, 0]


def test_route_far_logits(P):
    """Scores that are lost in 32 bits: shares of the chosen still have all digits."""
    l = rand(50, 16, t=torch.float32, std=40.0) - 300  # noqa: E741
    route_case(P, l, 3, "sigmoid")
    route_case(P, l, 3, "softmax")
    route_case(P, l + 600, 3, "sigmoid")


def test_route_nan_and_infinity(P):
    l = rand(6, 12, t=torch.float32)  # noqa: E741
    l[0, 3] = l[1, :] = math.nan
    l[2, 4] = math.inf
    experts, w = P.route(l, 2, renormalize=False)
    assert w[0].isnan().all() and w[1].isnan().all() and w[2].isnan().any() and w[3:].isfinite().all()
    assert 3 not in experts[0].tolist() and experts[1].tolist() == [0, 1] and experts[2, 0] == 4
    assert ((experts >= 0) & (experts < 12)).all()
    assert P.route_backward(torch.ones_like(w), l, experts, renormalize=False)[0].isnan().all()
    experts, w = P.route(l, 2, "sigmoid", bias=torch.zeros(12, device="cuda"))
    assert 3 not in experts[0].tolist() and w[0].isfinite().all() and w[1].isnan().all() and experts[2, 0] == 4 and w[2].isfinite().all()
    bias = torch.zeros(12, device="cuda")
    bias[5], bias[7] = math.nan, math.inf
    experts, _ = P.route(l[3:], 12, "sigmoid", bias=bias)
    assert (experts[:, 0] == 7).all() and (experts[:, -1] == 5).all()


@pytest.mark.parametrize("T,E", [(1, 4), (3, 8), (40, 16), (3000, 12), (2, 24), (3000, 24)])
def test_route_every_expert_where_one_is_nan(P, T, E):
    """NaN comes last, and every expert is chosen once: with scores that are compared in 32 bits first, and with logits."""
    for bias in (torch.linspace(-1, 1, E, device="cuda"), None):
        for groups in (1, 4):
            for at in (0, 3, E // 2, E - 1):
                l = rand(T, E, t=torch.float32)  # noqa: E741
                l[:, at] = math.nan
                experts, _ = P.route(l, E, "sigmoid", bias=bias, groups=groups)
                want = X.choose(l.double().cpu(), E, "sigmoid", None if bias is None else bias.double().cpu(), groups, groups, 2)
                assert (experts[:, -1] == at).all() and torch.equal(experts.cpu().long(), want), (groups, at)


@pytest.mark.parametrize("T", [5, 5000])
@pytest.mark.parametrize("at", [0, 3, 6, 7, 15])
def test_route_all_of_a_group_where_one_is_nan(P, T, at):
    l = rand(T, 64, t=torch.float32)  # noqa: E741
    l[:, at::16] = math.nan
    experts, _ = P.route(l, 16, "sigmoid", groups=4, keep_groups=1)
    assert torch.equal(experts.cpu().long(), X.choose(l.double().cpu(), 16, "sigmoid", None, 4, 1, 2)) and (experts[:, -1] % 16 == at).all()


def test_route_strides_shapes_and_gradient_of_several_axes(P):
    l = rand(3, 4, 20, t=torch.float16)  # noqa: E741
    experts, w = P.route(l, 3)
    assert experts.shape == (3, 4, 3) == w.shape
    flat = strided(l.view(12, 20), 9, 3)
    other = P.route(flat, 3)
    assert torch.equal(other[0], experts.view(12, 3)) and torch.equal(other[1], w.view(12, 3))
    dw = rand(3, 4, 3, t=torch.float32)
    assert torch.equal(P.route_backward(dw, l, experts).view(12, 20), P.route_backward(dw.view(12, 3), flat, other[0]))


def test_route_backward_of_choices_out_of_range_and_twice(P):
    l, dw = rand(4, 10, t=torch.float32), rand(4, 3, t=torch.float32)
    experts = torch.tensor([[0, -1, 5], [10, 2, 3], [1, 1, 4], [-2147483648, 2147483647, 9]], dtype=torch.int32, device="cuda")
    for score in ("softmax", "sigmoid"):
        d = P.route_backward(dw, l, experts, score, renormalize=False)
        leaf = l.double().requires_grad_()
        s = torch.softmax(leaf, 1) if score == "softmax" else torch.sigmoid(leaf)
        total = sum(s[t, e] * dw[t, j].double() for t, row in enumerate(experts.tolist()) for j, e in enumerate(row) if 0 <= e < 10)
        within(d, torch.autograd.grad(total, leaf)[0], torch.full_like(leaf, 1e-5), score)


def test_route_gradient_against_differences(P):
    l, dw = rand(16, 24, t=torch.float32), rand(16, 4, t=torch.float32)
    for score in ("softmax", "sigmoid"):
        for renormalize in (True, False):
            experts, _ = P.route(l, 4, score, renormalize=renormalize)
            g = P.route_backward(dw, l, experts, score, renormalize=renormalize).double().cpu()
            loss = lambda x: (X.weights(x, experts.cpu().long(), score, renormalize, 1.0) * dw.double().cpu()).sum()  # noqa: B023, E731
            d = torch.randn(16, 24, dtype=torch.float64)
            diff = (loss(l.double().cpu() + 1e-4 * d) - loss(l.double().cpu() - 1e-4 * d)) / 2e-4
            assert abs((g * d).sum() - diff) <= 1e-4


# ---- pairs in order ----------------------------------------------------------------------------------------
@pytest.mark.parametrize("T,k,of,E,first", [(1, 1, 1, 1, 0), (16, 2, 8, 8, 0), (700, 3, 60, 60, 0), (1024, 1, 7, 7, 0), (1025, 1, 9, 4, 3), (683, 3, 16, 4, 12),
                                            (4096, 2, 8, 8, 0), (5000, 3, 200, 50, 60), (777, 8, 1024, 1024, 0), (3000, 7, 300, 1000, -100), (0, 2, 4, 4, 0)])
def test_rows(P, T, k, of, E, first):
    experts = torch.randint(0, of, (T, k), dtype=torch.int32, device="cuda")
    if T > 10:
        experts[-T // 9:], experts[3, 0] = -1, 2147483647
        experts[5] = of - 1  # the same expert twice by one token
    offsets, rows, place = P.expert_rows(experts, E, first=first)
    want = X.in_order(experts, E, first)
    assert offsets.tolist() == want[0] and rows.tolist() == want[1] and place.reshape(-1).tolist() == want[2] and place.shape == experts.shape


def test_rows_of_many_pairs(P):
    n, E = 3_000_017, 96
    experts = (torch.rand(n, device="cuda") ** 3 * 100).int()
    offsets, rows, place = P.expert_rows(experts, E)
    here = experts < E
    order = torch.sort(torch.where(here, experts, E), stable=True)[1]
    m = int(here.sum())
    assert offsets.tolist() == [0] + torch.cumsum(torch.bincount(experts[here], minlength=E), 0).tolist()
    assert torch.equal(rows[:m], order[:m].int()) and (rows[m:] == -1).all()
    assert torch.equal(place[order[:m]], torch.arange(m, device="cuda", dtype=torch.int32)) and (place[~here] == -1).all()


def test_rows_all_of_one_expert_and_none(P):
    for n in (64, 2048, 2049, 40000):
        offsets, rows, place = P.expert_rows(torch.full((n, 1), 2, dtype=torch.int32, device="cuda"), 5)
        assert offsets.tolist() == [0, 0, 0, n, n, n] and torch.equal(rows, torch.arange(n, device="cuda", dtype=torch.int32)) and torch.equal(place[:, 0], rows)
        offsets, rows, place = P.expert_rows(torch.full((n, 1), 7, dtype=torch.int32, device="cuda"), 5)
        assert not offsets.any() and (rows == -1).all() and (place == -1).all()


# ---- products ----------------------------------------------------------------------------------------------
def division(T, k, E, of=None, skew=0.0):
    """(offsets, rows, place) of tokens that choose among `of` experts, as expert_rows lays them out."""
    of = of or E
    like = torch.rand(T, of) + skew * torch.linspace(1, 0, of)
    experts = torch.argsort(like, 1, descending=True)[:, :k].int()
    o, r, p = X.in_order(experts, E)
    return [torch.tensor(a, dtype=torch.int32, device="cuda").view(s) for a, s in ((o, (E + 1,)), (r, (-1,)), (p, (T, k)))]


def linear_case(P, T, k, E, N, K, act, t, gather=True, of=None, skew=0.0, bias=True, view=lambda a: a, wview=lambda a: a, need=("x", "w", "b")):
    u, tiny = U[t], TINY[t]
    offsets, rows, place = division(T, k, E, of, skew)
    R = T * k
    x, w, b, dy = view(rand(T if gather else R, K, t=t)), wview(rand(E, N, K, t=t, std=K ** -0.5)), rand(E, N, t=t), view(rand(R, N, t=t))
    out, dout = torch.full((R, N), 3.0, dtype=t, device="cuda"), torch.full((R, K), 3.0, dtype=t, device="cuda")
    kind = dict(rows=rows if gather else None, act=act)
    y, z = P.expert_linear(x, w, offsets, b if bias else None, keep=True, out=out, **kind)
    assert y is out and (z is None) == (act == "none")
    dx, dw, db = P.expert_linear_backward(dy, x, w, offsets, z, need=need, out=dout if "x" in need else None, **kind)
    at = offsets.tolist()
    token = (rows.long() // k if gather else torch.arange(R, device="cuda"))[: at[-1]]
    A, W, B = x.double()[token].requires_grad_(), w.double().requires_grad_(), (b if bias else torch.zeros_like(b)).double().requires_grad_()
    Z = torch.cat([A[a:z] @ W[e].t() + B[e] for e, (a, z) in enumerate(zip(at, at[1:]))]) if at[-1] else A @ W[0].t()
    Y = O.act(Z, act)
    m = at[-1]
    mine = lambda v: [v[a:z] for a, z in zip(at, at[1:])]  # noqa: E731
    sums = torch.cat([c.abs() @ W[e].detach().abs().t() + B[e].detach().abs() for e, c in enumerate(mine(A.detach()))])
    within(y[:m], Y.detach(), u * Y.detach().abs() + EPS * sums + tiny, "y")
    assert (y[m:] == 3).all()
    if not m:
        assert all(g is None or not g.any() for g in (dw, db))
        return
    D = dy[:m].double()
    want = torch.autograd.grad(Y, (A, W, B), D)
    Zd = Z.detach().requires_grad_()
    slope = torch.autograd.grad(O.act(Zd, act).sum(), Zd)[0]
    # dz is formed from z rounded (|act''| <= 1.2) and rounded itself, where there is an activation
    dz = (D * slope).abs()
    off = EPS * D.abs() + (0 if act == "none" else u * dz + 1.2 * u * D.abs() * Zd.detach().abs() + tiny)
    if act == "relu":  # a jump of the slope where z rounds to the other side of 0: nothing else
        off = off + D.abs() * (Zd.detach().abs() <= EPS * sums)
    off = off + EPS * dz
    if dx is not None:
        assert dx is dout and (dx[m:] == 3).all()
        bound = torch.cat([o @ W[e].detach().abs() for e, o in enumerate(mine(off))])
        within(dx[:m], want[0], bound + u * want[0].abs() + tiny, "dx")
    if dw is not None:
        bound = torch.stack([o.t() @ a.abs() for o, a in zip(mine(off), mine(A.detach()))])
        within(dw, want[1], bound + u * want[1].abs() + tiny, "dw")
    if db is not None:
        bound = torch.stack([o.sum(0) for o in mine(off)])
        within(db, want[2], bound + u * want[2].abs() + tiny, "db")
    for name, g in (("x", dx), ("w", dw), ("b", db)):
        assert (g is None) == (name not in need)


@pytest.mark.parametrize("t", HALF)
@pytest.mark.parametrize("T,k,E,N,K", [(1, 1, 1, 1, 1), (1, 1, 3, 8, 16), (16, 2, 8, 64, 128), (5, 3, 4, 7, 5), (64, 1, 2, 64, 64), (65, 2, 5, 63, 72), (130, 2, 4, 520, 200),
                                       (300, 3, 70, 40, 24), (33, 8, 128, 24, 40), (700, 2, 3, 130, 33)])
def test_linear_sizes(P, T, k, E, N, K, t):
    for gather in (True, False):
        linear_case(P, T, k, E, N, K, "none", t, gather)
        linear_case(P, T, k, E, N, K, "gelu_tanh", t, gather)


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
def test_linear_activations(P, act):
    for t in HALF:
        linear_case(P, 100, 2, 5, 72, 136, act, t)
        linear_case(P, 100, 2, 5, 72, 136, act, t, bias=False, gather=False)


@pytest.mark.parametrize("T,k,E,N,K", [(1024, 2, 4, 4096, 256), (2000, 1, 3, 4104, 192), (600, 2, 4, 2048, 520)])
def test_linear_large_tiles(P, T, k, E, N, K):
    linear_case(P, T, k, E, N, K, "silu", torch.bfloat16)
    linear_case(P, T, k, E, K, N, "none", torch.bfloat16, gather=False)


@pytest.mark.parametrize("skew", [0.0, 0.3, 1.0])
def test_linear_tiles_left_over(P, skew):
    """More large tiles than compute units: those of the last round have their depth divided among workgroups."""
    linear_case(P, 1024, 2, 4, 8184, 2056, "silu", torch.bfloat16, skew=skew, need=("w",))
    linear_case(P, 1024, 2, 4, 8184, 2056, "none", torch.float16, gather=False, bias=False, skew=skew, need=("b",))
    linear_case(P, 1024, 2, 4, 2056, 8184, "relu", torch.bfloat16, skew=skew, need=("x",))


def test_linear_shares_and_skewed_divisions(P):
    linear_case(P, 120, 3, 4, 72, 64, "silu", torch.bfloat16, of=16)            # most rows are elsewhere
    linear_case(P, 120, 3, 4, 72, 64, "silu", torch.bfloat16, of=16, gather=False)
    linear_case(P, 300, 1, 6, 72, 64, "relu", torch.float16, skew=20.0)          # all of the first expert, others have none
    linear_case(P, 40, 1, 1, 72, 64, "none", torch.float16, of=4000)             # hardly any row
    linear_case(P, 2, 1, 1000, 16, 24, "gelu", torch.bfloat16)


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("T,k,E,N,skew", [(2047, 1, 3, 65, 0.0), (2048, 1, 2, 64, 1.0), (2049, 1, 3, 63, 0.0), (1500, 3, 7, 520, 20.0)])
def test_linear_gradients_on_both_sides_of_few_rows(P, T, k, E, N, skew, act):
    linear_case(P, T, k, E, N, 24, act, torch.bfloat16, skew=skew)
    linear_case(P, T, k, E, N, 24, act, torch.float16, gather=False, skew=skew, need=("b",))


def test_linear_strides_and_parts(P):
    for at in (0, 1):
        linear_case(P, 90, 2, 3, 48, 40, "gelu", torch.float16, view=lambda a: strided(a, 8, at))
        linear_case(P, 90, 2, 3, 48, 40, "gelu", torch.float16, wview=lambda a: strided(a, 8, at))
    wide = lambda a: torch.cat([a, a], 1)[:, : a.shape[1]]  # noqa: E731  experts further apart than their rows say
    linear_case(P, 90, 2, 3, 48, 40, "silu", torch.bfloat16, wview=wide, gather=False)
    for need in (("x",), ("w",), ("b",), ("x", "w"), ("w", "b")):
        linear_case(P, 90, 2, 3, 48, 40, "gelu", torch.bfloat16, need=need)
        linear_case(P, 90, 2, 3, 48, 40, "none", torch.bfloat16, need=need)


def test_results_beside_what_is_read(P):
    """Results in columns of the matrix whose other columns are read."""
    offsets, rows, place = division(40, 1, 3)
    wide, w = rand(40, 16 + 24), rand(3, 24, 16)
    x, want = wide[:, :16], wide.clone()
    y = P.expert_linear(x.clone(), w, offsets)
    assert torch.equal(P.expert_linear(x, w, offsets, out=wide[:, 16:]), y) and torch.equal(wide[:, :16], want[:, :16])
    dx = P.expert_linear_backward(y, x.clone(), w, offsets)[0]
    assert torch.equal(P.expert_linear_backward(wide[:, 16:], x.clone(), w, offsets, out=x)[0], dx) and torch.equal(wide[:, 16:], y)


def test_linear_without_tokens(P):
    w, offsets = rand(3, 16, 24), torch.zeros(4, dtype=torch.int32, device="cuda")
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    for rows in (none, None):
        x = rand(0, 24)
        assert P.expert_linear(x, w, offsets, rows=rows).shape == (0, 16)
        dx, dw, db = P.expert_linear_backward(rand(0, 16), x, w, offsets, rows=rows)
        assert dx.shape == (0, 24) and dw.shape == w.shape and not dw.any() and not db.any()


def test_linear_offsets_rows_and_tokens_out_of_range(P):
    """What an offset or a row says out of range is never an address: such offsets are taken as the nearest in range, such rows as zeros."""
    T, k, E, N, K = 40, 2, 4, 24, 64
    _, rows, _ = division(T, k, E)
    x, w, dy = rand(T, K), rand(E, N, K), rand(T * k, N)
    rows[5], rows[6], rows[79] = -7, T * k, 2147483647
    offsets = torch.tensor([-5, 20, 20, 1 << 30, -1], dtype=torch.int32, device="cuda")  # 20 rows, none, 60, none
    y = P.expert_linear(x, w, offsets, rows=rows, out=torch.full((T * k, N), 3.0, device="cuda", dtype=x.dtype))
    token = rows.long().div(k, rounding_mode="floor")
    bad = (token < 0) | (token >= T)
    a = torch.where(bad[:, None], 0.0, x.double()[token.clamp(0, T - 1)])
    want = torch.cat([a[:20] @ w[0].double().t(), a[20:] @ w[2].double().t()])
    within(y, want, U[x.dtype] * want.abs() + EPS * (a.abs() @ w.double().abs().amax(0).t()) + 1e-30, "y")
    dx, dw, db = P.expert_linear_backward(dy, x, w, offsets, rows=rows)
    assert not dw[1].any() and not dw[3].any() and not db[1].any()
    g = dy.double()[20:].t() @ a[20:]
    within(dw[2], g, U[x.dtype] * g.abs() + EPS * dy.double()[20:].abs().t() @ a[20:].abs() + 1e-30, "dw")
    # offsets that fall: overlapping runs of rows, every access within the arrays
    for bad in ([0, 80, 0, 80, 0], [80, 0, 80, 0, 80], [7, 7, 7, 7, 7], [2147483647, -2147483648, 2147483647, 5, 2]):
        o = torch.tensor(bad, dtype=torch.int32, device="cuda")
        P.expert_linear(x, w, o, rows=rows)
        P.expert_linear_backward(dy, x, w, o, rows=rows)


def test_linear_poison_beside(P):
    """Rows behind the last expert's, and what lies beside the operands' rows, do not enter."""
    T, k, E, N, K = 50, 2, 3, 40, 72
    offsets, rows, _ = division(T, k, E, of=6)
    m = int(offsets[-1])
    x = torch.full((T * k, 104), math.inf, device="cuda", dtype=torch.bfloat16)
    x[:m, :K] = rand(m, K)
    dy = torch.full((T * k, 56), math.nan, device="cuda", dtype=torch.bfloat16)
    dy[:m, :N] = rand(m, N)
    w = rand(E, N, K)
    clean_x, clean_dy = torch.zeros(T * k, K, device="cuda", dtype=x.dtype), torch.zeros(T * k, N, device="cuda", dtype=x.dtype)
    clean_x[:m], clean_dy[:m] = x[:m, :K], dy[:m, :N]
    for act in ("none", "silu"):
        y, z = P.expert_linear(x[:, :K], w, offsets, act=act, keep=True)
        want, wz = P.expert_linear(clean_x, w, offsets, act=act, keep=True)
        assert torch.equal(y[:m], want[:m]) and torch.isfinite(y[:m]).all()
        if z is not None:
            z[m:] = math.nan
        got, ref = (P.expert_linear_backward(a, b, w, offsets, c, act=act) for a, b, c in ((dy[:, :N], x[:, :K], z), (clean_dy, clean_x, wz)))
        assert torch.equal(got[0][:m], ref[0][:m]) and all(torch.equal(a, b) and torch.isfinite(a).all() for a, b in zip(got[1:], ref[1:]))


def test_linear_gradient_against_differences(P):
    T, k, E, N, K, t = 30, 2, 3, 40, 24, torch.float16
    offsets, rows, place = division(T, k, E)
    x, w, b, dy = rand(T, K, t=t), rand(E, N, K, t=t, std=0.2), rand(E, N, t=t), rand(T * k, N, t=t)
    at, token = offsets.tolist(), rows.long() // k
    for act in ("gelu", "gelu_tanh", "silu"):
        _, z = P.expert_linear(x, w, offsets, b, rows=rows, act=act, keep=True)
        dx, dw, db = P.expert_linear_backward(dy, x, w, offsets, z, rows=rows, act=act)
        grads = P.expert_sum(dx, place), dw, db
        loss = lambda a, c, d: sum((O.act(a[token[i:j]] @ c[e].t() + d[e], act) * dy[i:j].double()).sum() for e, (i, j) in enumerate(zip(at, at[1:])))  # noqa: B023, E731
        base = [v.double() for v in (x, w, b)]
        for i, g in enumerate(grads):
            d, h = torch.randn_like(base[i]), 1e-4
            plus, minus = ([v + s * h * d if n == i else v for n, v in enumerate(base)] for s in (1, -1))
            diff = (loss(*plus) - loss(*minus)) / (2 * h)
            # each gradient has the error of two roundings of 16-bit values (z, dz) and its own; x's that of a second sum
            assert abs((g.double() * d).sum() - diff) <= 5 * U[t] * g.double().norm() * d.norm() + 1e-5


# ---- the weighted sum --------------------------------------------------------------------------------------
@pytest.mark.parametrize("t", ALL)
@pytest.mark.parametrize("T,k,C,of", [(1, 1, 1, 4), (16, 2, 2048, 4), (5, 8, 77, 4), (130, 3, 64, 9), (33, 9, 4100, 4), (700, 2, 8, 6), (3, 64, 2056, 64), (0, 2, 16, 4)])
def test_sum(P, T, k, C, of, t):
    E = 4 if k <= 4 else k
    offsets, rows, place = division(T, min(k, of), E, of) if T and k <= of else P.expert_rows(torch.randint(-1, E, (T, k), dtype=torch.int32, device="cuda"), E)
    R, u, tiny = T * k, U[t], TINY[t]
    for view in (lambda a: a, strided):
        y, res, w, d = view(rand(R, C, t=t)), view(rand(T, C, t=t)), rand(T, k, t=torch.float32), view(rand(T, C, t=t))
        for weights, residual in ((w, res), (w, None), (None, res), (None, None)):
            out = P.expert_sum(y, place, weights, residual=residual)
            here = (place >= 0).double()[:, :, None]
            parts = y.double()[place.clamp(min=0).long()] * here if T else y.double().view(0, k, C)
            v = parts * (1 if weights is None else w.double()[:, :, None])
            r = 0 if residual is None else res.double()
            want = v.sum(1) + r
            # k products and k + 1 additions in 32 bits, each rounded by at most 2^-24 of what the sizes add up to, and the result's rounding
            size = v.abs().sum(1) + (0 if residual is None else r.abs())
            within(out, want, u * want.abs() + (2 * k + 1) * 2.0 ** -24 * size + tiny, "out")
        target = torch.full((R, C), 3.0, dtype=t, device="cuda")
        dy, dw = P.expert_sum_backward(d, y, place, w, out=target)
        assert dy is target
        want = torch.full((R, C), 3.0, dtype=torch.float64, device="cuda")
        at = place >= 0
        want[place[at].long()] = (w.double()[:, :, None] * d.double()[:, None])[at]
        within(dy, want, 2 * u * want.abs() + tiny, "dy")
        want = (parts * d.double()[:, None]).sum(2)
        within(dw, want, 2.0 ** -24 * (C + 8) * (parts * d.double()[:, None]).abs().sum(2) + 1e-30, "dweights")
        only = P.expert_sum_backward(d, y, place, w, need=("weights",))
        assert only[0] is None and torch.equal(only[1], dw)
        if T:
            only = P.expert_sum_backward(d, y, place, None, need=("y",))
            assert only[1] is None and torch.equal(only[0][place[at].long()], d[:, None].expand(T, k, C)[at])


@pytest.mark.parametrize("t", ALL)
@pytest.mark.parametrize("C", [9, 17, 33, 72, 136, 264, 300, 513, 700, 1024, 1025])
def test_sum_of_every_number_of_tokens_a_workgroup(P, C, t):
    test_sum(P, 37, 3, C, 9, t)


def test_sum_places_out_of_range(P):
    y, w, d = rand(6, 40), rand(3, 2, t=torch.float32), rand(3, 40)
    place = torch.tensor([[0, -1], [6, 2147483647], [-2147483648, 5]], dtype=torch.int32, device="cuda")
    y[1:5] = math.nan  # nobody's
    out = P.expert_sum(y, place, w)
    assert torch.isfinite(out).all() and not out[1].any()
    target = torch.zeros_like(y)
    _, dw = P.expert_sum_backward(d, y, place, w, out=target)
    assert not target[1:5].any() and dw[1].tolist() == [0, 0] and dw[0, 1] == 0 and dw[2, 0] == 0


# ---- norm and clipping -------------------------------------------------------------------------------------
def tensors(kinds, sizes, std=1.0):
    return [rand(*s, t=kinds[i % len(kinds)], std=std) for i, s in enumerate(sizes)]


SIZES = [(1,), (7, 9), (0,), (32768,), (32769,), (3, 5, 1000), (70001,)]


@pytest.mark.parametrize("kinds", [[t] for t in ALL] + [ALL])
def test_clip(P, kinds):
    for sizes in (SIZES, [(1,)], [(0,), (3,)], [(65,)] * 300, [(2, 2049)] * 113):
        grads = tensors(kinds, sizes)
        before = [g.clone() for g in grads]
        want = math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))
        norm = P.gradient_norm(grads)
        assert norm.shape == () and norm.dtype == torch.float32 and abs(norm.item() - want) <= 2 ** -23 * want
        out = [torch.full_like(g, 5.0) for g in grads]
        got = P.clip_gradients(grads, 0.37 * want, out=out)
        assert torch.equal(got, norm) and all(torch.equal(a, b) for a, b in zip(grads, before))
        factor = 0.37 * want / norm.double().item()
        for g, o in zip(grads, out):
            w = g.double() * factor
            within(o, w, (U[g.dtype] + 4 * 2.0 ** -24) * w.abs() + TINY[g.dtype], "clipped")
        same = P.clip_gradients(grads, 0.37 * want)
        assert torch.equal(same, norm) and all(torch.equal(a, b) for a, b in zip(grads, out))
        P.clip_gradients(before, 1.01 * want + 1e-3)
        grads = tensors(kinds, sizes)
        copy = [torch.full_like(g, 5.0) for g in grads]
        P.clip_gradients(grads, 1e30, out=copy)
        assert all(torch.equal(a, b) for a, b in zip(grads, copy))


def test_clip_by_a_given_norm(P):
    grads = tensors(ALL, SIZES)
    before = [g.clone() for g in grads]
    given = torch.tensor(8.0, device="cuda")
    assert P.clip_gradients(grads, 2.0, norm=given) is given
    assert all(torch.equal(g, b * 0.25) for g, b in zip(grads, before))
    P.clip_gradients(grads, 9.0, norm=given)
    assert all(torch.equal(g, b * 0.25) for g, b in zip(grads, before))


def test_clip_views_off_alignment(P):
    for t in ALL:
        flat = rand(200_003, t=t)
        parts = [flat[1:70_000], flat[70_001: 70_004], flat[70_004: 200_002]]
        want = math.sqrt(sum(float((g.double() ** 2).sum()) for g in parts))
        copy = flat.clone()
        norm = P.clip_gradients(parts, 0.5 * want)
        assert abs(norm.item() - want) <= 2 ** -23 * want
        assert flat[0] == copy[0] and flat[70_000] == copy[70_000] and flat[-1] == copy[-1]
        w = copy.double() * 0.5
        within(flat[1:70_000], w[1:70_000], (U[t] + 4 * 2.0 ** -24) * w[1:70_000].abs() + TINY[t], "part")


def test_norm_of_large_and_small_values(P):
    """Squares beyond the range of 32 bits."""
    for t in (torch.bfloat16, torch.float32):
        for size in (1e30, 1e-30):
            g = rand(5000, t=t) * size
            want = float((g.double() ** 2).sum().sqrt())
            assert abs(P.gradient_norm([g]).item() - want) <= 2 ** -23 * want
            P.clip_gradients([g], size)
            assert abs(float((g.double() ** 2).sum().sqrt()) - size) <= 2 * U[t] * size
    assert P.gradient_norm([torch.zeros(0, device="cuda")]).item() == 0 and P.gradient_norm([torch.zeros(9, device="cuda")]).item() == 0


def test_clip_leaves_what_is_not_finite(P):
    for bad in (math.nan, math.inf, -math.inf):
        a, b = rand(100, t=torch.float32), rand(40_000, t=torch.bfloat16)
        b[39_999] = bad
        before = [a.clone(), b.clone()]
        norm = P.clip_gradients([a, b], 0.1)
        assert not math.isfinite(norm.item()) and torch.equal(a, before[0]) and torch.equal(b[:-1], before[1][:-1])


# ---- all of them together: a block with experts, streams, graphs --------------------------------------------
class Block:
    """Router, two products an expert, weighted sum: forward and backward as a layer runs them."""

    def __init__(self, P, C, F, E, k, t=torch.bfloat16):
        self.P, self.E, self.k = P, E, k
        self.router, self.up, self.down = rand(E, C, t=t, std=C ** -0.5), rand(E, F, C, t=t, std=C ** -0.5), rand(E, C, F, t=t, std=F ** -0.5)
        self.b = rand(E, F, t=t, std=0.1)

    def forward(self, x):
        P = self.P
        logits = P.linear(x, self.router)
        experts, w = P.route(logits, self.k)
        offsets, rows, place = P.expert_rows(experts, self.E)
        u, z = P.expert_linear(x, self.up, offsets, self.b, rows=rows, act="gelu_tanh", keep=True)
        v = P.expert_linear(u, self.down, offsets)
        return P.expert_sum(v, place, w, residual=x), (x, logits, experts, w, offsets, rows, place, u, z, v)

    def backward(self, dout, kept):
        P = self.P
        x, logits, experts, w, offsets, rows, place, u, z, v = kept
        dv, dw = P.expert_sum_backward(dout, v, place, w)
        du, down, _ = P.expert_linear_backward(dv, u, self.down, offsets, need=("x", "w"))
        dx, up, b = P.expert_linear_backward(du, x, self.up, offsets, z, rows=rows, act="gelu_tanh")
        dlogits = P.route_backward(dw, logits, experts)
        dr, router, _ = P.linear_backward(dlogits, x, self.router, need=("x", "w"))
        dx = P.expert_sum(dx, place, residual=dout) + dr
        grads = [router, up, b, down]
        return dx, grads, P.clip_gradients(grads, 1.0)


def test_block_with_experts_against_differentiation(P):
    T, C, F, E, k = 96, 64, 128, 6, 2
    block = Block(P, C, F, E, k)
    x, d = rand(T, C), rand(T, C)
    out, kept = block.forward(x)
    dx, grads, norm = block.backward(d, kept)
    leaf = [a.double().requires_grad_() for a in (x, block.router, block.up, block.b, block.down)]
    A, router, up, b, down = leaf
    w = X.weights(A @ router.t(), kept[2].long(), "softmax", True, 1.0)
    parts = []
    for j in range(k):
        e = kept[2][:, j].long()
        u = O.act(torch.bmm(up[e], A[:, :, None])[:, :, 0] + b[e], "gelu_tanh")
        parts.append(w[:, j, None] * torch.bmm(down[e], u[:, :, None])[:, :, 0])
    want = A + sum(parts)
    near = lambda a, b: (a.double() - b).norm() <= 16 * U[torch.bfloat16] * b.norm()  # noqa: E731  sixteen roundings in a row
    assert near(out, want.detach())
    gx, *gw = torch.autograd.grad(want, leaf, d.double())
    assert near(dx, gx)
    total = math.sqrt(sum(float((g ** 2).sum()) for g in gw))
    assert abs(norm.item() - total) <= 16 * U[torch.bfloat16] * total
    for got, g in zip(grads, gw):
        assert near(got, g / total)


def test_block_captured_and_replayed(P):
    T, C, F, E, k = 300, 64, 96, 5, 2
    block = Block(P, C, F, E, k)
    x, d = rand(T, C), rand(T, C)

    def step():
        out, kept = block.forward(x)
        dx, grads, norm = block.backward(d, kept)
        return [out, dx, *grads, norm]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):  # two graphs, each with workspaces of its own
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = step()
        graphs.append((g, out))
    for i in range(6):
        x.copy_(rand(T, C))
        d.copy_(rand(T, C))
        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        graph, out = graphs[i % 2]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), i


def test_streams_and_repeated_runs_give_the_same_bits(P):
    T, C, F, E, k = 2500, 128, 200, 12, 4
    block = Block(P, C, F, E, k)
    x, d = rand(T, C), rand(T, C)
    out, kept = block.forward(x)
    want = [out, *[t.clone() for t in block.backward(d, kept)[1]]]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    results = []
    for s in streams:
        with torch.cuda.stream(s):
            o, kp = block.forward(x)
            results.append([o, *block.backward(d, kp)[1]])
    torch.cuda.synchronize()
    for r in results:
        assert all(torch.equal(a, b) for a, b in zip(r, want))


# ---- more than 32 bits of elements or bytes --------------------------------------------------------------------
def test_far_rows_of_logits_sums_and_tensors(P):
    E = 1024
    l = torch.zeros(2_100_000, E, dtype=torch.bfloat16, device="cuda")  # noqa: E741  2.1e9 values
    l[-40:] = rand(40, E)
    experts, w = P.route(l, 4)
    last = P.route(l[-40:].clone(), 4)
    assert torch.equal(experts[-40:], last[0]) and torch.equal(w[-40:], last[1]) and experts[0].tolist() == [0, 1, 2, 3]
    d = P.route_backward(torch.ones_like(w), l, experts)
    assert torch.equal(d[-40:], P.route_backward(torch.ones_like(last[1]), l[-40:].clone(), last[0]))
    del d
    y = l.view(-1, 4096)  # 525 000 rows
    place = torch.tensor([[y.shape[0] - 1, 0], [y.shape[0] - 7, -1], [3, y.shape[0] - 2]], dtype=torch.int32, device="cuda")
    weights = rand(3, 2, t=torch.float32)
    rows = y[place.clamp(min=0).long()].double() * weights.double()[:, :, None] * (place >= 0)[:, :, None]
    within(P.expert_sum(y, place, weights), rows.sum(1), U[y.dtype] * rows.sum(1).abs() + 1e-6 * rows.abs().sum(1) + 1e-30, "sum")
    dy, _ = P.expert_sum_backward(rand(3, 4096), y, place, weights, out=torch.zeros_like(y))
    assert dy[-1].any() and dy[-7].any() and dy[-2].any() and not dy[-6:-2].any() and not dy[4:-7].any()
    del dy
    l.fill_(1.0)
    assert abs(P.gradient_norm([l]).item() - l.numel() ** 0.5) <= 1
    P.clip_gradients([l], 0.5 * l.numel() ** 0.5)
    assert float(l[0, 0]) == float(l[-1, -1]) == 0.5 and bool((l == 0.5).all())


def test_tokens_of_more_than_one_launch(P):
    T = (1 << 28) + 5  # eight lanes each
    l = torch.zeros(T, 8, dtype=torch.bfloat16, device="cuda")  # noqa: E741
    l[-40:] = rand(40, 8)
    last = l[-40:].clone()
    experts, w = P.route(l, 8)
    want = P.route(last, 8)
    assert torch.equal(experts[-40:], want[0]) and torch.equal(w[-40:], want[1])
    assert experts[:: 1 << 20][:-1].tolist() == [list(range(8))] * 256 and bool((w[:: 1 << 20][:-1] == 0.125).all())
    dw = torch.zeros_like(w)
    dw[-40:] = rand(40, 8, t=torch.float32)
    d = P.route_backward(dw, l, experts)
    assert torch.equal(d[-40:], P.route_backward(dw[-40:].clone(), last, want[0])) and not d[:-40].any()
    del l, experts, w, dw, d
    T = (1 << 23) + 9  # a workgroup each
    y, weights = rand(4, 1032), torch.ones(T, 1, device="cuda")
    place = torch.zeros(T, 1, dtype=torch.int32, device="cuda")
    place[-40:, 0] = torch.arange(40, device="cuda", dtype=torch.int32) % 4
    weights[-40:] = rand(40, 1, t=torch.float32)
    res = y[:1].expand(T, 1032).contiguous()
    out = P.expert_sum(y, place, weights, residual=res)
    assert torch.equal(out[-40:], P.expert_sum(y, place[-40:].clone(), weights[-40:].clone(), residual=res[-40:].clone())) and torch.equal(out[:: 1 << 15][:-1], (2 * res)[:: 1 << 15][:-1])
    dweights = P.expert_sum_backward(out, y, place, weights, need=("weights",))[1]
    want = P.expert_sum_backward(out[-40:].clone(), y, place[-40:].clone(), weights[-40:].clone(), need=("weights",))[1]
    assert torch.equal(dweights[-40:], want) and bool((dweights[:-40] == dweights[0]).all())


def test_linear_tokens_that_32_bit_offsets_do_not_reach(P):
    T, E, N, K = 1 << 18, 2, 16, 64
    wide = torch.zeros(T, 4104, dtype=torch.bfloat16, device="cuda")  # rows 8208 bytes apart: 2.15 GB
    x = wide[:, :K]
    x.copy_(rand(T, K))
    offsets, rows, _ = P.expert_rows(torch.randint(0, E, (T, 1), dtype=torch.int32, device="cuda"), E)
    w, dy = rand(E, N, K), rand(T, N)
    y, want = P.expert_linear(x, w, offsets, rows=rows), P.expert_linear(x.contiguous(), w, offsets, rows=rows)
    assert torch.equal(y, want)
    got, want = (P.expert_linear_backward(dy, a, w, offsets, rows=rows) for a in (x, x.contiguous()))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    big = torch.zeros(40, N, 4 << 20, dtype=torch.bfloat16, device="cuda")[:, :, :K]       # rows 8 MB apart: copied; experts 128 MB: 5 GB in all
    big.copy_(rand(40, N, K))
    offsets, rows, _ = P.expert_rows(torch.randint(0, 40, (300, 1), dtype=torch.int32, device="cuda"), 40)
    assert torch.equal(P.expert_linear(x[:300], big, offsets, rows=rows), P.expert_linear(x[:300], big.contiguous(), offsets, rows=rows))


# ---- refusals ----------------------------------------------------------------------------------------------
def test_refusals(P):
    l = rand(4, 8)  # noqa: E741
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    x, w, offsets, rows = rand(4, 16), rand(3, 24, 16), i32(4), i32(8)
    y, place, wt, both = rand(8, 24), i32(4, 2), torch.ones(4, 2, device="cuda"), rand(4, 40)
    for call in (lambda: P.route(l, 0), lambda: P.route(l, 9), lambda: P.route(l, 2, "relu"), lambda: P.route(l, 2, groups=3), lambda: P.route(l, 3, groups=4, keep_groups=1),
                 lambda: P.route(l, 2, groups=4, keep_groups=5), lambda: P.route(l, 2, groups=2, group_best=3), lambda: P.route(l.cpu(), 2), lambda: P.route(l.double(), 2),
                 lambda: P.route(l, 2, bias=rand(8)), lambda: P.route(l, 2, bias=torch.zeros(7, device="cuda")), lambda: P.route(l, 2, scale=math.inf), lambda: P.route(l.t(), 2),
                 lambda: P.route(rand(2, 1025), 2), lambda: P.route_backward(wt, l, i32(4, 2).long()), lambda: P.route_backward(wt.half(), l, i32(4, 2)),
                 lambda: P.route_backward(wt[:3], l, i32(4, 2)), lambda: P.expert_rows(i32(4, 2).long(), 4), lambda: P.expert_rows(i32(4, 4)[:, ::2], 4),
                 lambda: P.expert_rows(i32(4, 2), 0), lambda: P.expert_rows(i32(4, 2), 1025), lambda: P.expert_rows(i32(4, 2).cpu(), 4),
                 lambda: P.expert_linear(x, w[0], offsets), lambda: P.expert_linear(x, w, i32(3)), lambda: P.expert_linear(x, w, offsets.long()),
                 lambda: P.expert_linear(x, w.half(), offsets), lambda: P.expert_linear(x.float(), w.float(), offsets), lambda: P.expert_linear(x, w, offsets, rows=i32(7)),
                 lambda: P.expert_linear(x, w, offsets, rows=i32(0)), lambda: P.expert_linear(x, w, offsets, bias=rand(24)), lambda: P.expert_linear(x, w, offsets, act="tanh"),
                 lambda: P.expert_linear(x, w, offsets, out=rand(5, 24)), lambda: P.expert_linear(x, w, offsets, out=rand(1, 24).expand(4, 24)),
                 lambda: P.expert_linear(x, w.transpose(1, 2), offsets), lambda: P.expert_linear(y, w.new_empty(3, 24, 24), offsets, out=y),
                 lambda: P.expert_linear(both[:, :16], w, offsets, out=both[:, 8:32]), lambda: P.expert_linear(x, w, offsets, out=w.view(-1)[16:112].view(4, 24)),
                 lambda: P.expert_linear_backward(y, y, w.new_empty(3, 24, 24), offsets, out=y), lambda: P.expert_sum_backward(rand(4, 24), y, place, wt, out=y), lambda: P.expert_linear(x, rand(1025, 1, 16), i32(1026)),
                 lambda: P.expert_linear_backward(rand(4, 24), x, w, offsets, act="gelu"), lambda: P.expert_linear_backward(rand(5, 24), x, w, offsets),
                 lambda: P.expert_linear_backward(rand(4, 24), x, w, offsets, need=("z",)), lambda: P.expert_linear_backward(rand(4, 24), x, w, offsets, need=("w",), out=rand(4, 16)),
                 lambda: P.expert_sum(y, place.long()), lambda: P.expert_sum(y, place, wt[:3]), lambda: P.expert_sum(y, place, wt.half()),
                 lambda: P.expert_sum(y, place, residual=rand(4, 23)), lambda: P.expert_sum(y.double(), place), lambda: P.expert_sum(y, i32(1, 65)),
                 lambda: P.expert_sum_backward(rand(3, 24), y, place, wt), lambda: P.expert_sum_backward(rand(4, 24), y, place, wt, need=()),
                 lambda: P.expert_sum_backward(rand(4, 24), y, place, wt, need=("weights",), out=y),
                 lambda: P.gradient_norm([]), lambda: P.gradient_norm([l.double()]), lambda: P.gradient_norm([l.cpu()]), lambda: P.gradient_norm([l, rand(4, 4).t()]),
                 lambda: P.clip_gradients([l], -1.0), lambda: P.clip_gradients([l], math.nan), lambda: P.clip_gradients([l], 1.0, norm=torch.ones(2, device="cuda")),
                 lambda: P.clip_gradients([l], 1.0, norm=torch.ones(())), lambda: P.clip_gradients([l, l], 1.0), lambda: P.clip_gradients([l[:2], l[2:]], 1.0, out=[l[2:], l[:2]]),
                 lambda: P.clip_gradients([wt], 1.0, norm=wt[0, 0]), lambda: P.clip_gradients([l[:3], l[2:]], 1.0),
                 lambda: P.clip_gradients([l], 1.0, out=[]), lambda: P.clip_gradients([l], 1.0, out=[l[:3]]), lambda: P.clip_gradients([l], 1.0, out=[l.half()])):
        with pytest.raises(ValueError):
            call()
