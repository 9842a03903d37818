"""Calls of the experts' operators and of clipping at the edges of what their documentation allows: rows of stride 0, results between matrices, norms beyond 32
bits, experts that a bias rules out, results that the larger tests do not look at."""
import ctypes as C
import math

import pytest
import torch

import expert_oracle as X
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


def rand(*shape, t=torch.bfloat16, std=1.0):
    return (torch.randn(*shape, device="cuda") * std).to(t)


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


# ---- rows of stride 0: one row for all ------------------------------------------------------------------------
@pytest.mark.parametrize("K,N", [(64, 48), (33, 47)])
def test_linear_of_one_row_for_all(P, K, N):
    T, k, E = 70, 2, 3
    offsets, rows, _ = P.expert_rows(torch.randint(0, E, (T, k), dtype=torch.int32, device="cuda"), E)
    w = rand(E, N, K)
    for gather in (True, False):
        x, dy = rand(1, K).expand(T if gather else T * k, K), rand(1, N).expand(T * k, N)
        for act in ("none", "silu"):
            kind = dict(rows=rows if gather else None, act=act)
            (y, z), (want, _) = (P.expert_linear(a, w, offsets, keep=True, **kind) for a in (x, x.contiguous()))
            assert torch.equal(y, want)
            got, ref = (P.expert_linear_backward(d, a, w, offsets, z, **kind) for d, a in ((dy, x), (dy.contiguous(), x.contiguous())))
            assert all(torch.equal(a, b) for a, b in zip(got, ref))


def test_route_of_one_row_for_all(P):
    l, dw = rand(1, 20).expand(9, 20), rand(9, 3, t=torch.float32)  # noqa: E741
    experts, w = P.route(l, 3)
    want = P.route(l.contiguous(), 3)
    assert torch.equal(experts, want[0]) and torch.equal(w, want[1])
    assert torch.equal(P.route_backward(dw, l, experts), P.route_backward(dw, l.contiguous(), experts))


@pytest.mark.parametrize("C", [40, 37, 520])
def test_sum_of_one_row_for_all(P, C):
    place, w = torch.randperm(18, device="cuda").int().view(9, 2), rand(9, 2, t=torch.float32)
    for t in ALL:
        y, res, d = rand(1, C, t=t).expand(18, C), rand(1, C, t=t).expand(9, C), rand(1, C, t=t).expand(9, C)
        assert torch.equal(P.expert_sum(y, place, w, residual=res), P.expert_sum(y.contiguous(), place, w, residual=res.contiguous()))
        got, want = P.expert_sum_backward(d, y, place, w), P.expert_sum_backward(d.contiguous(), y.contiguous(), place, w)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


# ---- results in the place of what the call does not read --------------------------------------------------------
def test_gradient_of_y_in_its_place(P):
    """Without the weights' gradient y is not read: its gradient may take its place."""
    place, w = torch.randperm(18, device="cuda").int().view(9, 2), rand(9, 2, t=torch.float32)
    y, d = rand(18, 40), rand(9, 40)
    want = P.expert_sum_backward(d, y, place, w, need=("y",))[0]
    assert P.expert_sum_backward(d, y, place, w, need=("y",), out=y)[0] is y and torch.equal(y, want)
    with pytest.raises(ValueError, match="shares memory"):
        P.expert_sum_backward(d, y, place, w, out=y)


# ---- results between the experts' matrices --------------------------------------------------------------------
@pytest.mark.parametrize("T", [4, 3])
def test_results_between_matrices_far_apart(P, T):
    """Matrices with room between them: what lies in the room shares nothing with them."""
    wide = rand(3, 40, 16)
    w, room = wide[:, :24], wide[1, 24:].reshape(-1)
    x, offsets = rand(T, 16), ints(0, 1, 1, T)
    before = w.clone()
    out = room[8: 8 + T * 24].view(T, 24)
    y = P.expert_linear(x, w, offsets)
    assert P.expert_linear(x, w, offsets, out=out) is out and torch.equal(out, y) and torch.equal(w, before)
    out = room[8: 8 + T * 16].view(T, 16)
    dx = P.expert_linear_backward(y, x, w, offsets, need=("x",))[0]
    assert torch.equal(P.expert_linear_backward(y, x, w, offsets, need=("x",), out=out)[0], dx) and torch.equal(w, before)
    for bad in (wide.view(-1)[16 * 23: 16 * 23 + T * 24].view(T, 24), wide.view(-1)[16 * 40 - T * 24 + 1: 16 * 40 + 1].view(T, 24)):
        with pytest.raises(ValueError, match="shares memory"):
            P.expert_linear(x, w, offsets, out=bad)


# ---- norm and clipping ----------------------------------------------------------------------------------------
def test_clip_leaves_what_has_no_norm_in_32_bits(P):
    """Finite values whose norm passes 32 bits: it is an infinity, and they are left as they are, with the norm given or not."""
    for t in (torch.bfloat16, torch.float32):
        g = torch.full((4,), 3e38, device="cuda", dtype=t)
        before = g.clone()
        assert P.gradient_norm([g]).item() == math.inf
        assert P.clip_gradients([g], 1.0).item() == math.inf and torch.equal(g, before)
        out = torch.zeros_like(g)
        assert P.clip_gradients([g], 1.0, out=[out]).item() == math.inf and torch.equal(out, before)
        P.clip_gradients([g], 1.0, norm=P.gradient_norm([g]))
        assert torch.equal(g, before)


def test_clip_goes_by_the_norm_that_it_returns(P):
    """By its own norm or by the same one given: the same bits, at the bound too."""
    for n in range(1, 200):
        g = [rand(3 * n, t=torch.float32), rand(n, t=torch.bfloat16)]
        norm = P.gradient_norm(g)
        for bound in (0.37 * norm.item(), norm.item()):
            a, b = [torch.zeros_like(v) for v in g], [torch.zeros_like(v) for v in g]
            assert torch.equal(P.clip_gradients(g, bound, out=a), norm)
            P.clip_gradients(g, bound, norm=norm, out=b)
            assert all(torch.equal(u, v) for u, v in zip(a, b)), (n, bound)
        assert all(torch.equal(u, v) for u, v in zip(a, g)), n


def test_clip_by_factors_that_32_bits_hardly_hold(P):
    """max_norm / norm below the smallest normal float: the results are ordinary numbers and keep their digits."""
    for t in ALL[::2]:
        for bound in (1e-3, 1e-10):
            g = rand(5000, t=t, std=3e36)
            before = g.clone()
            norm = P.clip_gradients([g], bound).double().item()
            want = before.double() * (bound / norm)
            # the bound and the norm are rounded to 32 bits, the quotient and the product in 64
            within(g, want, (U[t] + 4 * 2.0 ** -24) * want.abs() + TINY[t], "clipped")


def test_clip_in_place_below_the_bound_changes_nothing(P):
    for t in ALL:
        for sizes in ([1], [70, 40_000], [65] * 300):
            g = [rand(n, t=t) for n in sizes]
            before = [a.clone() for a in g]
            norm = P.clip_gradients(g, 1.01 * float(P.gradient_norm(g)))
            assert all(torch.equal(a, b) for a, b in zip(g, before)) and torch.equal(norm, P.gradient_norm(before))


# ---- z of a product without activation --------------------------------------------------------------------------
@pytest.mark.parametrize("T,E,N,K", [(40, 3, 48, 64), (40, 3, 47, 33), (800, 4, 2048, 72), (2048, 4, 4096, 64), (2048, 4, 8192, 2048)])
def test_z_without_an_activation(P, T, E, N, K):
    """z[r] = x w^T + bias whatever the activation is: tiles of every size, and those whose depth is divided."""
    from paper_2309_08125_amd import expert

    lib = expert._load()
    offsets, rows, _ = P.expert_rows(torch.randint(0, E, (T, 1), dtype=torch.int32, device="cuda"), E)
    x, w, b = rand(T, K), rand(E, N, K, std=K ** -0.5), rand(E, N)
    y, z = torch.full((T, N), 3.0, dtype=x.dtype, device="cuda"), torch.full((T, N), 5.0, dtype=x.dtype, device="cuda")
    p = expert.oob_expert_linear_t(0, 0, E, 1, T, T, N, K, offsets.data_ptr(), rows.data_ptr(), x.data_ptr(), w.data_ptr(), b.data_ptr(), y.data_ptr(), z.data_ptr(),
                                   K, K, N * K, N, N)
    size = lib.oob_expert_linear_workspace_size(C.byref(p))
    ws = torch.empty(max(size, 1), dtype=torch.uint8, device="cuda")
    assert lib.oob_expert_linear(C.byref(p), ws.data_ptr(), size, torch.cuda.current_stream().cuda_stream) == P.OOB_OK
    torch.cuda.synchronize()
    assert torch.equal(y, P.expert_linear(x, w, offsets, b, rows=rows)) and torch.equal(z, y)


# ---- routing ----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("E", [8, 60, 256])
@pytest.mark.parametrize("T", [3, 3000])
def test_closed_experts_come_after_those_that_a_bias_rules_out(P, T, E):
    l = rand(T, E, t=torch.float32)  # noqa: E741
    closed = torch.rand(T, E, device="cuda") < 0.4
    l[closed] = -math.inf
    bias = rand(E, t=torch.float32, std=0.1)
    bias[torch.rand(E, device="cuda") < 0.5] = -math.inf
    k = min(E, 64)
    for score in ("softmax", "sigmoid"):
        experts, w = P.route(l, k, score, bias=bias)
        c = X.scores(l.double().cpu(), score) + bias.double().cpu()
        order = torch.tensor([sorted(range(E), key=lambda e: (bool(closed[t, e]), -float(c[t, e])))[:k] for t in range(min(T, 40))])  # noqa: B023
        order = torch.where(torch.gather(closed[: len(order)].cpu(), 1, order), -1, order)  # which of the closed ones does not count here
        got = experts[: len(order)].cpu().long()
        assert torch.equal(torch.where(torch.gather(closed[: len(order)].cpu(), 1, got), -1, got), order)
        at = torch.gather(closed, 1, experts.long())
        assert bool((at.int().cummax(1).values == at.int()).all()) and not bool(w[at].any())
        # closed ones follow one another by their numbers
        assert bool(((experts[:, 1:] > experts[:, :-1]) | ~at[:, :-1]).all())


@pytest.mark.parametrize("groups,per,keep,k", [(2, 2, 1, 1), (4, 2, 2, 3), (8, 32, 4, 8), (5, 3, 2, 4), (64, 16, 3, 9), (3, 341, 2, 6)])
def test_groups_that_hold_nan_come_after_all_others(P, groups, per, keep, k):
    """What a group's best add up to is NaN where a number is missing, and NaN comes after everything, a group of closed experts included."""
    for t in ALL:
        l = rand(60, groups, per, t=t)  # noqa: E741
        l[torch.rand(60, groups, device="cuda") < 0.3] = -math.inf
        nan = torch.rand(60, groups, device="cuda") < 0.4
        l[:, :, 1:][nan] = math.nan  # one number is left
        l[::7][nan[::7]] = math.nan  # or none
        l = l.view(60, -1)  # noqa: E741
        for best in (1, 2):
            for bias in (None, rand(groups * per, t=torch.float32, std=0.1)):
                experts, _ = P.route(l, k, "sigmoid", bias=bias, groups=groups, keep_groups=keep, group_best=best)
                want = X.choose(l.double().cpu(), k, "sigmoid", None if bias is None else bias.double().cpu(), groups, keep, best)
                assert torch.equal(experts.cpu().long(), want), (t, best)


@pytest.mark.parametrize("groups,per", [(33, 31), (3, 341), (64, 16), (1, 1000)])
def test_scores_closer_than_32_bits_tell(P, groups, per):
    """As many experts in one lane as there can be: scores that differ by less than their errors in 32 bits are compared in 64."""
    E = groups * per
    bias = torch.zeros(E, device="cuda")
    for step in (0.0, 1e-7, 3e-6, 1e-5, 1e-4, 1e-3, 1e-2):  # softmax scores around 1 / E, their differences from none to far beyond the errors
        l = (torch.randn(24, E, device="cuda") * step * E).clamp(-4, 4)  # noqa: E741
        for b in (bias, bias + 1.0, rand(E, t=torch.float32, std=0.2)):
            experts, _ = P.route(l, 7, "softmax", bias=b, groups=groups, keep_groups=max(1, groups // 3), group_best=2)
            want = X.choose(l.double().cpu(), 7, "softmax", b.double().cpu(), groups, max(1, groups // 3), 2)
            assert torch.equal(experts.cpu().long(), want), step


@pytest.mark.parametrize("E", [16, 60, 64, 100, 128, 129, 256, 500, 512, 1024])
def test_route_of_every_number_of_lanes(P, E):
    """As many tokens as fill the GPU, where a token's lanes are known when it is compiled, against the definition and against few tokens."""
    T = 64 * 2048 * 8 // E + 3
    for groups, keep in ((1, 1), (4, 3)):
        if E % groups:
            continue
        for t in ALL:
            l, bias = rand(T, E, t=t), rand(E, t=torch.float32, std=0.1)  # noqa: E741
            l[:: 3, :: 5], l[5, 1] = -math.inf, math.nan
            for score, b, renormalize in (("sigmoid", bias, True), ("softmax", bias, False), ("softmax", None, True)):
                kind = dict(score=score, bias=b, groups=groups, keep_groups=keep, renormalize=renormalize)
                (experts, w), (few, few_w) = P.route(l, 6, **kind), P.route(l[-40:], 6, **kind)
                assert torch.equal(experts[-40:], few)
                within(w[-40:], few_w.double(), 4e-6 * few_w.double().abs() + 1e-30, "weights")
                want = X.choose(l[:40].double().cpu(), 6, score, None if b is None else b.double().cpu(), groups, keep, 2)
                assert torch.equal(experts[:40].cpu().long(), want), (groups, t, score)


# ---- gradients with offsets and rows out of range ------------------------------------------------------------------
def test_dx_where_offsets_and_rows_are_out_of_range(P):
    T, k, E, N, K = 40, 2, 4, 24, 64
    x, w, dy = rand(T, K), rand(E, N, K), rand(T * k, N)
    rows = torch.randperm(T * k, device="cuda").int()
    rows[5], rows[6], rows[79] = -7, T * k, 2147483647
    out = torch.full((T * k, K), 3.0, dtype=x.dtype, device="cuda")
    dx, dw, db = P.expert_linear_backward(dy, x, w, ints(-5, 20, 20, 1 << 30, -1), rows=rows, out=out)
    want = torch.cat([dy[:20].double() @ w[0].double(), dy[20:].double() @ w[2].double()])  # dx goes by the rows of dy alone
    size = torch.cat([dy[:20].double().abs() @ w[0].double().abs(), dy[20:].double().abs() @ w[2].double().abs()])
    within(dx, want, U[x.dtype] * want.abs() + EPS * size + TINY[x.dtype], "dx")
    token = rows[:20].long().div(k, rounding_mode="floor")
    a = torch.where(((token < 0) | (token >= T))[:, None], 0.0, x.double()[token.clamp(0, T - 1)])
    want = dy[:20].double().t() @ a
    within(dw[0], want, U[x.dtype] * want.abs() + EPS * dy[:20].double().abs().t() @ a.abs() + TINY[x.dtype], "dw")
    for e, part in ((0, dy[:20]), (2, dy[20:])):
        want = part.double().sum(0)
        within(db[e], want, U[x.dtype] * want.abs() + EPS * part.double().abs().sum(0) + TINY[x.dtype], "db")
