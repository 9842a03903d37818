"""Host logic of the operators of a layer with experts and of clipping that needs no GPU: exported symbols, refusals, workspace sizes."""
import ctypes as C
import os
import re

import pytest

import paper_2309_08125_amd as P
from paper_2309_08125_amd import expert as X

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000  # never dereferenced: every call below fails its host-side checks or has nothing to do


def lib():
    return X._load()


def make(struct, **kw):
    s = struct()
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def test_library_exports_every_declared_symbol():
    text = open(os.path.join(ROOT, "paper_2309_08125_amd", "include", "oob_expert.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = sorted(set(re.findall(r"\b(oob_(?:expert|clip)_\w+)\s*\(", text)))
    assert names == sorted(P.EXPERT_SYMBOLS) and all(hasattr(lib(), n) for n in names)
    assert f"OOB_EXPERT_MAX {X.MAX_EXPERTS}" in text and f"OOB_EXPERT_MAX_CHOICES {X.MAX_CHOICES}" in text


ROUTE = dict(dtype=0, score=0, renormalize=1, E=16, k=4, groups=4, keep_groups=2, group_best=2, scale=1.0, T=5, logits=FAKE, logits_stride=16, experts=FAKE,
             weights=FAKE)


@pytest.mark.parametrize("bad", [dict(dtype=3), dict(dtype=-1), dict(score=2), dict(renormalize=2), dict(E=0), dict(E=1025, groups=1, logits_stride=1025), dict(k=0),
                                 dict(k=9), dict(E=128, k=65, groups=1, keep_groups=1, logits_stride=128), dict(groups=0), dict(groups=3), dict(E=650, groups=65, logits_stride=650),
                                 dict(keep_groups=0), dict(keep_groups=5), dict(group_best=0), dict(group_best=3), dict(scale=float("nan")), dict(scale=float("inf")),
                                 dict(T=-1), dict(T=1 << 31), dict(logits=0), dict(logits_stride=15), dict(experts=0), dict(weights=0), dict(logits=FAKE + 1),
                                 dict(dtype=2, logits=FAKE + 2), dict(experts=FAKE + 2), dict(weights=FAKE + 2), dict(bias=FAKE + 2)])
def test_route_refuses(bad):
    assert lib().oob_expert_route(C.byref(make(X.oob_route, **{**ROUTE, **bad})), None) == P.OOB_EINVAL


def test_route_backward_refuses():
    call = lambda p, dw=FAKE, dl=FAKE, ld=16: lib().oob_expert_route_backward(None if p is None else C.byref(p), dw, dl, ld, None)  # noqa: E731
    ok = make(X.oob_route, **ROUTE)
    assert call(None) == call(ok, dw=0) == call(ok, dl=0) == call(ok, ld=15) == call(ok, dw=FAKE + 2) == call(ok, dl=FAKE + 1) == P.OOB_EINVAL
    for bad in (dict(dtype=4), dict(k=17), dict(experts=0), dict(logits=0), dict(scale=float("nan")), dict(logits_stride=3)):
        assert call(make(X.oob_route, **{**ROUTE, **bad})) == P.OOB_EINVAL, bad
    none = make(X.oob_route, **{**ROUTE, "T": 0, "logits": 0, "experts": 0, "weights": 0})
    assert call(none, 0, 0) == P.OOB_OK and lib().oob_expert_route(C.byref(none), None) == P.OOB_OK


def test_rows_refuse_and_workspaces():
    call = lambda **k: lib().oob_expert_rows(k.get("experts", FAKE), k.get("n", 100000), 0, k.get("E", 8), k.get("offsets", FAKE), k.get("rows", FAKE),  # noqa: E731
                                             k.get("place", FAKE), k.get("ws", FAKE), k.get("bytes", 1 << 40), None)
    for bad in (dict(experts=0), dict(n=-1), dict(n=1 << 31), dict(E=0), dict(E=1025), dict(offsets=0), dict(rows=0), dict(place=0), dict(ws=FAKE + 4),
                dict(experts=FAKE + 2), dict(offsets=FAKE + 1), dict(rows=FAKE + 2), dict(place=FAKE + 2)):
        assert call(**bad) == P.OOB_EINVAL, bad
    size = lib().oob_expert_rows_workspace_size
    assert size(0, 8) == size(-1, 8) == size(8, 0) == size(8, 1025) == size(1000, 1024) == 0  # none, refused, one workgroup
    assert size(100000, 8) > 0 and call(bytes=size(100000, 8) - 1) == call(ws=0) == P.OOB_ECAPACITY
    assert size((1 << 31) - 1, 1024) <= 257 * 1024 * 4  # however many pairs there are, their runs are few


LINEAR = dict(dtype=0, act=0, E=3, per=2, R=8, T=4, N=16, K=8, offsets=FAKE, rows=FAKE, x=FAKE, w=FAKE, y=FAKE, x_stride=8, w_stride=8, expert_stride=128,
              y_stride=16)


@pytest.mark.parametrize("bad", [dict(dtype=2), dict(act=5), dict(act=-1), dict(E=0), dict(E=1025), dict(per=0), dict(per=3), dict(R=-8), dict(T=5), dict(N=0), dict(K=0),
                                 dict(N=1 << 21, y_stride=1 << 21), dict(K=1 << 21, x_stride=1 << 21, w_stride=1 << 21), dict(R=1 << 32, T=1 << 31), dict(rows=0),
                                 dict(offsets=0), dict(x=0), dict(w=0), dict(y=0), dict(x_stride=7), dict(w_stride=7), dict(y_stride=15), dict(expert_stride=-1),
                                 dict(z=FAKE, z_stride=15), dict(x=FAKE + 1), dict(y=FAKE + 1), dict(bias=FAKE + 1), dict(offsets=FAKE + 2), dict(rows=FAKE + 2)])
def test_linear_refuses(bad):
    assert lib().oob_expert_linear(C.byref(make(X.oob_expert_linear_t, **{**LINEAR, **bad})), FAKE, 1 << 60, None) == P.OOB_EINVAL


def test_linear_workspaces():
    size = lambda p, *g: (lib().oob_expert_linear_backward_workspace_size(C.byref(p), C.byref(g[0])) if g else lib().oob_expert_linear_workspace_size(C.byref(p)))  # noqa: E731
    ok = make(X.oob_expert_linear_t, **LINEAR)
    assert size(ok) == 0 and lib().oob_expert_linear(None, None, 0, None) == P.OOB_EINVAL
    assert lib().oob_expert_linear(C.byref(ok), FAKE + 8, 1 << 40, None) == P.OOB_EINVAL  # workspace off 256 bytes
    odd = make(X.oob_expert_linear_t, **{**LINEAR, "K": 7, "x_stride": 7, "w_stride": 7, "expert_stride": 112})  # rows that do not start at 16 bytes
    need = size(odd)
    assert need >= (3 * 16 + 8) * 8 * 2 and lib().oob_expert_linear(C.byref(odd), FAKE, need - 1, None) == P.OOB_ECAPACITY
    far = make(X.oob_expert_linear_t, **{**LINEAR, "T": 1 << 20, "R": 1 << 21, "x_stride": 1024})  # tokens that 32-bit offsets do not reach: rows are copied
    assert size(far) >= (1 << 21) * 8 * 2
    empty = make(X.oob_expert_linear_t, **{**LINEAR, "R": 0, "T": 0, "x": 0, "y": 0})
    assert lib().oob_expert_linear(C.byref(empty), None, 0, None) == P.OOB_OK
    many = make(X.oob_expert_linear_t, **{**LINEAR, "R": 1 << 30, "T": 1 << 29, "N": 1 << 20, "y_stride": 1 << 20, "expert_stride": 8 << 20})
    assert lib().oob_expert_linear(C.byref(many), FAKE, 1 << 62, None) == P.OOB_EINVAL  # more workgroups than a launch has

    p = make(X.oob_expert_linear_t, **{**LINEAR, "act": 3, "z": FAKE, "z_stride": 16})
    grad = dict(dy=FAKE, dx=FAKE, dw=FAKE, db=FAKE, dy_stride=16, dx_stride=8)
    both = size(p, make(X.oob_expert_linear_grad, **grad))
    parts = [size(p, make(X.oob_expert_linear_grad, **{**grad, n: 0})) for n in ("dx", "dw")]
    assert both >= max(parts) > 0
    call = lambda g, n=1 << 40, p=p: lib().oob_expert_linear_backward(C.byref(p), C.byref(make(X.oob_expert_linear_grad, **{**grad, **g})), FAKE, n, None)  # noqa: E731
    assert call({}, both - 1) == P.OOB_ECAPACITY
    for bad in (dict(dy=0), dict(dy_stride=15), dict(dx_stride=7), dict(dy=FAKE + 1), dict(dx=FAKE + 1), dict(dw=FAKE + 1), dict(db=FAKE + 1)):
        assert call(bad) == P.OOB_EINVAL, bad
    for bad in (dict(z=0), dict(z_stride=15), dict(w=0), dict(x=0), dict(offsets=0)):
        assert call({}, p=make(X.oob_expert_linear_t, **{**LINEAR, "act": 3, "z": FAKE, "z_stride": 16, **bad})) == P.OOB_EINVAL, bad


SUM = dict(dtype=0, k=2, T=4, R=8, C=16, y=FAKE, place=FAKE, out=FAKE, y_stride=16, out_stride=16)


@pytest.mark.parametrize("bad", [dict(dtype=3), dict(k=0), dict(k=65), dict(T=-1), dict(R=-1), dict(C=0), dict(T=1 << 31), dict(R=1 << 31), dict(C=1 << 30), dict(y=0), dict(place=0),
                                 dict(out=0), dict(y_stride=15), dict(out_stride=15), dict(residual=FAKE, residual_stride=15), dict(y=FAKE + 1), dict(place=FAKE + 2),
                                 dict(weights=FAKE + 2), dict(dtype=2, out=FAKE + 2), dict(residual=FAKE + 1, residual_stride=16)])
def test_sum_refuses(bad):
    assert lib().oob_expert_sum(C.byref(make(X.oob_expert_sum_t, **{**SUM, **bad})), None) == P.OOB_EINVAL


def test_sum_backward_refuses():
    p = make(X.oob_expert_sum_t, **SUM)
    call = lambda p=p, d=FAKE, ld=16, dy=FAKE, ldy=16, dw=FAKE: lib().oob_expert_sum_backward(C.byref(p), d, ld, dy, ldy, dw, None)  # noqa: E731
    assert {call(d=0), call(ld=15), call(ldy=15), call(dy=0, dw=0), call(d=FAKE + 1), call(dy=FAKE + 1), call(dw=FAKE + 2)} == {P.OOB_EINVAL}
    assert call(make(X.oob_expert_sum_t, **{**SUM, "T": 0, "place": 0}), 0, 0, 0, 0, 0) == P.OOB_OK


def test_clip_refuses():
    arrays = lambda n, at=FAKE, size=100, kind=0: ((C.c_void_p * n)(*[at + i * 4096 for i in range(n)]), (C.c_int64 * n)(*[size] * n), (C.c_int * n)(*[kind] * n))  # noqa: E731
    ptr, sizes, types = arrays(3)
    size = lib().oob_clip_workspace_size
    need = size(3, sizes)
    assert need > 0 and size(-1, sizes) == size(3, None) == 0 and size(0, sizes) == 0
    norm = lambda n=3, p=ptr, s=sizes, t=types, out=FAKE, ws=FAKE, b=need: lib().oob_clip_norm(n, p, s, t, out, ws, b, None)  # noqa: E731
    assert {norm(n=-1), norm(p=None), norm(s=None), norm(t=None), norm(out=0), norm(out=FAKE + 2), norm(ws=FAKE + 8)} == {P.OOB_EINVAL}
    assert norm(b=need - 1) == norm(ws=0) == P.OOB_ECAPACITY
    assert norm(p=arrays(3, FAKE + 1)[0]) == norm(s=arrays(3, size=-1)[1]) == norm(t=arrays(3, kind=3)[2]) == P.OOB_EINVAL
    scale = lambda to=ptr, m=1.0, given=None, out=FAKE, ws=FAKE, b=need: lib().oob_clip_scale(3, ptr, to, sizes, types, m, given, out, ws, b, None)  # noqa: E731
    assert {scale(to=None), scale(m=-1.0), scale(m=float("nan")), scale(out=0), scale(out=FAKE + 2), scale(given=FAKE + 2, out=0)} == {P.OOB_EINVAL}
    assert scale(b=need - 1) == P.OOB_ECAPACITY
    same = (C.c_void_p * 3)(FAKE, FAKE + 4096, FAKE + 4096 + 198)  # two that share two bytes
    overlap = lambda to, given=None: lib().oob_clip_overlap(3, ptr, to, sizes, types, given)  # noqa: E731
    at = lambda *a: (C.c_void_p * 3)(*a)  # noqa: E731
    assert overlap(same) == 1 and scale(to=same) == P.OOB_EINVAL
    far = FAKE + (1 << 20)
    assert overlap(ptr) == overlap(at(far, far + 200, far + 400)) == 0
    # what is written lies on another's input, or beside its own by one value; or on the given norm
    for to in (at(FAKE + 4096, FAKE, FAKE + 8192), at(FAKE + 2, far, far + 200), at(FAKE - 198, far, far + 200), at(far, far + 200, FAKE + 4096 + 198)):
        assert overlap(to) == 1 and scale(to=to) == P.OOB_EINVAL
    assert overlap(at(FAKE + 200, far, FAKE + 4096 - 200)) == 0
    for given, shares in ((FAKE - 4, 0), (FAKE, 1), (FAKE + 196, 1), (FAKE + 200, 0), (FAKE + 8192 + 196, 1), (FAKE + 8192 + 200, 0)):
        assert overlap(ptr, given) == shares
        assert not shares or scale(given=given, out=0) == P.OOB_EINVAL


def test_results_on_what_is_read_are_refused():
    """Of the calls that are refused nothing is enqueued; those that would be let through are not made here."""
    at = lambda i: FAKE + i * (1 << 16)  # noqa: E731
    apart = dict(LINEAR, x=at(0), w=at(1), bias=at(2), y=at(3), z=at(4), z_stride=LINEAR["y_stride"])
    run = lambda **kw: lib().oob_expert_linear(C.byref(make(X.oob_expert_linear_t, **{**apart, **kw})), None, 0, None)  # noqa: E731
    w = 2 * (2 * LINEAR["expert_stride"] + (LINEAR["N"] - 1) * LINEAR["w_stride"] + LINEAR["K"])  # bytes of three matrices
    for kw in (dict(y=at(0)), dict(z=at(0)), dict(y=at(0) + 2), dict(y=at(1)), dict(y=at(1) + w - 2), dict(z=at(2)), dict(y=at(2) + 2 * 3 * LINEAR["N"] - 2)):
        assert run(**kw) == P.OOB_EINVAL, kw
    back = lambda dx, **kw: lib().oob_expert_linear_backward(  # noqa: E731
        C.byref(make(X.oob_expert_linear_t, **{**apart, **kw})), C.byref(X.oob_expert_linear_grad(at(5), dx, at(6), None, LINEAR["N"], LINEAR["K"])), FAKE, 1 << 40, None)
    for kw in (dict(dx=at(5)), dict(dx=at(1)), dict(dx=at(0) + 2), dict(dx=at(4), act=4)):
        assert back(**kw) == P.OOB_EINVAL, kw
