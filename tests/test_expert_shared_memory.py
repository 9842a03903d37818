"""Results of the experts' operators and of clipping on memory that the call reads, or writes to for another result: refused before anything is enqueued.  Calls that
would be let through are not made here: nothing at these addresses is anybody's."""
import ctypes as C

import paper_2309_08125_amd as P
from paper_2309_08125_amd import expert as X

BASE = 0x100000


def at(i):
    """Addresses far enough apart for every array below."""
    return BASE + i * (1 << 16)


def make(struct, **kw):
    s = struct()
    for k, v in kw.items():
        setattr(s, k, v)
    return s


SUM = dict(dtype=0, k=2, T=4, R=8, C=16, y=at(0), place=at(1), weights=at(2), residual=at(3), out=at(4), y_stride=16, residual_stride=16, out_stride=16)


def test_sum_on_what_it_reads():
    call = lambda **kw: X._load().oob_expert_sum(C.byref(make(X.oob_expert_sum_t, **{**SUM, **kw})), None)  # noqa: E731
    for kw in (dict(out=at(0)), dict(out=at(0) + 8 * 32 - 2), dict(out=at(0) - 4 * 32 + 2), dict(out=at(0) + 32, y_stride=32, out_stride=20),  # rows of y
               dict(out=at(1)), dict(out=at(1) + 28), dict(out=at(2) - 100), dict(out=at(2) + 28),  # places, weights
               dict(out=at(3), out_stride=17), dict(out=at(3), residual_stride=17), dict(out=at(3) + 2), dict(out=at(3) - 32)):  # the residual, not in its place
        assert call(**kw) == P.OOB_EINVAL, kw


LINEAR = dict(dtype=0, act=0, E=3, per=2, R=8, T=4, N=16, K=8, offsets=at(0), rows=at(1), x=at(2), w=at(3), bias=at(4), y=at(5), z=at(6), x_stride=8, w_stride=8,
              expert_stride=128, y_stride=16, z_stride=16)


def test_products_on_what_they_read():
    call = lambda **kw: X._load().oob_expert_linear(C.byref(make(X.oob_expert_linear_t, **{**LINEAR, **kw})), None, 0, None)  # noqa: E731
    for name in ("y", "z"):
        for first, size in ((at(0), 16), (at(1), 32)):  # offsets, rows: later tiles read them too
            for where in (first, first + size - 2, first - 8 * 32 + 2):
                assert call(**{name: where}) == P.OOB_EINVAL, (name, where - BASE)
    for kw in (dict(y=at(6)), dict(y=at(6) + 30), dict(y=at(6) + 32, y_stride=24), dict(z=at(5) + 8 * 32 - 2)):  # one another
        assert call(**kw) == P.OOB_EINVAL, kw


def test_products_in_order_have_as_many_tokens_as_rows():
    """Without rows x is [R][K]: a smaller T would leave the end of x out of what results are held against."""
    in_order = dict(LINEAR, rows=0, per=1)
    for T in (0, 4, 7, 9):
        p = make(X.oob_expert_linear_t, **{**in_order, "T": T, "y": at(2) + 7 * 16})  # on the last row of x
        assert X._load().oob_expert_linear(C.byref(p), None, 0, None) == P.OOB_EINVAL, T
        g = X.oob_expert_linear_grad(at(7), at(2) + 7 * 16, at(8), 0, 16, 8)
        assert X._load().oob_expert_linear_backward(C.byref(p), C.byref(g), at(9), 1 << 40, None) == P.OOB_EINVAL, T
        assert X._load().oob_expert_linear_workspace_size(C.byref(p)) == 0


def test_gradients_of_products_on_what_is_read_and_on_one_another():
    grad = dict(dy=at(7), dx=at(8), dw=at(9), db=at(10), dy_stride=16, dx_stride=8)

    def call(p=(), **kw):
        q = make(X.oob_expert_linear_t, **{**LINEAR, "act": 4, **dict(p)})
        return X._load().oob_expert_linear_backward(C.byref(q), C.byref(make(X.oob_expert_linear_grad, **{**grad, **kw})), at(11), 1 << 40, None)

    sizes = {at(7): 8 * 32, at(6): 8 * 32, at(3): 3 * 256, at(2): 4 * 16, at(0): 16, at(1): 32}  # dy, z, w, x, offsets, rows
    results = dict(dx=8 * 16, dw=3 * 256, db=3 * 32)
    for name, mine in results.items():
        for first, size in sizes.items():
            for where in (first, first + size - 2, first - mine + 2):
                assert call(**{name: where}) == P.OOB_EINVAL, (name, where - BASE)
        for other in results.keys() - {name}:
            for where in (grad[other], grad[other] + results[other] - 2):
                assert call(**{name: where}) == P.OOB_EINVAL, (name, other)


def test_gradients_of_sums_on_what_is_read_and_on_one_another():
    p = make(X.oob_expert_sum_t, **SUM)
    call = lambda dy=at(6), dw=at(7): X._load().oob_expert_sum_backward(C.byref(p), at(5), 16, dy, 16, dw, None)  # noqa: E731
    for first, size in ((at(0), 8 * 32), (at(1), 32), (at(2), 32), (at(5), 4 * 32)):  # y, places, weights, dout
        for where in (first, first + size - 4, first - 28):
            assert call(dy=where) == call(dw=where) == P.OOB_EINVAL, where - BASE
    assert call(dw=at(6)) == call(dw=at(6) + 8 * 32 - 4) == call(dy=at(7) - 8 * 32 + 2) == P.OOB_EINVAL


def test_norm_on_tensors_that_are_scaled():
    """The norm is written while other workgroups still read and write the tensors."""
    n, sizes, types = 2, (C.c_int64 * 2)(100, 50), (C.c_int * 2)(0, 2)
    arrays = lambda *a: (C.c_void_p * 2)(*a)  # noqa: E731
    need = X._load().oob_clip_workspace_size(n, sizes)
    for to in (arrays(at(0), at(1)), arrays(at(2), at(3))):
        for first in (at(0), at(1), to[0], to[1]):
            for where in (first, first + 196):
                assert X._load().oob_clip_scale(n, arrays(at(0), at(1)), to, sizes, types, 1.0, None, where, at(4), need, None) == P.OOB_EINVAL, where - BASE
