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
