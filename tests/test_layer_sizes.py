"""Launches of the matrix products of a transformer layer (csrc/oob_layer_sizes.h), compiled for the host."""
import ctypes as C
import os
import subprocess

import pytest

import paper_2309_08125_amd as P
from paper_2309_08125_amd import layer as L
from test_layer_abi import FAKE, LINEAR, attention, lib, make

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2309_08125_amd", "csrc")
WRAPPERS = r"""
#include "oob_layer_sizes.h"
using namespace layer;
extern "C" {
int largest(int ak, int64_t a_rows, int64_t a_ld, int bk, int64_t b_rows, int64_t b_ld) { return largest_tile(Extent{ak != 0, a_rows, a_ld}, Extent{bk != 0, b_rows, b_ld}); }
void chosen(int64_t M, int64_t N, int64_t K, int most, int *to) {
    const Shape s = choose(M, N, K, most);
    to[0] = s.tile, to[1] = s.splits, to[2] = s.full, to[3] = s.rest;
}
}
"""


@pytest.fixture(scope="module")
def sizes(tmp_path_factory):
    at = tmp_path_factory.mktemp("layer_sizes")
    (at / "w.cpp").write_text(WRAPPERS)
    subprocess.run(["g++", "-std=c++17", "-O2", "-shared", "-fPIC", "-I", CSRC, "-o", str(at / "w.so"), str(at / "w.cpp")], check=True)
    so = C.CDLL(str(at / "w.so"))
    so.largest.argtypes = [C.c_int, C.c_int64, C.c_int64] * 2
    so.chosen.argtypes = [C.c_int64] * 3 + [C.c_int, C.POINTER(C.c_int * 4)]
    return so


def chosen(sizes, M, N, K, most=256):
    s = (C.c_int * 4)()
    sizes.chosen(M, N, K, most, C.byref(s))
    return tuple(s)


def test_offsets_of_a_tile_stay_below_the_buffers_end(sizes):
    """A lane's last byte, row by row and at the row's end, over long rows of few and of many."""
    for ld in [8, 1 << 20, (1 << 21) - 8, 1 << 22, (1 << 22) + 8, 1 << 23, (1 << 24) - 8, 1 << 24, 17043512, 17043520, 1 << 25, 1 << 27, (1 << 31) - 8]:
        for rows in [1, 2, 31, 32, 33, 63, 64, 65, 127, 129, 255, 256, 1 << 20]:
            for kc in (0, 1):
                got = sizes.largest(kc, rows, ld, 1, 1, 8)
                ends = {t: (min(rows, t if kc else 64) - 1) * ld * 2 + (128 if kc else 2 * t) for t in (64, 128, 256)}
                assert got == max((t for t, e in ends.items() if e < 1 << 31), default=0), (ld, rows, kc)
                assert got or ld > 1 << 24  # rows below 2^24 are never refused
    for most in (64, 128, 256):
        for M, N, K in ((4096, 4096, 4096), (4096, 6144, 12288), (1000, 2000, 1 << 24)):
            tile, splits, full, rest = chosen(sizes, M, N, K, most)
            assert tile <= most and full + rest == -(-M // tile) * -(-N // tile) and (splits > 1) == (rest > 0)


# (T, N, K) of a product and its gradients: (tile, parts of k, whole tiles, split tiles) of y, dx and dw.  The GPU tests run these.
LARGE = {
    (4000, 6100, 5128): ((256, 2, 256, 128), (256, 2, 256, 80), (256, 1, 504, 0)),  # whole and split tiles in one launch, joined
    (5200, 2501, 2499): ((256, 1, 210, 0), (256, 1, 210, 0), (256, 2, 0, 100)),     # all tiles split; rows that have to be copied
    (2000, 2000, 2000): ((128, 1, 256, 0), (128, 1, 256, 0), (128, 1, 256, 0)),
    (1990, 1985, 2003): ((128, 1, 256, 0), (128, 1, 256, 0), (128, 1, 256, 0)),
    (300, 260, 2100): ((64, 8, 0, 25), (64, 1, 165, 0), (64, 1, 165, 0)),
}


def test_sizes_of_the_gpu_tests_reach_every_kind_of_launch(sizes):
    got = {s: tuple(chosen(sizes, *mnk) for mnk in ((s[0], s[1], s[2]), (s[0], s[2], s[1]), (s[1], s[2], s[0]))) for s in LARGE}
    assert got == LARGE
    for product in range(3):  # each product (its layout is its own kernel) in the middle and the large tile
        assert {c[product][0] for c in got.values()} == {64, 128, 256}
    assert any(c[0][1] > 1 and c[0][0] == 256 for c in got.values()) and any(c[1][1] > 1 for c in got.values()) and any(c[2][1] > 1 for c in got.values())


def test_rows_that_the_loads_do_not_reach_are_refused():
    long = 1 << 25
    p = make(L.oob_linear, **{**LINEAR, "T": 1, "N": 64, "K": long, "x_stride": long, "w_stride": long, "y_stride": 64})
    assert lib().oob_layer_linear(C.byref(p), FAKE, 1 << 50, None) == P.OOB_EINVAL
    p = make(L.oob_linear, **{**LINEAR, "T": 64, "N": 1, "K": long, "x_stride": long, "w_stride": long, "y_stride": 1})
    assert lib().oob_layer_linear(C.byref(p), FAKE, 1 << 50, None) == P.OOB_EINVAL
    grad = dict(dtype=0, act=0, T=64, N=64, K=64, dy=FAKE, x=FAKE, w=FAKE, dy_stride=64, x_stride=64, w_stride=64, dx_stride=64, dw_stride=64)
    for bad in (dict(N=long, dy_stride=long, dx=FAKE), dict(N=long, dy_stride=long, dw=FAKE), dict(K=long, w_stride=long, dx_stride=long, dx=FAKE),
                dict(K=long, x_stride=long, dw_stride=long, dw=FAKE), dict(N=long, dy_stride=long, z=FAKE, z_stride=long, act=3, dx=FAKE)):
        g = make(L.oob_linear_grad, **{**grad, **bad})
        assert lib().oob_layer_linear_backward(C.byref(g), FAKE, 1 << 50, None) == P.OOB_EINVAL, bad


@pytest.mark.parametrize("bad", [dict(B=1 << 30, H=1 << 30, G=1, Sq=240, Sk=8), dict(B=1 << 29), dict(B=(1 << 31) - 1), dict(B=1 << 15, H=1 << 16, G=1)])
def test_attention_sizes_whose_products_pass_their_integers_are_refused(bad):
    """The first passes 64 bits to the very 0."""
    p = attention(**bad)
    assert lib().oob_layer_attention(C.byref(p), FAKE, 1 << 62, None) == P.OOB_EINVAL
    assert lib().oob_layer_attention_workspace_size(C.byref(p)) == 0


def test_attention_heads_whose_copies_the_loads_do_not_reach_are_refused():
    """2^19 heads of 128 values: copied rows of 2^27 bytes, 40 of them.  The backward pass reads q and dout the same way."""
    N, odd = 1 << 19, (1 << 30, (1 << 26) + 1, 128)
    sizes = dict(B=1, Sq=40, Sk=40, H=N, D=128)
    for bad in (dict(G=N, k_stride=odd), dict(G=N, v_stride=odd)):
        p = attention(**sizes, **bad)
        assert lib().oob_layer_attention(C.byref(p), FAKE, 1 << 62, None) == P.OOB_EINVAL, bad
    strides = lambda *s: [(C.c_int64 * 3)(*x) for x in s]  # noqa: E731
    even = (1 << 30, 128 * 8, 128)
    for bad, dout in ((dict(q_stride=odd), even), ({}, odd)):
        p = attention(**sizes, G=1, **bad)
        g = L.oob_attention_grad(FAKE, FAKE, FAKE, FAKE, *strides(dout, even, even, even))
        assert lib().oob_layer_attention_backward(C.byref(p), C.byref(g), FAKE, 1 << 62, None) == P.OOB_EINVAL, (bad, dout)


def test_attention_results_that_lie_on_themselves_are_refused():
    """Expanded tensors: strides of 0.  Inputs may be such."""
    for bad in ((0, 64, 16), (512, 0, 16), (512, 64, 0)):
        p = attention(B=2, o_stride=bad)
        assert lib().oob_layer_attention(C.byref(p), FAKE, 1 << 40, None) == P.OOB_EINVAL, bad
        for n in range(3):
            g = L.oob_attention_grad(FAKE, FAKE, FAKE, FAKE, *[(C.c_int64 * 3)(*(bad if k == n else (512, 64, 16))) for k in (3, 0, 1, 2)])
            assert lib().oob_layer_attention_backward(C.byref(attention(B=2)), C.byref(g), FAKE, 1 << 40, None) == P.OOB_EINVAL, (bad, n)
    expanded = attention(B=2, q_stride=(0, 64, 16), k_stride=(0, 0, 16), v_stride=(512, 64, 0))
    g = L.oob_attention_grad(FAKE, FAKE, FAKE, FAKE, *[(C.c_int64 * 3)(*s) for s in ((0, 0, 0), (512, 64, 16), (512, 64, 16), (512, 64, 16))])
    assert lib().oob_layer_attention_backward_workspace_size(C.byref(expanded), C.byref(g)) > 0
    assert lib().oob_layer_attention_workspace_size(C.byref(attention(B=1, o_stride=(0, 64, 16)))) == 0  # one sequence: its stride is not used
