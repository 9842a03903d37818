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
