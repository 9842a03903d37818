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
