"""The example's layer with experts: its gradients against differentiation of the plain form, its captured passes, and the whole of it."""
import os
import sys

import pytest
import torch

import expert_oracle as X
import layer_oracle as O

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_block_with_experts_of_the_example_against_the_plain_form():
    import measured_profile as E

    B, S, C, experts, choices = 2, 96, 128, 6, 2
    layer = E.ExpertLayerShare(C, 4, 1, B, S, [[40, 30], [96]], experts=experts, choices=choices)
    layer.w["router"] *= 20  # logits as far apart as a trained router's
    h, dy = (torch.randn(B, S, C, device="cuda").bfloat16() for _ in range(2))
    y, kept = layer.block(h)
    dh, grads = layer.block_backward(dy, h, kept)
    names = ["router", "up", "up_b", "down", "down_b"]
    leaves = {n: t.double().requires_grad_() for n, t in zip(names, (layer.w["router"], layer.w["up"], layer.b["up"], layer.w["down"], layer.b["down"]))}
    x = h.double().view(-1, C).requires_grad_()
    w = X.weights(x @ leaves["router"].t(), kept[1].long(), "softmax", True, 1.0)
    out = 0
    for j in range(choices):
        e = kept[1][:, j].long()
        u = O.act(torch.bmm(leaves["up"][e], x[:, :, None])[:, :, 0] + leaves["up_b"][e], "gelu_tanh")
        out = out + w[:, j, None] * (torch.bmm(leaves["down"][e], u[:, :, None])[:, :, 0] + leaves["down_b"][e])
    near = lambda a, b: (a.double().reshape(b.shape) - b).norm() <= 16 * O.U[torch.bfloat16] * b.norm()  # noqa: E731  sixteen roundings in a row
    assert near(y, out.detach())
    want = torch.autograd.grad(out, [x, *leaves.values()], dy.double().view(-1, C))
    for n, got, g in zip(["h", *names], [dh, *(grads[n] for n in names)], want):
        assert near(got, g), n


def test_captured_passes_with_experts_give_what_the_calls_give():
    import measured_profile as E

    B, S, C = 2, 96, 128
    layer = E.ExpertLayerShare(C, 4, 2, B, S, [[40, 30], [96]], experts=5, choices=3)
    x, z, dx, dy = (torch.randn(B, S, C, device="cuda").bfloat16() for _ in range(4))
    (forward, out), (backward, grads) = E.captured(layer, x, z, dx, dy, seed=3)
    for _ in range(4):
        for t in (x, z, dx, dy):
            t.copy_(torch.randn(B, S, C, device="cuda"))
        want = layer.forward(x, z, 3)
        want_grads = layer.backward(dx, dy, want[2])
        torch.cuda.synchronize()
        forward.replay()
        backward.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out[:2] + grads[:2], want[:2] + want_grads[:2]))
        assert all(torch.equal(grads[2][n], g) for n, g in want_grads[2].items())


def test_example_measures_a_layer_with_experts_and_plans(capsys):
    import measured_profile as E

    res = E.main(["--hidden", "256", "--width", "64", "--layers", "4", "--gpus", "2", "--tokens", "128", "--nodes-min", "1", "--nodes-max", "2", "--runs", "2",
                  "--experts", "4", "--choices", "2"])
    assert res["feasible"].all() and (res["T"] > 0).all() and "2 nodes:" in capsys.readouterr().out
    with pytest.raises(ValueError):
        E.ExpertLayerShare(256, 4, 1, 1, 64, [[64]], experts=4, choices=5)
