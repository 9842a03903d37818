"""The example that measures a layer's profile and plans with it: its layer's gradients against differentiation of the plain form, and
the whole of it at a small size."""
import os
import sys

import pytest
import torch

import layer_oracle as O

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_layer_of_the_example_against_the_plain_form():
    import measured_profile as E

    B, S, C, heads, p, seed = 2, 96, 128, 4, 0.1, 5
    documents = [[40, 30], [96]]
    layer = E.LayerShare(C, heads, 1, B, S, documents, p=p)
    x, z, dx, dy = (torch.randn(B, S, C, device="cuda").bfloat16() for _ in range(4))
    x2, y, kept = layer.forward(x, z, seed)
    gx, gz, grads = layer.backward(dx, dy, kept)

    names = ["qkv", "out", "up", "down"]
    leaf = lambda t: t.double().requires_grad_()  # noqa: E731
    X, Z = leaf(x).view(-1, C), leaf(z).view(-1, C)
    W, Bs = {n: leaf(layer.w[n]) for n in names}, {n: leaf(layer.b[n]) for n in names}
    N = [{k: leaf(v) for k, v in n.items()} for n in layer.n]
    kept64 = [O.keep(B * S * C, p, seed, k * B * S * C).view(-1, C).cuda() for k in (0, 1)]
    n1 = O.residual_norm(X, Z, N[0]["weight"], N[0]["bias"], "layer", "none", None, None, None, 1.0, 1e-5, kept64[0])
    q, k, v = (n1[1] @ W["qkv"].t() + Bs["qkv"]).view(B, S, 3, heads, C // heads).unbind(2)
    m = O.seen(B, S, S, False, layer.ranges["key_begin"], layer.ranges["key_end"], "cuda")
    o = O.attention(q, k, v, m, (C // heads) ** -0.5, None, 0.0)[0].reshape(-1, C)
    n2 = O.residual_norm(n1[0], o @ W["out"].t() + Bs["out"], N[1]["weight"], N[1]["bias"], "layer", "none", None, None, None, 1.0, 1e-5, kept64[1])
    out = O.act(n2[1] @ W["up"].t() + Bs["up"], "gelu_tanh") @ W["down"].t() + Bs["down"]
    near = lambda a, b: (a.double().reshape(b.shape) - b).norm() <= 16 * O.U[torch.bfloat16] * b.norm()  # noqa: E731  sixteen roundings in a row
    assert near(x2, n2[0].detach()) and near(y, out.detach())
    leaves = {"x": X, "z": Z, **W, **{n + "_b": t for n, t in Bs.items()}, "norm1": N[0]["weight"], "norm1_b": N[0]["bias"], "norm2": N[1]["weight"], "norm2_b": N[1]["bias"]}
    want = dict(zip(leaves, torch.autograd.grad((n2[0], out), list(leaves.values()), (dx.double().view(-1, C), dy.double().view(-1, C)))))
    for n, g in {"x": gx, "z": gz, **grads}.items():
        assert near(g, want[n]), n


def test_example_measures_and_plans(capsys):
    import measured_profile as E

    res = E.main(["--hidden", "256", "--width", "64", "--layers", "4", "--gpus", "4", "--tokens", "128", "--nodes-min", "1", "--nodes-max", "2", "--runs", "2"])
    said = capsys.readouterr().out
    assert res["feasible"].all() and (res["T"] > 0).all()
    assert "layer on 1 GPU(s): forward" in said and "layer on 3 GPU(s): heads do not divide" in said and "2 nodes:" in said


def test_profile_is_the_gpus_time_not_the_calls(monkeypatch):
    """Calls that take the host 2 ms each do not enter: a pass of this share runs for some 0.1 ms."""
    import time

    import measured_profile as E

    layer = E.LayerShare(128, 4, 2, 1, 64, [[64]])
    for name in ("residual_norm", "residual_norm_backward"):
        call = getattr(E.P, name)
        monkeypatch.setattr(E.P, name, lambda *a, call=call, **k: (time.sleep(2e-3), call(*a, **k))[1])
    assert all(0 < ns < 2_000_000 for ns in E.measure(layer, 128, runs=5))


def test_captured_passes_give_what_the_calls_give():
    import measured_profile as E

    B, S, C = 2, 96, 128
    layer = E.LayerShare(C, 4, 2, B, S, [[40, 30], [96]])
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
