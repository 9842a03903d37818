"""A layer profile measured on this GPU, planned.

The planner wants the forward and backward time of every layer on d = 1..M GPUs of a node.  This runs one GPU's share of a
GPT-shaped layer (pre-norm, attention, feed-forward block of four times the width, residual dropout) with 1/d of the heads and
columns, forward and backward, through the package's operators, adds the all-reduce of the two partial sums over the node's
links by the rule of inputs.make_profile, and plans pipeline templates with the result.  With --experts the feed-forward block is one of
several for each token, chosen by a router.

    python examples/measured_profile.py                       # 1.3B-shaped: hidden width 2048, 24 layers, 4 GPUs a node
    python examples/measured_profile.py --hidden 4096 --layers 32 --gpus 8
    python examples/measured_profile.py --experts 8 --choices 2
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import inputs  # noqa: E402
import paper_2309_08125_amd as P  # noqa: E402

LINK = 25 * 10**9  # bytes a second between nodes; eight times that within one


class LayerShare:
    """One GPU's part of a layer on d GPUs, for B sequences of S tokens packed with documents."""

    def __init__(self, hidden, heads, d, B, S, documents, p=0.1, seed=0):
        if heads % d or hidden % heads:
            raise ValueError(f"{heads} heads do not divide among {d} GPUs, or {hidden} columns among the heads")
        g = torch.Generator(device="cuda").manual_seed(seed)
        new = lambda *shape, std: (torch.randn(*shape, generator=g, device="cuda") * std).bfloat16()  # noqa: E731
        C, self.heads, self.width, self.p, self.B, self.S = hidden, heads // d, hidden // heads, p, B, S
        own = self.heads * self.width
        self.w = {"qkv": new(3 * own, C, std=0.02), "out": new(C, own, std=0.02), "up": new(4 * C // d, C, std=0.02), "down": new(C, 4 * C // d, std=0.02)}
        self.b = {"qkv": new(3 * own, std=0.02), "out": new(C, std=0.02), "up": new(4 * C // d, std=0.02), "down": new(C, std=0.02)}
        self.n = [{"weight": 1 + new(C, std=0.02), "bias": new(C, std=0.02)} for _ in range(2)]
        self.ranges = dict(zip(("key_begin", "key_end"), P.document_ranges(documents, S)))

    def heads_of(self, t):
        t = t.view(self.B, self.S, 3, self.heads, self.width)
        return t[:, :, 0], t[:, :, 1], t[:, :, 2]

    def forward(self, x, z, seed):
        """x: the residual stream, z: the output of the layer before, dropped and added here.  (stream, this layer's output, kept)."""
        x1, h1, s1 = P.residual_norm(x, z, p=self.p, seed=seed, offset=0, **self.n[0])
        qkv = P.linear(h1, self.w["qkv"], self.b["qkv"])
        o, lse = P.attention(*self.heads_of(qkv), **self.ranges)
        a = P.linear(o.view(self.B, self.S, -1), self.w["out"], self.b["out"])  # a partial sum where d > 1
        x2, h2, s2 = P.residual_norm(x1, a, p=self.p, seed=seed, offset=a.numel(), **self.n[1])
        y, block = self.block(h2)
        return x2, y, (z, x1, h1, s1, qkv, o, lse, a, x2, h2, s2, block, seed)

    def block(self, h):
        """The feed-forward block: (output, kept)."""
        u, uz = P.linear(h, self.w["up"], self.b["up"], act="gelu_tanh", keep=True)
        return P.linear(u, self.w["down"], self.b["down"]), (u, uz)

    def block_backward(self, dy, h, kept):
        """(dh, gradients of the block's weights)."""
        (u, uz), grads = kept, {}
        du, grads["down"], grads["down_b"] = P.linear_backward(dy, u, self.w["down"])
        dh, grads["up"], grads["up_b"] = P.linear_backward(du, h, self.w["up"], uz, act="gelu_tanh")
        return dh, grads

    def backward(self, dx2, dy, kept):
        """From the gradients of forward's results: those of x and z, and of every weight."""
        z, x1, h1, s1, qkv, o, lse, a, x2, h2, s2, block, seed = kept
        dh2, grads = self.block_backward(dy, h2, block)
        d = P.residual_norm_backward(dx2, dh2, x2, a, s2, p=self.p, seed=seed, offset=a.numel(), **self.n[1])
        grads["norm2"], grads["norm2_b"] = d["weight"], d["bias"]
        do, grads["out"], grads["out_b"] = P.linear_backward(d["z"], o.view(self.B, self.S, -1), self.w["out"])
        dqkv = torch.empty_like(qkv)
        P.attention_backward(do.view(o.shape), *self.heads_of(qkv), o, lse, out=self.heads_of(dqkv), **self.ranges)
        dh1, grads["qkv"], grads["qkv_b"] = P.linear_backward(dqkv, h1, self.w["qkv"])
        d = P.residual_norm_backward(d["x"], dh1, x1, z, s1, p=self.p, seed=seed, offset=0, **self.n[0])
        grads["norm1"], grads["norm1_b"] = d["weight"], d["bias"]
        return d["x"], d["z"], grads


class ExpertLayerShare(LayerShare):
    """A layer share whose feed-forward block is `choices` of `experts` blocks for each token: every GPU has 1/d of all their columns."""

    def __init__(self, hidden, heads, d, B, S, documents, p=0.1, seed=0, experts=8, choices=2):
        super().__init__(hidden, heads, d, B, S, documents, p, seed)
        if not 1 <= choices <= experts:
            raise ValueError(f"{choices} choices among {experts} experts")
        g = torch.Generator(device="cuda").manual_seed(seed + 1)
        new = lambda *shape: (torch.randn(*shape, generator=g, device="cuda") * 0.02).bfloat16()  # noqa: E731
        C, F, self.experts, self.choices = hidden, 4 * hidden // d, experts, choices
        self.w.update(router=new(experts, C), up=new(experts, F, C), down=new(experts, C, F))
        self.b.update(up=new(experts, F), down=new(experts, C))

    def block(self, h):
        logits = P.linear(h.view(-1, h.shape[-1]), self.w["router"])
        chosen, weights = P.route(logits, self.choices)
        offsets, rows, place = P.expert_rows(chosen, self.experts)
        u, uz = P.expert_linear(h, self.w["up"], offsets, self.b["up"], rows=rows, act="gelu_tanh", keep=True)
        v = P.expert_linear(u, self.w["down"], offsets, self.b["down"])
        return P.expert_sum(v, place, weights).view(h.shape), (logits, chosen, weights, offsets, rows, place, u, uz, v)

    def block_backward(self, dy, h, kept):
        (logits, chosen, weights, offsets, rows, place, u, uz, v), grads = kept, {}
        dv, dweights = P.expert_sum_backward(dy.view(-1, dy.shape[-1]), v, place, weights)
        du, grads["down"], grads["down_b"] = P.expert_linear_backward(dv, u, self.w["down"], offsets)
        dx, grads["up"], grads["up_b"] = P.expert_linear_backward(du, h, self.w["up"], offsets, uz, rows=rows, act="gelu_tanh")
        dlogits = P.route_backward(dweights, logits, chosen)
        dh, grads["router"], _ = P.linear_backward(dlogits, h.view(-1, h.shape[-1]), self.w["router"], need=("x", "w"))
        return P.expert_sum(dx, place, residual=dh).view(h.shape), grads


def captured(layer, x, z, dx, dy, seed=0):
    """(graph, results) of the forward pass and of the backward pass on these tensors."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):  # once outside a graph: libraries and kernels are loaded
        layer.backward(dx, dy, layer.forward(x, z, seed)[2])
    torch.cuda.current_stream().wait_stream(side)
    graphs = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graphs[0]):
        out = layer.forward(x, z, seed)
    with torch.cuda.graph(graphs[1], pool=graphs[0].pool()):
        grads = layer.backward(dx, dy, out[2])
    return (graphs[0], out), (graphs[1], grads)


def measure(layer, hidden, runs=10):
    """(forward, backward) of the share in ns of the GPU: graphs, replayed in a row behind one another, since the calls of a small share
    take the host longer than their kernels run."""
    x, z, dx, dy = (torch.randn(layer.B, layer.S, hidden, device="cuda").bfloat16() for _ in range(4))
    ns = []
    passes = captured(layer, x, z, dx, dy)
    for graph, _ in passes:
        marks = [[torch.cuda.Event(enable_timing=True) for _ in range(2)] for _ in range(3)]
        for _ in range(3):
            graph.replay()
        for first, last in marks:
            first.record()
            for _ in range(runs):
                graph.replay()
            last.record()
        torch.cuda.synchronize()
        ns.append(int(np.median([first.elapsed_time(last) for first, last in marks]) / runs * 1e6))
    return ns


def profile(hidden, heads, layers, gpus, B, S, documents, emb=3, state_bytes=None, runs=10, experts=0, choices=2):
    """Times per layer and GPU count as the planner takes them: layers between an embedding and a head of `emb` layers' cost."""
    fwd, bwd = np.zeros((layers + 2, gpus), dtype=np.int64), np.zeros((layers + 2, gpus), dtype=np.int64)
    boundary = B * S * hidden * 2
    for d in range(1, gpus + 1):
        if heads % d or 4 * hidden % d:
            fwd[:, d - 1] = bwd[:, d - 1] = P.OOB_FORBIDDEN  # the heads do not divide among so many GPUs
            continue
        share = ExpertLayerShare(hidden, heads, d, B, S, documents, experts=experts, choices=choices) if experts else LayerShare(hidden, heads, d, B, S, documents)
        f, b = measure(share, hidden, runs)
        reduce = -(-2 * (d - 1) * boundary * 10**9 // (d * 8 * LINK)) if d > 1 else 0
        fwd[:, d - 1], bwd[:, d - 1] = f + 2 * reduce, b + 2 * reduce  # two partial sums a layer each way
    fwd[[0, -1]] = np.where(fwd[[0, -1]] == P.OOB_FORBIDDEN, P.OOB_FORBIDDEN, fwd[[0, -1]] * emb)
    bwd[[0, -1]] = np.where(bwd[[0, -1]] == P.OOB_FORBIDDEN, P.OOB_FORBIDDEN, bwd[[0, -1]] * emb)
    weights = (4 + 8 * max(experts, 1)) * hidden * hidden
    mem = np.full(layers + 2, (state_bytes or weights * 16) + 16 * boundary, dtype=np.int64)
    bnd = np.full(layers + 2, 2 * -(-boundary * 10**9 // LINK), dtype=np.int64)
    return fwd, bwd, mem, bnd


def main(argv=None):
    a = argparse.ArgumentParser()
    for name, value in (("hidden", 2048), ("width", 128), ("layers", 24), ("gpus", 4), ("sequences", 2), ("tokens", 2048), ("nodes-min", 2),
                        ("nodes-max", 8), ("microbatches", 32), ("f", 1), ("runs", 10), ("experts", 0), ("choices", 2)):
        a.add_argument("--" + name, type=int, default=value)
    a = a.parse_args(argv)
    documents = [[a.tokens // 3, a.tokens // 2], [a.tokens]][: a.sequences] + [[a.tokens]] * max(0, a.sequences - 2)
    fwd, bwd, mem, bnd = profile(a.hidden, a.hidden // a.width, a.layers, a.gpus, a.sequences, a.tokens, documents, runs=a.runs,
                                 experts=a.experts, choices=a.choices)
    for d in range(a.gpus):
        print(f"layer on {d + 1} GPU(s): " + ("heads do not divide" if fwd[1, d] == P.OOB_FORBIDDEN else f"forward {fwd[1, d] / 1e3:.0f} us, backward {bwd[1, d] / 1e3:.0f} us"))
    job = inputs.PlanInput("measured", fwd, bwd, mem, bnd, a.nodes_min, a.nodes_max, a.gpus, a.microbatches, 192 << 30, a.f)
    res = P.Planner(job.L, job.n_max, job.gpus_per_node).plan(job)
    for i, n in enumerate(range(a.nodes_min, a.nodes_max + 1)):
        if res["feasible"][i]:
            stages, per = P.template_stages(res, i)
            print(f"{n} nodes: {len(per)} stages, {res['T'][i] / 1e6:.1f} ms an iteration, first layers {stages[:-1]}, GPUs {per}")
    return res


if __name__ == "__main__":
    main()
