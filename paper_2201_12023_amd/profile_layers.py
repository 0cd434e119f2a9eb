"""Profiles layers on this GPU and plans with what it measured.

    python -m paper_2201_12023_amd.profile_layers [--layers 8 --width 2048 ...]

A model of dense and expert layers with a loss over a vocabulary at its end runs one training step, forward and backward, on the
operators of ``layers``, with every submesh's share of the work in turn; the times, with the shares' memory, are the options of
``alpa_dp_create_from_profiles``, and the dynamic program cuts the model into stages with them.

A share is one device's of d, in two ways: "rows" (a d-th of the rows, all weights) or "weights" (all rows, a d-th of the inner
width and of the words).  One GPU stands for each device of the mesh; what devices exchange is not run but added as bytes over
``link`` bytes/s: the gradients of all weights once a batch for "rows", the layer's result and its gradient once a microbatch for
"weights" (not what the loss exchanges where its words are split).

A layer is its two products with their activation; what else a block has, its attention, is not timed.  Times are between events around a
layer's calls, so where the GPU waits for launches, some 12 us a call, they are the host's.
"""
from __future__ import annotations

import argparse
from dataclasses import dataclass

import numpy as np

from . import binding, workloads

INF = 2 ** 31 - 1                    # an option that does not exist
SPLITS = ("rows", "weights")


@dataclass(frozen=True)
class Model:
    """``layers`` layers, every ``expert_every``-th (0: none) of experts, the last one with the loss; sizes of one microbatch."""
    layers: int = 8
    rows: int = 4096
    width: int = 2048
    inner: int = 8192
    experts: int = 8
    expert_every: int = 2
    words: int = 51200
    dtype: str = "bfloat16"

    def kind(self, k):
        return "experts" if self.expert_every and (k + 1) % self.expert_every == 0 else "dense"

    def weights(self, k):
        n = (2 * self.width * self.inner + self.inner + self.width) * (self.experts if self.kind(k) == "experts" else 1)
        return n + (self.words * self.width if k == self.layers - 1 else 0)

    def share(self, d, split):
        """One device's part as a model of its own, None if it cannot be cut so."""
        cut = dict(rows=self.rows // d) if split == "rows" else dict(inner=self.inner // d, words=self.words // d)
        if any(getattr(self, name) % d for name in cut):
            return None
        return Model(**{**self.__dict__, **cut})


class Layer:
    """y = x + act(x w1^T + b1) w2^T + b2 on ``rows`` rows; an expert layer's rows are sorted by expert."""

    def __init__(self, model, k, device, generator):
        import torch
        self.dtype, self.offsets = getattr(torch, model.dtype), None
        many = ()
        if model.kind(k) == "experts":
            many = (model.experts,)
            cuts = torch.sort(torch.randint(0, model.rows + 1, (model.experts - 1,), generator=generator, device=device))[0]
            ends = torch.tensor([0, model.rows], device=device)
            self.offsets = torch.cat([ends[:1], cuts, ends[1:]]).to(torch.int32)
        new = lambda *size, scale: (torch.randn(size, generator=generator, device=device) * scale).to(self.dtype)
        self.w1, self.b1 = new(*many, model.inner, model.width, scale=model.width ** -0.5), new(*many, model.inner, scale=0.02)
        self.w2, self.b2 = new(*many, model.width, model.inner, scale=model.inner ** -0.5), new(*many, model.width, scale=0.02)

    def forward(self, x):
        from . import layers as L
        if self.offsets is None:
            h, z = L.alpa_linear_forward(x, self.w1, self.b1, act=L.ALPA_ACT_GELU_TANH, keep_z=True)
            y = L.alpa_linear_forward(h, self.w2, self.b2, residual=x)
        else:
            h, z = L.alpa_experts_forward(x, self.w1, self.offsets, self.b1, act=L.ALPA_ACT_GELU_TANH, keep_z=True)
            y = L.alpa_experts_forward(h, self.w2, self.offsets, self.b2, residual=x)
        self.saved = x, z, h
        return y

    def backward(self, dy):
        """dx; the weights' gradients are kept in ``grads``."""
        from . import layers as L
        x, z, h = self.saved
        if self.offsets is None:
            dh, dw2, db2 = L.alpa_linear_backward(dy, h, self.w2)
            dx, dw1, db1 = L.alpa_linear_backward(dh, x, self.w1, z, L.ALPA_ACT_GELU_TANH)
        else:
            dh, dw2, db2 = L.alpa_experts_backward(dy, h, self.w2, self.offsets)
            dx, dw1, db1 = L.alpa_experts_backward(dh, x, self.w1, self.offsets, z, L.ALPA_ACT_GELU_TANH)
        self.grads = dw1, db1, dw2, db2
        return dx.add_(dy)


class Step:
    """One training step of a share of the model: weights, inputs and the order of its layers."""

    def __init__(self, model, device="cuda", seed=0):
        import torch
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        self.model = model
        self.layers = [Layer(model, k, device, g) for k in range(model.layers)]
        self.x = torch.randn(model.rows, model.width, generator=g, device=device).to(self.layers[0].dtype)
        self.words = (torch.randn(model.words, model.width, generator=g, device=device) * model.width ** -0.5).to(self.x.dtype)
        self.target = torch.randint(0, model.words, (model.rows,), generator=g, device=device)
        self.dloss = torch.full((model.rows,), 1.0 / model.rows, device=device)

    def run(self, mark=lambda: None):
        """(loss of each row, dx); ``mark`` is called at the beginning and behind each layer of both directions, the loss being the
        last layer's."""
        from . import layers as L
        mark()
        x = self.x
        for layer in self.layers[:-1]:
            x = layer.forward(x)
            mark()
        x = self.layers[-1].forward(x)
        loss, lse = L.alpa_vocab_loss_forward(x, self.words, self.target)
        mark()
        dx, self.dwords = L.alpa_vocab_loss_backward(self.dloss, x, self.words, self.target, lse)
        for layer in reversed(self.layers):
            dx = layer.backward(dx)
            mark()
        return loss, dx

    def microseconds(self, repeats=5):
        """Forward and backward of each layer, the least of ``repeats`` runs."""
        import torch
        times = []
        for n in range(repeats + 1):                     # (the first is not counted)
            events = []

            def mark():
                events.append(torch.cuda.Event(enable_timing=True))
                events[-1].record()
            self.run(mark)
            torch.cuda.synchronize()
            spans = [a.elapsed_time(b) * 1e3 for a, b in zip(events, events[1:])]
            K = len(self.layers)
            if n:
                times.append([spans[k] + spans[2 * K - 1 - k] for k in range(K)])
        return np.min(np.array(times), axis=0)


def measure(model):
    """Microseconds of each layer of a share on this GPU."""
    return Step(model).microseconds()


def profiles(model, shapes, microbatches, link, measure=measure):
    """(t_l, mem_stage, mem_act), arrays [K, K, S, 2]: the options of SPLITS for every stage of layers and every submesh shape.

    Memory: weights and gradients in ``dtype`` and twelve bytes a weight for the optimizer; for a microbatch a layer's input,
    z and h, which the backward pass reads."""
    K, es = model.layers, 4 if model.dtype == "float32" else 2
    size = (K, K, len(shapes), len(SPLITS))
    t_l, mem_stage, mem_act = np.full(size, INF, np.int32), np.zeros(size, np.int64), np.zeros(size, np.int64)
    known = {}
    for q, (n, m) in enumerate(shapes):
        d = int(n) * int(m)
        for o, split in enumerate(SPLITS):
            share = model.share(d, split)
            if share is None:
                continue
            if share not in known:
                known[share] = measure(share)
            ring = 2.0 * (d - 1) / d / link * 1e6                       # microseconds a byte
            exchanged = [es * (model.weights(k) / microbatches if split == "rows" else 2 * model.rows * model.width) for k in range(K)]
            time = [known[share][k] + ring * exchanged[k] for k in range(K)]
            weights = [(2 * es + 12) * share.weights(k) for k in range(K)]
            kept = [es * share.rows * (share.width + 2 * share.inner) for k in range(K)]
            for k in range(K):
                for i in range(k, K):
                    t_l[k, i, q, o] = int(np.ceil(sum(time[k:i + 1])))
                    mem_stage[k, i, q, o] = sum(weights[k:i + 1])
                    mem_act[k, i, q, o] = sum(kept[k:i + 1])
    return t_l, mem_stage, mem_act


def plan(model, nodes, devices, microbatches, mem_device, link, measure=measure):
    """The plan for a mesh of nodes x devices (``alpa_dp_solve``'s, with "shapes": the submesh of each stage)."""
    shapes = workloads.submesh_shapes(nodes, devices)
    tables = profiles(model, shapes, microbatches, link, measure)
    h = binding.alpa_dp_create_from_profiles(*tables, mem_device, model.layers, nodes, devices, microbatches, shapes)
    try:
        found = binding.alpa_dp_solve(h, None, 0, binding.ALPA_DP_PRUNE, want_T=False)[1]
    finally:
        binding.alpa_dp_destroy(h)
    found["shapes"] = [tuple(int(v) for v in shapes[q]) for q in found["shape_idx"]]
    return found, tables, shapes


def main(argv=None):
    p = argparse.ArgumentParser(prog="python -m paper_2201_12023_amd.profile_layers", description=__doc__.split("\n")[0])
    for name, value in Model().__dict__.items():
        p.add_argument("--" + name.replace("_", "-"), type=type(value), default=value)
    p.add_argument("--nodes", type=int, default=1)
    p.add_argument("--devices", type=int, default=8, help="of a node")
    p.add_argument("--microbatches", type=int, default=32)
    p.add_argument("--memory", type=float, default=288e9, help="bytes of a device")
    p.add_argument("--link", type=float, default=153e9, help="bytes/s between devices")
    a = p.parse_args(argv)
    model = Model(**{name: getattr(a, name) for name in Model().__dict__})
    found, (t_l, _, _), shapes = plan(model, a.nodes, a.devices, a.microbatches, int(a.memory), a.link)
    print("microseconds of a microbatch, forward and backward (" + ", ".join(SPLITS) + "):")
    for k in range(model.layers):
        cells = ["x".join(map(str, s)) + " " + "/".join("-" if t == INF else str(t) for t in t_l[k, k, q])
                 for q, s in enumerate(shapes)]
        print(f"  layer {k:2d} {model.kind(k) + (' + loss' if k == model.layers - 1 else ''):14s} " + "  ".join(cells))
    if found["num_stages"] == 0:
        print("no plan fits the memory")
        return 1
    print(f"{a.microbatches} microbatches in {found['T_star']} us, {found['num_stages']} stages:")
    for s, shape in enumerate(found["shapes"]):
        print(f"  layers {found['first_layer'][s]} .. {found['first_layer'][s + 1] - 1} on {shape[0]} x {shape[1]}")
    return 0


if __name__ == "__main__":
    raise SystemExit(main())
