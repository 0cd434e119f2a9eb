"""A training step of blocks, attention and layer norm among them, against automatic differentiation in 64 bits, and the plan from its times."""
import math

import numpy as np
import pytest
import torch

import oracle
from paper_2201_12023_amd import profile_layers as P

pytestmark = pytest.mark.gpu
D = torch.float64


def norm(x, weight, bias):
    d = x - x.mean(1, keepdim=True)
    return d / torch.sqrt((d * d).mean(1, keepdim=True) + 1e-5) * weight + bias


def turned(x, positions, dim):
    half = torch.arange(dim // 2, dtype=D)
    u = positions[:, None, None] * 10000.0 ** (-2.0 * half / dim)
    a, b = x[..., :dim // 2], x[..., dim // 2:]
    return torch.cat([a * torch.cos(u) - b * torch.sin(u), a * torch.sin(u) + b * torch.cos(u)], -1)


def attend(q, k, v, cuts):
    """Causal attention within the sequences."""
    rows, group = q.shape[0], q.shape[1] // k.shape[1]
    row = torch.arange(rows)
    of = torch.bucketize(row, torch.tensor(cuts[1:]), right=True)
    seen = (of[:, None] == of) & (row[:, None] >= row)
    k, v = (t.repeat_interleave(group, 1).transpose(0, 1) for t in (k, v))
    s = (q.transpose(0, 1) @ k.transpose(1, 2)) * q.shape[2] ** -0.5
    return (torch.softmax(s.masked_fill(~seen, -math.inf), -1) @ v).transpose(0, 1)


def exact(step):
    """(loss, dx, each layer's gradients, those of attention) of the same step in 64 bits"""
    leaf = lambda t: t.detach().cpu().to(D).requires_grad_()
    x = x0 = leaf(step.x)
    weights = []
    for layer in step.layers:
        a = layer.attention
        w = [leaf(t) for t in (layer.w1, layer.b1, layer.w2, layer.b2, a.wqkv, a.wo, *a.norms[0], *a.norms[1])]
        weights.append(w)
        w1, b1, w2, b2, wqkv, wo, n1, m1, n2, m2 = w
        qkv = (norm(x, n1, m1) @ wqkv.t()).view(x.shape[0], -1, a.dim)
        place = a.positions.cpu().to(D)
        q, k = turned(qkv[:, :a.heads], place, a.dim), turned(qkv[:, a.heads:a.heads + a.kv], place, a.dim)
        x = x + attend(q, k, qkv[:, a.heads + a.kv:], a.offsets.tolist()).flatten(1) @ wo.t()
        inside = norm(x, n2, m2)
        cuts = [0, x.shape[0]] if layer.offsets is None else layer.offsets.tolist()
        parts = []
        for e, (i, j) in enumerate(zip(cuts, cuts[1:])):
            at = (lambda t: t) if layer.offsets is None else (lambda t: t[e])
            z = inside[i:j] @ at(w1).t() + at(b1)
            h = z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))) / 2
            parts.append(x[i:j] + h @ at(w2).t() + at(b2))
        x = torch.cat(parts)
    words = leaf(step.words)
    loss = torch.nn.functional.cross_entropy(x @ words.t(), step.target.cpu(), reduction="none")
    loss.backward(step.dloss.cpu().to(D))
    return loss.detach(), x0.grad, [[t.grad for t in w] for w in weights], words.grad


def test_step_against_automatic_differentiation():
    """In 32 bits a sum of n products is off by at most n 2^-23 of its operands' norms; of a block's forward and backward pass twelve lie one behind the other
    (norm, product, scores, weighted sum, product, norm, two products, and as many back are counted with them), n <= 320, in two blocks and the loss, each with a
    gain of at most two: 2 * 24 * 320 * 2^-23 * 2."""
    bound = 2 * 24 * 320 * 2.0 ** -23 * 2
    step = P.Step(P.Model(layers=2, rows=150, width=72, inner=200, experts=3, expert_every=2, words=320, dtype="float32", heads=6, kv_heads=2, dim=20, context=64))
    loss, dx = step.run()
    ref_loss, ref_dx, ref_weights, ref_words = exact(step)

    def close(name, got, ref):
        off = float((got.cpu().double() - ref).norm() / ref.norm())
        assert off <= bound, (name, off)
    close("loss", loss, ref_loss)
    close("dx", dx, ref_dx)
    close("words", step.dwords, ref_words)
    names = ("w1", "b1", "w2", "b2", "wqkv", "wo", "norm 1 weight", "norm 1 bias", "norm 2 weight", "norm 2 bias")
    for k, (layer, ref) in enumerate(zip(step.layers, ref_weights)):
        for name, g, r in zip(names, (*layer.grads, *layer.attention.grads), ref):
            close(f"layer {k} {name}", g, r)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_the_step_twice_gives_the_same(dtype):
    step = P.Step(P.Model(layers=2, rows=600, width=128, inner=264, experts=4, words=1000, heads=8, kv_heads=2, dim=64, context=250, dtype=dtype))
    kept = lambda: [g for layer in step.layers for g in (*layer.grads, *layer.attention.grads)]
    first = [t.clone() for t in step.run()] + [g.clone() for g in kept()]
    again = list(step.run()) + kept()
    assert all(torch.equal(a, b) and bool(torch.isfinite(a.float()).all()) for a, b in zip(first, again))


def test_plan_from_measured_times():
    model = P.Model(layers=4, rows=512, width=256, inner=1024, experts=4, words=4096, heads=8, kv_heads=4, dim=64, context=128)
    found, tables, shapes = P.plan(model, 1, 4, 8, 1 << 36, 153e9)
    table = oracle.build_table(*tables, 1 << 36)
    _, ref = oracle.solve(table, 1, 4, 8, shapes, oracle.all_candidates(table, shapes), True)
    assert (found["T_star"], found["t_max"], found["num_stages"], found["first_layer"], found["shape_idx"]) == \
           (ref.T_star, ref.t_max, ref.num_stages, ref.first_layer, ref.shape_idx)
    used = tables[0][np.triu_indices(4)]
    assert (used > 0).all() and (used < P.INF).all()


def test_command(capsys):
    sizes = ["--layers", "2", "--rows", "64", "--width", "64", "--inner", "128", "--experts", "2", "--words", "512", "--devices", "2", "--heads", "4",
             "--dim", "32", "--context", "32"]
    assert P.main(sizes) == 0
    assert "32 microbatches in" in capsys.readouterr().out
