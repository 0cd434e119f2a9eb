"""A training step on the layer operators against automatic differentiation in 64 bits, and the plan from measured times."""
import math

import numpy as np
import pytest
import torch

import oracle
from paper_2201_12023_amd import profile_layers as P

pytestmark = pytest.mark.gpu


def exact(step):
    """(loss, {name: gradient}) of the same step in 64 bits"""
    D = torch.float64
    leaf = lambda t: t.detach().cpu().to(D).requires_grad_()
    x = x0 = leaf(step.x)
    weights = []
    for layer in step.layers:
        w1, b1, w2, b2 = w = [leaf(t) for t in (layer.w1, layer.b1, layer.w2, layer.b2)]
        weights.append(w)
        cuts = [0, x.shape[0]] if layer.offsets is None else layer.offsets.cpu().tolist()
        parts = []
        for e, (a, b) in enumerate(zip(cuts, cuts[1:])):
            at = (lambda t: t) if layer.offsets is None else (lambda t: t[e])
            z = x[a:b] @ at(w1).t() + at(b1)
            h = z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))) / 2
            parts.append(x[a:b] + h @ at(w2).t() + at(b2))
        x = torch.cat(parts)
    words = leaf(step.words)
    loss = torch.nn.functional.cross_entropy(x @ words.t(), step.target.cpu(), reduction="none")
    loss.backward(step.dloss.cpu().to(D))
    return loss.detach(), x0.grad, [[t.grad for t in w] for w in weights], words.grad


def test_step_against_automatic_differentiation():
    """In 32 bits a product of n terms is off by at most n 2^-23 of its operands' norms; sixteen of them with n <= 320 lie one behind the
    other, each with a gain of at most two (weights are scaled to keep norms, and a layer adds its input): 16 * 320 * 2^-23 * 2."""
    bound = 16 * 320 * 2.0 ** -23 * 2
    step = P.Step(P.Model(layers=3, rows=150, width=72, inner=200, experts=3, expert_every=2, words=320, dtype="float32"))
    loss, dx = step.run()
    ref_loss, ref_dx, ref_weights, ref_words = exact(step)

    def close(name, got, ref):
        off = float((got.cpu().double() - ref).norm() / ref.norm())
        assert off <= bound, (name, off)
    close("loss", loss, ref_loss)
    close("dx", dx, ref_dx)
    close("words", step.dwords, ref_words)
    for k, (layer, ref) in enumerate(zip(step.layers, ref_weights)):
        for name, g, r in zip(("w1", "b1", "w2", "b2"), layer.grads, ref):
            close(f"layer {k} {name}", g, r)


def test_the_step_twice_gives_the_same():
    step = P.Step(P.Model(layers=2, rows=300, width=64, inner=264, experts=4, words=1000))
    first = [t.clone() for t in step.run()] + [g.clone() for layer in step.layers for g in layer.grads]
    again = list(step.run()) + [g for layer in step.layers for g in layer.grads]
    assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_plan_from_measured_times():
    model = P.Model(layers=4, rows=256, width=256, inner=1024, experts=4, words=4096)
    found, tables, shapes = P.plan(model, 1, 4, 8, 1 << 36, 153e9)
    table = oracle.build_table(*tables, 1 << 36)
    _, ref = oracle.solve(table, 1, 4, 8, shapes, oracle.all_candidates(table, shapes), True)
    assert (found["T_star"], found["t_max"], found["num_stages"], found["first_layer"], found["shape_idx"]) == \
           (ref.T_star, ref.t_max, ref.num_stages, ref.first_layer, ref.shape_idx)
    used = tables[0][np.triu_indices(4)]
    assert (used > 0).all() and (used[used < P.INF] < 1_000_000).all()


def test_command(capsys):
    sizes = ["--layers", "2", "--rows", "64", "--width", "64", "--inner", "128", "--experts", "2", "--words", "512", "--devices", "2"]
    assert P.main(sizes) == 0
    out = capsys.readouterr().out
    assert "layer  1 experts + loss" in out and "32 microbatches in" in out
    assert P.main(sizes + ["--memory", "1000"]) == 1
    assert "no plan fits" in capsys.readouterr().out
