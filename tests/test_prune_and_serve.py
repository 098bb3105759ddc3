"""The example that prunes a little network, limits its gradients and serves it in 8-bit integers."""
import math
import os
import sys

import pytest

from gpu_util import say

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def load():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import prune_and_serve
    finally:
        sys.path.pop(0)
    return prune_and_serve


@pytest.mark.gpu
def test_the_example_trains_and_serves():
    import torch
    say("[case] examples/prune_and_serve.py")
    E = load()
    norms, right, far = E.main(steps=60, say=say)
    assert norms.shape == (60,) and bool(torch.isfinite(norms).all()) and float(norms.max()) > 1.0     # the limit was met
    # Two layers, each with activations and weights rounded to 127 steps of a row's largest: rms 1/440 of it an operand, some
    # four times that of the rms value, four operands: 2 %.  One class in ten by chance.
    assert far < 0.06 and right > 0.5


@pytest.mark.gpu
def test_gradients_are_limited_as_the_formula_says():
    """One step of the example's: its gradients against those computed apart, limited by elementary operations."""
    import torch
    import torch.nn.functional as F
    import paper_1909_05073_amd as P
    say("[case] a step of examples/prune_and_serve.py")
    E = load()
    p = E.parameters(3)
    x, label = E.images(32, seed=5)
    want = torch.autograd.grad(F.cross_entropy(E.forward(p, x), label), list(p.values()))
    total = math.sqrt(sum(float(g.double().square().sum()) for g in want))
    grads = [g.clone() for g in want]
    norm = P.clip_grad_norm(grads, 0.25 * total)
    assert abs(float(norm) - total) <= 1.1 * 2.0 ** -24 * total
    for g, w in zip(grads, want):
        exact = w.double() * (0.25 * total / (total + 1e-6))
        assert bool(((g.double() - exact).abs() <= 4 * 2.0 ** -24 * exact.abs() + 1e-40).all())
