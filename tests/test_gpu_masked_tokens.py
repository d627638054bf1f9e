"""The token operators together, as examples/masked_tokens.py uses them around a GGNN."""
from __future__ import annotations

import math
import os
import sys

import numpy as np
import pytest
import torch

from gpu_common import ensure_built

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    ensure_built()


def test_masked_token_training_learns():
    """The loss starts near that of guessing (log V; logits of unit states against rows of norm 1) and
    falls below half of it: a hidden token follows from its neighbour's."""
    import masked_tokens as mt
    losses = mt.train(steps=120)
    assert abs(losses[0] - math.log(60)) < 2.0
    assert np.mean(losses[-10:]) < 0.5 * math.log(60), losses[::10]


def test_a_step_is_repeatable_and_its_gradient_descends():
    """The same step gives the same bits twice (no order of additions is left to chance outside the
    GGNN's own kernels), and a small step against the gradient lowers the same loss."""
    import masked_tokens as mt
    net = mt.MaskedTokenModel(p=0.2)
    ids, target, dloss = net.hide(np.random.default_rng(3))
    n = int((target >= 0).sum())
    net.loss_and_gradients(ids, target, dloss)
    first, grads = net.loss.clone(), {k: v.clone() for k, v in net.grad.items()}
    net.call = 0
    net.loss_and_gradients(ids, target, dloss)
    assert torch.equal(first, net.loss)
    for k, v in grads.items():
        assert torch.equal(v, net.grad[k]), k
    assert float(first.sum()) / n > 1.0
    # along the table's gradient: the loss changes by -step |g|^2 to first order
    g = grads["table"]
    step = 0.02 * float(first.sum()) / n / float((g * g).sum())
    net.work["table"] = (net.master["table"] - step * g).to(torch.bfloat16)
    net.call = 0
    net.loss_and_gradients(ids, target, dloss)
    fall = (float(first.sum()) - float(net.loss.sum())) / float(first.sum())
    # bf16 rounding of the table and of the states moves the loss by less than the 2% that is asked for
    assert 0.005 < fall < 0.04, fall
