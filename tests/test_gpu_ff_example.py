"""The example that trains and serves with the feed-forward operators."""
import math

import pytest
import torch

from ff_util import act, slope
from gpu_util import announce

pytestmark = pytest.mark.gpu


def test_trains_and_answers_single_tokens():
    from paper_2011_05630_amd import ff_example
    announce("ff_example")
    losses, off = ff_example.main(["--blocks", "2", "--width", "256", "--hidden", "712", "--classes", "100", "--tokens", "1024", "--steps", "12"])
    assert all(math.isfinite(v) for v in losses)
    assert losses[0] > 0.5 * math.log(100) and losses[-1] < 0.5 * losses[0]
    # two residual blocks and the classifier round activations and logits to bf16: a handful of roundings of 2^-8, in another order of sums
    assert off <= 8 * 2.0 ** -8


def test_gradients_of_the_stack():
    """Against the formulas in 64 bits on the operators' own weights: every tensor on the way is rounded to bf16 (2^-8 of its values at
    most), which a handful of products carry on: 5 % of the gradient's norm bounds them."""
    from paper_2011_05630_amd import ff_example
    net = ff_example.Stack(1, 64, 136, 24)
    x, target = ff_example.synthetic(96, 64, 24, 5)
    announce("ff_example gradients")
    _, grads, dbias = net.gradients(x, target)
    wg, wu, wd, wh = (w.double().cpu() for w in net.weights)
    x64 = x.double().cpu()
    g, u = x64 @ wg.t(), x64 @ wu.t()
    h = act("silu", g) * u
    y = x64 + h @ wd.t()
    dz = torch.softmax(y @ wh.t(), 1)
    dz[torch.arange(96), target.cpu()] -= 1
    dy = dz @ wh
    dh = dy @ wd
    dg, du = dh * u * slope("silu", g), dh * act("silu", g)
    for got, want in zip(grads + [dbias], (dg.t() @ x64, du.t() @ x64, dy.t() @ h, dz.t() @ y, dz.sum(0))):
        assert got.shape == want.shape
        assert float((got.double().cpu() - want).norm()) <= 0.05 * float(want.norm())
