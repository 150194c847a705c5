"""A step of training as a program makes it: blocks, cross entropy, the gradients' norm and AdamW, one behind the other, eager and captured."""
import math

import numpy as np
import pytest
import torch

from ff_util import act, slope
from gpu_util import announce
from opt_util import Plain

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("optimizer", ["adamw", "adamw8"])
def test_the_command_runs(optimizer):
    from paper_2011_05630_amd import ff_example
    announce(optimizer)
    losses, off = ff_example.main(["--blocks", "2", "--width", "256", "--hidden", "712", "--classes", "100", "--tokens", "1024", "--steps", "6",
                                   "--optimizer", optimizer])
    assert len(losses) == 6 and all(math.isfinite(v) for v in losses)
    assert off <= 8 * 2.0 ** -8             # (as of the same example with the plain update)


def want_gradients(net, x, target):
    """Of the mean over the rows with a target, in 64 bits on the weights as they are."""
    wg, wu, wd, wh = (w.double().cpu() for w in net.weights)
    x64, t = x.double().cpu(), target.cpu()
    g, u = x64 @ wg.t(), x64 @ wu.t()
    h = act("silu", g) * u
    y = x64 + h @ wd.t()
    z = y @ wh.t() + net.bias.double().cpu()
    counted = t >= 0
    p = torch.softmax(z, 1)
    loss = -(torch.log_softmax(z, 1).gather(1, t.clamp_min(0)[:, None]).squeeze(1))[counted].mean()
    dz = p.scatter_add(1, t.clamp_min(0)[:, None], -torch.ones_like(p[:, :1])) * (counted / counted.sum())[:, None]
    dy = dz @ wh
    dh = dy @ wd
    dg, du = dh * u * slope("silu", g), dh * act("silu", g)
    return loss, (dg.t() @ x64, du.t() @ x64, dy.t() @ h, dz.t() @ y, dz.sum(0))


@pytest.mark.parametrize("state", ["fp32", "8bit"])
def test_a_step(state):
    """Gradients within 5 % of their norm (every tensor on the way is rounded to bf16, 2^-8 of its values at most, which a handful of products carry on), then
    the step on those very gradients: states bit for bit, weights within AdamW's bounds."""
    from paper_2011_05630_amd import ff_example, optimizer
    net = ff_example.Stack(1, 64, 136, 24)
    trainer = ff_example.Trainer(net, state=state, most=0.25, decay=0.1, seed=9)
    x, target = ff_example.synthetic(96, 64, 24, 5)
    target[::5] = -1
    announce(state)
    loss, grads = trainer.gradients(x, target)
    want_loss, want = want_gradients(net, x, target)
    assert abs(float(loss) - float(want_loss)) <= 0.05 * float(want_loss)
    for got, w in zip(grads, want):
        assert got.shape == w.shape and float((got.double().cpu() - w).norm()) <= 0.05 * float(w.norm())
    norm, factor = optimizer.gradient_norm(grads, most=0.25)
    size = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
    assert abs(float(norm) / size - 1) < 2.0 ** -23 and size > 0.25
    params = net.master + [net.bias]
    plain = [Plain(np.zeros(p.numel()), at, (0.9, 0.95), 1e-8, d, state == "8bit", 9)
             for p, at, d in zip(params, trainer.optimizer.offsets, [0.1] * 4 + [0.0])]
    before = [p.double().cpu().numpy().reshape(-1) for p in params]
    again = float(trainer.step(x, target, 0.01))
    assert again == float(loss)
    for i, (p, q) in enumerate(zip(params, plain)):
        value, bound = q.step(before[i], grads[i].float().cpu().numpy().reshape(-1), 0, 0.01, float(factor))
        assert (np.abs(p.double().cpu().numpy().reshape(-1) - value) <= bound).all()
        if i < 4:
            assert torch.equal(net.weights[i], p.bfloat16())
        at = trainer.optimizer.offsets[i]
        m = trainer.optimizer.m[at:at + q.m.size]
        if state == "8bit":
            assert np.array_equal(m.view(torch.uint8).cpu().numpy(), q.mc)
        else:
            assert np.array_equal(m.cpu().numpy(), q.m)


@pytest.mark.parametrize("state", ["fp32", "8bit"])
def test_a_captured_step(state):
    """A whole step in a graph, on new tokens from replay to replay, the same bits as eager steps."""
    from paper_2011_05630_amd import ff_example
    pair = []
    for _ in range(2):
        net = ff_example.Stack(2, 64, 136, 1000, seed=3)
        pair.append((net, ff_example.Trainer(net, state=state, seed=4)))
    data = [ff_example.synthetic(200, 64, 1000, s) for s in range(4)]
    x, target = data[0][0].clone(), data[0][1].clone()
    (net, trainer), (net2, trainer2) = pair
    for t in (trainer, trainer2):
        t.step(x, target, 0.01)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = trainer.step(x, target, 0.01)
    for s in (1, 2, 3, 1):
        x.copy_(data[s][0])
        target.copy_(data[s][1])
        graph.replay()
        torch.cuda.synchronize()
        assert float(loss) == float(trainer2.step(data[s][0], data[s][1], 0.01))
        for a, b in zip(net.master + net.weights + [net.bias], net2.master + net2.weights + [net2.bias]):
            assert torch.equal(a, b)
    assert int(trainer.optimizer.count) == 5


def test_fp16_with_a_loss_scale():
    """A loss scaled so far that gradients overflow leaves everything as it was; scaled less, the step is the unscaled one's within its roundings."""
    from paper_2011_05630_amd import ff_example, loss, optimizer
    t = torch.float16
    net = ff_example.Stack(1, 64, 136, 24, dtype=t)
    x, target = ff_example.synthetic(96, 64, 24, 6, dtype=t)
    op = loss.CrossEntropy(net.head.weight, net.bias)
    params = [net.master[-1], net.bias]
    opt = optimizer.AdamW(params, [net.weights[-1], None])
    before = [p.clone() for p in params]
    for scale in (2.0 ** 24, 2.0 ** 10):
        _, _, dw, db = op.gradients(x, target, scale / 96)
        norm, factor = optimizer.gradient_norm([dw, db], most=1.0, scale=1.0 / scale)
        opt.step([dw, db], 0.01, factor=factor)
        if scale > 2.0 ** 20:
            assert dw.isinf().any() and factor.isnan() and int(opt.count) == 0
            assert all(torch.equal(a, b) for a, b in zip(before, params))
    assert int(opt.count) == 1 and torch.isfinite(norm)
    # the first step moves every element by the rate, against its gradient
    for p, b, g in zip(params, before, (dw, db)):
        assert torch.equal((p - b).sign()[g != 0], -g.float().sign()[g != 0])
