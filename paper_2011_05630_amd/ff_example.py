"""The feed-forward operators as a program uses them: a stack of gated residual blocks and a classifier, trained on synthetic
tokens with hand-written gradients, then answering single tokens.

    python -m paper_2011_05630_amd.ff_example [--blocks 2] [--width 512] [--hidden 1408] [--classes 1000] [--tokens 2048] [--steps 30]
                                              [--optimizer sgd|adamw|adamw8] [--rate 1.0]

sgd: the loss written out in PyTorch, a plain update.  adamw, adamw8: the cross entropy and its gradients in one call, the gradients' norm brought down to 1 and
AdamW with states in 32 or in 8 bits, by the library.  Prints the loss as it trains, the time of a step and of a single token, and how far the single token's logits are from the same row of
a whole batch.
"""
import argparse
import math
import time

import torch

from .feedforward import FeedForward, GatedLinear, Linear
from .loss import CrossEntropy
from .optimizer import AdamW, gradient_norm


class Stack:
    """x -> x + block_1(x) -> ... -> logits.  Weights of type `dtype` for the products, fp32 copies for the updates."""

    def __init__(self, blocks, width, hidden, classes, dtype=torch.bfloat16, seed=0):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.master, self.weights = [], []

        def weight(o, i, scale=1.0):
            m = torch.randn(o, i, generator=gen, device="cuda") * (scale / math.sqrt(i))
            self.master.append(m)
            self.weights.append(m.to(dtype))
            return self.weights[-1]

        self.blocks = []
        for _ in range(blocks):
            gate, up, down = weight(hidden, width), weight(hidden, width), weight(width, hidden, 1 / math.sqrt(blocks))
            self.blocks.append(FeedForward(GatedLinear(gate, up, act="silu"), Linear(down)))
        self.bias = torch.zeros(classes, device="cuda")
        self.head = Linear(weight(classes, width), self.bias)

    def run(self, x):
        for b in self.blocks:
            x = b.run(x, residual=x)
        return self.head.run(x)

    def _run_saved(self, x):
        """-> (what the classifier reads, what each block's backward pass needs)."""
        kept = []
        for b in self.blocks:
            y, saved = b.run_saved(x, residual=x)
            kept.append((x, saved))
            x = y
        return x, kept

    def _backward(self, dx, dw, kept):
        """Gradients of the weights, from those of what the classifier reads and of its weight."""
        grads = [dw]
        for b, (x, saved) in zip(reversed(self.blocks), reversed(kept)):
            through, gated, down = b.backward(dx, x, saved)
            grads += [down[0], gated[1], gated[0]]
            dx = dx + through                               # the residual's part
        return grads[::-1]

    def gradients(self, x, target):
        """-> (mean cross entropy, gradients of the weights in the order of `weights`, gradient of the bias)."""
        x, kept = self._run_saved(x)
        logits, _ = self.head.run_saved(x)
        z = logits.float()
        z = z - z.amax(1, keepdim=True)
        logp = z - z.exp().sum(1, keepdim=True).log()
        rows = torch.arange(x.shape[0], device=x.device)
        loss = -logp[rows, target].mean()
        dz = logp.exp()
        dz[rows, target] -= 1.0
        # the gradient of the rows' sum: of their mean it would be too small for the type.  The updates divide.
        dx, dw, dbias = self.head.backward(dz.to(x.dtype), x, None)
        return loss, self._backward(dx, dw, kept), dbias

    def step(self, x, target, rate):
        loss, grads, dbias = self.gradients(x, target)
        scale = rate / x.shape[0]
        for m, w, g in zip(self.master, self.weights, grads):
            m.sub_(g.float(), alpha=scale)
            w.copy_(m)                                      # in place: the operators read the weights where they lie
        self.bias.sub_(dbias, alpha=scale)
        return loss


class Trainer:
    """A stack's steps by the library's operators: `state` "fp32" or "8bit", the gradients' norm at most `most`."""

    def __init__(self, net, state="fp32", most=1.0, decay=0.01, seed=0):
        self.net, self.most = net, most
        self.loss = CrossEntropy(net.head.weight, net.bias)
        # 32-bit weights, and beside them those that the products read; no decay of the bias
        self.optimizer = AdamW(net.master + [net.bias], net.weights + [None], decay=[decay] * len(net.master) + [0.0], state=state, seed=seed)

    def gradients(self, x, target):
        """-> (mean cross entropy, the mean's gradients of the weights in the order of `weights` and of the bias).  Targets below zero are passed over."""
        counted = (target >= 0).sum().clamp_min(1).float()
        x, kept = self.net._run_saved(x)
        loss, dx, dw, dbias = self.loss.gradients(x, torch.where(target >= 0, target, self.loss.ignore_index), 1.0 / counted)
        return loss.sum() / counted, self.net._backward(dx, dw, kept) + [dbias]

    def step(self, x, target, rate):
        loss, grads = self.gradients(x, target)
        norm, factor = gradient_norm(grads, most=self.most)
        self.optimizer.step(grads, rate, factor=factor)
        return loss


def synthetic(tokens, width, classes, seed, dtype=torch.bfloat16):
    """Tokens around one centre per class."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    centres = torch.randn(classes, width, generator=gen, device="cuda")
    gen.manual_seed(seed)
    target = torch.randint(classes, (tokens,), generator=gen, device="cuda")
    return (centres[target] + 0.5 * torch.randn(tokens, width, generator=gen, device="cuda")).to(dtype), target


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("blocks", 2), ("width", 512), ("hidden", 1408), ("classes", 1000), ("tokens", 2048), ("steps", 30)):
        p.add_argument("--" + name, type=int, default=value)
    p.add_argument("--optimizer", choices=("sgd", "adamw", "adamw8"), default="sgd")
    p.add_argument("--rate", type=float, help="1.0 for sgd, 0.003 for the others")
    a = p.parse_args(argv)
    net = Stack(a.blocks, a.width, a.hidden, a.classes)
    trained = net if a.optimizer == "sgd" else Trainer(net, "8bit" if a.optimizer == "adamw8" else "fp32")
    rate = a.rate if a.rate is not None else 1.0 if a.optimizer == "sgd" else 0.003
    losses = []
    for s in range(a.steps):
        x, target = synthetic(a.tokens, a.width, a.classes, 100 + s)
        torch.cuda.synchronize()
        t = time.perf_counter()
        losses.append(float(trained.step(x, target, rate)))
        print("step %d: loss %.4f, %.0f us" % (s, losses[-1], (time.perf_counter() - t) * 1e6), flush=True)
    whole, one = net.run(x), net.run(x[:1])
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(100):
        net.run(x[:1])
    torch.cuda.synchronize()
    us = (time.perf_counter() - t) * 1e4
    off = float((whole[:1].float() - one.float()).abs().max() / whole[:1].float().abs().max())
    print("one token: %.1f us; its logits differ from the batch's by %.2g of the largest" % (us, off))
    return losses, off


if __name__ == "__main__":
    main()
