"""The cross entropy of a linear layer in 64 bits, from its formulas, with elementwise bounds of what a computation in 32 bits may be off by.

Bounds, with U = 2^-23 (a whole step of the last place) as in ff_util: a logit is a sum of K products, off by (K + 2) U sum |terms|.  An exponential of d is off by its
argument's error and (2 |d| + 8) U of its value (d rounded, multiplied by log2 e, rounded, the instruction); a row's sum of them takes
at most 64 additions in a lane, then one for each part of the classes and a rescaling by another exponential of no larger |d|.  A rounding to type t is
off by half_eps(t) of the value, in fp16 at least by half the least number, 2^-25."""
import torch

from ff_util import U, half_eps

IGNORE = -100


def floor_of(t):
    """Half the least number of type t."""
    return 2.0 ** -25 if t == torch.float16 else 0.0


def reference(x, w, b, target, ignore=IGNORE):
    """All in 64 bits on the CPU: -> dict of z, lse, loss, p and the bounds of z, lse and loss."""
    k, v = w.shape[1], w.shape[0]
    z, size = x @ w.t(), x.abs() @ w.abs().t()
    if b is not None:
        z, size = z + b, size + b.abs().nan_to_num(posinf=0.0)
    ez = (k + 2) * U * size
    lse = torch.logsumexp(z, 1)
    p = torch.exp(z - lse[:, None])
    far = torch.where(p > 0, (z - z.max(1, keepdim=True).values).abs(), 0.0)
    e_sum = (64 + v / 16 + 32 + 4 * (p * far).sum(1)) * U
    e_lse = (p * ez).sum(1) + e_sum + 4 * U * (lse.abs() + 1 + far.max(1).values.clamp_max(90))
    counted = target != ignore
    at = torch.where(counted, target, 0)
    loss = torch.where(counted, lse - z.gather(1, at[:, None]).squeeze(1), 0.0)
    e_loss = torch.where(counted, e_lse + ez.gather(1, at[:, None]).squeeze(1) + U * loss.abs(), 0.0)
    return dict(z=z, lse=lse, p=p, loss=loss, ez=ez, e_lse=e_lse, e_loss=e_loss, counted=counted, at=at)


def gradients(ref, x, w, dloss, dlse, t, kept=False):
    """-> dx, dw, db with their bounds, for tensors of type t.  kept: the exponentials are rounded to 11 bits behind the point on the way."""
    own = torch.where(ref["counted"], dloss, 0.0)
    total = own + dlse
    p = ref["p"]
    dz = total[:, None] * p
    e = dz.abs() * (ref["ez"] + ref["e_lse"][:, None] + (2 * torch.where(p > 0, (ref["z"] - ref["lse"][:, None]).abs(), 0.0) + 16) * U)
    if kept:
        # 2^-12 of an exponential, 2^-31 of the largest of its part, whose probability is at most 1
        e = e + dz.abs() * 2.0 ** -12 + total.abs()[:, None] * 2.0 ** -31
    dz = dz.scatter_add(1, ref["at"][:, None], -own[:, None])
    e = e + U * dz.abs() + 2 * U * own.abs()[:, None] * (dz != 0)
    out = {"db": (dz.sum(0), e.sum(0) + (dz.shape[0] + 4) * U * dz.abs().sum(0))}
    rounded = e + half_eps(t) * (dz.abs() + e)
    if t == torch.float16:
        # dz is scaled by what brings the largest |dloss| + |dlse| to at least 2^13
        rounded = rounded + 2.0 ** -25 * float((own.abs() + dlse.abs()).max()) / 2.0 ** 13
    for name, a, ea, c in (("dx", dz, rounded, w), ("dw", dz.t(), rounded.t(), x)):
        value, terms = a @ c, a.abs() @ c.abs()
        bound = ea @ c.abs() + (a.shape[1] + 4) * U * (terms + ea @ c.abs())
        out[name] = (value, bound + half_eps(t) * (value.abs() + bound) + floor_of(t))
    return out
