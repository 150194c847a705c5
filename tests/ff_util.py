"""Shared helpers of the feed-forward operators' tests: inputs whose results are exact, the plain operators in 64 bits, and
elementwise error bounds.

Whole numbers of small size make every product and sum of the operators exact in 32 bits (all partial sums stay below 2^24), so
the only rounding is the one to the output's type, and outputs have to be equal bit for bit in any order of summation.

Bounds: a sum of K terms in 32 bits is off by at most (K + 2) * U * sum |terms|, with U = 2^-23 (a whole step of the last
place: the matrix unit's adders may truncate); a rounding to type t by eps(t) / 2 of the value; an activation evaluated in 32 bits by
E_ACT * (|z| + 1) (four units of its largest intermediate term); a slope by E_ACT * (|z| + 1)^2."""
import math

import torch

U = 2.0 ** -23
E_ACT = 8 * U
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
SLOPE = 1.2        # largest |act'| of the activations (GELU: 1.13)
CURVE = 1.0        # largest |act''| (GELU: 0.80, its tanh form 0.81)


def half_eps(t):
    return torch.finfo(t).eps / 2


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def rows_of(values, t, gap=0, offset=0, device="cuda"):
    """`values` as a tensor of type t on the GPU whose rows lie `gap` elements apart, `offset` elements behind an allocation's
    start; what lies between the rows is NaN."""
    m, n = values.shape
    buf = torch.full((offset + m * (n + gap) + 8,), float("nan"), dtype=t, device=device)
    v = buf[offset:offset + m * (n + gap)].view(m, n + gap)[:, :n]
    v.copy_(values.to(t))
    return v


def whole(m, n, seed, top=2):
    """Whole numbers of at most `top`, in 64 bits on the CPU."""
    return torch.randint(-top, top + 1, (m, n), generator=gen(seed)).double()


def normal(m, n, seed, t, scale=1.0):
    """Normal values as type t holds them, in 64 bits on the CPU."""
    return (torch.randn(m, n, generator=gen(seed)) * scale).to(t).double()


def act(name, z):
    if name == "none":
        return z
    if name == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if name == "relu6":
        return z.clamp(0, 6)
    if name == "gelu":
        return 0.5 * z * torch.erfc(-z / math.sqrt(2))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    s = 1 / (1 + torch.exp(-z))
    return z * s if name == "silu" else s


def slope(name, z):
    """act'(z); 0 on a step."""
    if name == "none":
        return torch.ones_like(z)
    if name == "relu":
        return (z > 0).double()
    if name == "relu6":
        return ((z > 0) & (z < 6)).double()
    if name == "gelu":
        return 0.5 * torch.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    s = 1 / (1 + torch.exp(-z))
    return s * (1 + z * (1 - s)) if name == "silu" else s * (1 - s)


def same(got, want, what):
    """Equal values where all is exact but the last rounding, which `want` (64 bits) gets here."""
    w = want.to(got.dtype)
    g = got.cpu()
    assert g.shape == w.shape, (what, g.shape, w.shape)
    bad = ~((g == w) | (g.isnan() & w.isnan()))
    assert not bad.any(), "%s: %d of %d values differ, first at %s: %s for %s" % (
        what, int(bad.sum()), bad.numel(), bad.nonzero()[0].tolist(), float(g[bad][0]), float(w[bad][0]))


def within(got, want, bound, what):
    """|got - want| <= bound, elementwise."""
    g = got.double().cpu()
    assert g.shape == want.shape, (what, g.shape, want.shape)
    assert torch.isfinite(g).all(), what + ": not finite"
    over = ((g - want).abs() - bound)
    i = int(over.argmax())
    assert float(over.max()) <= 0, "%s: off by %.4g, bound %.4g, value %.4g" % (
        what, float((g - want).abs().flatten()[i]), float(bound.flatten()[i]), float(want.flatten()[i]))
