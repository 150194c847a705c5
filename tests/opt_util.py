"""AdamW in plain form, on the CPU: states by the very roundings that are documented, parameters in 64 bits with a bound."""
import numpy as np
import torch

BLOCK = 64
U = 2.0 ** -23      # a whole step of fp32's last place


def stir(h):
    h = np.uint64(h) if np.isscalar(h) else h.astype(np.uint64)
    m = np.uint64(0xFFFFFFFF)
    h = ((h ^ h >> np.uint64(16)) * np.uint64(0x9E3779B9)) & m
    h = ((h ^ h >> np.uint64(15)) * np.uint64(0x6A09E667)) & m
    return h ^ h >> np.uint64(16)


def noise_of(seed, count, first, n):
    """The hash of the elements first .. first + n of the state arrays in the step behind `count`."""
    at = np.arange(first, first + n, dtype=np.uint64)
    key = stir((int(stir(seed)) + count) & 0xFFFFFFFF)
    return stir((at & np.uint64(0xFFFFFFFF)) ^ key ^ stir(at >> np.uint64(32)))


def values(mantissa, low, top):
    """The numbers from zero on that a code of 8 bits stands for, by code: `mantissa` bits, least normal number 2^low, the last one `top`."""
    got, step = [], 2.0 ** (low - mantissa)
    got += [i * step for i in range(1 << mantissa)]
    e = low
    while True:
        for i in range(1 << mantissa):
            v = 2.0 ** e * (1 + i / (1 << mantissa))
            if v > top:
                return np.array(got)
            got.append(v)
        e += 1


E4M3, E5M2 = values(3, -6, 448.0), values(2, -14, 57344.0)


def scale_of(x, top):
    """Each block's scale: the least power of two from 2^-110 on by which its largest finite value comes to at most 1.75 * 2^top."""
    a = np.abs(x.astype(np.float64)).reshape(-1, BLOCK)
    a = np.where(np.isfinite(a), a, 0).max(1)
    e = np.ceil(np.log2(np.maximum(a, 2.0 ** -150) / 1.75)) - top
    e = np.where(np.maximum(a, 2.0 ** -150) / 1.75 <= 2.0 ** (e + top - 1), e - 1, e)
    e = np.where(np.maximum(a, 2.0 ** -150) / 1.75 > 2.0 ** (e + top), e + 1, e)
    return 2.0 ** np.maximum(e, -110)


def codes_of(x, scale, table, noise, kept):
    """x (fp32) as codes of `table`: down to the next number, up where the missing part of the step and the noise come to a whole one."""
    y = np.abs(x.astype(np.float64)) / np.repeat(scale, BLOCK)
    fine = np.isfinite(x)
    y = np.where(fine, y, 0)
    at = np.clip(np.searchsorted(table, y, side="right") - 1, 0, len(table) - 1)
    mantissa = 3 if len(table) == len(E4M3) else 2
    up = np.minimum(at + 1, len(table) - 1)
    # the part of the step that is missing, as 32 bits hold the number (below the least normal one: the number plus that)
    low = table[1 << mantissa]
    held = np.where(y < low, (y + low).astype(np.float32).astype(np.float64) - low, y)
    at = np.where(y < low, np.clip(np.searchsorted(table, held, side="right") - 1, 0, len(table) - 1), at)
    up = np.minimum(at + 1, len(table) - 1)
    part = np.where(up > at, (held - table[at]) / np.where(up > at, table[up] - table[at], 1), 0)
    code = np.where(part + (noise.astype(np.float64) + 0.5) / 65536 >= 1, up, at)
    if kept:
        code = np.where((y > 0) & (code == 0), 1, code)
    return np.where(fine, code + np.where(np.signbit(x), 128, 0), 0x7F).astype(np.uint8)


def decode(codes, scale, table):
    c = codes & 0x7F
    v = np.where(c < len(table), table[np.minimum(c, len(table) - 1)], np.nan)
    return (np.where(codes & 0x80, -v, v) * np.repeat(scale, BLOCK)).astype(np.float32)


class Plain:
    """One parameter, flat; values as numpy arrays of 32 bits."""

    def __init__(self, p, first, betas, eps, decay, small, seed):
        self.n, self.first, self.betas, self.eps, self.decay, self.small, self.seed = p.size, first, betas, eps, decay, small, seed
        pad = -(-self.n // BLOCK) * BLOCK
        self.m, self.v = np.zeros(pad, np.float32), np.zeros(pad, np.float32)
        self.mc = self.vc = np.zeros(pad, np.uint8)
        self.ms = self.vs = np.ones(pad // BLOCK)

    def step(self, p, g, count, rate, factor=None):
        """p (64 bits of what the parameter holds), g (32 bits) -> (new p in 64 bits, bound)."""
        f = np.float32
        b1, b2 = self.betas
        g = np.concatenate([g.astype(f), np.zeros(self.m.size - self.n, f)])
        with np.errstate(all="ignore"):
            if factor is not None:
                g = g * f(factor)
            self.m = f(b1) * self.m + f(1 - b1) * g
            self.v = f(b2) * self.v + f(1 - b2) * g * g
            t = count + 1
            m, v = self.m[:self.n].astype(np.float64), self.v[:self.n].astype(np.float64)
            new = f(rate).astype(np.float64) / (1 - b1 ** t) * m / (np.sqrt(v / (1 - b2 ** t)) + float(f(self.eps)))
            away = float(f(rate)) * float(f(self.decay))
            want = p - (away * p + new)
            # by, root, their product with m and v, the root, the sum with eps, the quotient: a step each, and two for the difference
            bound = 12 * U * np.abs(new) + 4 * U * np.abs(away * p) + U / 2 * np.abs(want)
            if self.small:
                noise = noise_of(self.seed, count, self.first, self.m.size)
                self.ms, self.vs = scale_of(self.m, 8), scale_of(self.v, 15)
                self.mc = codes_of(self.m, self.ms, E4M3, noise >> np.uint64(16), False)
                self.vc = codes_of(self.v, self.vs, E5M2, noise & np.uint64(0xFFFF), True)
                self.m, self.v = decode(self.mc, self.ms, E4M3), decode(self.vc, self.vs, E5M2)
        return want, bound
