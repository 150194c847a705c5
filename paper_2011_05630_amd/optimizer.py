"""The end of a step of training on libdlf, many tensors at once: the norm of all gradients with the factor that clips them, and AdamW with
states in 32 or in 8 bits.

Parameters, gradients and copies are the caller's own tensors, fp16, bf16 or fp32 in any mixture, each with its elements next to each
other (in any order of its dimensions, a gradient's the same as its parameter's).  Calls run on the current stream of their device,
asynchronously, and may be captured into a graph: the count of steps lies on the device, and so may the rate and the factor.  A
tensor that another stream wrote or will overwrite is ordered by the caller, as for any kernel.
"""
import torch

from .feedforward import _native, _need, _stream

_STATES = {"fp32": 0, "8bit": 1}
BLOCK = 64          # elements of the states that share a scale
_norm = None        # the native step, looked for once


def _list(x, name):
    _need(not isinstance(x, torch.Tensor), "%s: a list of tensors expected", name)
    return x if isinstance(x, (list, tuple)) else list(x)


def gradient_norm(gradients, most=float("inf"), scale=1.0):
    """-> (norm, factor), an fp32 element each on the gradients' device: norm = |scale| * sqrt(sum of all their squares), factor = scale, brought
    down by most / norm where the norm is above `most`, and NaN where it is not finite (`AdamW.step` leaves a step with such a factor out).
    scale: what the gradients are to be multiplied by, 1 / (loss scale) among others.  None among the gradients is passed over."""
    global _norm
    gradients = _list(gradients, "gradients")
    index = -1
    for g in gradients:
        if g is not None:
            index = g.get_device() if isinstance(g, torch.Tensor) else -1
            break
    _need(index >= 0, "gradients: tensors on the GPU expected")
    if _norm is None:
        _norm = _native().gradient_norm
    return _norm(gradients, most, scale, _stream(index))


class AdamW:
    """g = factor * gradient;  m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g g;  t = steps
    parameter -= rate * (decay * parameter + m / (1 - b1^t) / (sqrt(v / (1 - b2^t)) + eps))

    copies: for fp32 parameters an fp16 or bf16 tensor each (or None) that gets the new values rounded: what the products read.
    decay: a number, or one for each parameter.  state: "fp32", or "8bit": m as e4m3 and v as e5m2 times a power of two for every BLOCK of
    them, rounded up or down at random as `seed`, the step and the place say, so that they follow what moves them by less than a rounding; a byte
    and a sixteenth an element instead of four.

    The states are one tensor each over all parameters, `m` and `v` (and `m_scale`, `v_scale`): parameter i's begin at `offsets[i]`, in the order in which
    its elements lie in memory, zeros between its end and the next block.  The object is made on the
    stream that is current then; what follows, its steps one after the other, is on the same stream, or ordered by the caller.
    A parameter whose memory, type or form has changed is refused: make another object.  The states' values may be read and written, their tensors
    not exchanged."""

    def __init__(self, params, copies=None, betas=(0.9, 0.95), eps=1e-8, decay=0.0, state="fp32", seed=0):
        params = _list(params, "params")
        _need(state in _STATES, "state: one of %s expected", ", ".join(sorted(_STATES)))
        _need(all(isinstance(p, torch.Tensor) and p.is_cuda for p in params), "params: tensors on the GPU expected")
        b1, b2 = betas
        _need(0 <= b1 < 1 and 0 <= b2 < 1, "betas: numbers from 0 to below 1 expected")
        _need(eps == 0 or 2.0 ** -126 <= eps <= 2.0 ** 126, "eps: 0, or a number from 2^-126 to 2^126, expected")
        _need(isinstance(seed, int) and 0 <= seed < 1 << 32, "seed: a whole number below 2^32 expected")
        decays = [float(d) for d in decay] if isinstance(decay, (list, tuple)) else [float(decay)] * len(params)
        self._make(params, None if copies is None else _list(copies, "copies"), decays, b1, b2, eps, state, seed)

    def _make(self, params, copies, decays, b1, b2, eps, state, seed):
        native = _native().AdamW(params, copies, decays, b1, b2, eps, _STATES[state], seed)
        self.betas, self.eps, self.state, self.seed = (b1, b2), eps, state, seed
        self.device, self.offsets, at = params[0].device, [], 0
        for p in params:
            self.offsets.append(at)
            at += -(-p.numel() // BLOCK) * BLOCK
        self.m, self.v, self.m_scale, self.v_scale, self._counter = native.m, native.v, native.m_scale, native.v_scale, native.counter
        self._index, self._step = params[0].get_device(), native.step

    def step(self, gradients, rate, factor=None):
        """One step.  gradients: a list with one for each parameter, None where a parameter is to stay as it is.  rate: a number, or an
        fp32 tensor of one element on the device; factor: one of those, by which the gradients are multiplied; where it is not finite, everything
        stays as it is, the count of steps too."""
        self._step(_list(gradients, "gradients"), rate, factor, _stream(self._index))

    @property
    def count(self):
        """Steps done, an int64 element on the device."""
        return self._counter[0].long()

    @property
    def powers(self):
        """{steps done, b1, b2, b1^steps, b2^steps} in 64 bits, on the device: the powers as the steps multiplied them."""
        return torch.cat([self._counter[:1], torch.full((1,), self.betas[0], dtype=torch.float64, device=self.device),
                          torch.full((1,), self.betas[1], dtype=torch.float64, device=self.device), self._counter[1:3]])

    def _states(self):
        return {n: getattr(self, n) for n in ("m", "v", "m_scale", "v_scale") if getattr(self, n) is not None}

    def save_state(self):
        """-> copies of the states, the count and `powers`, for `load_state` of an object over parameters of the same sizes."""
        return dict({n: t.clone() for n, t in self._states().items()}, count=self.count, powers=self.powers)

    def load_state(self, state):
        """Takes over the values of `state`, as save_state returns it (the count may be a number).  Without `powers`, or with those of another count or
        other betas, the powers are formed from the count, which may differ in the last places of 64 bits."""
        mine = self._states()
        _need(set(state) - {"powers"} == set(mine) | {"count"}, "state: %s expected", ", ".join(sorted(set(mine) | {"count", "powers"})))
        for n, t in mine.items():
            s = state[n]
            _need(isinstance(s, torch.Tensor) and s.shape == t.shape and s.dtype == t.dtype, "%s: a %s tensor %s expected", n, t.dtype, list(t.shape))
        count = state["count"]
        if isinstance(count, torch.Tensor):
            _need(count.numel() == 1 and count.dtype == torch.int64, "count: a whole number expected")
            count = count.reshape(()).to(self.device)
        else:
            _need(isinstance(count, int) and count >= 0, "count: a whole number expected")
            count = torch.full((), count, dtype=torch.int64, device=self.device)
        powers = state.get("powers")
        if powers is not None:
            _need(isinstance(powers, torch.Tensor) and powers.shape == (5,) and powers.dtype == torch.float64, "powers: an fp64 tensor [5] expected")
            powers = powers.to(self.device)
        with torch.no_grad():
            for n, t in mine.items():
                t.copy_(state[n])
            c = count.double()
            now = torch.stack([c, self.betas[0] ** c, self.betas[1] ** c, torch.zeros_like(c)])
            if powers is not None:
                same = (powers[:3] == torch.cat([now[:1], self.powers[1:3]])).all()
                now[1:3] = torch.where(same, powers[3:], now[1:3])
            self._counter.copy_(now)
