"""Performance cases of the feed-forward operators: the matrix product with bias, activation and residual in its epilogue
(`feedforward.Linear`) and the gated pair of projections (`feedforward.GatedLinear`), forward, forward and backward, and both as one
block (`feedforward.FeedForward`), from a single token to a long prompt.

A case is {"kind", "m", "k", "n", "dtype", "act", "bias", "residual", "gap"}: `m` rows of `k` features in rows of k + `gap` elements,
`n` output features (of the gated pair: features of either projection); "kind" is

    linear        y = act(x w^T + bias) + residual
    linear_grad   the same without a residual, then the gradients of x, w and bias for a given gradient of y
    gated         h = act(x wg^T + bg) * (x wu^T + bu)
    gated_grad    the same, then the gradients of x, wg, wu, bg and bu for a given gradient of h
    block         y = x + gated(x) wd^T + bd

The gradient cases keep to smooth activations: a derivative with a step turns the last bit of a sum next to it into an output that
differs by a whole term.
"""
import math

import torch

own = False

DTYPE = {"fp16": torch.float16, "bf16": torch.bfloat16}
KINDS = ("linear", "linear_grad", "gated", "gated_grad", "block")
SMOOTH = ("none", "gelu", "gelu_tanh", "silu", "sigmoid")


def _case(kind, m, k, n, dtype, act, bias=False, residual=False, gap=0):
    return dict(kind=kind, m=m, k=k, n=n, dtype=dtype, act=act, bias=bias, residual=residual, gap=gap)


def listed():
    return [
        # one new token through an output projection of a small model: nothing but latency
        dict(_case("linear", 1, 1024, 1024, "bf16", "none", residual=True), name="linear_token"),
        # the classifier of ResNet-50 at its throughput batch
        dict(_case("linear", 32, 2048, 1000, "fp16", "none", bias=True), name="linear_classes_b32"),
        # five requests' logits over a vocabulary of odd size: rows of the output start anywhere
        dict(_case("linear", 5, 2048, 32001, "bf16", "none"), name="linear_logits_m5"),
        # a prompt of 4096 tokens through one projection with everything in the epilogue
        dict(_case("linear", 4096, 4096, 4096, "bf16", "gelu", bias=True, residual=True), name="linear_prompt"),
        # sizes and strides nobody tuned for: no row starts on a 16-byte line
        dict(_case("linear", 601, 1003, 777, "fp16", "relu", bias=True, residual=True, gap=5), name="linear_odd"),
        # a training step of one projection
        dict(_case("linear_grad", 4096, 2048, 2048, "bf16", "gelu_tanh", bias=True), name="linear_train"),
        # ... of odd sizes, its input a part of wider rows
        dict(_case("linear_grad", 333, 520, 1001, "fp16", "silu", bias=True, gap=24), name="linear_train_odd"),
        # one new token through the two projections of a large model: the weights' bytes
        dict(_case("gated", 1, 4096, 10880, "bf16", "silu"), name="gated_token"),
        # sixteen requests through a whole block
        dict(_case("block", 16, 2048, 5632, "bf16", "silu"), name="block_requests_m16"),
        # a prompt through the two projections
        dict(_case("gated", 4096, 4096, 10880, "bf16", "silu"), name="gated_prompt"),
        # a training step of the gated pair
        dict(_case("gated_grad", 4096, 2048, 5632, "bf16", "silu"), name="gated_train"),
        # ... of odd sizes
        dict(_case("gated_grad", 515, 770, 1031, "fp16", "gelu", bias=True), name="gated_train_odd"),
    ]


def _log_int(rng, lo, hi):
    return int(min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def _size(rng, lo, hi):
    """A size over the logarithm of the range: a multiple of 64, a multiple of 8, or any."""
    s, unit = _log_int(rng, lo, hi), rng.choice((64, 64, 8, 1))
    return min(hi, max(lo, s // unit * unit))


def draw(rng):
    kind = rng.choice(KINDS)
    grad, gated = kind.endswith("_grad"), kind in ("gated", "gated_grad", "block")
    k, n = _size(rng, 64, 4096), _size(rng, 64, 10880 if gated else 8192)
    most = work(max(listed(), key=lambda c: work(c)["flops"]))["flops"]
    m = _log_int(rng, 16 if grad else 1, 4096)
    one = work(_case(kind, 1, k, n, "bf16", "none"))["flops"]
    m = max(1, min(m, int(most / one)))
    return _case(kind, m, k, n, rng.choice(("fp16", "bf16")), rng.choice(SMOOTH if grad else SMOOTH + ("relu",)), bias=rng.random() < 0.5,
                 residual=kind == "linear" and rng.random() < 0.5, gap=rng.choice((0, 0, 0, 8, 5)))


def work(case):
    m, k, n = case["m"], case["k"], case["n"]
    b = 4 * n if case["bias"] else 0
    kind = case["kind"]
    if kind == "linear":
        return {"bytes": 2 * (m * k + n * k + m * n * (2 if case["residual"] else 1)) + b, "flops": 2 * m * n * k}
    if kind == "linear_grad":
        return {"bytes": 2 * (2 * m * k + 2 * n * k + 2 * m * n) + 2 * b, "flops": 6 * m * n * k}
    if kind == "gated":
        return {"bytes": 2 * (m * k + 2 * n * k + m * n) + 2 * b, "flops": 4 * m * n * k}
    if kind == "gated_grad":
        return {"bytes": 2 * (2 * m * k + 4 * n * k + 2 * m * n) + 4 * b, "flops": 12 * m * n * k}
    return {"bytes": 2 * (2 * m * k + 3 * n * k) + 2 * b + (4 * k if case["bias"] else 0), "flops": 6 * m * n * k}


def prepare(case, seed):
    dev, t = torch.device("cuda"), DTYPE[case["dtype"]]
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)

    def normal(*shape, scale=1.0, dtype=t):
        return (torch.randn(*shape, generator=gen, device=dev) * scale).to(dtype)

    m, k, n, kind = case["m"], case["k"], case["n"], case["kind"]
    # activations as they leave a norm, weights that keep their size
    s = {"case": case, "x": normal(m, k + case["gap"])[:, :k]}
    w, bias = (lambda o, i: normal(o, i, scale=i ** -0.5)), (lambda o: normal(o, scale=0.2, dtype=torch.float32) if case["bias"] else None)
    if kind in ("linear", "linear_grad"):
        s["w"], s["b"] = w(n, k), bias(n)
        s["r"] = normal(m, n) if case["residual"] else None
    else:
        s["wg"], s["wu"], s["bg"], s["bu"] = w(n, k), w(n, k), bias(n), bias(n)
    if kind == "block":
        s["wd"], s["bd"] = w(k, n), bias(k)
    if kind.endswith("_grad"):
        s["dy"] = normal(m, n)
    if own:  # the objects that a program makes once around its weights; they hold no copy of them
        from paper_2011_05630_amd import feedforward as F
        if kind in ("linear", "linear_grad"):
            s["op"] = F.Linear(s["w"], s["b"], act=case["act"])
        else:
            s["op"] = F.GatedLinear(s["wg"], s["wu"], s["bg"], s["bu"], act=case["act"])
        if kind == "block":
            s["op"] = F.FeedForward(s["op"], F.Linear(s["wd"], s["bd"]))
    return s


# ---- plain form: elementary operations in 32 bits, one rounding at the end ----------------------

GELU_C, GELU_A = math.sqrt(2.0 / math.pi), 0.044715


def _act(name, z):
    if name == "none":
        return z
    if name == "relu":
        return torch.clamp_min(z, 0.0)
    if name == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(GELU_C * (z + GELU_A * z * z * z)))
    s = 1.0 / (1.0 + torch.exp(-z))
    return s if name == "sigmoid" else z * s


def _act_grad(name, z):
    if name == "none":
        return torch.ones_like(z)
    if name == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    if name == "gelu_tanh":
        t = torch.tanh(GELU_C * (z + GELU_A * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * (GELU_C * (1.0 + 3.0 * GELU_A * z * z))
    s = 1.0 / (1.0 + torch.exp(-z))
    return s * (1.0 - s) if name == "sigmoid" else s * (1.0 + z * (1.0 - s))


def _proj(x, w, b):
    z = x @ w.float().t()
    return z if b is None else z + b


def _plain(s):
    c, t = s["case"], s["x"].dtype
    kind, act, x = c["kind"], c["act"], s["x"].float()
    if kind in ("linear", "linear_grad"):
        z = _proj(x, s["w"], s["b"])
        y = _act(act, z)
        if kind == "linear":
            return {"y": (y if s["r"] is None else y + s["r"].float()).to(t)}
        dz = s["dy"].float() * _act_grad(act, z)
        out = {"y": y.to(t), "dx": (dz @ s["w"].float()).to(t), "dw": (dz.t() @ x).to(t)}
        return out if s["b"] is None else dict(out, db=dz.sum(0))
    g, u = _proj(x, s["wg"], s["bg"]), _proj(x, s["wu"], s["bu"])
    a = _act(act, g)
    h = a * u
    if kind == "gated":
        return {"h": h.to(t)}
    if kind == "block":
        return {"y": (x + _proj(h, s["wd"], s["bd"])).to(t)}
    dh = s["dy"].float()
    dg, du = dh * u * _act_grad(act, g), dh * a
    out = {"h": h.to(t), "dx": (dg @ s["wg"].float() + du @ s["wu"].float()).to(t),
           "dwg": (dg.t() @ x).to(t), "dwu": (du.t() @ x).to(t)}
    return out if s["bg"] is None else dict(out, dbg=dg.sum(0), dbu=du.sum(0))


def run(state):
    s = state
    if not own:
        return _plain(s)
    kind, op = s["case"]["kind"], s["op"]
    if kind == "linear":
        return {"y": op.run(s["x"], residual=s["r"])}
    if kind == "linear_grad":
        y, saved = op.run_saved(s["x"])
        dx, dw, db = op.backward(s["dy"], s["x"], saved)
        out = {"y": y, "dx": dx, "dw": dw}
        return out if db is None else dict(out, db=db)
    if kind == "gated":
        return {"h": op.run(s["x"])}
    if kind == "block":
        return {"y": op.run(s["x"], residual=s["x"])}
    h, saved = op.run_saved(s["x"])
    dx, dwg, dwu, dbg, dbu = op.backward(s["dy"], s["x"], saved)
    out = {"h": h, "dx": dx, "dwg": dwg, "dwu": dwu}
    return out if dbg is None else dict(out, dbg=dbg, dbu=dbu)


# ---- in 64 bits, from the definitions: the gradients are those of automatic differentiation ----

def exact(case, seed):
    s = prepare(case, seed)
    phi = {"none": lambda v: v, "relu": torch.relu, "gelu": lambda v: v * torch.special.ndtr(v), "sigmoid": torch.sigmoid,
           "silu": lambda v: v * torch.sigmoid(v),
           "gelu_tanh": lambda v: v * torch.sigmoid(math.sqrt(8.0 / math.pi) * (v + 0.044715 * v ** 3))}[case["act"]]
    grad = case["kind"].endswith("_grad")
    names = [q for q in ("x", "w", "wg", "wu", "b", "bg", "bu") if s.get(q) is not None]
    v = {q: s[q].double().requires_grad_(grad) for q in names}

    def affine(inp, weight, b):
        z = torch.matmul(inp, weight.transpose(0, 1))
        return z + b if b is not None else z

    with torch.set_grad_enabled(grad):
        if "w" in v:
            key, res = "y", phi(affine(v["x"], v["w"], v.get("b")))
            if s["r"] is not None:
                res = res + s["r"].double()
        else:
            key, res = "h", phi(affine(v["x"], v["wg"], v.get("bg"))) * affine(v["x"], v["wu"], v.get("bu"))
            if case["kind"] == "block":
                key, res = "y", s["x"].double() + affine(res, s["wd"].double(), None if s["bd"] is None else s["bd"].double())
        out = {key: res.detach()}
        if grad:
            out.update(zip(["d" + q for q in names], torch.autograd.grad(res, [v[q] for q in names], s["dy"].double())))
    return out
