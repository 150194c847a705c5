"""Performance cases of what stands around the feed-forward operators in a step of training: the softmax cross entropy of a linear layer over a
vocabulary, without keeping its logits, and its gradients (`loss.CrossEntropy`), the norm of all gradients with the factor that clips them
(`optimizer.gradient_norm`), and an AdamW step over many tensors with states in 32 or 8 bits (`optimizer.AdamW`).

A case has a "kind":

    loss       loss[r] = log sum_c exp z[r][c] - z[r][target], z = x w^T + bias, `m` rows of `k` features in rows of k + `gap` elements,
               `v` classes; a share `ignored` of the rows has no target
    loss_grad  the loss and, for the same gradient of every row's loss (their mean's, times `scale`), the gradients of x, w and bias
    loss_back  the loss and log sum exp, then, for given gradients of both, the gradients of x, w and bias
    norm       the norm of all gradients and the factor that brings it down to a given one
    adamw      a step of AdamW: `state` "fp32" or "8bit", parameters of type `param`, gradients `grad`, 16-bit `copy` of the parameters or none,
               gradients times a factor on the device where `factor`

The tensors of the last two: `tensors` of them of sizes up to `largest`, packed one behind the other so that they start anywhere, or (tensors = 0) those
of a stack of `blocks` gated feed-forward blocks and a classifier, `width`, `hidden` and `classes` wide.
"""
import math
import random

import torch

own = False

DTYPE = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
IGNORE = -100
B1, B2, EPS, DECAY, RATE = 0.9, 0.95, 1e-8, 0.1, 3e-4
COUNT, RANDOM_SEED = 1000, 12345
BLOCK = 64                      # elements that share a scale of the 8-bit states


def _loss(kind, m, k, v, dtype, bias=False, ignored=0.0, gap=0, scale=1.0):
    return dict(kind=kind, m=m, k=k, v=v, dtype=dtype, bias=bias, ignored=ignored, gap=gap, scale=scale)


def _stack(kind, blocks, width, hidden, classes, grad, **kw):
    return dict(kw, kind=kind, blocks=blocks, width=width, hidden=hidden, classes=classes, tensors=0, largest=0, sizes=0, grad=grad)


def _ragged(kind, tensors, largest, sizes, grad, **kw):
    return dict(kw, kind=kind, blocks=0, width=0, hidden=0, classes=0, tensors=tensors, largest=largest, sizes=sizes, grad=grad)


def listed():
    return [
        # how likely one answer is, among the thousand classes of the example: nothing but latency
        dict(_loss("loss", 1, 512, 1000, "bf16", bias=True), name="loss_token"),
        # five candidates scored over a vocabulary of odd size: the weights' bytes
        dict(_loss("loss", 5, 2048, 32001, "bf16"), name="loss_requests_m5"),
        # a long text evaluated
        dict(_loss("loss", 4096, 2048, 32001, "fp16"), name="loss_text"),
        # a step of training: loss and gradients of 4096 tokens
        dict(_loss("loss_grad", 4096, 4096, 32000, "bf16"), name="loss_train"),
        # ... of odd sizes, with a bias, the loss scaled as fp16 needs it
        dict(_loss("loss_grad", 515, 770, 5003, "fp16", bias=True, ignored=0.1, gap=5, scale=1024.0), name="loss_train_odd"),
        # ... in two calls, as a chain of automatic differentiation makes them, half of the tokens a prompt without targets
        dict(_loss("loss_back", 2048, 2048, 32001, "bf16", ignored=0.5), name="loss_train_two_calls"),
        # the gradients of a small stack: a bias among its weights
        dict(_stack("norm", 2, 512, 1408, 1000, "bf16"), name="norm_small"),
        # those of a larger one
        dict(_stack("norm", 6, 2048, 5632, 32000, "bf16"), name="norm_large"),
        # a step of the small stack
        dict(_stack("adamw", 2, 512, 1408, 1000, "bf16", state="fp32", param="fp32", copy="bf16", factor=True), name="adamw_small"),
        # many tensors, most of them small, starting anywhere, of odd sizes
        dict(_ragged("adamw", 200, 1 << 20, 7, "fp32", state="8bit", param="fp32", copy="fp16", factor=True), name="adamw8_ragged"),
        # a step of a larger stack
        dict(_stack("adamw", 2, 2048, 5632, 8000, "bf16", state="fp32", param="fp32", copy="bf16", factor=False), name="adamw_large"),
        # ... with states in 8 bits
        dict(_stack("adamw", 2, 2048, 5632, 8000, "bf16", state="8bit", param="fp32", copy="bf16", factor=False), name="adamw8_large"),
    ]


def _log_int(rng, lo, hi):
    return int(min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def _size(rng, lo, hi):
    """A size over the logarithm of the range: a multiple of 64, a multiple of 8, or any."""
    s, unit = _log_int(rng, lo, hi), rng.choice((64, 64, 8, 1))
    return min(hi, max(lo, s // unit * unit))


MOST_LOGITS, MOST_ELEMENTS = 1 << 28, 100 * 1000 * 1000


def draw(rng):
    kind = rng.choice(("loss", "loss_grad", "loss_grad", "loss_back", "norm", "adamw", "adamw"))
    if kind.startswith("loss"):
        k, v = _size(rng, 64, 4096), _size(rng, 100, 131072)
        most = 6 * 4096 * 4096 * 32000 // (2 if kind == "loss" else 6)
        m = max(1, min(_log_int(rng, 1, 8192), MOST_LOGITS // v, most // (k * v)))
        dtype = rng.choice(("fp16", "bf16"))
        return _loss(kind, m, k, v, dtype, bias=rng.random() < 0.4, ignored=rng.choice((0.0, 0.1, 0.5)), gap=rng.choice((0, 0, 0, 8, 5)),
                     scale=1024.0 if dtype == "fp16" else 1.0)
    grad = rng.choice(("bf16", "bf16", "fp16", "fp32"))
    more = {}
    if kind == "adamw":
        param = rng.choice(("fp32", "fp32", "fp32", "bf16"))
        more = dict(state=rng.choice(("fp32", "8bit")), param=param, copy=rng.choice(("none", "bf16", "fp16")) if param == "fp32" else "none",
                    factor=rng.random() < 0.5)
    if rng.random() < 0.5:
        n = _log_int(rng, 1, 300)
        return _ragged(kind, n, _log_int(rng, 1, min(1 << 24, 6 * MOST_ELEMENTS // n)), rng.randrange(1 << 30), grad, **more)
    width, classes = _size(rng, 64, 2048), _size(rng, 10, 32000)
    hidden = max(1, width * 11 // 4)
    blocks = max(1, min(_log_int(rng, 1, 20), (MOST_ELEMENTS - width * classes) // (3 * width * hidden)))
    return _stack(kind, blocks, width, hidden, classes, grad, **more)


def _counts(case):
    """Elements of each tensor."""
    if case["tensors"]:
        rng = random.Random(case["sizes"])
        got = [_log_int(rng, 1, case["largest"]) for _ in range(case["tensors"])]
        return [n if sum(got[:i + 1]) <= MOST_ELEMENTS else 1 for i, n in enumerate(got)]
    w, h, c = case["width"], case["hidden"], case["classes"]
    return [h * w, h * w, w * h] * case["blocks"] + [c * w, c]


def work(case):
    kind = case["kind"]
    if kind.startswith("loss"):
        m, k, v = case["m"], case["k"], case["v"]
        b = 4 * v if case["bias"] else 0
        if kind == "loss":
            return {"bytes": 2 * (m * k + v * k) + b + 12 * m, "flops": 2 * m * k * v}
        return {"bytes": 4 * (m * k + v * k) + 2 * b + 12 * m + (12 * m if kind == "loss_back" else 0), "flops": 6 * m * k * v}
    n = sum(_counts(case))
    g = 4 if case["grad"] == "fp32" else 2
    if kind == "norm":
        return {"bytes": g * n, "flops": 2 * n}
    p, c = (4 if case["param"] == "fp32" else 2), (0 if case["copy"] == "none" else 2)
    return {"bytes": n * (g + 2 * p + c) + (16 * n if case["state"] == "fp32" else 4 * n + 16 * (n // BLOCK)), "flops": 16 * n}


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)

    def normal(*shape, scale=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=gen, device=dev) * scale).to(dtype)

    s = {"case": case}
    if case["kind"].startswith("loss"):
        m, k, v, t = case["m"], case["k"], case["v"], DTYPE[case["dtype"]]
        s["w"], s["b"] = normal(v, k, scale=k ** -0.5, dtype=t), normal(v, scale=0.2) if case["bias"] else None
        s["target"] = torch.randint(v, (m,), generator=gen, device=dev)
        # as a model that has learned something leaves them: the target's logit is about ten above the others' mean
        x = normal(m, k + case["gap"])
        x[:, :k] += 10.0 * s["w"][s["target"]].float()
        s["x"] = x.to(t)[:, :k]
        s["target"][torch.rand(m, generator=gen, device=dev) < case["ignored"]] = IGNORE
        s["dloss"] = case["scale"] / (s["target"] != IGNORE).sum().clamp_min(1).float()
        if case["kind"] == "loss_back":
            s["dloss"] = s["dloss"] * (0.5 + torch.rand(m, generator=gen, device=dev))
            s["dlse"] = 0.01 * s["dloss"] * normal(m)
        if own:                 # made once around the weights, of which it holds no copy
            from paper_2011_05630_amd import loss
            s["op"] = loss.CrossEntropy(s["w"], s["b"], ignore_index=IGNORE)
        return s

    counts, t = _counts(case), DTYPE[case["grad"]]
    s["grads"] = [normal(n, scale=1e-3, dtype=t) for n in counts]
    if case["kind"] == "norm":
        return s
    # parameters and their copies as a program keeps them: one allocation, a view for each tensor
    unit = 1 if case["tensors"] else BLOCK
    at, starts = 0, []
    for n in counts:
        starts.append(at)
        at += -(-n // unit) * unit
    s["p"] = normal(at, scale=0.02, dtype=DTYPE[case["param"]])
    s["c"] = None if case["copy"] == "none" else s["p"].to(DTYPE[case["copy"]])
    s["counts"] = counts
    s["params"], s["copies"] = ([None if f is None else f[a:a + n] for a, n in zip(starts, counts)] for f in (s["p"], s["c"]))
    # states: each tensor's start on a block, zeros behind its last element
    at, s["at"] = 0, []
    for n in counts:
        s["at"].append(at)
        at += -(-n // BLOCK) * BLOCK
    inside = torch.zeros(at, dtype=torch.bool, device=dev)
    for a, n in zip(s["at"], counts):
        inside[a:a + n] = True
    m = normal(at, scale=3e-4) * inside
    v = (0.3 + torch.rand(at, generator=gen, device=dev)) * 1e-6 * inside
    if case["state"] == "8bit":
        s["ms"], s["vs"] = _scale(m, 8), _scale(v, 15)
        m = (m.view(-1, BLOCK) / s["ms"][:, None]).to(torch.float8_e4m3fn).view(-1)
        v = (v.view(-1, BLOCK) / s["vs"][:, None]).clamp_min(2.0 ** -16).mul(inside.view(-1, BLOCK)).to(torch.float8_e5m2).view(-1)
    s["m"], s["v"], s["count"] = m, v, torch.full((), COUNT, dtype=torch.int64, device=dev)
    s["factor"] = torch.full((), 0.37, device=dev) if case["factor"] else None
    if own:
        from paper_2011_05630_amd import optimizer
        s["op"] = optimizer.AdamW(s["params"], None if s["c"] is None else s["copies"], betas=(B1, B2), eps=EPS, decay=DECAY,
                                  state=case["state"], seed=RANDOM_SEED)
        s["op"].load_state({q: s[q2] for q, q2 in (("count", "count"), ("m", "m"), ("v", "v"), ("m_scale", "ms"), ("v_scale", "vs")) if q2 in s})
    return s


# ---- plain forms: elementary operations in 32 bits, one rounding at the end ---------------------

def _logits(s):
    z = s["x"].float() @ s["w"].float().t()
    return z if s["b"] is None else z + s["b"]


def _plain_loss(s):
    kind, t = s["case"]["kind"], s["x"].dtype
    z = _logits(s)
    top = z.max(1, keepdim=True).values
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    lse = (top + torch.log(total)).squeeze(1)
    counted = s["target"] != IGNORE
    at = torch.where(counted, s["target"], 0)
    loss = torch.where(counted, lse - z.gather(1, at[:, None]).squeeze(1), 0.0)
    if kind == "loss":
        return {"loss": loss}
    dloss = torch.where(counted, s["dloss"].expand(loss.shape), 0.0)
    dz = e.div_(total).mul_((dloss + s["dlse"] if kind == "loss_back" else dloss)[:, None])
    dz.scatter_add_(1, at[:, None], -dloss[:, None])
    out = {"loss": loss, "dx": (dz @ s["w"].float()).to(t), "dw": (dz.t() @ s["x"].float()).to(t)}
    if kind == "loss_back":
        out["lse"] = lse
    return out if s["b"] is None else dict(out, db=dz.sum(0))


def _plain_norm(grads):
    norm = torch.sqrt(torch.cat(grads).double().square().sum()).float()
    return {"norm": norm, "factor": torch.where(norm > 1.0, 1.0 / norm, torch.ones_like(norm))}


def _mix(h):
    """32 bits, in int64, stirred."""
    h = (h ^ h >> 16) * 0x9E3779B9 & 0xFFFFFFFF
    h = (h ^ h >> 15) * 0x6A09E667 & 0xFFFFFFFF
    return h ^ h >> 16


def _scale(x, top):
    """For every block the least power of two (from 2^-110 on) by which its largest finite value comes to at most 1.75 * 2^top."""
    b = x.abs().view(torch.int32).view(-1, BLOCK)
    b = torch.where(b < 0x7F800000, b, 0).max(1).values
    return (((b + 0x1FFFFF >> 23) - top).clamp_min(17) << 23).view(torch.float32)


def _to_8_bits(x, scale, noise, mantissa, low, kept):
    """x / scale rounded to floating-point numbers of `mantissa` bits and least normal number 2^low, up where `noise` (in steps, of 16 bits)
    makes up for what is missing, as their codes; kept: nothing but zero becomes zero."""
    cut, first = 23 - mantissa, (127 + low) << mantissa
    y = x.abs() / scale
    small = y < 2.0 ** low
    r = (noise << cut - 16) + (1 << cut - 17)
    code = (torch.where(small, y + 2.0 ** low, y).view(torch.int32).long() + r >> cut) - first + torch.where(small, 0, 1 << mantissa)
    if kept:
        code = torch.where(x > 0, code.clamp_min(1), code)
    code = torch.where(torch.isfinite(x), code, 0x7F)
    return torch.where(x.view(torch.int32) < 0, code + 128, code).to(torch.uint8)


def _on_blocks(tensors):
    """The tensors one behind the other, each filled up with zeros to a whole number of blocks, in 32 bits."""
    return torch.cat([q for t in tensors for q in (t, t.new_zeros(-t.numel() % BLOCK))]).float()


def _plain_step(s):
    small = s["case"]["state"] == "8bit"
    m, v = s["m"], s["v"]
    g, p = _on_blocks(s["grads"]), _on_blocks(s["params"])
    if s["factor"] is not None:
        g = g * s["factor"]
    if small:
        m, v = ((a.float().view(-1, BLOCK) * b[:, None]).view(-1) for a, b in ((m, s["ms"]), (v, s["vs"])))
    m = B1 * m + (1 - B1) * g
    v = B2 * v + (1 - B2) * g * g
    t = (s["count"] + 1).double()
    p = p * (1 - RATE * DECAY) - RATE / (1 - B1 ** t) * m / (torch.sqrt(v / (1 - B2 ** t)) + EPS)
    new = torch.cat([p[a:a + n] for a, n in zip(s["at"], s["counts"])])
    torch._foreach_copy_(s["params"], list(new.split(s["counts"])))
    if s["c"] is not None:
        torch._foreach_copy_(s["copies"], s["params"])
    if small:
        s["ms"].copy_(_scale(m, 8))
        s["vs"].copy_(_scale(v, 15))
        key = _mix(_mix(torch.full_like(s["count"], RANDOM_SEED)) + s["count"] & 0xFFFFFFFF)
        noise = _mix(torch.arange(m.numel(), device=m.device) ^ key)
        for_m, for_v = (b.repeat_interleave(BLOCK) for b in (s["ms"], s["vs"]))
        s["m"].view(torch.uint8).copy_(_to_8_bits(m, for_m, noise >> 16, 3, -6, False))
        s["v"].view(torch.uint8).copy_(_to_8_bits(v, for_v, noise & 0xFFFF, 2, -14, True))
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    s["count"] += 1


def _state(s, src):
    out = {"p": s["p"], **src}
    return out if s["c"] is None else dict(out, c=s["c"])


def run(state):
    s = state
    c = s["case"]
    kind = c["kind"]
    if kind.startswith("loss"):
        if not own:
            return _plain_loss(s)
        op = s["op"]
        if kind == "loss":
            return {"loss": op.run(s["x"], s["target"])}
        if kind == "loss_grad":
            loss, dx, dw, db = op.gradients(s["x"], s["target"], s["dloss"])
            out = {"loss": loss, "dx": dx, "dw": dw}
        else:
            loss, lse = op.run_saved(s["x"], s["target"])
            dx, dw, db = op.backward(s["dloss"], s["x"], s["target"], lse, dlse=s["dlse"])
            out = {"loss": loss, "lse": lse, "dx": dx, "dw": dw}
        return out if db is None else dict(out, db=db)
    if kind == "norm":
        if not own:
            return _plain_norm(s["grads"])
        from paper_2011_05630_amd import optimizer
        norm, factor = optimizer.gradient_norm(s["grads"], most=1.0)
        return {"norm": norm, "factor": factor}
    names = ("m", "v", "m_scale", "v_scale") if c["state"] == "8bit" else ("m", "v")
    if own:
        op = s["op"]
        op.step(s["grads"], RATE, factor=s["factor"])
        return _state(s, {q: getattr(op, q) for q in names})
    _plain_step(s)
    return _state(s, dict(zip(names, (s["m"], s["v"], s.get("ms"), s.get("vs")))))


# ---- in 64 bits, from the definitions: the gradients are those of automatic differentiation ----

def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind.startswith("loss"):
        grad = kind != "loss"
        leaf = {q: s[q].double().requires_grad_(grad) for q in ("x", "w", "b") if s[q] is not None}
        with torch.set_grad_enabled(grad):
            z = torch.matmul(leaf["x"], leaf["w"].transpose(0, 1))
            if "b" in leaf:
                z = z + leaf["b"]
            lse = torch.logsumexp(z, 1)
            rows = torch.nonzero(s["target"] != IGNORE).squeeze(1)
            loss = torch.zeros_like(lse).index_put((rows,), lse[rows] - z[rows, s["target"][rows]])
            out = {"loss": loss.detach()}
            if grad:
                whole = (loss * s["dloss"].double()).sum()
                if kind == "loss_back":
                    whole, out["lse"] = whole + (lse * s["dlse"].double()).sum(), lse.detach()
                del z
                out.update(zip(["d" + q for q in leaf], torch.autograd.grad(whole, list(leaf.values()))))
        return out
    flat = torch.cat([g.double() for g in s["grads"]])
    if kind == "norm":
        norm = torch.linalg.vector_norm(flat)
        return {"norm": norm, "factor": torch.clamp(1.0 / norm, max=1.0)}
    if s["factor"] is not None:
        flat = flat * s["factor"].double()
    counts = [g.numel() for g in s["grads"]]
    where = torch.cat([torch.arange(a, a + n, device=flat.device) for a, n in zip(s["at"], counts)])
    m, v = s["m"].double(), s["v"].double()
    if case["state"] == "8bit":
        m, v = m * s["ms"].double().repeat_interleave(BLOCK), v * s["vs"].double().repeat_interleave(BLOCK)
    m[where] += (flat - m[where]) * (1.0 - B1)
    v[where] += (flat ** 2 - v[where]) * (1.0 - B2)
    new = m[where] / (1.0 - B1 ** (COUNT + 1)) / (torch.sqrt(v[where] / (1.0 - B2 ** (COUNT + 1))) + EPS)
    p = s["p"].double()
    starts = [q.storage_offset() for q in s["params"]]
    at = torch.cat([torch.arange(a, a + n, device=flat.device) for a, n in zip(starts, counts)])
    p[at] = p[at] - RATE * (DECAY * p[at] + new)
    small = case["state"] == "8bit"
    out = {"p": p, "m": None if small else m, "v": None if small else v}
    if small:
        out.update(m_scale=None, v_scale=None)
    return out if s["c"] is None else dict(out, c=p)
