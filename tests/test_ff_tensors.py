"""What the feed-forward operators do with tensors that changed, on CPU tensors without rows: nothing is launched, and no GPU is needed."""
import pytest
import torch

from paper_2011_05630_amd import binding as B
from paper_2011_05630_amd import feedforward as F

N, K = 24, 16
X = torch.zeros(0, K, dtype=torch.bfloat16)
DY = torch.zeros(0, N, dtype=torch.bfloat16)
SAVED = {False: torch.zeros(0, N), True: torch.zeros(2, 0, N)}


def operands(gated):
    """Weights, then biases, under the names that refusals use."""
    names = (("w_gate", "w_up"), ("b_gate", "b_up")) if gated else (("weight",), ("bias",))
    return {n: torch.zeros(N, K, dtype=torch.bfloat16) for n in names[0]}, {n: torch.zeros(N) for n in names[1]}


def native(gated, w, b):
    pair = lambda d: tuple(d.values()) if gated else tuple(d.values()) + (None,)
    return F._native().Op(gated, B.FF_ACT["silu"], *pair(w), *pair(b), K)


def calls(op, gated, x=X, dy=DY):
    return (lambda: op.forward(x, None, None, False, 0), lambda: op.forward(x, None, None, True, 0),
            lambda: op.backward(dy, x, SAVED[gated], True, True, True, 0), lambda: op.backward(dy, x, SAVED[gated], False, False, False, 0))


OTHER_WEIGHTS = {
    "fewer rows": lambda: torch.zeros(2, K, dtype=torch.bfloat16), "fewer columns": lambda: torch.zeros(N, K - 1, dtype=torch.bfloat16),
    "transposed": lambda: torch.zeros(K, N, dtype=torch.bfloat16).t(), "one dimension": lambda: torch.zeros(N * K, dtype=torch.bfloat16),
    "farther rows": lambda: torch.zeros(N, K + 8, dtype=torch.bfloat16)[:, :K], "one row": lambda: torch.zeros(1, K, dtype=torch.bfloat16).expand(N, K),
    "fp32": lambda: torch.zeros(N, K), "fp16": lambda: torch.zeros(N, K, dtype=torch.float16)}
OTHER_BIASES = {
    "shorter": lambda: torch.zeros(N - 1), "two dimensions": lambda: torch.zeros(1, N), "strided": lambda: torch.zeros(2 * N)[::2],
    "bf16": lambda: torch.zeros(N, dtype=torch.bfloat16), "fp64": lambda: torch.zeros(N, dtype=torch.float64)}


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("other", sorted(OTHER_WEIGHTS))
def test_weights_of_another_form_are_refused(gated, other):
    """`.data = ` exchanges sizes, strides, type and device within the tensor that the operator holds; so do a module's conversions."""
    for name in operands(gated)[0]:
        w, b = operands(gated)
        op = native(gated, w, b)
        w[name].data = OTHER_WEIGHTS[other]()
        for call in calls(op, gated):
            with pytest.raises(ValueError, match="^%s: " % name):
                call()


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("other", sorted(OTHER_BIASES))
def test_biases_of_another_form_are_refused(gated, other):
    for name in operands(gated)[1]:
        w, b = operands(gated)
        op = native(gated, w, b)
        b[name].data = OTHER_BIASES[other]()
        for call in calls(op, gated):
            with pytest.raises(ValueError, match="^%s: " % name):
                call()


@pytest.mark.parametrize("gated", [False, True])
def test_values_of_the_same_form_are_followed(gated):
    """New storage of the same form is a change that the next call sees; one row's distance to the next says nothing."""
    w, b = operands(gated)
    op = native(gated, w, b)
    for t in list(w.values()) + list(b.values()):
        t.data = torch.ones_like(t)
    for call in calls(op, gated)[:2]:
        call()
    one = torch.zeros(1, K, dtype=torch.bfloat16)
    op = F._native().Op(False, B.FF_ACT["none"], one, None, None, None, K)
    one.data = torch.zeros(3, K + 5, dtype=torch.bfloat16)[1:2, :K]
    assert op.forward(X, None, None, False, 0).shape == (0, 1)


def test_a_module_that_converts_its_parameters():
    m = torch.nn.Linear(K, N, bias=False, dtype=torch.bfloat16)
    op = F._native().Op(False, B.FF_ACT["none"], m.weight.data, None, None, None, K)
    held = F._native().Op(False, B.FF_ACT["none"], m.weight, None, None, None, K)
    m.float()
    op.forward(X, None, None, False, 0)                     # `.data` of before: a tensor of its own, unchanged
    with torch.no_grad(), pytest.raises(ValueError, match="^weight: "):
        held.forward(X, None, None, False, 0)


def forward_and_backward(gated, **kw):
    """Each call, with the named operands in place of the usual ones: [(name, call)]."""
    w, b = operands(gated)
    w.update({k: v for k, v in kw.items() if k in w})
    b.update({k: v for k, v in kw.items() if k in b})
    op = native(gated, w, b)
    x, saved, dy = kw.get("x", X), kw.get("saved", SAVED[gated]), kw.get("dh" if gated else "dy", DY)
    forward = lambda save: op.forward(x, kw.get("residual"), kw.get("out"), save, 0)
    backward = lambda: op.backward(dy, x, saved, False, False, False, 0)
    out = []
    if not {"saved", "dy", "dh"} & set(kw):
        out += [lambda: forward(False), lambda: forward(True)]
    if not {"residual", "out"} & set(kw):
        out.append(backward)
    return out


NAMES = [(g, n) for g in (False, True) for n in (["x", "residual", "out", "saved"] + (["dh", "w_gate", "w_up", "b_gate", "b_up"] if g else ["dy", "weight", "bias"]))
         if not (g and n == "residual")]


def usual(gated, name):
    w, b = operands(gated)
    return dict(w, **b, x=X, residual=DY, out=DY, saved=SAVED[gated], dy=DY, dh=DY)[name].clone()


@pytest.mark.parametrize("gated,name", NAMES)
def test_operands_that_require_a_gradient_are_refused(gated, name):
    """The operators stand outside automatic differentiation: a result without a graph would be a wrong gradient without a word."""
    for t in (usual(gated, name).requires_grad_(), usual(gated, name).requires_grad_() * 1):
        for call in forward_and_backward(gated, **{name: t}):
            with pytest.raises(ValueError, match="^%s: .*no_grad" % name):
                call()
        with torch.no_grad():
            for call in forward_and_backward(gated, **{name: t})[:1 if name in ("saved", "dy", "dh") else 2]:
                try:
                    call()
                except B.DlfError as e:                     # (a backward call goes on to the GPU)
                    assert e.status == B.DLF_ERR_HIP
    with torch.inference_mode():
        for call in forward_and_backward(gated, x=X)[:2]:
            call()


@pytest.mark.parametrize("gated,name", NAMES)
def test_operands_with_a_tangent_are_refused(gated, name):
    import torch.autograd.forward_ad as fw
    t = usual(gated, name)
    with fw.dual_level():
        d = fw.make_dual(t, torch.ones_like(t))
        for call in forward_and_backward(gated, **{name: d}):
            with pytest.raises(ValueError, match="^%s: .*tangent" % name):
                call()
        with fw._set_fwd_grad_enabled(False):
            for call in forward_and_backward(gated, x=X)[:2]:
                call()


def test_function_transforms_are_refused():
    op = native(False, *operands(False))
    x = torch.zeros(3, K, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="^x: "):
        torch.func.grad(lambda v: op.forward(v, None, None, False, 0).sum())(x)
    with pytest.raises(ValueError, match="^x: "):
        torch.func.jvp(lambda v: op.forward(v, None, None, False, 0), (x,), (x,))


def test_outputs_raise_their_version():
    """PyTorch tells by its version whether a tensor kept for a backward pass was written since."""
    for gated in (False, True):
        op = native(gated, *operands(gated))
        out = DY.clone()
        before = out._version
        op.forward(X, None, out, False, 0)
        assert out._version == before + 1
        op.forward(X, None, out, True, 0)
        assert out._version == before + 2
    a = torch.zeros(0, N, requires_grad=True)
    y = a.bfloat16()
    loss = (y * y).sum()                                    # keeps y
    with torch.no_grad():
        op.forward(X, None, y, False, 0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    with torch.inference_mode():
        out = DY.clone()
        op.forward(X, None, out, False, 0)                  # counts nothing
    op.forward(X, None, out, False, 0)
    big = F._native().Op(False, B.FF_ACT["none"], torch.empty(1, (1 << 20) + 1, dtype=torch.bfloat16), None, None, None, (1 << 20) + 1)
    out = torch.zeros(0, 1, dtype=torch.bfloat16)
    before = out._version
    with pytest.raises(B.DlfError):
        big.forward(torch.empty(0, (1 << 20) + 1, dtype=torch.bfloat16), None, out, False, 0)
    assert out._version == before                           # refused, not written


def on_cpu(gated):
    """The Python object around CPU tensors, which its constructor refuses."""
    w, b = operands(gated)
    op = object.__new__(F.GatedLinear if gated else F.Linear)
    for name, t in dict(w, **b).items():
        setattr(op, name, t)
    pair = lambda d: tuple(d.values()) if gated else tuple(d.values()) + (None,)
    op._setup(gated, "silu", pair(w), pair(b))
    return op


@pytest.mark.parametrize("gated", [False, True])
def test_what_an_operator_was_made_of_is_fixed(gated):
    """The native operator would not see another tensor in a weight's place."""
    op = on_cpu(gated)
    for name in list(operands(gated)[0]) + list(operands(gated)[1]) + ["act", "dtype", "device", "in_features", "out_features"]:
        have = getattr(op, name)
        with pytest.raises(AttributeError, match="^%s: " % name):
            setattr(op, name, torch.zeros(N, K, dtype=torch.bfloat16))
        with pytest.raises(AttributeError, match="^%s: " % name):
            delattr(op, name)
        assert getattr(op, name) is have
    op.label = "up"                                         # a caller's own
    op.label = "down"
    del op.label


def test_unknown_gradients_are_refused():
    """A misspelled gradient would come back as None."""
    for op in (on_cpu(False), on_cpu(True)):
        for bad in (("weights",), ("x", "b"), "w", "bias, x", (1,)):
            with pytest.raises(ValueError, match="^need: "):
                op.backward(DY, X, SAVED[isinstance(op, F.GatedLinear)], need=bad)
    block = object.__new__(F.FeedForward)
    with pytest.raises(ValueError, match="^need: "):
        block.backward(DY, X, (DY, SAVED[True], None), need=("weights",))


def test_pending_negations_are_refused():
    """A view whose elements are the negated ones of its memory."""
    neg = torch._neg_view
    for gated, name in NAMES:
        t = neg(usual(gated, name))
        for call in forward_and_backward(gated, **{name: t}):
            with pytest.raises(ValueError, match="^%s: " % name):
                call()
    column = torch.zeros(0, 1, dtype=torch.complex32).conj().imag
    op = F._native().Op(False, B.FF_ACT["none"], torch.zeros(2, 1, dtype=torch.float16), None, None, None, 1)
    with pytest.raises(ValueError, match="^x: "):
        op.forward(column, None, None, False, 0)
    op.forward(column.resolve_neg(), None, None, False, 0)


@pytest.mark.parametrize("gated,name", NAMES)
def test_storage_that_was_taken_away_is_refused(gated, name):
    """A freed or shortened storage leaves a tensor its sizes: behind an offset its address is not even null."""
    w, b = operands(gated)
    dy = "dh" if gated else "dy"
    all_of = dict(w, **b, x=torch.zeros(5, K, dtype=torch.bfloat16), saved=torch.zeros(2, 5, N) if gated else torch.zeros(5, N),
                  **{n: torch.zeros(5, N, dtype=torch.bfloat16) for n in ("residual", "out", "dy", "dh")})
    usual = all_of[name]
    for left in (0, 16, (2 * usual.numel() - 1) * usual.itemsize):
        buf = torch.zeros(2 * usual.numel(), dtype=usual.dtype)
        t = buf[usual.numel():].view(usual.shape)
        kw = dict(all_of, **{name: t})
        op = native(gated, {n: kw[n] for n in w}, {n: kw[n] for n in b})
        buf.untyped_storage().resize_(left)
        if name not in ("saved", dy):
            with pytest.raises(ValueError, match="^%s: .*storage" % name):
                op.forward(kw["x"], kw["residual"] if name == "residual" else None, kw["out"] if name == "out" else None, True, 0)
        if name not in ("residual", "out"):
            with pytest.raises(ValueError, match="^%s: .*storage" % name):
                op.backward(kw[dy], kw["x"], kw["saved"], True, True, True, 0)
