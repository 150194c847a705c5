"""What the cross entropy refuses, and the sizes it accepts, without a GPU."""
import ctypes

import pytest
import torch

from paper_2011_05630_amd import binding as B
from paper_2011_05630_amd import feedforward as F

P, Q = 0x10000, 0x20000      # never read: every call here is refused before a launch
BIG = 1 << 40


def desc(**kw):
    d = dict(dtype="bf16", rows=4, in_features=16, classes=24)
    d.update(kw)
    return B.dlf_ce_desc(**d)


def status(f, *a):
    with pytest.raises(B.DlfError) as e:
        f(*a)
    assert str(e.value)
    return e.value.status


def loss(d, x=P, w=P, b=None, t=P, out=Q, lse=None, ws=P, n=BIG):
    return lambda: B.dlf_cross_entropy(d, x, w, b, t, out, lse, ws, n)


def backward(d, x=P, w=P, b=None, t=P, lse=P, dloss=P, ds=1, value=0.0, dlse=None, es=0, dx=Q, dw=Q, db=None, ws=P, n=BIG):
    return lambda: B.dlf_cross_entropy_backward(d, x, w, b, t, lse, dloss, ds, value, dlse, es, dx, dw, db, ws, n)


def gradients(d, x=P, w=P, b=None, t=P, dloss=P, ds=1, value=0.0, out=Q, dx=Q, dw=Q, db=None, ws=P, n=BIG):
    return lambda: B.dlf_cross_entropy_gradients(d, x, w, b, t, dloss, ds, value, out, dx, dw, db, ws, n)


CALLS = (loss, backward, gradients)
SIZES = (B.dlf_cross_entropy_workspace_bytes, B.dlf_cross_entropy_backward_workspace_bytes, B.dlf_cross_entropy_gradients_workspace_bytes)
BAD = [dict(rows=-1), dict(rows=(1 << 30) + 1), dict(in_features=0), dict(classes=0), dict(in_features=(1 << 20) + 1), dict(classes=(1 << 20) + 1),
       dict(x_stride=15), dict(w_stride=-16), dict(x_stride=1 << 24), dict(w_stride=1 << 40), dict(piece_bytes=-1), dict(piece_bytes=(1 << 50) + 1)]


@pytest.mark.parametrize("kw", BAD)
def test_bad_descriptions(kw):
    d = desc(**kw)
    for call in CALLS:
        assert status(call(d)) == B.DLF_ERR_INVALID_ARG
    for f in SIZES:
        status(f, d)


@pytest.mark.parametrize("field,value", [("dtype", 2), ("dtype", -1), ("dbias", 2), ("dbias", -1)])
def test_bad_fields(field, value):
    d = desc()
    setattr(d, field, value)
    for call in CALLS:
        assert status(call(d)) == B.DLF_ERR_INVALID_ARG


def test_a_bias_gradient_that_the_description_does_not_name():
    d, e = desc(), desc(dbias=1)
    assert status(gradients(d, db=Q)) == B.DLF_ERR_INVALID_ARG
    # backward keeps nothing for it
    assert SIZES[0](d) == SIZES[0](e) and SIZES[1](d) == SIZES[1](e)


def test_null_description():
    L = B.lib()
    assert L.dlf_cross_entropy(None, P, P, None, P, Q, None, P, BIG, None) == B.DLF_ERR_INVALID_ARG
    for n in ("", "_backward", "_gradients"):
        assert getattr(L, "dlf_cross_entropy%s_workspace_bytes" % n)(None) == ctypes.c_size_t(-1).value


@pytest.mark.parametrize("i,o", [(1, 1 << 20), (1 << 20, 1), (4096, 1 << 17), (1 << 20, 500), (1000, 50257)])
def test_most_features_and_classes(i, o):
    """As include/dlf.h states them: any number of rows, and 2 i o + 2 o + 4 i below 2^24 - 16 in 64s."""
    def stated(i, o):
        i, o = (i + 63) // 64, (o + 63) // 64
        return 2 * i * o + 2 * o + 4 * i < (1 << 24) - 16

    for a, c in ((i, o), (i, min(1 << 20, 2 * o)), (min(1 << 20, 2 * i), o), (min(1 << 20, 16 * i), min(1 << 20, 16 * o))):
        for rows in (1, 1000, 1 << 20):
            got = []
            for f in SIZES:
                try:
                    got.append(f(desc(rows=rows, in_features=a, classes=c)) > 0)
                except B.DlfError as e:
                    assert e.status in (B.DLF_ERR_INVALID_ARG, B.DLF_ERR_UNSUPPORTED)
                    got.append(False)
            assert set(got) == {stated(a, c)}, (a, c, rows, got)


def test_null_and_misaligned_operands():
    d = desc()
    for call in CALLS:
        for kw in (dict(x=None), dict(w=None), dict(t=None), dict(x=P + 1), dict(w=P + 1), dict(b=P + 2), dict(t=P + 4)):
            assert status(call(d, **kw)) == B.DLF_ERR_INVALID_ARG
    for call in (loss, gradients):
        for kw in (dict(out=None), dict(out=Q + 2)):
            assert status(call(d, **kw)) == B.DLF_ERR_INVALID_ARG
    assert status(loss(d, lse=Q + 2)) == B.DLF_ERR_INVALID_ARG
    assert status(backward(d, lse=None)) == B.DLF_ERR_INVALID_ARG
    for call in (backward, gradients):
        for kw in (dict(dloss=P + 2), dict(ds=-1), dict(ds=(1 << 24) + 1), dict(dloss=None, value=float("nan")), dict(dloss=None, value=float("inf")),
                   dict(dx=Q + 1), dict(dw=Q + 1), dict(db=Q + 2)):
            assert status(call(d, **kw)) == B.DLF_ERR_INVALID_ARG
    assert status(backward(d, dlse=P + 2, es=1)) == B.DLF_ERR_INVALID_ARG
    assert status(backward(d, dlse=P, es=-1)) == B.DLF_ERR_INVALID_ARG


@pytest.mark.parametrize("rows", [3, 100, 5000])
def test_workspaces(rows):
    for k in (16, 41):
        d = desc(rows=rows, in_features=k, piece_bytes=1)
        for call, f in zip(CALLS, SIZES):
            need = f(d)
            assert need > 0
            assert status(call(d, n=need - 1)) == B.DLF_ERR_OOM
            assert status(call(d, ws=None, n=need)) == B.DLF_ERR_INVALID_ARG
            assert status(call(d, ws=P + 128, n=need)) == B.DLF_ERR_INVALID_ARG


def test_workspaces_are_bounded_by_the_piece():
    """131072 classes, 65536 rows: what the logits alone would take is 32 GiB in 32 bits; dz of a piece takes what piece_bytes say."""
    for piece in (1 << 28, 1 << 30):
        got = B.dlf_cross_entropy_gradients_workspace_bytes(desc(rows=65536, in_features=64, classes=131072, piece_bytes=piece))
        assert piece * 0.7 < got < 1.3 * piece + (64 << 20)
        # ... and the logits, where the bias's gradient is wanted, twice that
        got = B.dlf_cross_entropy_gradients_workspace_bytes(desc(rows=65536, in_features=64, classes=131072, piece_bytes=piece, dbias=1))
        assert piece * 2.1 < got < 3.9 * piece + (64 << 20)
    assert B.dlf_cross_entropy_workspace_bytes(desc(rows=65536, in_features=64, classes=131072)) < 1 << 30


def test_no_rows_is_no_error_forward():
    B.dlf_cross_entropy(desc(rows=0), None, None, None, None, None)


# ---- the native step, on CPU tensors --------------------------------------------------------

K, V = 16, 24
X, T = torch.zeros(6, K, dtype=torch.bfloat16), torch.zeros(6, dtype=torch.int64)


def op(bias=False, t=torch.bfloat16, w=None, b=None):
    w = torch.zeros(V, K, dtype=t) if w is None else w
    b = torch.zeros(V) if bias and b is None else b
    return F._native().CrossEntropy(w, b, w.stride(0), -100, 1 << 30)


BAD_X = {"not a tensor": [1.0], "type": X.half(), "width": X[:, :15], "no dimension": X[0, 0], "strided row": torch.zeros(K, 6, dtype=torch.bfloat16).t(),
         "overlapping": X[:1].expand(6, K), "gap between blocks": torch.zeros(4, 6, K, dtype=torch.bfloat16)[:, :5]}
BAD_TARGET = {"not a tensor": 3, "type": T.int(), "fewer": T[:5], "another shape": T.view(2, 3), "strided": torch.zeros(12, dtype=torch.int64)[::2],
              "expanded": T[:1].expand(6), "fp32": T.float()}
GIVEN = {"None": None, "text": "1", "type": torch.zeros(6, dtype=torch.float64), "fewer": torch.zeros(5), "two": torch.zeros(2), "strided": torch.zeros(12)[::2],
         "another shape": torch.zeros(3, 2), "not finite": float("nan")}


def calls(o, x=X, t=T, dloss=1.0, lse=torch.zeros(6), dlse=None):
    return (lambda: o.forward(x, t, False, 0), lambda: o.forward(x, t, True, 0), lambda: o.backward(dloss, x, t, lse, dlse, True, True, True, 0),
            lambda: o.gradients(x, t, dloss, True, True, True, 0))


@pytest.mark.parametrize("what", sorted(BAD_X))
def test_inputs(what):
    for call in calls(op(), x=BAD_X[what]):
        with pytest.raises(ValueError, match="^x: "):
            call()


@pytest.mark.parametrize("what", sorted(BAD_TARGET))
def test_targets(what):
    for call in calls(op(), t=BAD_TARGET[what]):
        with pytest.raises(ValueError, match="^target: "):
            call()


@pytest.mark.parametrize("what", sorted(GIVEN))
def test_gradients_given(what):
    for call in calls(op(), dloss=GIVEN[what])[2:]:
        with pytest.raises(ValueError, match="^dloss: "):
            call()
    if what != "None":
        with pytest.raises(ValueError, match="^dlse: "):
            calls(op(), dlse=GIVEN[what])[2]()
    with pytest.raises(ValueError, match="^dlse: "):
        calls(op(), dlse=1.0)[2]()


def test_lse():
    for bad in (None, torch.zeros(5), torch.zeros(6).double(), torch.zeros(12)[::2], torch.zeros(2, 3)):
        with pytest.raises(ValueError, match="^lse: "):
            calls(op(), lse=bad)[2]()


OTHER = {"weight": [lambda: torch.zeros(V - 1, K, dtype=torch.bfloat16), lambda: torch.zeros(V, K, dtype=torch.float16), lambda: torch.zeros(K, V, dtype=torch.bfloat16).t(),
                    lambda: torch.zeros(V, K + 8, dtype=torch.bfloat16)[:, :K], lambda: torch.zeros(V * K, dtype=torch.bfloat16)],
         "bias": [lambda: torch.zeros(V - 1), lambda: torch.zeros(V).double(), lambda: torch.zeros(2 * V)[::2], lambda: torch.zeros(1, V)]}


@pytest.mark.parametrize("name", sorted(OTHER))
def test_operands_of_another_form_are_refused(name):
    for other in OTHER[name]:
        w, b = torch.zeros(V, K, dtype=torch.bfloat16), torch.zeros(V)
        o = op(w=w, b=b)
        (w if name == "weight" else b).data = other()
        for call in calls(o):
            with pytest.raises(ValueError, match="^%s: " % name):
                call()


def test_what_automatic_differentiation_follows_is_refused():
    for name, kw in (("x", dict(x=X.clone().requires_grad_())), ("dloss", dict(dloss=torch.zeros(6, requires_grad=True)))):
        for call in calls(op(), **kw)[2 if name == "dloss" else 0:]:
            with pytest.raises(ValueError, match="^%s: requires a gradient" % name):
                call()
    w = torch.zeros(V, K, dtype=torch.bfloat16, requires_grad=True)
    for call in calls(op(w=w)):
        with pytest.raises(ValueError, match="^weight: requires a gradient"):
            call()


def test_storages_that_no_longer_hold_their_tensors():
    for name in ("x", "target", "weight", "bias"):
        x, t, w, b = X.clone(), T.clone(), torch.zeros(V, K, dtype=torch.bfloat16), torch.zeros(V)
        o = op(w=w, b=b)
        dict(x=x, target=t, weight=w, bias=b)[name].untyped_storage().resize_(8)
        for call in calls(o, x=x, t=t):
            with pytest.raises(ValueError, match="^%s: its storage" % name):
                call()


def test_no_rows():
    o = op(bias=True)
    for shape in ((0, K), (3, 0, K)):
        x, t = torch.zeros(shape, dtype=torch.bfloat16), torch.zeros(shape[:-1], dtype=torch.int64)
        value, lse = o.forward(x, t, True, 0)
        assert value.shape == lse.shape == shape[:-1] and value.dtype == lse.dtype == torch.float32


def test_construction():
    from paper_2011_05630_amd import loss
    with pytest.raises(ValueError, match="^weight: "):
        loss.CrossEntropy(torch.zeros(V, K, dtype=torch.bfloat16))
