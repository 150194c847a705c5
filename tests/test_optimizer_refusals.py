"""What AdamW and the gradients' norm refuse, and what they keep where, without a GPU."""
import ctypes

import numpy as np
import pytest
import torch

from opt_util import E4M3, E5M2, codes_of, decode, noise_of, scale_of, stir
from paper_2011_05630_amd import binding as B
from paper_2011_05630_amd import feedforward as F

P, Q = 0x10000, 0x20000      # never read: every call here is refused before a launch


def status(f, *a, **kw):
    with pytest.raises(B.DlfError) as e:
        f(*a, **kw)
    assert str(e.value)
    return e.value.status


def one(p=P, c=None, n=100, t="fp32", ct=None, decay=0.0):
    return B.dlf_adamw_tensors([(p, c, n, t, ct, decay)])


def step(tensors=None, n=1, d=None, table=P, g=(P,), gt=("bf16",), m=P, v=P, ms=None, vs=None, counter=P, rate=0.1, rate_at=None, factor=None):
    return status(B.dlf_adamw_step, B.dlf_adamw_desc() if d is None else d, one() if tensors is None else tensors, n, table, g, gt, m, v, ms, vs, counter, rate,
                  rate_at, factor)


def test_steps():
    for kw in (dict(table=None), dict(m=None), dict(v=None), dict(m=P + 8), dict(v=P + 4), dict(table=P + 8), dict(counter=None), dict(counter=P + 4), dict(g=(P + 1,)),
               dict(rate=float("nan")), dict(rate=float("inf")), dict(rate_at=P + 2), dict(factor=P + 1), dict(g=(P + 2,), gt=("fp32",))):
        assert step(**kw) == B.DLF_ERR_INVALID_ARG
    d = B.dlf_adamw_desc(state="8bit")
    for kw in (dict(), dict(ms=P), dict(vs=P), dict(ms=P + 4, vs=P)):
        assert step(d=d, **kw) == B.DLF_ERR_INVALID_ARG
    assert B.lib().dlf_adamw_step(None, one(), 1, P, None, None, P, P, None, None, P, 0.1, None, None, None) == B.DLF_ERR_INVALID_ARG
    assert B.lib().dlf_adamw_step(B.dlf_adamw_desc(), one(), 1, P, None, None, P, P, None, None, P, 0.1, None, None, None) == B.DLF_ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(betas=(1.0, 0.9)), dict(betas=(-0.1, 0.9)), dict(betas=(0.9, 1.0)), dict(betas=(0.9, float("nan"))), dict(eps=-1.0),
                                dict(eps=float("inf")), dict(eps=float("nan"))])
def test_descriptions(kw):
    assert step(d=B.dlf_adamw_desc(**kw)) == B.DLF_ERR_INVALID_ARG


# (a reciprocal of less than 2^-126, or that is less, is none on the device: m = 0 times infinity would be NaN)
@pytest.mark.parametrize("eps", [1e-45, 1e-40, 2.0 ** -127, 2.0 ** 126 * 1.001, 3e38])
def test_eps_outside_the_range_of_reciprocals(eps):
    from paper_2011_05630_amd import optimizer
    assert step(d=B.dlf_adamw_desc(eps=eps)) == B.DLF_ERR_INVALID_ARG
    with pytest.raises(ValueError, match="^eps: "):
        optimizer.AdamW([], eps=eps)
    if eps < 1:
        with pytest.raises(ValueError, match="^eps: "):
            optimizer.AdamW([], eps=1e-60)                  # (0 in 32 bits)


@pytest.mark.parametrize("field,value", [("state", 2), ("state", -1), ("reserved", 1)])
def test_bad_fields(field, value):
    d = B.dlf_adamw_desc()
    setattr(d, field, value)
    assert step(d=d) == B.DLF_ERR_INVALID_ARG


BAD = {"null": one(p=None), "misaligned": one(p=P + 2), "negative": one(n=-1), "huge": one(n=(1 << 40) + 1), "decay": one(decay=float("nan")),
       "copy of bf16": one(t="bf16", c=Q, ct="bf16"), "fp32 copy": one(c=Q, ct="fp32"), "misaligned copy": one(c=Q + 1, ct="bf16")}


@pytest.mark.parametrize("what", sorted(BAD))
def test_tensors(what):
    t = BAD[what]
    assert step(t) == B.DLF_ERR_INVALID_ARG
    for f in (B.dlf_adamw_state_elements, B.dlf_adamw_table_bytes):
        status(f, t, 1)
    assert status(B.dlf_adamw_table, t, 1, P, 1 << 20) == B.DLF_ERR_INVALID_ARG


def test_bad_fields_of_tensors():
    for field, value in (("param_dtype", 3), ("param_dtype", -1), ("reserved", 1)):
        t = one()
        setattr(t[0], field, value)
        assert step(t) == B.DLF_ERR_INVALID_ARG
    many = B.dlf_adamw_tensors([(P, None, 1 << 40, "fp32", None, 0.0)] * 5)
    assert step(many, n=5, g=(P,) * 5, gt=("bf16",) * 5) == B.DLF_ERR_UNSUPPORTED
    assert step(n=-1, g=(), gt=()) == B.DLF_ERR_INVALID_ARG


def test_table():
    """Chunks of 4096 elements, tensors' states on whole blocks of 64."""
    sizes = [1, 64, 65, 0, 4096, 4097, 10000]
    t = B.dlf_adamw_tensors([(0x1000000 * (i + 1), 0x80000000 + 0x1000000 * i if i % 2 else None, n, "fp32", "bf16" if i % 2 else None, 0.5 * i) for i, n in enumerate(sizes)])
    assert B.dlf_adamw_state_elements(t, len(sizes)) == sum(-(-n // 64) * 64 for n in sizes)
    need, chunks = B.dlf_adamw_table_bytes(t, len(sizes)), sum(-(-n // 4096) for n in sizes)
    size = need // chunks
    buf = ctypes.create_string_buffer(need + 1)
    assert status(B.dlf_adamw_table, t, len(sizes), ctypes.addressof(buf), need - 1) == B.DLF_ERR_OOM
    B.dlf_adamw_table(t, len(sizes), ctypes.addressof(buf) + 1, need)       # (any alignment)
    kind = np.dtype([("p", "u8"), ("c", "u8"), ("state", "i8"), ("at", "i8"), ("n", "i4"), ("tensor", "i4"), ("decay", "f4"), ("types", "u4")])
    assert kind.itemsize == size
    got, k, state = np.frombuffer(buf.raw[1:], kind), 0, 0
    for i, n in enumerate(sizes):
        for at in range(0, n, 4096):
            e = got[k]
            assert (e["p"], e["state"], e["at"], e["n"], e["tensor"], e["decay"]) == (0x1000000 * (i + 1) + 4 * at, state + at, at, min(4096, n - at), i, 0.5 * i)
            assert e["c"] == (0x80000000 + 0x1000000 * i + 2 * at if i % 2 else 0)
            k += 1
        state += -(-n // 64) * 64
    assert k == chunks


def test_norms():
    def call(g=(P,), n=(100,), t=("bf16",), most=1.0, scale=1.0, norm=Q, factor=Q, ws=P, size=1 << 20):
        return status(B.dlf_gradient_norm, g, n, t, most, scale, norm, factor, ws, size)
    for kw in (dict(g=(None,)), dict(g=(P + 1,)), dict(n=(-1,)), dict(n=((1 << 40) + 1,)), dict(most=-1.0), dict(most=float("nan")), dict(scale=float("inf")),
               dict(norm=None), dict(norm=Q + 2), dict(factor=Q + 1), dict(ws=None), dict(ws=P + 8)):
        assert call(**kw) == B.DLF_ERR_INVALID_ARG
    need = B.dlf_gradient_norm_workspace_bytes([100])
    assert call(size=need - 1) == B.DLF_ERR_OOM
    assert B.dlf_gradient_norm_workspace_bytes([]) == 0 == B.dlf_gradient_norm_workspace_bytes([0, 0])
    assert B.lib().dlf_gradient_norm(None, None, None, 1, 1.0, 1.0, Q, Q, P, 1 << 20, None) == B.DLF_ERR_INVALID_ARG


# ---- the native step, on CPU tensors --------------------------------------------------------

def make(params, copies=None, decay=None, state="fp32"):
    return F._native().AdamW(params, copies, decay or [0.0] * len(params), 0.9, 0.95, 1e-8, {"fp32": 0, "8bit": 1}[state], 0)


def pair():
    return [torch.zeros(100), torch.zeros(30, 10)]


def test_states_begin_as_zeros():
    for state in ("fp32", "8bit"):
        o = make(pair() + [torch.zeros(0)], state=state)
        assert o.m.shape == o.v.shape == (128 + 320,) and o.counter.tolist() == [0, 1, 1, 0]
        assert o.m.dtype == (torch.float8_e4m3fn if state == "8bit" else torch.float32) and o.v.dtype == (torch.float8_e5m2 if state == "8bit" else torch.float32)
        assert (o.m.view(torch.uint8) == 0).all() and (o.v.view(torch.uint8) == 0).all()
        assert (o.m_scale is None) == (o.v_scale is None) == (state == "fp32")
        assert state == "fp32" or (o.m_scale.shape == (7,) and (o.m_scale == 1).all())


BAD_PARAMS = {"none": [], "not a list": torch.zeros(3), "not a tensor": [1.0], "type": [torch.zeros(3).double()], "strided": [torch.zeros(20)[::2]],
              "expanded": [torch.zeros(1).expand(5)], "the same twice": None, "overlapping": None}


@pytest.mark.parametrize("what", sorted(BAD_PARAMS))
def test_parameters(what):
    base = torch.zeros(20)
    p = {"the same twice": [base, base], "overlapping": [base[:10], base[9:]]}.get(what, BAD_PARAMS[what])
    with pytest.raises(ValueError, match="overlap$" if what in ("the same twice", "overlapping") else "^param"):
        make(p, decay=[0.0] * (2 if BAD_PARAMS[what] is None else 1))


def test_copies():
    p = pair()
    c = [torch.zeros(100).bfloat16(), torch.zeros(30, 10).half()]
    make(p, c)
    make(p, [None, c[1]])
    with pytest.raises(ValueError, match="^copies: "):
        make(p, c[:1])
    for bad in (torch.zeros(100), torch.zeros(99).half(), torch.zeros(200).half()[::2], 1.0, torch.zeros(100, dtype=torch.int16)):
        with pytest.raises(ValueError, match="^copy 0: "):
            make(p, [bad, c[1]])
    with pytest.raises(ValueError, match="^copy 1: "):
        make([p[0], p[1].bfloat16()], c)
    with pytest.raises(ValueError, match="^copy 1: "):
        make(p, [c[0], torch.zeros(10, 30).half().t()])
    raw = torch.zeros(400, dtype=torch.uint8)
    with pytest.raises(ValueError, match="overlap$"):
        make([raw.view(torch.float32)], [raw[:200].view(torch.bfloat16)])
    with pytest.raises(ValueError, match="^decay: "):
        make(p, decay=[0.0])


def test_gradients():
    p = pair()
    o = make(p)
    good = [torch.zeros(100).half(), torch.zeros(30, 10)]
    for bad in (good[:1], good + good, torch.zeros(2), iter(good)):
        with pytest.raises(ValueError, match="^gradients: "):
            o.step(bad, 0.1, None, 0)
    for bad in (1.0, torch.zeros(100).double(), torch.zeros(99), torch.zeros(100, 1), torch.zeros(200)[::2], torch.zeros(1).expand(100), torch.zeros(100, requires_grad=True),
                p[0], p[0][:50], o.m[:100]):
        with pytest.raises(ValueError, match="^gradient 0: "):
            o.step([bad, good[1]], 0.1, None, 0)
    with pytest.raises(ValueError, match="^gradient 1: the sizes and strides"):
        o.step([good[0], torch.zeros(10, 30).t()], 0.1, None, 0)
    for bad in ("1", None, float("nan"), float("inf"), torch.zeros(2), torch.zeros(1).double(), p[0][:1]):
        with pytest.raises(ValueError, match="^rate: "):
            o.step(good, bad, None, 0)
    for bad in (1.0, torch.zeros(2), torch.zeros(1).half(), o.v[:1]):
        with pytest.raises(ValueError, match="^factor: "):
            o.step(good, 0.1, bad, 0)


def test_tensors_that_changed():
    for change in ("data", "size", "type", "storage"):
        p, c = pair(), [torch.zeros(100).bfloat16(), None]
        o = make(p, c)
        which = c[0] if change == "type" else p[0]
        if change == "data":
            p[0].data = torch.zeros(100)
        elif change == "size":
            p[0].data = p[0].data[:50]
        elif change == "type":
            c[0].data = torch.zeros(100).half()
        else:
            p[0].untyped_storage().resize_(0)
        with pytest.raises(ValueError, match="^copy 0: " if which is c[0] else "^parameter 0: "):
            o.step([torch.zeros(100), None], 0.1, None, 0)


CHANGED = {"transposed": lambda t: t.t(), "reshaped": lambda t: t.reshape(20, 15), "flat": lambda t: t.reshape(300), "another dimension": lambda t: t[None]}


@pytest.mark.parametrize("what", sorted(CHANGED))
def test_tensors_whose_form_changed(what):
    """The same memory with other sizes or strides: the gradient's order would be the new one, the copy's the old one."""
    change = CHANGED[what]
    for which in ("parameter", "copy", "both"):
        p, c = pair(), [None, torch.zeros(30, 10).bfloat16()]
        o = make(p, c)
        if which != "copy":
            p[1].data = change(p[1].data)
        if which != "parameter":
            c[1].data = change(c[1].data)
        with pytest.raises(ValueError, match="^copy 1: no longer" if which == "copy" else "^parameter 1: no longer"):
            o.step([None, torch.empty_like(p[1])], 0.1, None, 0)
    square = [torch.zeros(10, 10)]
    o = make(square)
    square[0].data = square[0].data.t()
    with pytest.raises(ValueError, match="^parameter 0: no longer"):
        o.step([torch.empty_like(square[0])], 0.1, None, 0)


@pytest.mark.parametrize("name", ["m", "v", "m_scale", "v_scale", "counter"])
def test_states_that_changed(name):
    """The states are the object's own tensors, which a program may read and write, but not exchange: a step writes as many elements as there were."""
    for change in ("memory", "size", "type", "storage"):
        o = make(pair(), state="8bit")
        t = getattr(o, name)
        if change == "memory":
            t.data = t.data.clone()
        elif change == "size":
            t.data = t.data[:-1]
        elif change == "type":
            t.data = t.data.view(torch.uint8)
        else:
            t.untyped_storage().resize_(0)
        with pytest.raises(ValueError, match="^%s: no longer the tensor, or the memory" % name if change != "storage" else "^%s: " % name):
            o.step([torch.zeros(100), None], 0.1, None, 0)


def test_a_parameter_that_automatic_differentiation_computed():
    leaf = torch.zeros(100, requires_grad=True)
    o = make([leaf * 2])
    with pytest.raises(ValueError, match="^parameter 0: automatic differentiation"):
        o.step([torch.zeros(100)], 0.1, None, 0)


def test_python_refuses():
    from paper_2011_05630_amd import optimizer
    with pytest.raises(ValueError, match="^params: "):
        optimizer.AdamW([torch.zeros(3)])
    with pytest.raises(ValueError, match="^params: a list"):
        optimizer.AdamW(torch.zeros(3))
    for kw in (dict(state="16bit"), dict(betas=(1.0, 0.5)), dict(eps=-1), dict(seed=-1), dict(seed=1 << 32), dict(seed=0.5)):
        with pytest.raises(ValueError):
            optimizer.AdamW([], **kw)
    for bad in ([], [None], torch.zeros(3), [torch.zeros(3)]):
        with pytest.raises(ValueError, match="^gradients: "):
            optimizer.gradient_norm(bad)
    with pytest.raises(ValueError, match="^gradient 1: "):
        F._native().gradient_norm([torch.zeros(3), torch.zeros(6)[::2]], 1.0, 1.0, 0)


# ---- the codes of 8 bits, as the plain form has them -----------------------------------------

def test_codes_are_the_types_that_pytorch_has():
    for table, t in ((E4M3, torch.float8_e4m3fn), (E5M2, torch.float8_e5m2)):
        have = torch.arange(256, dtype=torch.uint8).view(t).float().numpy()
        assert np.array_equal(have[:len(table)], table) and np.array_equal(have[128:128 + len(table)], -table)
        assert np.isnan(decode(np.full(64, 0x7F, np.uint8), np.ones(1), table)).all() and np.isnan(have[0x7F])


@pytest.mark.parametrize("table,top,kept", [(E4M3, 8, False), (E5M2, 15, True)])
def test_rounding_is_unbiased(table, top, kept):
    """Over many draws of the noise a code stands for its value: within five standard deviations of a mean of 65536, a step's part each, and 2^-17 of a step."""
    x = np.array([1.0, 0.999, 0.3, 0.01, 1.7e-3, 2e-5, 3.3e-6] + [0.0] * 57, np.float32)
    s = scale_of(x, top)
    n = 1 << 16
    got = np.zeros(64)
    square = np.zeros(64)
    for k in range(0, n, 1024):
        noise = noise_of(3, 7, k * 64, 64 * 1024) >> np.uint64(16)
        v = decode(codes_of(np.tile(x, 1024), np.repeat(s, 1024), table, noise, False), np.repeat(s, 1024), table).astype(np.float64).reshape(1024, 64)
        got += v.sum(0)
        square += (v ** 2).sum(0)
    mean = got / n
    dev = np.sqrt(np.maximum(square / n - mean ** 2, 0) / n)
    step = np.maximum(np.abs(x), table[1] * s) / 4
    assert (np.abs(mean - x) <= 5 * dev + 2.0 ** -17 * step + 2.0 ** -24 * table[1 << (3 if top == 8 else 2)] * s).all(), (mean - x, dev)


def test_the_hash_spreads():
    """Bits of neighbouring places, steps and seeds: each is set half of the time and pairs agree half of the time, within five standard deviations."""
    n = 1 << 16
    def bits(h):
        return (h[:, None] >> np.arange(32, dtype=np.uint64)) & np.uint64(1)
    a = bits(noise_of(1, 5, 0, n)).astype(np.int64)
    limit = 5 * 0.5 * np.sqrt(n)
    assert (np.abs(a.sum(0) - n / 2) < limit).all()
    for other in (noise_of(1, 5, 1, n), noise_of(1, 5, 64, n), noise_of(1, 6, 0, n), noise_of(2, 5, 0, n), noise_of(1, 5, 1 << 32, n)):
        assert (np.abs((a == bits(other)).sum(0) - n / 2) < limit).all()
    for d in range(1, 32):
        assert (np.abs((a == np.roll(a, d, 1)).sum(0) - n / 2) < limit).all()
    assert int(stir(0)) == 0
