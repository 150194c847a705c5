"""The cross entropy of a linear layer on the GPU against its formulas in 64 bits, within bounds of its roundings (ce_util)."""
import pytest
import torch

from ce_util import IGNORE, gradients, reference
from ff_util import TYPES, U, gen, half_eps, rows_of, within
from gpu_util import announce

pytestmark = pytest.mark.gpu

SIZES = [(1, 1, 1), (1, 64, 1000), (2, 3, 5), (5, 72, 33), (16, 128, 64), (17, 40, 129), (33, 256, 2049), (64, 136, 257), (65, 100, 300), (129, 64, 1000),
         (257, 136, 513), (300, 520, 1001), (520, 65, 129), (700, 256, 2500), (1, 2048, 5003), (48, 1003, 777)]


def inputs(m, k, v, t, seed, bias=False, ignored=0.0, gap=0, offset=0, sure=4.0):
    """Values as the type holds them, in 64 bits on the CPU, and the same on the GPU: rows that have learned something."""
    g = gen(seed)
    w = (torch.randn(v, k, generator=g) * k ** -0.5).to(t)
    target = torch.randint(v, (m,), generator=g)
    x = (torch.randn(m, k, generator=g) + sure * w.float()[target]).to(t)
    b = torch.randn(v, generator=g) * 0.3 if bias else None
    target[torch.rand(m, generator=g) < ignored] = IGNORE
    on = dict(x=rows_of(x.double(), t, gap, offset), w=rows_of(w.double(), t, gap, offset), b=None if b is None else b.cuda(), target=target.cuda())
    return x.double(), w.double(), None if b is None else b.double(), target, on


def given(m, seed):
    """Gradients of loss and lse as 32 bits hold them."""
    g = gen(seed)
    return (0.5 + torch.rand(m, generator=g)) / m, torch.randn(m, generator=g) * 0.1 / m


def check_all(m, k, v, dtype, seed, bias, ignored, gap=0, offset=0, piece_bytes=1 << 30):
    from paper_2011_05630_amd import loss
    t = TYPES[dtype]
    announce(m, k, v, dtype, seed, bias, ignored, gap, offset, piece_bytes)
    x, w, b, target, on = inputs(m, k, v, t, seed, bias, ignored, gap, offset)
    scale = 256.0 if dtype == "fp16" else 1.0
    dloss, dlse = (q * scale for q in given(m, seed + 1))
    ref = reference(x, w, b, target)
    op = loss.CrossEntropy(on["w"], on["b"], ignore_index=IGNORE, piece_bytes=piece_bytes)
    within(op.run(on["x"], on["target"]), ref["loss"], ref["e_loss"], "loss alone")
    got, lse = op.run_saved(on["x"], on["target"])
    within(got, ref["loss"], ref["e_loss"], "loss")
    within(lse, ref["lse"], ref["e_lse"], "lse")
    names = ("dx", "dw", "db")
    want = gradients(ref, x, w, dloss.double(), dlse.double(), t)
    for name, value in zip(names, op.backward(dloss.cuda(), on["x"], on["target"], lse, dlse=dlse.cuda())):
        assert (value is None) == (name == "db" and b is None)
        if value is not None:
            within(value, *want[name], name + " in two calls")
    mean = torch.full((), scale / m)
    want = gradients(ref, x, w, mean.double().expand(m), torch.zeros(m).double(), t, kept=b is None)
    got, *grads = op.gradients(on["x"], on["target"], mean.cuda())
    within(got, ref["loss"], ref["e_loss"], "loss with gradients")
    for name, value in zip(names, grads):
        if value is not None:
            within(value, *want[name], name + " in one call")


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("m,k,v", SIZES)
def test_sizes(m, k, v, dtype):
    check_all(m, k, v, dtype, m + v, bias=(m + k + v) % 2 == 1, ignored=0.3 if m > 1 else 0.0)
    check_all(m, k, v, dtype, m + v + 7, bias=(m + k + v) % 2 == 0, ignored=0.0, gap=(5 if m % 2 else 8), offset=(3 if m % 2 else 8))


@pytest.mark.parametrize("kernel", [1, 2, 3, 4, 5, 6])
@pytest.mark.parametrize("bias", [False, True])
def test_every_kernel(kernel, bias):
    """Each tile shape where the rule would take another, and the kernel for few rows that start anywhere."""
    from paper_2011_05630_amd import binding as B
    B.dlf_debug_ff_kernel(kernel)
    try:
        for m, k, v in ((3, 72, 100), (70, 200, 333), (300, 136, 700)):
            check_all(m, k, v, "bf16", kernel, bias, 0.2)
            check_all(m, k, v, "fp16", kernel + 50, bias, 0.2)
    finally:
        B.dlf_debug_ff_kernel()


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("bias", [False, True])
def test_pieces(dtype, bias):
    """Rows in three pieces, the last one short: the weight's gradient is summed over them in 32 bits."""
    check_all(700, 72, 500, dtype, 3, bias, 0.2, piece_bytes=1)
    check_all(513, 41, 130, dtype, 4, bias, 0.0, gap=5, offset=1, piece_bytes=1)


@pytest.mark.parametrize("m,k,v,gap,offset,bias,piece_bytes", [(1500, 520, 3000, 5, 3, False, 1 << 30), (1500, 521, 3000, 0, 0, True, 1 << 30),
                                                               (1300, 521, 3000, 8, 1, False, 1), (1300, 523, 2999, 3, 0, True, 1), (4000, 1001, 3000, 0, 0, False, 1 << 30)])
def test_operands_copied_to_whole_lines(m, k, v, gap, offset, bias, piece_bytes):
    """Sizes at which rows that start anywhere are copied first: x alone, both, the weight once for several pieces, and for a loss alone."""
    check_all(m, k, v, "bf16", 61, bias, 0.2, gap=gap, offset=offset, piece_bytes=piece_bytes)


@pytest.mark.parametrize("m", [1, 3, 64, 65, 130])
@pytest.mark.parametrize("bias", [False, True])
def test_many_classes(m, bias):
    """So many that a row's parts are joined by a launch of their own."""
    check_all(m, 16, 60001, "bf16", 62, bias, 0.0)


def test_leading_dimensions_and_gradients_of_one_element():
    from paper_2011_05630_amd import loss
    x, w, b, target, on = inputs(24, 40, 100, torch.bfloat16, 11, bias=True, ignored=0.3)
    op = loss.CrossEntropy(on["w"], on["b"])
    xs, ts = on["x"].view(2, 3, 4, 40), on["target"].view(2, 3, 4)
    whole, lse = op.run_saved(on["x"], on["target"])
    part, lse3 = op.run_saved(xs, ts)
    assert part.shape == lse3.shape == (2, 3, 4) and torch.equal(part.flatten(), whole) and torch.equal(lse3.flatten(), lse)
    # one row, without leading dimensions
    one, _ = op.run_saved(on["x"][0], on["target"][0])
    assert one.shape == () and float(one) == float(op.run(on["x"][:1], on["target"][:1])[0])
    ways = [0.25, torch.full((), 0.25).cuda(), torch.full((1,), 0.25).cuda(), torch.full((1,), 0.25).cuda().expand(24), torch.full((24,), 0.25).cuda()]
    first = op.backward(ways[0], on["x"], on["target"], lse)
    for way in ways[1:]:
        for a, c in zip(first, op.backward(way, on["x"], on["target"], lse)):
            assert torch.equal(a, c)
    ways = ways[:3] + [w_.reshape(-1)[:1].expand(2, 3, 4) if w_.dim() else w_ for w_ in ways[3:4]] + [ways[4].view(2, 3, 4)]
    first = op.gradients(xs, ts, ways[0])
    assert first[1].shape == xs.shape and first[0].shape == (2, 3, 4)
    for way in ways[1:]:
        for a, c in zip(first, op.gradients(xs, ts, way)):
            assert torch.equal(a, c)


@pytest.mark.parametrize("bias", [False, True])
def test_subsets_of_the_gradients(bias):
    from paper_2011_05630_amd import loss
    x, w, b, target, on = inputs(150, 72, 333, torch.float16, 12, bias=bias, ignored=0.1)
    op = loss.CrossEntropy(on["w"], on["b"])
    _, lse = op.run_saved(on["x"], on["target"])
    ref = reference(x, w, b, target)
    want = gradients(ref, x, w, torch.full((150,), 2.0).double(), torch.zeros(150).double(), torch.float16, kept=True)
    order = ("x", "weight", "bias")
    for mask in range(8):
        need = tuple(n for i, n in enumerate(order) if mask >> i & 1)
        for got in (op.backward(2.0, on["x"], on["target"], lse, need=need), op.gradients(on["x"], on["target"], 2.0, need=need)[1:]):
            for i, (name, value) in enumerate(zip(("dx", "dw", "db"), got)):
                assert (value is not None) == (order[i] in need and (i < 2 or bias))
                if value is not None:
                    within(value, *want[name], name)


def test_targets_that_are_no_class_give_nan_in_their_rows():
    from paper_2011_05630_amd import loss
    for m in (5, 200):
        x, w, b, target, on = inputs(m, 64, 100, torch.bfloat16, 13)
        bad = on["target"].clone()
        bad[1], bad[2], bad[3] = 100, -1, 1 << 40
        op = loss.CrossEntropy(on["w"])
        for need in ("x", ("x", "weight")):
            got, dx, dw, _ = op.gradients(on["x"], bad, 1.0, need=need)
            good, gx, _, _ = op.gradients(on["x"], on["target"], 1.0, need="x")
            assert got[1:4].isnan().all() and dx[1:4].isnan().all()
            keep = torch.ones(m, dtype=torch.bool, device="cuda")
            keep[1:4] = False
            assert torch.equal(got[keep], good[keep]) and torch.equal(dx[keep], gx[keep])
            assert dw is None or dw.isnan().all()
        _, lse = op.run_saved(on["x"], bad)
        assert torch.isfinite(lse).all()
        dx = op.backward(1.0, on["x"], bad, lse, need="x")[0]
        assert dx[1:4].isnan().all() and torch.isfinite(dx[keep]).all()


@pytest.mark.parametrize("m", [5, 200])
def test_another_value_to_ignore(m):
    """A class that is ignored, and the usual value, which then is no class."""
    from paper_2011_05630_amd import loss
    x, w, b, target, on = inputs(m, 64, 30, torch.bfloat16, 14)
    t = target.clone()
    t[0], t[1] = 7, 8
    op = loss.CrossEntropy(on["w"], ignore_index=7)
    got, dx, dw, _ = op.gradients(on["x"], t.cuda(), 1.0)
    none = (t == 7).cuda()
    assert (got[none] == 0).all() and (dx[none] == 0).all() and (got[~none] != 0).all()
    t[1] = IGNORE
    assert op.run(on["x"], t.cuda())[1].isnan()


@pytest.mark.parametrize("m", [3, 150])
def test_all_rows_ignored(m):
    """Zero losses and exactly zero gradients, also where logits are infinite."""
    from paper_2011_05630_amd import loss
    x, w, b, target, on = inputs(m, 64, 90, torch.float16, 15, bias=True)
    on["target"].fill_(IGNORE)
    on["b"].fill_(float("-inf"))
    for bias in (None, on["b"]):
        op = loss.CrossEntropy(on["w"], bias)
        got, dx, dw, db = op.gradients(on["x"], on["target"], 1.0)
        assert (got == 0).all() and (dx == 0).all() and (dw == 0).all() and (db is None or (db == 0).all())
        _, lse = op.run_saved(on["x"], on["target"])
        dx, dw, db = op.backward(torch.ones(m).cuda(), on["x"], on["target"], lse)
        assert (dx == 0).all() and (dw == 0).all() and (db is None or (db == 0).all())


@pytest.mark.parametrize("m", [4, 150])
@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_classes_that_take_no_part(m, dtype):
    """A bias of -inf: as if the class were not there; a row of nothing else has lse -inf and loss NaN."""
    from paper_2011_05630_amd import loss
    t = TYPES[dtype]
    x, w, b, target, on = inputs(m, 72, 400, t, 16, bias=True)
    off = torch.zeros(400, dtype=torch.bool)
    off[:130] = True
    off[200::3] = True
    target = torch.where(off[target], torch.tensor(150), target)
    b[off] = float("-inf")
    on["b"].copy_(b)
    op = loss.CrossEntropy(on["w"], on["b"])
    ref = reference(x, w, b, target)
    want = gradients(dict(ref, ez=torch.where(off, 0.0, ref["ez"])), x, w, torch.ones(m).double(), torch.zeros(m).double(), t)
    got, dx, dw, db = op.gradients(on["x"], target.cuda(), 1.0)
    within(got, ref["loss"], ref["e_loss"], "loss")
    for name, value in (("dx", dx), ("dw", dw), ("db", db)):
        within(value, *want[name], name)
    assert (db[off.cuda()] == 0).all() and (dw[off.cuda()] == 0).all()
    # a target among them: infinitely unlikely, and its gradient finite
    target[0] = 0
    got, dx, _, db = op.gradients(on["x"], target.cuda(), 1.0)
    assert got[0] == float("inf") and torch.isfinite(got[1:]).all() and torch.isfinite(dx).all() and db[0] == -1
    on["b"].fill_(float("-inf"))
    got, lse = op.run_saved(on["x"], target.cuda())
    assert (lse == float("-inf")).all() and got.isnan().all()


@pytest.mark.parametrize("m", [4, 150])
def test_infinities_and_nan_stay_in_their_rows(m):
    from paper_2011_05630_amd import loss
    x, w, b, target, on = inputs(m, 64, 300, torch.bfloat16, 17)
    op = loss.CrossEntropy(on["w"])
    good, gx = op.gradients(on["x"], on["target"], 1.0, need="x")[:2]
    on["x"][1, 5], on["x"][2, 6] = float("nan"), float("inf")
    got, dx = op.gradients(on["x"], on["target"], 1.0, need="x")[:2]
    assert not torch.isfinite(got[1:3]).any() and dx[1:3].isnan().all()
    keep = torch.ones(m, dtype=torch.bool, device="cuda")
    keep[1:3] = False
    assert torch.equal(got[keep], good[keep]) and torch.equal(dx[keep], gx[keep])


@pytest.mark.parametrize("m", [8, 300])
def test_large_logits(m):
    """Logits of hundreds: no exponential overflows, sure targets lose nothing."""
    from paper_2011_05630_amd import loss
    t = torch.bfloat16
    x, w, b, target, on = inputs(m, 64, 500, t, 18, sure=300.0)
    ref = reference(x, w, b, target)
    assert float(ref["z"].abs().max()) > 200
    op = loss.CrossEntropy(on["w"])
    got, lse = op.run_saved(on["x"], on["target"])
    within(got, ref["loss"], ref["e_loss"], "loss")
    within(lse, ref["lse"], ref["e_lse"], "lse")
    want = gradients(ref, x, w, torch.ones(m).double(), torch.zeros(m).double(), t, kept=True)
    _, dx, dw, _ = op.gradients(on["x"], on["target"], 1.0)
    within(dx, *want["dx"], "dx")
    within(dw, *want["dw"], "dw")


def sure_rows(m, v, t, seed):
    """Logits of 4000 to 17000 that are the same in any order of their sums, whole numbers of quarters: a feature that all classes share, and fifteen of +-1 that tell them
    apart, a row's being 2 to 2.5 times its target's."""
    g = gen(seed)
    w = torch.randint(0, 2, (v, 16), generator=g).double() * 2 - 1
    w[:, 0] = 64
    target = torch.randint(v, (m,), generator=g)
    x = w[target] * (2.0 + 0.25 * torch.randint(0, 3, (m, 1), generator=g))
    x[:, 0] = torch.randint(64, 257, (m,), generator=g).double()
    return x, w, target, dict(x=x.to(t).cuda(), w=w.to(t).cuda(), target=target.cuda())


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("m", [40, 300, 2100])
def test_sure_targets_of_large_logits(m, bias, dtype):
    """In one call 1 - p of a sure target does not see how large its logit is.  Bounds: the logits are exact, so p is off by its row's sum
    (ce_util's e_sum), its own exponential and quotient, where exponentials are kept by 2^-12 of it and 2^-31 of the row's, but not the largest, which is 1."""
    from paper_2011_05630_amd import loss
    announce(m, bias, dtype)
    t, v = TYPES[dtype], 500
    x, w, target, on = sure_rows(m, v, t, 26)
    b = torch.zeros(v) if bias else None
    ref = reference(x, w, b, target)
    assert float(ref["lse"].min()) > 4000 and float((1 - ref["p"].gather(1, target[:, None])).median()) < 2e-3
    far = ref["z"].max(1, keepdim=True).values - ref["z"]
    e_sum = (64 + v / 16 + 32 + 4 * (ref["p"] * far).sum(1)) * U
    kept = torch.where((far > 0) & (ref["p"] > 0), 2.0 ** -12 + 2.0 ** -31 / ref["p"], 0.0) if not bias else torch.zeros_like(far)
    own = dict(ref, e_lse=e_sum, ez=kept)
    op = loss.CrossEntropy(on["w"], None if b is None else b.cuda())
    for dloss in (1.0, (0.5 + torch.rand(m, generator=gen(27))).cuda()):
        each = torch.full((m,), dloss) if isinstance(dloss, float) else dloss.cpu()
        want = gradients(own, x, w, each.double(), torch.zeros(m).double(), t)
        _, dx, dw, db = op.gradients(on["x"], on["target"], dloss)
        within(dx, *want["dx"], "dx")
        within(dw, *want["dw"], "dw")
        if bias:
            within(db, *want["db"], "db")


@pytest.mark.parametrize("scale", [1e-20, 1e-6, 1.0, 3e4, 1e20])
def test_fp16_gradients_of_any_size(scale):
    """dz is scaled by a power of two on its way through fp16: what counts is whether the results fit the type."""
    from paper_2011_05630_amd import loss
    m = 130
    x, w, b, target, on = inputs(m, 40, 210, torch.float16, 19, bias=True)
    on["x"] = on["x"] * 2.0 ** -2
    x = on["x"].double().cpu()
    ref = reference(x, w, b, target)
    dloss = torch.full((m,), scale)
    op = loss.CrossEntropy(on["w"], on["b"])
    _, lse = op.run_saved(on["x"], on["target"])
    want = gradients(ref, x, w, dloss.double(), torch.zeros(m).double(), torch.float16)
    for dx, dw, db in (op.backward(dloss.cuda(), on["x"], on["target"], lse), op.gradients(on["x"], on["target"], dloss.cuda())[1:]):
        within(db, *want["db"], "db")
        for got, (value, bound) in ((dx, want["dx"]), (dw, want["dw"])):
            fits = value.abs() + bound < 65504
            g = got.double().cpu()
            assert ((g - value).abs() <= bound)[fits].all()
            assert (g[value.abs() - bound > 65520].isinf()).all()


@pytest.mark.parametrize("scale", [2.0 ** 20, 2.0 ** 40, 1e30])
@pytest.mark.parametrize("m", [130, 2100])
def test_bf16_gradients_of_any_size(m, scale):
    """Gradients of each row's own, far above 1, without the bias's: exponentials lost beside their part's largest, and classes that take no part, stay
    zeros."""
    from paper_2011_05630_amd import loss
    announce(m, scale)
    t, v = torch.bfloat16, 210
    x, w, b, target, on = inputs(m, 40, v, t, 24, bias=True, ignored=0.1, sure=60.0)
    off = torch.arange(v) % 5 == 3
    target = torch.where(off[target.clamp_min(0)] & (target >= 0), target + 1, target)
    dloss = (0.5 + torch.rand(m, generator=gen(25))) * scale
    for bias in (None, torch.where(off, float("-inf"), b).float()):
        ref = reference(x, w, None if bias is None else bias.double(), target)
        want = gradients(ref, x, w, dloss.double(), torch.zeros(m).double(), t, kept=True)
        op = loss.CrossEntropy(on["w"], None if bias is None else bias.cuda())
        got, dx, dw, _ = op.gradients(on["x"], target.cuda(), dloss.cuda(), need=("x", "weight"))
        within(got, ref["loss"], ref["e_loss"], "loss")
        within(dx, *want["dx"], "dx")
        within(dw, *want["dw"], "dw")


@pytest.mark.parametrize("m", [8, 130, 700])
@pytest.mark.parametrize("bias", [False, True])
def test_gradients_given_for_ignored_rows_scale_nothing(m, bias):
    """fp16: the power of two that dz is scaled by comes from what counts."""
    from paper_2011_05630_amd import loss
    announce(m, bias)
    t = torch.float16
    x, w, b, target, on = inputs(m, 40, 210, t, 28, bias=bias, ignored=0.3)
    target[m // 2] = IGNORE
    on["target"].copy_(target)
    ref = reference(x, w, b, target)
    dloss, dlse = given(m, 29)
    op = loss.CrossEntropy(on["w"], on["b"], piece_bytes=1)
    _, lse = op.run_saved(on["x"], on["target"])
    for away in (1e9, 1e30):
        away = torch.where(target == IGNORE, away, dloss)
        names = ("dx", "dw", "db")
        want = gradients(ref, x, w, dloss.double(), torch.zeros(m).double(), t, kept=not bias)
        for grads in (op.backward(away.cuda(), on["x"], on["target"], lse), op.gradients(on["x"], on["target"], away.cuda())[1:]):
            for name, value in zip(names, grads):
                if value is not None:
                    within(value, *want[name], name)
        want = gradients(ref, x, w, dloss.double(), dlse.double(), t)
        for name, value in zip(names, op.backward(away.cuda(), on["x"], on["target"], lse, dlse=dlse.cuda())):
            if value is not None:
                within(value, *want[name], name + " with dlse")
    # no row counts: dlse alone
    none = torch.full((m,), IGNORE)
    ref = reference(x, w, b, none)
    for e in (dlse, torch.full((1,), 0.125)):
        want = gradients(ref, x, w, torch.zeros(m).double(), e.double().expand(m), t)
        for d in (1e30, torch.full((m,), 1e30).cuda()):
            for name, value in zip(names, op.backward(d, on["x"], none.cuda(), lse, dlse=e.cuda())):
                if value is not None:
                    within(value, *want[name], name + " of dlse alone")


def test_differences():
    """The gradients against differences of the losses themselves: steps of 2^-6 that the type holds exactly.  A row's loss along such a step has a third derivative of at most R^3,
    R the range of the step's logits, which costs a difference R^3 / 6; each loss is off by its bound."""
    from paper_2011_05630_amd import loss
    m, k, v = 40, 16, 50
    g = gen(20)
    x = torch.randint(-32, 33, (m, k), generator=g).double() / 32
    w = torch.randint(-16, 17, (v, k), generator=g).double() / 32
    target = torch.randint(v, (m,), generator=g)
    b = torch.randn(v, generator=g)
    on = {n: a.half().cuda() for n, a in (("x", x), ("w", w))}
    op = loss.CrossEntropy(on["w"], b.cuda())
    weight = torch.rand(m, generator=g) + 0.5
    _, dx, dw, db = op.gradients(on["x"], target.cuda(), weight.cuda())
    want = gradients(reference(x, w, b.double(), target), x, w, weight.double(), torch.zeros(m).double(), torch.float16)

    def total(x_, w_, b_):
        o = loss.CrossEntropy(w_.half().cuda(), b_.float().cuda())
        e = reference(x_, w_, b_.float().double(), target)["e_loss"]
        return float((o.run(x_.half().cuda(), target.cuda()).double().cpu() * weight).sum()), float((e * weight).sum())

    h = 2.0 ** -6
    for n, (base, grad) in {"x": (x, dx), "w": (w, dw), "b": (b.double(), db)}.items():
        for trial in range(4):
            step = torch.randint(-1, 2, base.shape, generator=g).double()
            at = dict(x=x, w=w, b=b.double())
            up, e1 = total(**{q + "_": t + (h * step if q == n else 0) for q, t in at.items()})
            down, e2 = total(**{q + "_": t - (h * step if q == n else 0) for q, t in at.items()})
            z = {"x": step @ w.t() if n == "x" else None, "w": x @ step.t() if n == "w" else None, "b": step.expand(m, v) if n == "b" else None}[n] * h
            curve = float((weight * (z.max(1).values - z.min(1).values) ** 3).sum()) / 6
            bias_rounding = 2.0 ** -23 * float(b.abs().max()) * float(weight.sum()) if n == "b" else 0.0
            bound = (curve + (e1 + e2) / 2 + bias_rounding) / h + float((want["d" + n][1] * step.abs()).sum())
            assert abs((up - down) / (2 * h) - float((grad.double().cpu() * step).sum())) <= bound, (n, trial)


def test_equal_calls_give_equal_bits():
    from paper_2011_05630_amd import loss
    x, w, b, target, on = inputs(300, 200, 1500, torch.bfloat16, 21, bias=True, ignored=0.2)
    for bias in (None, on["b"]):
        op = loss.CrossEntropy(on["w"], bias, piece_bytes=1)
        first = op.gradients(on["x"], on["target"], 1.0)
        for _ in range(3):
            for a, c in zip(first, op.gradients(on["x"], on["target"], 1.0)):
                assert a is c or torch.equal(a, c)


def test_no_rows():
    from paper_2011_05630_amd import loss
    x, w, b, target, on = inputs(4, 64, 100, torch.bfloat16, 22, bias=True)
    op = loss.CrossEntropy(on["w"], on["b"])
    xs, ts = on["x"][:0], on["target"][:0]
    got, lse = op.run_saved(xs, ts)
    assert got.shape == lse.shape == (0,)
    for grads in (op.backward(1.0, xs, ts, lse), op.gradients(xs, ts, 1.0)[1:]):
        assert grads[0].shape == (0, 64)
        assert grads[1].shape == (100, 64) and (grads[1] == 0).all() and (grads[2] == 0).all()
    db = op.backward(1.0, xs, ts, lse, need="bias")[2]
    assert (db == 0).all()


def test_what_lies_around_the_operands_is_not_touched():
    """Gaps between rows, the weight's and the inputs' surroundings are NaN in rows_of; here they are looked at after the calls."""
    from paper_2011_05630_amd import loss
    for dtype in sorted(TYPES):
        x, w, b, target, on = inputs(70, 41, 133, TYPES[dtype], 23, gap=7, offset=3, bias=True, ignored=0.2)
        whole = [torch.empty(0, dtype=on[n].dtype, device="cuda").set_(on[n].untyped_storage()).clone() for n in ("x", "w")]
        op = loss.CrossEntropy(on["w"], on["b"], piece_bytes=1)
        op.gradients(on["x"], on["target"], 1.0)
        for n, before in zip(("x", "w"), whole):
            now = torch.empty(0, dtype=on[n].dtype, device="cuda").set_(on[n].untyped_storage())
            assert torch.equal(now.view(torch.int16), before.view(torch.int16))


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("m", [6, 300])
def test_a_captured_call_follows_its_inputs(m, bias):
    from paper_2011_05630_amd import loss
    t = torch.float16
    sets = [inputs(m, 72, 333, t, 30 + i, bias=True, ignored=0.2)[4] for i in range(3)]
    x, w, b, target = (sets[0][n].clone() for n in ("x", "w", "b", "target"))
    op = loss.CrossEntropy(w, b if bias else None, piece_bytes=1)
    dloss = torch.full((), 1.0).cuda()
    op.gradients(x, target, dloss)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        op.gradients(x, target, dloss)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = op.gradients(x, target, dloss)
        again, lse = op.run_saved(x, target)
        back = op.backward(dloss, x, target, lse)
    for i in (1, 2, 0, 2):
        for a, n in ((x, "x"), (w, "w"), (b, "b"), (target, "target")):
            a.copy_(sets[i][n])
        dloss.fill_(0.5 + i)
        graph.replay()
        torch.cuda.synchronize()
        want = op.gradients(x, target, dloss)
        loss2, lse2 = op.run_saved(x, target)
        for a, c in zip(tuple(out) + (again, lse) + tuple(back), tuple(want) + (loss2, lse2) + tuple(op.backward(dloss, x, target, lse2))):
            assert a is c or torch.equal(a, c)


def test_other_streams():
    """Two calls of one object on two streams at once: workspaces of their own."""
    from paper_2011_05630_amd import loss
    a, c = (inputs(400, 256, 2000, torch.bfloat16, s)[4] for s in (40, 41))
    op = loss.CrossEntropy(a["w"])
    want = [op.gradients(q["x"], q["target"], 1.0) for q in (a, c)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        got = []
        for s, q in zip(streams, (a, c)):
            with torch.cuda.stream(s):
                got.append(op.gradients(q["x"], q["target"], 1.0))
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            for u, v in zip(g, w):
                assert u is v or torch.equal(u, v)


def test_inside_a_function_of_automatic_differentiation():
    from paper_2011_05630_amd import loss

    class Loss(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w, target):
            op = loss.CrossEntropy(w.detach())
            value, lse = op.run_saved(x, target)
            ctx.save_for_backward(x, w, target, lse)
            return value, lse

        @staticmethod
        def backward(ctx, dloss, dlse):
            x, w, target, lse = ctx.saved_tensors
            dx, dw, _ = loss.CrossEntropy(w.detach()).backward(dloss, x.detach(), target, lse, dlse=dlse)
            return dx, dw, None

    x, w, b, target, on = inputs(90, 64, 200, torch.bfloat16, 50, ignored=0.1)
    xs, ws = on["x"].clone().requires_grad_(), on["w"].clone().requires_grad_()
    value, lse = Loss.apply(xs, ws, on["target"])
    (value.sum() + 0.1 * lse.sum()).backward()              # (gradients expanded from one element)
    want = gradients(reference(x, w, b, target), x, w, torch.ones(90).double(), torch.full((90,), 0.1).float().double(), torch.bfloat16)
    within(xs.grad, *want["dx"], "dx")
    within(ws.grad, *want["dw"], "dw")
