"""The feed-forward operators against the plain ones in 64 bits: bit for bit on whole numbers over sizes, strides, alignments and types,
within derived bounds with smooth activations (ff_util); gradients also against differences."""
import pytest
import torch

from ff_util import (CURVE, E_ACT, SLOPE, TYPES, U, act, half_eps, normal, rows_of, same, slope, whole, within)
from gpu_util import announce

pytestmark = pytest.mark.gpu

# (rows, in, out): one of everything, one token, sizes around every multiple of a tile, odd ones, long sums
SIZES = [(1, 1, 1), (1, 8, 8), (1, 1000, 65), (1, 1024, 1024), (2, 7, 3), (3, 4097, 17), (8, 64, 640), (15, 520, 130), (16, 2048, 48), (17, 96, 257),
         (31, 72, 128), (33, 1003, 64), (64, 64, 64), (65, 63, 66), (100, 2056, 200), (128, 128, 128), (129, 264, 255), (250, 512, 384),
         (256, 64, 256), (257, 72, 264), (300, 1024, 776), (513, 520, 520), (1025, 136, 1032), (40, 24, 4104)]
# (gap between rows, offset of the first): aligned, 16-byte rows in wider ones, rows that start anywhere
LAYOUTS = [(0, 0), (8, 0), (24, 8), (3, 0), (0, 1), (5, 3)]


def F():
    from paper_2011_05630_amd import feedforward
    return feedforward


def layout(i):
    return LAYOUTS[i % len(LAYOUTS)]


def f32(v):
    return v.float().cuda()


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("t", sorted(TYPES))
def test_linear_whole_numbers(size, t):
    m, k, n = size
    i = SIZES.index(size)
    for j, (a, has_bias, has_res) in enumerate((("none", False, False), ("relu", True, True), ("relu6", True, False), ("none", False, True))):
        if j and i % 3 != j % 3 and m * k * n > 1 << 20:
            continue
        announce("linear", t, size, a, layout(i + j))
        x, w, b, r = whole(m, k, 1), whole(n, k, 2), whole(1, n, 3, 9)[0], whole(m, n, 4, 9)
        xd, wd, rd = (rows_of(v, TYPES[t], *layout(i + q)) for v, q in ((x, j), (w, j // 2), (r, j + 1)))
        op = F().Linear(wd, f32(b) if has_bias else None, a)
        out = rows_of(torch.zeros(m, n), TYPES[t], *layout(j)) if j % 2 else None
        z = x @ w.t() + (b if has_bias else 0)
        want = act(a, z) + (r if has_res else 0)
        y = op.run(xd, rd if has_res else None, out)
        same(y, want, "y")
        y, saved = op.run_saved(xd, rd if has_res else None)
        same(y, want, "y")
        if a == "none":
            assert saved is None
        else:
            same(saved, z, "saved")
        if out is not None and layout(j)[0]:            # nothing is written between the rows
            gap = out.as_strided((m, layout(j)[0]), (out.stride(0), 1), out.storage_offset() + n)
            assert gap.isnan().all()


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("t", sorted(TYPES))
def test_gated_whole_numbers(size, t):
    m, k, n = size
    i = SIZES.index(size)
    for j, (a, has_bias) in enumerate((("none", True), ("relu", False))):
        announce("gated", t, size, a, layout(i + j))
        x, wg, wu, bg, bu = whole(m, k, 1, 1), whole(n, k, 2, 1), whole(n, k, 3, 1), whole(1, n, 4, 9)[0], whole(1, n, 5, 9)[0]
        xd, gd, ud = (rows_of(v, TYPES[t], *layout(i + q)) for v, q in ((x, j), (wg, j + 1), (wu, j + 1)))
        op = F().GatedLinear(gd, ud, f32(bg) if has_bias else None, f32(bu) if has_bias else None, a)
        g, u = x @ wg.t() + (bg if has_bias else 0), x @ wu.t() + (bu if has_bias else 0)
        same(op.run(xd), act(a, g) * u, "h")
        h, saved = op.run_saved(xd)
        same(h, act(a, g) * u, "h")
        same(saved, torch.stack((g, u)), "saved")


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("t", sorted(TYPES))
def test_linear_backward_whole_numbers(size, t):
    m, k, n = size
    i = SIZES.index(size)
    for j, (a, has_bias) in enumerate((("none", True), ("relu", True))):
        announce("linear backward", t, size, a, layout(i + j))
        x, w, b, dy = whole(m, k, 1), whole(n, k, 2), whole(1, n, 3, 9)[0], whole(m, n, 4)
        xd, wd, dd = (rows_of(v, TYPES[t], *layout(i + q)) for v, q in ((x, j), (w, j + 1), (dy, j + 2)))
        op = F().Linear(wd, f32(b) if has_bias else None, a)
        _, saved = op.run_saved(xd)
        dz = dy * slope(a, x @ w.t() + b)
        dx, dw, db = op.backward(dd, xd, saved)
        same(dx, dz @ w, "dx")
        same(dw, dz.t() @ x, "dw")
        same(db, dz.sum(0), "db")


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("t", sorted(TYPES))
def test_gated_backward_whole_numbers(size, t):
    m, k, n = size
    i = SIZES.index(size)
    for j, a in enumerate(("none", "relu")):
        announce("gated backward", t, size, a, layout(i + j))
        # few values differ from zero, so that dg and du stay whole numbers of the type and every sum below 2^24
        x, wg, wu, dh = whole(m, k, 1, 1), whole(n, k, 2, 1), whole(n, k, 3, 1), whole(m, n, 4, 1)
        x *= (torch.rand(m, k, generator=torch.Generator().manual_seed(7)) < min(1.0, 32.0 / k)).double()
        xd, gd, ud, dd = (rows_of(v, TYPES[t], *layout(i + q)) for v, q in ((x, j), (wg, j + 1), (wu, j + 1), (dh, j + 2)))
        zero = torch.zeros(n)
        op = F().GatedLinear(gd, ud, f32(zero), f32(zero), a)
        _, saved = op.run_saved(xd)
        g, u = x @ wg.t(), x @ wu.t()
        dg, du = dh * u * slope(a, g), dh * act(a, g)
        assert dg.abs().max() <= 256 and du.abs().max() <= 256
        dx, dwg, dwu, dbg, dbu = op.backward(dd, xd, saved)
        same(dx, dg @ wg + du @ wu, "dx")
        same(dwg, dg.t() @ x, "dw_gate")
        same(dwu, du.t() @ x, "dw_up")
        same(dbg, dg.sum(0), "db_gate")
        same(dbu, du.sum(0), "db_up")


SMOOTH = ("gelu", "gelu_tanh", "silu", "sigmoid")


def sum_err(k, terms):
    return (k + 2) * U * terms


@pytest.mark.parametrize("a", SMOOTH)
@pytest.mark.parametrize("t", sorted(TYPES))
@pytest.mark.parametrize("size", [(1, 256, 96), (7, 1000, 136), (70, 300, 257), (384, 512, 640)], ids=str)
def test_linear_smooth(size, t, a):
    m, k, n = size
    announce("linear", t, size, a)
    ty, he = TYPES[t], half_eps(TYPES[t])
    x, w, b, dy = normal(m, k, 1, ty), normal(n, k, 2, ty, 2 * k ** -0.5), normal(1, n, 3, torch.float32)[0], normal(m, n, 4, ty)
    op = F().Linear(rows_of(w, ty), f32(b), a)
    z = x @ w.t() + b
    ez = sum_err(k, x.abs() @ w.abs().t() + b.abs())
    xd = rows_of(x, ty)
    y, saved = op.run_saved(xd)
    within(saved, z, ez, "saved")
    ya = act(a, z)
    ey = SLOPE * ez + E_ACT * (z.abs() + 1)
    within(y, ya, ey + he * (ya.abs() + ey) + torch.finfo(ty).smallest_normal, "y")
    dx, dw, db = op.backward(rows_of(dy, ty), xd, saved)
    d = slope(a, z)
    dz = dy * d
    ed = dy.abs() * (CURVE * ez + E_ACT * (z.abs() + 1) ** 2)       # of dz in 32 bits
    within(db, dz.sum(0), ed.sum(0) + sum_err(m, (dz.abs() + ed).sum(0)), "db")
    tiny = torch.finfo(ty).smallest_normal
    ed = ed + he * (dz.abs() + ed) + tiny
    for got, want, terms, err, q in ((dx, dz @ w, (dz.abs() + ed) @ w.abs(), ed @ w.abs(), n), (dw, dz.t() @ x, (dz.abs() + ed).t() @ x.abs(), ed.t() @ x.abs(), m)):
        e = err + sum_err(q, terms)
        within(got, want, e + he * (want.abs() + e) + tiny, "gradient")


@pytest.mark.parametrize("a", SMOOTH)
@pytest.mark.parametrize("t", sorted(TYPES))
@pytest.mark.parametrize("size", [(1, 256, 96), (7, 1000, 136), (70, 300, 257), (384, 512, 640)], ids=str)
def test_gated_smooth(size, t, a):
    m, k, n = size
    announce("gated", t, size, a)
    ty, he, tiny = TYPES[t], half_eps(TYPES[t]), torch.finfo(TYPES[t]).smallest_normal
    x, wg, wu, dh = normal(m, k, 1, ty), normal(n, k, 2, ty, 2 * k ** -0.5), normal(n, k, 3, ty, k ** -0.5), normal(m, n, 4, ty)
    bg, bu = normal(1, n, 5, torch.float32)[0], normal(1, n, 6, torch.float32)[0]
    op = F().GatedLinear(rows_of(wg, ty), rows_of(wu, ty), f32(bg), f32(bu), a)
    g, u = x @ wg.t() + bg, x @ wu.t() + bu
    eg, eu = sum_err(k, x.abs() @ wg.abs().t() + bg.abs()), sum_err(k, x.abs() @ wu.abs().t() + bu.abs())
    xd = rows_of(x, ty)
    h, saved = op.run_saved(xd)
    within(saved, torch.stack((g, u)), torch.stack((eg, eu)), "saved")
    ag, dga = act(a, g), slope(a, g)
    ea = SLOPE * eg + E_ACT * (g.abs() + 1)
    eh = ea * (u.abs() + eu) + ag.abs() * eu + U * (ag * u).abs()
    within(h, ag * u, eh + he * ((ag * u).abs() + eh) + tiny, "h")
    dx, dwg, dwu, dbg, dbu = op.backward(rows_of(dh, ty), xd, saved)
    dg, du = dh * u * dga, dh * ag
    es = CURVE * eg + E_ACT * (g.abs() + 1) ** 2
    edg = dh.abs() * (es * (u.abs() + eu) + dga.abs() * eu) + 2 * U * dg.abs()
    edu = dh.abs() * ea + U * du.abs()
    for got, d, e in ((dbg, dg, edg), (dbu, du, edu)):
        within(got, d.sum(0), e.sum(0) + sum_err(m, (d.abs() + e).sum(0)), "db")
    edg, edu = edg + he * (dg.abs() + edg) + tiny, edu + he * (du.abs() + edu) + tiny
    checks = [(dx, dg @ wg + du @ wu, (dg.abs() + edg) @ wg.abs() + (du.abs() + edu) @ wu.abs(), edg @ wg.abs() + edu @ wu.abs(), 2 * n)]
    checks += [(got, d.t() @ x, (d.abs() + e).t() @ x.abs(), e.t() @ x.abs(), m) for got, d, e in ((dwg, dg, edg), (dwu, du, edu))]
    for got, want, terms, err, q in checks:
        e = err + sum_err(q, terms)
        within(got, want, e + he * (want.abs() + e) + tiny, "gradient")


@pytest.mark.parametrize("t", sorted(TYPES))
def test_gradients_against_differences(t):
    """The operators without an activation are linear in x and in every weight: a difference of any size is the gradient's, exactly on
    whole numbers.  With one, the central difference of the forward call is off by its step's square and the outputs' roundings."""
    ty = TYPES[t]
    m, k, n = 19, 40, 35
    x, w, dy, ex, ew = whole(m, k, 1), whole(n, k, 2), whole(m, n, 3, 1), whole(m, k, 4, 1), whole(n, k, 5, 1)
    op = F().Linear(rows_of(w, ty))
    dx, dw, _ = op.backward(rows_of(dy, ty), rows_of(x, ty), None)
    y0 = op.run(rows_of(x, ty)).double().cpu()
    assert float((dy * (op.run(rows_of(x + ex, ty)).double().cpu() - y0)).sum()) == float((dx.double().cpu() * ex).sum())
    y1 = F().Linear(rows_of(w + ew, ty)).run(rows_of(x, ty)).double().cpu()
    assert float((dy * (y1 - y0)).sum()) == float((dw.double().cpu() * ew).sum())
    # gated, SiLU: along one direction of x.  The step is a power of two that both points hold exactly.
    x, wg, wu = whole(m, k, 6, 1) / 4, whole(n, k, 7, 1) / 4, whole(n, k, 8, 1) / 4
    op = F().GatedLinear(rows_of(wg, ty), rows_of(wu, ty), act="silu")
    h, saved = op.run_saved(rows_of(x, ty))
    dx = op.backward(rows_of(dy, ty), rows_of(x, ty), saved)[0].double().cpu()
    step = 2.0 ** -3
    hp, hm = (op.run(rows_of(x + s * step * ex, ty)).double().cpu() for s in (1, -1))
    diff = float((dy * (hp - hm)).sum()) / (2 * step)
    # third derivative along the direction: h = s(g) u with g' = wg ex, u' = wu ex, |s''| <= 1/2, |s'''| <= 1
    gp, up, um = (ex @ wg.t()).abs(), (ex @ wu.t()).abs(), (x @ wu.t()).abs() + step * (ex @ wu.t()).abs()
    third = gp ** 3 * um + 1.5 * gp ** 2 * up
    bound = float((dy.abs() * (third * step ** 2 / 6 + half_eps(ty) * (hp.abs() + hm.abs()) / (2 * step))).sum())
    # ... and dx: one rounding of its own, one of dg and du on the way
    g, u = x @ wg.t(), x @ wu.t()
    mid = ((dy * u * slope("silu", g)).abs() @ wg.abs() + (dy * act("silu", g)).abs() @ wu.abs())
    bound += float((ex.abs() * half_eps(ty) * 1.1 * (dx.abs() + mid)).sum())
    assert abs(diff - float((dx * ex).sum())) <= bound, (diff, float((dx * ex).sum()), bound)


def test_values_out_of_the_ordinary():
    """Infinities and NaN stay in their row (forward) and do not reach others; activations at large arguments."""
    t = torch.bfloat16
    for m in (3, 70, 300):
        for gated in (False, True):
            x, w = whole(m, 72, 1), whole(130, 72, 2)
            x[1, 5], x[2, 7] = float("nan"), float("inf")
            xd, wd = rows_of(x, t), rows_of(w, t)
            y = (F().GatedLinear(wd, wd, act="none") if gated else F().Linear(wd)).run(xd)
            z = x @ w.t()
            same(y, z * z if gated else z, "y")
    z = torch.tensor([[0.0, -0.0, 1e-30, -1e-30, 20, -20, 88, -88, 104, -104, 1e4, -1e4, 1e19, -1e19, 3e38, -3e38, float("inf"), float("nan")]]).double()
    x = rows_of(z.t().contiguous(), t)                 # one feature: the pre-activation is x itself
    zx = x.double().cpu()
    for a in ("relu", "relu6", "gelu", "gelu_tanh", "silu", "sigmoid"):
        op = F().Linear(torch.ones(1, 1, dtype=t, device="cuda"), act=a)
        y, saved = op.run_saved(x)
        want = act(a, zx)
        want = torch.where(zx == float("inf"), torch.tensor(6.0 if a == "relu6" else 1.0 if a == "sigmoid" else float("inf")).double(), want)
        want[-1] = float("nan")
        got = y.double().cpu()
        assert got[-1].isnan()
        assert (got[-2] == want[-2]).all(), (a, got[-2], want[-2])
        within(got[:-2], want[:-2], half_eps(t) * 1.01 * want[:-2].abs() + E_ACT * 1e-3 + torch.finfo(t).smallest_normal, a)
        dx = op.backward(torch.ones(18, 1, dtype=t, device="cuda"), x, saved)[0].double().cpu()
        within(dx[:-2], torch.nan_to_num(slope(a, zx[:-2].clamp(-1e4, 1e4))), torch.full((16, 1), 2.0 ** -8 * 1.2).double(), a + " slope")
        assert dx[-1].isnan()


def test_no_rows():
    t = torch.bfloat16
    w = rows_of(whole(20, 24, 1), t)
    x = torch.empty(0, 24, dtype=t, device="cuda")
    b = torch.zeros(20, device="cuda")
    for a in ("none", "silu"):
        op = F().Linear(w, b, a)
        y, saved = op.run_saved(x)
        assert y.shape == (0, 20)
        dx, dw, db = op.backward(y, x, saved)
        assert dx.shape == (0, 24) and not dw.any() and not db.any()
    op = F().GatedLinear(w, w, b, b)
    h, saved = op.run_saved(x)
    assert h.shape == (0, 20)
    g = op.backward(h, x, saved)
    assert g[0].shape == (0, 24) and not any(v.any() for v in g[1:])


def test_leading_dimensions_and_what_is_left_out():
    t = torch.float16
    x, w, dy = whole(30, 40, 1), whole(24, 40, 2), whole(30, 24, 3)
    xd, wd, dd = rows_of(x, t).view(2, 3, 5, 40), rows_of(w, t), rows_of(dy, t).view(2, 3, 5, 24)
    op = F().Linear(wd, torch.zeros(24, device="cuda"))
    same(op.run(xd).view(30, 24), x @ w.t(), "y")
    same(op.run(xd[0, 0, 1]).view(1, 24), x[1:2] @ w.t(), "one row")
    dx, dw, db = op.backward(dd, xd, None, need=("weight",))
    assert dx is None and db is None
    same(dw, dy.t() @ x, "dw")
    dx, dw, db = op.backward(dd, xd, None, need=("x", "bias"))
    assert dw is None and dx.shape == xd.shape
    same(db, dy.sum(0), "db")
    with pytest.raises(ValueError):
        op.run(xd.transpose(0, 1))
    with pytest.raises(ValueError):
        op.run(rows_of(x, t).t().contiguous().t())
    with pytest.raises(ValueError):
        op.run(rows_of(x, torch.bfloat16))
    with pytest.raises(ValueError):
        op.run(xd, residual=dd[:1])
    with pytest.raises(ValueError):
        op.run(rows_of(x[:1], t).expand(4, 40))
    with pytest.raises(ValueError):
        F().Linear(wd, act="tanh")
    with pytest.raises(ValueError):
        F().Linear(wd, torch.zeros(24, dtype=t, device="cuda"))
    with pytest.raises(ValueError):
        F().GatedLinear(wd, rows_of(w, t, 8))
    g = F().GatedLinear(wd, wd, act="none")
    _, saved = g.run_saved(xd)
    out = g.backward(dd, xd, saved, need=("x",))
    assert out[1:] == (None, None, None, None)
    with pytest.raises(ValueError):
        g.backward(dd, xd, saved[:1])


@pytest.mark.parametrize("m", [1, 16, 200, 700])
def test_block_and_residual_in_place(m):
    """The block, its output written over its input, which is the residual."""
    t = torch.bfloat16
    d, f = 136, 264
    x, wg, wu, wd = whole(m, d, 1, 1), whole(f, d, 2, 1), whole(f, d, 3, 1), whole(d, f, 4, 1)
    x *= (torch.rand(m, d, generator=torch.Generator().manual_seed(7)) < 0.1).double()
    block = F().FeedForward(F().GatedLinear(rows_of(wg, t), rows_of(wu, t), act="relu"), F().Linear(rows_of(wd, t)))
    h = act("relu", x @ wg.t()) * (x @ wu.t())
    assert h.abs().max() <= 256                       # whole numbers that bf16 holds
    want = h @ wd.t() + x
    xd = rows_of(x, t)
    same(block.run(xd, residual=xd), want, "y")
    y, saved = block.run_saved(xd, residual=xd)
    same(y, want, "y")
    dy = whole(m, d, 5, 1)
    dx, dgate, ddown = block.backward(rows_of(dy, t), xd, saved)
    dh = (dy @ wd).to(t).double()
    same(ddown[0], dy.t() @ h, "dw_down")
    g, u = x @ wg.t(), x @ wu.t()
    dg, du = (dh * u * slope("relu", g)).to(t).double(), (dh * act("relu", g)).to(t).double()
    same(dx, dg @ wg + du @ wu, "dx")
    same(dgate[0], dg.t() @ x, "dw_gate")
    same(dgate[1], du.t() @ x, "dw_up")
    same(block.run(xd, residual=xd, out=xd), want, "in place")
    same(xd, want, "in place")


@pytest.mark.parametrize("m,k,n", [(1, 512, 256), (48, 520, 264), (600, 1024, 512)])
def test_captured_into_a_graph(m, k, n):
    """Forward and backward calls in a graph: every replay, on inputs changed in place, equals the eager calls; calls on another stream too."""
    t = torch.bfloat16
    op = F().GatedLinear(rows_of(normal(n, k, 1, t, k ** -0.5), t), rows_of(normal(n, k, 2, t, k ** -0.5), t),
                         torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"))
    lin = F().Linear(rows_of(normal(k, n, 3, t, n ** -0.5), t), act="gelu")
    x, dy = rows_of(normal(m, k, 4, t), t), rows_of(normal(m, k, 5, t), t)

    def step():
        h, saved = op.run_saved(x)
        y, saved2 = lin.run_saved(h, residual=x)
        dh, dw, _ = lin.backward(dy, h, saved2)
        return (y, dw) + op.backward(dh, x, saved)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        first = step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        static = step()
    for k2 in range(4):
        if k2:
            x.copy_(normal(m, k, 10 + k2, t))
        eager = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(static, eager):
            assert torch.equal(a, b)
        if k2 == 0:
            for a, b in zip(first, eager):
                assert torch.equal(a, b)
