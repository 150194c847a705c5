"""Calls of the feed-forward operators beyond the usual ones: some of the gradients, rows far apart, the C calls themselves.  Whole numbers, bit for bit."""
import itertools

import pytest
import torch

from ff_util import TYPES, act, rows_of, same, slope, whole
from gpu_util import announce

pytestmark = pytest.mark.gpu

T = torch.bfloat16
SUBSETS = [s for n in (1, 2, 3) for s in itertools.combinations(("x", "weight", "bias"), n)]


def F():
    from paper_2011_05630_amd import feedforward
    return feedforward


@pytest.fixture
def force():
    from paper_2011_05630_amd import binding as B
    yield B.dlf_debug_ff_kernel
    B.dlf_debug_ff_kernel(0)


def few_values(m, k, seed):
    """Whole numbers, few of them not zero: sums of products of products stay whole numbers of the type."""
    x = whole(m, k, seed, 1)
    return x * (torch.rand(m, k, generator=torch.Generator().manual_seed(7)) < min(1.0, 32.0 / k)).double()


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("kernel", [(0, 0), (2, 3), (3, 5), (4, 3), (5, 4), (6, 3)], ids=str)
@pytest.mark.parametrize("size", [(300, 264, 520), (259, 1031, 517), (1288, 136, 776), (40, 24, 4104)], ids=str)
@pytest.mark.parametrize("layouts", [((0, 0), (0, 0)), ((3, 0), (0, 0)), ((0, 0), (5, 1))], ids=str)
def test_some_of_the_gradients(layouts, size, kernel, gated, force):
    """Their layout in the workspace and their cuts differ; so does the number of launches where only one of x and the weights lies in lines."""
    m, k, n = size
    announce("subsets", size, kernel, gated, layouts)
    force(*kernel)
    x, wg, wu, dh = few_values(m, k, 1), whole(n, k, 2, 1), whole(n, k, 3, 1), whole(m, n, 4, 1)
    xd, gd, ud, dd = rows_of(x, T, *layouts[0]), rows_of(wg, T, *layouts[1]), rows_of(wu, T, *layouts[1]), rows_of(dh, T)
    zero = torch.zeros(n, device="cuda")
    g, u = x @ wg.t(), x @ wu.t()
    if gated:
        op = F().GatedLinear(gd, ud, zero, zero, "relu")
        dz = [dh * u * slope("relu", g), dh * act("relu", g)]
        want = [dz[0] @ wg + dz[1] @ wu, dz[0].t() @ x, dz[1].t() @ x, dz[0].sum(0), dz[1].sum(0)]
    else:
        op = F().Linear(gd, zero, "relu")
        dz = dh * slope("relu", g)
        want = [dz @ wg, dz.t() @ x, dz.sum(0)]
    part = ["x", "weight", "weight", "bias", "bias"] if gated else ["x", "weight", "bias"]
    _, saved = op.run_saved(xd)
    for need in SUBSETS:
        for got, w, p in zip(op.backward(dd, xd, saved, need=need), want, part):
            if p in need:
                same(got, w, "%s of %s" % (p, need))
            else:
                assert got is None


def far_rows(values, t, stride):
    """The rows `stride` elements apart."""
    m, n = values.shape
    v = torch.empty((m - 1) * stride + n, dtype=t, device="cuda").as_strided((m, n), (stride, 1))
    v.copy_(values.to(t))
    return v


@pytest.mark.parametrize("m", [20, 140])
@pytest.mark.parametrize("stride", [(1 << 22) - 8, 1 << 22, (1 << 24) - 8, (1 << 24) - 1])
def test_rows_far_apart(stride, m):
    """Up to the largest distance that is accepted: 32-bit offsets within a tile, 64-bit ones between tiles."""
    announce("rows far apart", stride, m)
    k, n = 72, 136
    x, w, r, dy = whole(m, k, 1), whole(n, k, 2), whole(m, n, 3, 9), whole(m, n, 4)
    dz = dy * slope("relu", x @ w.t())
    for which in ("x", "w", "residual", "out", "dy"):
        place = lambda v, name: far_rows(v, T, stride) if name == which else rows_of(v, T)
        xd, wd, rd, dd = place(x, "x"), place(w, "w"), place(r, "residual"), place(dy, "dy")
        op = F().Linear(wd, act="relu")
        y, saved = op.run_saved(xd, rd, place(torch.zeros(m, n), "out"))
        same(y, act("relu", x @ w.t()) + r, "y, %s far" % which)
        dx, dw, _ = op.backward(dd, xd, saved)
        same(dx, dz @ w, "dx, %s far" % which)
        same(dw, dz.t() @ x, "dw, %s far" % which)
        del xd, wd, rd, dd, op, y, saved
    torch.cuda.empty_cache()


def test_rows_farther_apart_are_refused():
    from paper_2011_05630_amd.binding import DlfError
    op = F().Linear(rows_of(whole(8, 16, 1), T))
    buf = torch.empty((1 << 24) + 16, dtype=T, device="cuda")
    with pytest.raises(DlfError, match="apart"):
        op.run(buf.as_strided((2, 16), (1 << 24, 1)))


@pytest.mark.parametrize("t", sorted(TYPES))
@pytest.mark.parametrize("size", [(7, 72, 40), (300, 264, 517)], ids=str)
def test_the_c_calls(size, t):
    """Through the ctypes binding, on the default stream, with workspaces of exactly the size asked for; gradients one by one."""
    from paper_2011_05630_amd import binding as B
    m, k, n = size
    announce("C calls", size, t)
    ty = TYPES[t]
    x, wg, wu, dh, bg, bu = few_values(m, k, 1), whole(n, k, 2, 1), whole(n, k, 3, 1), whole(m, n, 4, 1), whole(1, n, 5, 1)[0], whole(1, n, 6, 1)[0]
    xd, gd, ud, dd, bgd, bud = rows_of(x, ty, 8), rows_of(wg, ty), rows_of(wu, ty), rows_of(dh, ty, 3), bg.float().cuda(), bu.float().cuda()
    d = B.dlf_ff_desc(t, "relu", m, k, n, x_stride=k + 8, y_stride=n + 2, dy_stride=n + 3, res_stride=n + 3)
    keep = []

    def ws(f):
        need = f(d)
        keep.append(torch.full((need + 256,), 0xA5, dtype=torch.uint8, device="cuda"))
        return keep[-1].data_ptr(), need

    def untouched():
        for w in keep:
            assert (w[-256:] == 0xA5).all()

    y = rows_of(torch.zeros(m, n), ty, 2)
    z = x @ wg.t() + bg
    saved = torch.empty(m, n, device="cuda")
    torch.cuda.synchronize()
    B.dlf_linear(d, xd.data_ptr(), gd.data_ptr(), bgd.data_ptr(), dd.data_ptr(), y.data_ptr(), saved.data_ptr(), *ws(B.dlf_linear_workspace_bytes))
    torch.cuda.synchronize()
    same(y, act("relu", z) + dh, "y")
    same(saved, z, "saved")
    dz = dh * slope("relu", z)
    want = [dz @ wg, dz.t() @ x, dz.sum(0)]
    for some in itertools.product((0, 1), repeat=3):
        got = [torch.full((m, k), 7, dtype=ty, device="cuda"), torch.full((n, k), 7, dtype=ty, device="cuda"), torch.full((n,), 7.0, device="cuda")]
        torch.cuda.synchronize()
        B.dlf_linear_backward(d, dd.data_ptr(), xd.data_ptr(), gd.data_ptr(), saved.data_ptr(), *(g.data_ptr() if s else None for g, s in zip(got, some)),
                              *ws(B.dlf_linear_backward_workspace_bytes))
        torch.cuda.synchronize()
        for g, w, s in zip(got, want, some):
            if s:
                same(g, w, "gradient")
            else:
                assert (g == 7).all()
    g, u = z, x @ wu.t() + bu
    h = rows_of(torch.zeros(m, n), ty, 2)
    saved = torch.empty(2, m, n, device="cuda")
    torch.cuda.synchronize()
    B.dlf_gated(d, xd.data_ptr(), gd.data_ptr(), ud.data_ptr(), bgd.data_ptr(), bud.data_ptr(), h.data_ptr(), saved.data_ptr(), *ws(B.dlf_gated_workspace_bytes))
    torch.cuda.synchronize()
    same(h, act("relu", g) * u, "h")
    same(saved, torch.stack((g, u)), "saved")
    dg, du = dh * u * slope("relu", g), dh * act("relu", g)
    assert max(dg.abs().max(), du.abs().max()) <= 256
    want = [dg @ wg + du @ wu, dg.t() @ x, du.t() @ x, dg.sum(0), du.sum(0)]
    for some in itertools.product((0, 1), repeat=5):
        got = [torch.full(s, 7, dtype=q, device="cuda") for s, q in (((m, k), ty), ((n, k), ty), ((n, k), ty), ((n,), torch.float32), ((n,), torch.float32))]
        torch.cuda.synchronize()
        B.dlf_gated_backward(d, dd.data_ptr(), xd.data_ptr(), gd.data_ptr(), ud.data_ptr(), saved.data_ptr(),
                             *(v.data_ptr() if s else None for v, s in zip(got, some)), *ws(B.dlf_gated_backward_workspace_bytes))
        torch.cuda.synchronize()
        for v, w, s in zip(got, want, some):
            if s:
                same(v, w, "gradient")
            else:
                assert (v == 7).all()
    untouched()
