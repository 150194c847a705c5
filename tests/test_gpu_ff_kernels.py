"""Every kernel that the feed-forward operators' products may run on, forced, against the plain operators in 64 bits: bit for bit on
whole numbers, at sizes around the kernels' tiles and at sums of every length modulo their steps."""
import pytest
import torch

from ff_util import TYPES, act, rows_of, same, slope, whole
from gpu_util import announce

pytestmark = pytest.mark.gpu

# (kernel, workgroups that share a tile's k)
KERNELS = {"few": (1, 0), "tile256": (2, 1), "tile256_split3": (2, 3), "tile128": (3, 1), "tile128_split5": (3, 5), "any": (4, 1), "any_split2": (4, 2), "deep": (5, 1), "deep_split4": (5, 4), "any64": (6, 1), "any64_split3": (6, 3),
           "any64_gated": (7, 1), "any64_gated_split3": (7, 3)}
# (rows, in, out)
SIZES = [(8, 8, 8), (64, 72, 40), (128, 64, 128), (136, 72, 120), (256, 128, 256), (264, 192, 264), (504, 840, 520), (1288, 64, 776), (700, 1032, 1304),
         (1, 5, 1), (131, 77, 67), (259, 1031, 517)]


@pytest.fixture
def force():
    from paper_2011_05630_amd import binding as B
    yield B.dlf_debug_ff_kernel
    B.dlf_debug_ff_kernel(0)


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("t", sorted(TYPES))
@pytest.mark.parametrize("kernel", sorted(KERNELS))
def test_linear(kernel, t, size, force):
    from paper_2011_05630_amd import feedforward as F
    announce("linear", kernel, t, size)
    force(*KERNELS[kernel])
    m, k, n = size
    ty = TYPES[t]
    x, w, b, r, dy = whole(m, k, 1), whole(n, k, 2), whole(1, n, 3, 9)[0], whole(m, n, 4, 9), whole(m, n, 5)
    xd, wd = rows_of(x, ty, 8), rows_of(w, ty)
    z = x @ w.t() + b
    op = F.Linear(wd, b.float().cuda(), "relu")
    y, saved = op.run_saved(xd, rows_of(r, ty, 3))
    same(y, act("relu", z) + r, "y")
    same(saved, z, "saved")
    dz = dy * slope("relu", z)
    dx, dw, db = op.backward(rows_of(dy, ty, 8), xd, saved)
    same(dx, dz @ w, "dx")
    same(dw, dz.t() @ x, "dw")
    same(db, dz.sum(0), "db")
    same(F.Linear(wd).run(xd), x @ w.t(), "plain")


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("t", sorted(TYPES))
@pytest.mark.parametrize("kernel", sorted(KERNELS))
def test_gated(kernel, t, size, force):
    from paper_2011_05630_amd import feedforward as F
    announce("gated", kernel, t, size)
    force(*KERNELS[kernel])
    m, k, n = size
    ty = TYPES[t]
    x, wg, wu, dh = whole(m, k, 1, 1), whole(n, k, 2, 1), whole(n, k, 3, 1), whole(m, n, 4, 1)
    x *= (torch.rand(m, k, generator=torch.Generator().manual_seed(7)) < min(1.0, 32.0 / k)).double()
    xd = rows_of(x, ty)
    both = rows_of(torch.cat((wg, wu)), ty)                # two halves of one tensor
    op = F.GatedLinear(both[:n], both[n:], act="relu")
    g, u = x @ wg.t(), x @ wu.t()
    h, saved = op.run_saved(xd)
    same(h, act("relu", g) * u, "h")
    same(saved, torch.stack((g, u)), "saved")
    same(op.run(xd), act("relu", g) * u, "h")
    dg, du = dh * u * slope("relu", g), dh * act("relu", g)
    assert dg.abs().max() <= 256 and du.abs().max() <= 256
    dx, dwg, dwu, _, _ = op.backward(rows_of(dh, ty), xd, saved)
    same(dx, dg @ wg + du @ wu, "dx")
    same(dwg, dg.t() @ x, "dw_gate")
    same(dwu, du.t() @ x, "dw_up")
