"""The few-rows kernels of the feed-forward operators where every wave goes round its ring many times, against the plain operators in 64 bits: bit
for bit on whole numbers.

A workgroup has eight waves while there are at most 256 of them, else four; each wave takes its share of k in stages of 64 (operands of whole
lines: two in LDS, so three stages reuse a slot) or of 32 (rows that start anywhere: six or eight requested ahead, so the loop that
requests while it multiplies takes twelve or sixteen).  k = 4104 gives eight waves 8 stages or 16 steps each, four as many
of 2056."""
import pytest
import torch

from ff_util import TYPES, act, rows_of, same, whole
from gpu_util import announce

pytestmark = pytest.mark.gpu

# (rows, in, out): every count of blocks of 16 rows, features over and under 16, 256 groups and more of them
SIZES = [(1, 4104, 40), (5, 8200, 17), (7, 4096, 72), (16, 4104, 24), (17, 4104, 130), (24, 2056, 100), (24, 2056, 4200), (32, 8200, 72), (33, 4104, 33),
         (40, 4104, 72), (48, 4104, 72), (48, 2056, 4200), (64, 4096, 130), (64, 8200, 1000), (9, 2056, 4200)]
# (gap between rows, offset of the first) of x and of the weights
LAYOUTS = {"lines": ((0, 0), (8, 0)), "x anywhere": ((3, 0), (0, 0)), "weights anywhere": ((0, 0), (5, 1)), "both anywhere": ((1, 1), (0, 3))}


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("layout", sorted(LAYOUTS))
@pytest.mark.parametrize("t", sorted(TYPES))
def test_linear(t, layout, size):
    from paper_2011_05630_amd import feedforward as F
    m, k, n = size
    announce("few rows linear", t, layout, size)
    ty, (lx, lw) = TYPES[t], LAYOUTS[layout]
    for odd in (0, 1):                                          # the last stage whole or not, the last step too
        x, w, b, r = whole(m, k - odd, 1), whole(n, k - odd, 2), whole(1, n, 3, 9)[0], whole(m, n, 4, 9)
        op = F.Linear(rows_of(w, ty, *lw), b.float().cuda(), "relu")
        z = x @ w.t() + b
        y, saved = op.run_saved(rows_of(x, ty, *lx), rows_of(r, ty))
        same(y, act("relu", z) + r, "y")
        same(saved, z, "saved")


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("layout", sorted(LAYOUTS))
@pytest.mark.parametrize("t", sorted(TYPES))
def test_gated(t, layout, size):
    from paper_2011_05630_amd import feedforward as F
    m, k, n = size
    announce("few rows gated", t, layout, size)
    ty, (lx, lw) = TYPES[t], LAYOUTS[layout]
    for odd in (0, 1):
        # few values of x differ from zero, so that the products of both sums stay within fp16's range
        x, wg, wu, bg, bu = whole(m, k - odd, 1, 1), whole(n, k - odd, 2, 1), whole(n, k - odd, 3, 1), whole(1, n, 4, 9)[0], whole(1, n, 5, 9)[0]
        x *= (torch.rand(m, k - odd, generator=torch.Generator().manual_seed(7)) < 0.25).double()
        op = F.GatedLinear(rows_of(wg, ty, *lw), rows_of(wu, ty, *lw), bg.float().cuda(), bu.float().cuda(), "relu")
        g, u = x @ wg.t() + bg, x @ wu.t() + bu
        h, saved = op.run_saved(rows_of(x, ty, *lx))
        same(h, act("relu", g) * u, "h")
        same(saved, torch.stack((g, u)), "saved")
