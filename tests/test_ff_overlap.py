"""An output that lies on an operand is refused, however the rows of the two interleave, without a GPU: addresses that nobody reads, calls that
ask for a workspace and give none, so that what is not refused for its overlap is refused for that."""
import random

import numpy as np
import pytest

from paper_2011_05630_amd import binding as B

BASE, FAR = 1 << 30, 1 << 40
K, N = 1024, 24


@pytest.fixture(autouse=True)
def split():
    B.dlf_debug_ff_kernel(3, 2)                     # any number of rows needs a workspace
    yield
    B.dlf_debug_ff_kernel(0)


def refused(rows, gated=False, x=FAR, xs=K, w=2 * FAR, ws=K, w2=3 * FAR, bias=None, bias2=None, res=None, rs=N, y=BASE, ys=N):
    d = B.dlf_ff_desc("bf16", "none", rows, K, N, xs, ws, ys, rs)
    with pytest.raises(B.DlfError) as e:
        if gated:
            B.dlf_gated(d, x, w, w2, bias, bias2, y)
        else:
            B.dlf_linear(d, x, w, bias, res, y)
    assert e.value.status in (B.DLF_ERR_INVALID_ARG, B.DLF_ERR_OOM), e.value
    if e.value.status == B.DLF_ERR_OOM:
        return None
    assert "overlaps" in str(e.value)
    return str(e.value)


def test_the_plain_cases():
    assert refused(9) is None
    assert "overlaps x" in refused(9, x=BASE)
    assert "overlaps weight" in refused(9, w=BASE)
    assert "overlaps bias" in refused(9, bias=BASE + 4)
    assert "residual" in refused(9, res=BASE + 2)
    assert refused(9, res=BASE) is None             # the residual itself
    assert "residual" in refused(9, res=BASE, rs=N + 8)
    assert refused(1, res=BASE, rs=N + 8) is None   # one row has no distance
    assert "overlaps x" in refused(9, x=BASE, res=BASE)
    for kw, what in ((dict(x=BASE), "h overlaps x"), (dict(w=BASE), "h overlaps w_gate"), (dict(w2=BASE), "h overlaps w_up"),
                     (dict(bias=BASE), "h overlaps b_gate"), (dict(bias2=BASE), "h overlaps b_up")):
        assert what in refused(9, gated=True, **kw)
    assert refused(9, gated=True) is None


def test_columns_of_one_matrix():
    """x and y side by side in wider rows share no element."""
    s = K + N + 8
    for rows in (1, 2, 70):
        assert refused(rows, x=BASE + 2 * N, xs=s, ys=s) is None
        assert refused(rows, x=BASE - 2 * K, xs=s, ys=s) is None
        assert "overlaps x" in refused(rows, x=BASE + 2 * N - 2, xs=s, ys=s)
        assert "overlaps x" in refused(rows, x=BASE - 2 * K + 2, xs=s, ys=s)


def bytes_of(p, rows, row, stride):
    return (p + stride * np.arange(rows)[:, None] + np.arange(row)[None, :]).ravel()


def test_against_the_bytes_themselves():
    rng = random.Random(5)
    seen = {True: 0, False: 0}
    for _ in range(4000):
        rows = rng.choice((1, 2, 3, 7, 70))
        ys, rs = N + rng.choice((0, 0, 8, N, 30, 64)), N + rng.choice((0, 0, 8, N, 30, 64))
        if ys != rs and N not in (ys, rs) and rows > 1:
            continue                                # two distances, neither the row: taken as apart
        at = 2 * rng.choice((rng.randint(-N - 2, N + 2), rng.randint(-rows * rs - 4, rows * ys + 4)))
        if at == 0:
            continue
        a, b = bytes_of(0, rows, 2 * N, 2 * ys), bytes_of(at, rows, 2 * N, 2 * rs)
        want = np.intersect1d(a, b, assume_unique=True).size > 0
        assert (refused(rows, res=BASE + at, rs=rs, ys=ys) is not None) == want, (rows, ys, rs, at)
        seen[want] += 1
    assert min(seen.values()) > 300


def test_rows_that_lie_far_apart():
    """Distances whose extents pass 32 bits."""
    s = (1 << 24) - 1
    rows = 70
    y = 1 << 45
    for j in (0, 1, 68, 69):
        assert refused(rows, y=y, ys=s, w=y + 2 * j * s) is not None
        assert refused(rows, y=y, ys=s, w=y + 2 * j * s + 2 * N) is None
    assert refused(rows, y=y, ys=s, w=y + 2 * 70 * s) is None
