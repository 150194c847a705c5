"""The sizes that the feed-forward operators accept, as include/dlf.h states them, without a GPU."""
import pytest

from paper_2011_05630_amd import binding as B


def accepted(**kw):
    d = dict(dtype="fp16", act="relu", rows=4, in_features=16, out_features=24)
    d.update(kw)
    got = []
    for f in (B.dlf_linear_workspace_bytes, B.dlf_linear_backward_workspace_bytes, B.dlf_gated_workspace_bytes, B.dlf_gated_backward_workspace_bytes):
        try:
            f(B.dlf_ff_desc(**d))
            got.append(True)
        except B.DlfError:
            got.append(False)
    assert len(set(got)) == 1, (kw, got)                    # one rule for all four calls
    return got[0]


def stated(rows, i, o):
    m, i, o = ((v + 63) // 64 for v in (rows, i, o))
    return max(2 * m * o, m * i + 2 * i * o + 2 * o) < (1 << 24) - 16


@pytest.mark.parametrize("i,o", [(1, 1), (64, 64), (65, 1), (1, 65), (4096, 4096), (1000, 50257), (1 << 20, 1), (1, 1 << 20), (1 << 20, 512)])
def test_most_rows(i, o):
    """The largest number of rows by the stated bound, and one more."""
    lo, hi = 0, 1 << 30
    while lo < hi:
        mid = (lo + hi + 1) // 2
        lo, hi = (mid, hi) if stated(mid, i, o) else (lo, mid - 1)
    assert lo > 0
    assert accepted(rows=lo, in_features=i, out_features=o)
    assert not accepted(rows=lo + 1, in_features=i, out_features=o)


def test_features():
    assert accepted(in_features=1 << 20) and not accepted(in_features=(1 << 20) + 1)
    assert accepted(out_features=1 << 20) and not accepted(out_features=(1 << 20) + 1)
    assert not accepted(in_features=1 << 20, out_features=1 << 20)


@pytest.mark.parametrize("name", ["x_stride", "w_stride", "y_stride", "res_stride", "dy_stride"])
def test_row_distances(name):
    assert accepted(**{name: (1 << 24) - 1}) and not accepted(**{name: 1 << 24})
