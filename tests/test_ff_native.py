"""What the feed-forward operators' native step refuses before anything is launched: on CPU tensors, without a GPU."""
import pytest
import torch

from paper_2011_05630_amd import binding as B
from paper_2011_05630_amd import feedforward as F


def op(gated=False, act="silu", n=24, k=16, bias=False, t=torch.bfloat16):
    w = torch.zeros(n, k, dtype=t)
    b = torch.zeros(n) if bias else None
    return F._native().Op(gated, B.FF_ACT[act], w, w if gated else None, b, b if gated else None, k)


X = torch.zeros(6, 16, dtype=torch.bfloat16)
BAD_X = {
    "not a tensor": [1.0], "type": X.half(), "width": X[:, :15], "no dimension": X[0, 0], "strided row": torch.zeros(16, 6, dtype=torch.bfloat16).t(),
    "overlapping": X[:1].expand(6, 16), "two distances": torch.zeros(4, 6, 16, dtype=torch.bfloat16)[:, :5].transpose(0, 1),
    "gap between blocks": torch.zeros(4, 6, 16, dtype=torch.bfloat16)[:, :5],
}


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("what", sorted(BAD_X))
def test_operands(what, gated):
    with pytest.raises(ValueError, match="^x: "):
        op(gated).forward(BAD_X[what], None, None, False, 0)
    with pytest.raises(ValueError, match="^x: "):
        op(gated).backward(X, BAD_X[what], None, True, True, True, 0)


def test_residual_out_and_gradients():
    r = torch.zeros(6, 24, dtype=torch.bfloat16)
    for bad in (r[:5], r[:, :23], r.view(2, 3, 24), r.float(), r[:1].expand(6, 24)):
        with pytest.raises(ValueError, match="^residual: "):
            op().forward(X, bad, None, False, 0)
        with pytest.raises(ValueError, match="^out: "):
            op().forward(X, None, bad, False, 0)
        with pytest.raises(ValueError, match="^dy: "):
            op().backward(bad, X, torch.zeros(6, 24), True, True, True, 0)
        with pytest.raises(ValueError, match="^dh: "):
            op(True).backward(bad, X, torch.zeros(2, 6, 24), True, True, True, 0)
    for bad in (None, torch.zeros(6, 23), torch.zeros(6, 24).double(), torch.zeros(6, 48)[:, ::2], torch.zeros(2, 6, 24)):
        with pytest.raises(ValueError, match="^saved: "):
            op().backward(r, X, bad, True, True, True, 0)
    with pytest.raises(ValueError, match="^saved: "):
        op(True).backward(r, X, torch.zeros(6, 24), True, True, True, 0)


def test_no_rows():
    """Nothing to compute, nothing launched: shapes and types of the outputs."""
    for shape in ((0, 16), (3, 0, 16)):
        x = torch.zeros(shape, dtype=torch.bfloat16)
        y, saved = op().forward(x, None, None, True, 0)
        assert y.shape == shape[:-1] + (24,) and y.dtype == torch.bfloat16 and saved.shape == (0, 24) and saved.dtype == torch.float32
        y, saved = op(act="none").forward(x, None, None, True, 0)
        assert saved is None
        h, saved = op(True).forward(x, None, None, True, 0)
        assert h.shape == shape[:-1] + (24,) and saved.shape == (2, 0, 24)
        out = torch.zeros(shape[:-1] + (24,), dtype=torch.bfloat16)
        assert op().forward(x, None, out, False, 0) is out


def test_refusals_of_the_library_carry_their_status():
    big = F._native().Op(False, B.FF_ACT["none"], torch.empty(1, (1 << 20) + 1, dtype=torch.bfloat16), None, None, None, (1 << 20) + 1)
    with pytest.raises(B.DlfError) as e:
        big.forward(torch.empty(1, (1 << 20) + 1, dtype=torch.bfloat16), None, None, False, 0)
    assert e.value.status == B.DLF_ERR_INVALID_ARG
    assert "features" in str(e.value)
