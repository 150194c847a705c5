"""What the feed-forward operators refuse, and the sizes they ask for, without a GPU."""
import ctypes

import pytest
import torch

from paper_2011_05630_amd import binding as B

P, Q = 0x10000, 0x20000      # never read: every call here is refused before a launch


def desc(**kw):
    d = dict(dtype="bf16", act="silu", rows=4, in_features=16, out_features=24)
    d.update(kw)
    return B.dlf_ff_desc(**d)


def status(f, *a):
    with pytest.raises(B.DlfError) as e:
        f(*a)
    assert str(e.value)
    return e.value.status


BAD_DESCS = [dict(rows=-1), dict(rows=(1 << 30) + 1), dict(in_features=0), dict(out_features=0), dict(in_features=(1 << 20) + 1),
             dict(out_features=-5), dict(x_stride=15), dict(w_stride=-16), dict(y_stride=23), dict(dy_stride=23), dict(res_stride=1),
             dict(x_stride=1 << 24), dict(dy_stride=1 << 40)]


@pytest.mark.parametrize("kw", BAD_DESCS)
def test_bad_descriptions(kw):
    d = desc(**kw)
    assert status(B.dlf_linear, d, P, P, None, None, Q) == B.DLF_ERR_INVALID_ARG
    assert status(B.dlf_gated, d, P, P, P, None, None, Q) == B.DLF_ERR_INVALID_ARG
    assert status(B.dlf_linear_backward, d, P, P, P, P, Q, Q, None, P, 1 << 40) == B.DLF_ERR_INVALID_ARG
    assert status(B.dlf_gated_backward, d, P, P, P, P, P, Q, Q, Q, None, None, P, 1 << 40) == B.DLF_ERR_INVALID_ARG
    for f in (B.dlf_linear_workspace_bytes, B.dlf_gated_workspace_bytes, B.dlf_linear_backward_workspace_bytes, B.dlf_gated_backward_workspace_bytes):
        status(f, d)


@pytest.mark.parametrize("field,value", [("dtype", 2), ("dtype", -1), ("act", 7), ("act", -1)])
def test_bad_enumerators(field, value):
    d = desc()
    setattr(d, field, value)
    assert status(B.dlf_linear, d, P, P, None, None, Q) == B.DLF_ERR_INVALID_ARG
    assert status(B.dlf_gated_workspace_bytes, d) == B.DLF_ERR_INVALID_ARG


def test_null_description():
    L = B.lib()
    assert L.dlf_linear(None, P, P, None, None, Q, None, None, 0, None) == B.DLF_ERR_INVALID_ARG
    assert L.dlf_linear_workspace_bytes(None) == ctypes.c_size_t(-1).value
    assert L.dlf_gated_backward_workspace_bytes(None) == ctypes.c_size_t(-1).value


def test_more_tiles_than_a_launch_holds():
    d = desc(rows=1 << 30, in_features=1 << 20, out_features=1 << 20)
    assert status(B.dlf_linear, d, P, P, None, None, Q) == B.DLF_ERR_UNSUPPORTED


def test_null_and_misaligned_tensors():
    d = desc()
    for bad in ((None, P, None, None, Q), (P, None, None, None, Q), (P, P, None, None, None), (P + 1, P, None, None, Q), (P, P + 1, None, None, Q),
                (P, P, P + 2, None, Q), (P, P, None, P + 1, Q), (P, P, None, None, Q + 1), (P, P, None, None, Q, P + 2)):
        assert status(B.dlf_linear, d, *bad) == B.DLF_ERR_INVALID_ARG
    for i in range(3):
        a = [P, P, P, None, None, Q]
        a[i] = None
        assert status(B.dlf_gated, d, *a) == B.DLF_ERR_INVALID_ARG
    ws = B.dlf_gated_backward_workspace_bytes(d)
    ok = [P, P, P, P, P, Q, Q, Q, None, None]
    for i in range(5):
        a = list(ok)
        a[i] = None
        assert status(B.dlf_gated_backward, d, *a, P, ws) == B.DLF_ERR_INVALID_ARG
    for i, off in ((0, 1), (4, 2), (5, 1), (8, 2)):
        a = list(ok)
        a[i] = (a[i] or P) + off
        assert status(B.dlf_gated_backward, d, *a, P, ws) == B.DLF_ERR_INVALID_ARG


def test_workspace_refusals():
    d = desc(rows=100)
    for f, args, need in ((B.dlf_linear_backward, (P, P, P, P, Q, Q, None), B.dlf_linear_backward_workspace_bytes(d)),
                          (B.dlf_gated_backward, (P, P, P, P, P, Q, Q, Q, None, None), B.dlf_gated_backward_workspace_bytes(d))):
        assert need > 0
        assert status(f, d, *args, P, need - 1) == B.DLF_ERR_OOM
        assert status(f, d, *args, None, need) == B.DLF_ERR_INVALID_ARG
        assert status(f, d, *args, P + 128, need) == B.DLF_ERR_INVALID_ARG


def test_no_rows_is_no_error_forward():
    d = desc(rows=0)
    B.dlf_linear(d, None, None, None, None, None)
    B.dlf_gated(d, None, None, None, None, None, None)


def test_network_layers_keep_their_activations():
    """The new activations belong to the feed-forward operators: a network layer with one is refused as before."""
    from synth import nets
    net = nets.two_layer_block()
    layer = dict(net["layers"][0])
    d = (B.LayerDesc * 1)()
    d[0].op, d[0].cin, d[0].cout, d[0].kh, d[0].kw, d[0].stride, d[0].pad = 0, layer["cin"], layer["cout"], 3, 3, 1, 1
    d[0].input_from = d[0].residual_from = -1
    h = ctypes.c_void_p()
    for act in (3, 4, 5, 6):
        d[0].act = act
        assert B.lib().dlf_net_create(d, 1, net["in_h"], net["in_w"], net["in_c"], ctypes.byref(h)) == B.DLF_ERR_INVALID_ARG


def test_python_refuses_host_tensors():
    from paper_2011_05630_amd import feedforward as F
    with pytest.raises(ValueError):
        F.Linear(torch.zeros(4, 8, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        F.GatedLinear(torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(4, 8, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        F.FeedForward(None, None)
