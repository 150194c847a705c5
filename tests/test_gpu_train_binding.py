"""The C calls of the cross entropy, the gradients' norm and AdamW through the Python binding, on device addresses: the bits of the operators on tensors."""
import pytest
import torch

from ff_util import TYPES
from test_gpu_loss import given, inputs

pytestmark = pytest.mark.gpu


def room(n):
    """A workspace of as many bytes as the call asks for."""
    return torch.empty(max(1, n), dtype=torch.uint8, device="cuda")


def at(t):
    return None if t is None else t.data_ptr()


def here():
    return torch.cuda.current_stream().cuda_stream


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("m,bias", [(7, True), (150, False), (150, True)])
def test_cross_entropy(m, bias, dtype):
    from paper_2011_05630_amd import binding as B, loss
    k, v = 72, 333
    x, w, b, target, on = inputs(m, k, v, TYPES[dtype], 70, bias=bias, ignored=0.2, gap=8)
    dloss, dlse = (q.cuda() for q in given(m, 71))
    op = loss.CrossEntropy(on["w"], on["b"])
    d = B.dlf_ce_desc(dtype, m, k, v, x_stride=on["x"].stride(0), w_stride=on["w"].stride(0), dbias=int(bias))
    got, lse = (torch.full((m,), float("nan"), device="cuda") for _ in range(2))
    n = B.dlf_cross_entropy_workspace_bytes(d)
    ws = room(n)
    B.dlf_cross_entropy(d, at(on["x"]), at(on["w"]), at(on["b"]), at(on["target"]), at(got), at(lse), at(ws), n, here())
    for a, c in zip((got, lse), op.run_saved(on["x"], on["target"])):
        assert torch.equal(a, c)

    def outputs():
        return (torch.full((m, k), float("nan"), dtype=TYPES[dtype], device="cuda"), torch.full((v, k), float("nan"), dtype=TYPES[dtype], device="cuda"),
                torch.full((v,), float("nan"), device="cuda") if bias else None)

    def same(out, want):
        for a, c in zip(out, want):
            assert a is c or torch.equal(a, c)

    out = outputs()
    n = B.dlf_cross_entropy_backward_workspace_bytes(d)
    ws = room(n)
    B.dlf_cross_entropy_backward(d, at(on["x"]), at(on["w"]), at(on["b"]), at(on["target"]), at(lse), at(dloss), 1, 0.0, at(dlse), 1, *map(at, out),
                                 workspace=at(ws), workspace_bytes=n, stream=here())
    same(out, op.backward(dloss, on["x"], on["target"], lse, dlse=dlse))
    for step, value in ((1, 0.0), (0, 0.25)):               # each row's own, and a number for all
        out = outputs()
        got.fill_(float("nan"))
        n = B.dlf_cross_entropy_gradients_workspace_bytes(d)
        ws = room(n)
        B.dlf_cross_entropy_gradients(d, at(on["x"]), at(on["w"]), at(on["b"]), at(on["target"]), at(dloss) if step else None, step, value, at(got), *map(at, out),
                                      workspace=at(ws), workspace_bytes=n, stream=here())
        same((got,) + out, op.gradients(on["x"], on["target"], dloss if step else value))


@pytest.mark.parametrize("state", ["fp32", "8bit"])
def test_a_step(state):
    from paper_2011_05630_amd import binding as B, optimizer
    sizes, types = [5000, 1, 0, 130], ["fp32", "fp32", "bf16", "fp16"]
    t = {"fp32": torch.float32, **TYPES}
    torch.manual_seed(72)
    params = [torch.randn(n, device="cuda").to(t[q]) for n, q in zip(sizes, types)]
    copies = [torch.zeros(sizes[0], dtype=torch.bfloat16, device="cuda"), None, None, None]
    mine, mine_copies = [p.clone() for p in params], [None if c is None else c.clone() for c in copies]
    grad_types = ["bf16", "fp32", "fp32", "fp16"]
    grads = [torch.randn(n, device="cuda").to(t[q]) for n, q in zip(sizes, grad_types)]
    decays = [0.1, 0.0, 0.2, 0.3]
    op = optimizer.AdamW(mine, mine_copies, betas=(0.8, 0.9), eps=1e-6, decay=decays, state=state, seed=9)

    table = B.dlf_adamw_tensors([(at(p), at(c), n, q, None if c is None else "bf16", e) for p, c, n, q, e in zip(params, copies, sizes, types, decays)])
    elements = B.dlf_adamw_state_elements(table, 4)
    assert elements == op.m.numel()
    host = torch.empty(B.dlf_adamw_table_bytes(table, 4), dtype=torch.uint8)
    B.dlf_adamw_table(table, 4, host.data_ptr(), host.numel())
    filled = host.cuda()
    small = state == "8bit"
    m, v = (torch.zeros(elements, dtype=torch.uint8 if small else torch.float32, device="cuda") for _ in range(2))
    ms, vs = (torch.ones(elements // optimizer.BLOCK, device="cuda") if small else None for _ in range(2))
    counter = torch.tensor([0.0, 1.0, 1.0, 0.0], dtype=torch.float64).cuda()
    d = B.dlf_adamw_desc((0.8, 0.9), 1e-6, 9, state)
    rate = torch.full((), 0.02).cuda()
    for s in range(3):
        n = B.dlf_gradient_norm_workspace_bytes(sizes)
        ws, norm, factor = room(n), torch.empty((), device="cuda"), torch.empty((), device="cuda")
        B.dlf_gradient_norm([at(g) for g in grads], sizes, grad_types, 1.0, 0.5, at(norm), at(factor), at(ws), n, here())
        want, by = optimizer.gradient_norm(grads, most=1.0, scale=0.5)
        assert float(norm) == float(want) and float(factor) == float(by) < 0.5
        given_ = [None if s == 1 and i == 1 else g for i, g in enumerate(grads)]
        B.dlf_adamw_step(d, table, 4, at(filled), [at(g) for g in given_], grad_types, at(m), at(v), at(ms), at(vs), at(counter), 0.02, at(rate) if s == 2 else None,
                         at(factor), here())
        op.step(given_, rate if s == 2 else 0.02, factor=by)
    assert float(counter[0]) == int(op.count) == 3
    for a, c in zip(params + copies[:1] + [m, v] + ([ms, vs] if small else []), mine + mine_copies[:1] + [op.m, op.v] + ([op.m_scale, op.v_scale] if small else [])):
        assert torch.equal(a.view(torch.uint8), c.view(torch.uint8))
