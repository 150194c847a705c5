"""The cross entropy and the optimizer where places pass 2^31 and 2^32 elements: wrong 32-bit offsets would write or read elsewhere."""
import numpy as np
import pytest
import torch

from ce_util import IGNORE, gradients, reference
from ff_util import gen, half_eps, within
from gpu_util import announce
from opt_util import BLOCK, Plain

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def give_memory_back():
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("bias", [False, True])
def test_a_piece_of_more_than_32_bits(bias):
    """One piece of 65536 rows of 50000 classes: 3.3 * 10^9 elements of dz and of the logits.  Rows on both sides of 2^31 and, in bytes of either, 2^32 have a
    target, the others none: the gradients are those rows' alone."""
    from paper_2011_05630_amd import loss
    m, k, v, t = 65536, 16, 50000, torch.bfloat16
    announce(m, k, v, bias)
    g = gen(70)
    some = sorted({0, 1, 21474, 21475, 42949, 42950, 65534, 65535} | {int(i) for i in torch.randint(m, (56,), generator=g)})
    w = (torch.randn(v, k, generator=g) * k ** -0.5).to(t)
    x = torch.randn(m, k, generator=g).to(t)
    b = torch.randn(v, generator=g) * 0.3 if bias else None
    target = torch.full((m,), IGNORE)
    target[some] = torch.randint(v, (len(some),), generator=g)
    on = dict(x=x.cuda(), w=w.cuda(), target=target.cuda())
    xs, ws = x[some].double(), w.double()
    ref = reference(xs, ws, None if b is None else b.double(), target[some])
    op = loss.CrossEntropy(on["w"], None if b is None else b.cuda(), ignore_index=IGNORE, piece_bytes=1 << 40)
    one, none = torch.ones(len(some)).double(), torch.zeros(len(some)).double()

    def check(got, grads, kept):
        assert int((got != 0).sum()) == len(some)
        within(got[some], ref["loss"], ref["e_loss"], "loss")
        want = gradients(ref, xs, ws, one, none, t, kept=kept)
        dx, dw, db = grads
        assert int((dx != 0).any(1).sum()) == len(some)
        within(dx[some], *want["dx"], "dx")
        within(dw, *want["dw"], "dw")
        assert (db is None) == (b is None)
        if db is not None:
            within(db, *want["db"], "db")

    got, *grads = op.gradients(on["x"], on["target"], 1.0)
    check(got, grads, kept=b is None)
    got, lse = op.run_saved(on["x"], on["target"])
    assert torch.isfinite(lse).all()
    check(got, op.backward(1.0, on["x"], on["target"], lse), kept=False)


@pytest.mark.parametrize("state", ["fp32", "8bit"])
def test_a_tensor_of_more_than_32_bits(state):
    """2^32 + 12365 elements: the norm of all of them, and two steps, looked at around 2^31, 2^32 and at the end."""
    from paper_2011_05630_amd import optimizer
    n, t, betas, eps, rate, width = (1 << 32) + 12365, torch.bfloat16, (0.9, 0.95), 1e-8, 1e-2, 1024
    announce(n, state)
    p, grad = torch.zeros(n, dtype=t, device="cuda"), torch.full((n,), 2.0 ** -10, dtype=t, device="cuda")
    norm, factor = optimizer.gradient_norm([grad], most=1.0)
    want = n ** 0.5 * 2.0 ** -10                            # (the sum of squares is exact)
    assert abs(float(norm) - want) <= 2.0 ** -24 * want and abs(float(factor) - 1 / want) <= 2.0 ** -23 / want
    windows = [(a, min(n, a + width)) for a in (0, (1 << 31) - 512, (1 << 32) - 512, (n // BLOCK) * BLOCK - 512)]
    g = gen(71)
    op = optimizer.AdamW([p], betas=betas, eps=eps, state=state, seed=5)
    plain = [Plain(np.zeros(b - a), a, betas, eps, 0.0, state == "8bit", 5) for a, b in windows]
    for s in range(2):
        for a, b in windows:
            grad[a:b] = (torch.randn(b - a, generator=g) * 10.0 ** -s).to(t).cuda()
        before = [p[a:b].double().cpu().numpy() for a, b in windows]
        op.step([grad], rate)
        for (a, b), old, q in zip(windows, before, plain):
            want, bound = q.step(old, grad[a:b].float().cpu().numpy(), s, rate)
            bound = bound + half_eps(t) * (np.abs(want) + bound)
            assert (np.abs(p[a:b].double().cpu().numpy() - want) <= bound).all(), (s, a)
            end = a + q.m.size
            if state == "8bit":
                assert np.array_equal(op.m[a:end].view(torch.uint8).cpu().numpy(), q.mc) and np.array_equal(op.v[a:end].view(torch.uint8).cpu().numpy(), q.vc)
            else:
                assert np.array_equal(op.m[a:end].cpu().numpy()[:q.n], q.m[:q.n]) and np.array_equal(op.v[a:end].cpu().numpy()[:q.n], q.v[:q.n])
    assert int(op.count) == 2
