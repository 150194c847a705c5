"""AdamW and the gradients' norm on the GPU against their plain forms: states bit for bit, parameters within bounds of their roundings."""
import math

import numpy as np
import pytest
import torch

from ff_util import gen, half_eps
from gpu_util import announce
from opt_util import BLOCK, Plain

pytestmark = pytest.mark.gpu

T = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
SIZES = [1, 7, 8, 9, 63, 64, 65, 127, 0, 2047, 2048, 2049, 4095, 4096, 4097, 12289, 70001]


def tensors(sizes, t, seed, scale=1.0, offset=0, device="cuda"):
    """Views of one allocation, one behind the other, so that they start anywhere; NaN around them."""
    g = gen(seed)
    buf = torch.full((offset + sum(sizes) + 8,), float("nan"), dtype=t, device=device)
    got, at = [], offset
    for n in sizes:
        v = buf[at:at + n]
        v.copy_((torch.randn(n, generator=g) * scale).to(t))
        got.append(v)
        at += n
    return got


def numbers(t):
    return t.detach().double().cpu().numpy().reshape(-1)


def bits(t):
    return t.cpu().view(torch.uint8).numpy()


def check_states(op, plain):
    for q, at in zip(plain, op.offsets):
        end = at + q.m.size
        if op.state == "8bit":
            assert np.array_equal(bits(op.m)[at:end], q.mc) and np.array_equal(bits(op.v)[at:end], q.vc)
            assert np.array_equal(op.m_scale.cpu().numpy()[at // BLOCK:end // BLOCK], q.ms.astype(np.float32))
            assert np.array_equal(op.v_scale.cpu().numpy()[at // BLOCK:end // BLOCK], q.vs.astype(np.float32))
        else:
            assert np.array_equal(op.m.cpu().numpy()[at:end], q.m, equal_nan=True) and np.array_equal(op.v.cpu().numpy()[at:end], q.v, equal_nan=True)


def run_steps(sizes, grad, param, copy, state, seed, steps=3, offset=0, decay=0.1, factor=None, betas=(0.9, 0.95), eps=1e-8, rate=1e-2, grads=None):
    from paper_2011_05630_amd import optimizer
    announce(sizes[:3], grad, param, copy, state, seed, offset, factor)
    params = tensors(sizes, T[param], seed, 0.1, offset)
    copies = None if copy is None else tensors(sizes, T[copy], seed + 1, offset=offset)
    decays = [decay * (i % 3) for i in range(len(sizes))]
    op = optimizer.AdamW(params, copies, betas=betas, eps=eps, decay=decays, state=state, seed=77)
    plain = [Plain(numbers(p), at, betas, eps, d, state == "8bit", 77) for p, at, d in zip(params, op.offsets, decays)]
    for s in range(steps):
        g = grads(s) if grads else tensors(sizes, T[grad], seed + 10 + s, 10.0 ** (-s), offset)
        skip = [s == 1 and i % 4 == 3 for i in range(len(sizes))]
        before = [numbers(p) for p in params]
        f = None if factor is None else torch.full((), factor).cuda()
        r = rate if s % 2 == 0 else torch.full((), rate).cuda()
        op.step([None if k else q for q, k in zip(g, skip)], r, factor=f)
        assert int(op.count) == s + 1
        for i, (p, q) in enumerate(zip(params, plain)):
            if skip[i]:
                assert np.array_equal(numbers(p), before[i])
                continue
            want, bound = q.step(before[i], g[i].float().cpu().numpy(), s, rate, factor)
            if param != "fp32":
                bound = bound + half_eps(T[param]) * (np.abs(want) + bound) + (2.0 ** -25 if param == "fp16" else 0)
            got = numbers(p)
            fine = np.isfinite(want)
            assert np.array_equal(np.isfinite(got), fine)
            assert (np.abs(got - want) <= bound)[fine].all(), (i, np.abs(got - want)[fine].max())
            if copies is not None:
                assert np.array_equal(numbers(copies[i]), numbers(p.to(T[copy])), equal_nan=True)
        check_states(op, plain)
    return op, params, plain


@pytest.mark.parametrize("state", ["fp32", "8bit"])
@pytest.mark.parametrize("param,copy", [("fp32", None), ("fp32", "bf16"), ("fp32", "fp16"), ("bf16", None), ("fp16", None)])
@pytest.mark.parametrize("grad", ["bf16", "fp16", "fp32"])
def test_types(state, param, copy, grad):
    run_steps(SIZES, grad, param, copy, state, 1)
    run_steps(SIZES[::-1], grad, param, copy, state, 2, offset=3, factor=0.37)


@pytest.mark.parametrize("state", ["fp32", "8bit"])
def test_more_tensors_than_a_launch_holds(state):
    """900 tensors are three launches; the step is counted once."""
    sizes = [1 + (i * 37) % 300 for i in range(900)]
    run_steps(sizes, "bf16", "fp32", "bf16", state, 3, steps=2)


@pytest.mark.parametrize("state", ["fp32", "8bit"])
def test_more_chunks_than_workgroups(state):
    run_steps([9 * 1000 * 1000 + 5, 77], "bf16", "fp32", "bf16", state, 4, steps=2)


@pytest.mark.parametrize("betas", [(0.0, 0.0), (0.9, 0.999), (0.0, 0.99)])
@pytest.mark.parametrize("state", ["fp32", "8bit"])
def test_betas(betas, state):
    run_steps([100, 1000], "fp32", "fp32", None, state, 5, betas=betas)


@pytest.mark.parametrize("state", ["fp32", "8bit"])
def test_values_of_any_size(state):
    """Gradients over the whole range of fp32, zeros, infinities and NaN among them: states follow them bit for bit, in their own places."""
    def grads(s):
        g = gen(90 + s)
        e = torch.rand(3000, generator=g) * 36 - 18
        v = 10.0 ** e * torch.where(torch.rand(3000, generator=g) < 0.5, -1.0, 1.0)
        v[::7] = 0.0
        v[1::64] = -0.0
        if s == 1:
            v[100], v[700], v[701] = float("inf"), float("nan"), float("-inf")
        small = torch.full((200,), 1e-25)
        small[3:9] = 1e-22
        return [v.float().cuda(), small.cuda()]
    run_steps([3000, 200], "fp32", "fp32", None, state, 6, steps=4, grads=grads, eps=1e-3)


@pytest.mark.parametrize("eps", [2.0 ** -126, 2.0 ** 126])
@pytest.mark.parametrize("state", ["fp32", "8bit"])
def test_eps_at_the_ends_of_its_range(eps, state):
    """Beside second moments of zero, whose gradients were zero or had no square."""
    def grads(s):
        g = gen(95 + s)
        v = torch.randn(300, generator=g) * 10.0 ** (torch.rand(300, generator=g) * 12 - 12)
        v[::3] = 0.0
        v[1::9] = 1e-25
        return [v.cuda()]
    run_steps([300], "fp32", "fp32", None, state, 8, grads=grads, eps=eps)


def test_a_second_moment_above_zero_stays_above_zero():
    """Elements far below their block's largest would get a root of zero under their first moment."""
    from paper_2011_05630_amd import optimizer
    p = torch.zeros(64, device="cuda")
    g = torch.full((64,), 1e-12, device="cuda")
    g[0] = 1e3
    op = optimizer.AdamW([p], state="8bit", eps=0.0)
    for _ in range(20):
        op.step([g], 1.0)
    assert (op.v.float() > 0).all() and torch.isfinite(p).all() and float(p.abs().max()) < 25


def test_8bit_states_follow_what_moves_them_by_less_than_a_rounding():
    """v decays by 0.1 % a step, its codes lie 12 to 25 % apart: after 700 steps without gradients it is at e^-0.7 of where it was.  A step moves a
    code's value by a random amount of mean zero and at most a step of 25 % with a variance of at most 0.001 * 0.25 of its square; over 700 of them, by the mean
    of 65536 elements: a standard deviation of at most sqrt(700 * 0.00025 / 65536) = 0.0016 of the mean; five of them and what 16 bits of noise leave (700 * 2^-17 of a step)."""
    from paper_2011_05630_amd import optimizer
    n = 65536
    p = torch.zeros(n, device="cuda")
    op = optimizer.AdamW([p], betas=(0.9, 0.999), state="8bit", seed=5)
    g = torch.ones(n, device="cuda")
    for _ in range(10):
        op.step([g], 0.0)
    before = float((op.v.float().view(-1, BLOCK) * op.v_scale[:, None]).mean())
    g.zero_()
    for _ in range(700):
        op.step([g], 0.0)
    after = float((op.v.float().view(-1, BLOCK) * op.v_scale[:, None]).mean())
    assert abs(after / before / 0.999 ** 700 - 1) < 5 * 0.0016 + 700 * 2.0 ** -17 * 0.25


def test_strided_parameters_and_gradients():
    """Elements in any order of the dimensions, the same in all of a parameter's tensors."""
    from paper_2011_05630_amd import optimizer
    base = torch.randn(30, 50, generator=gen(8)).cuda()
    grad = torch.randn(30, 50, generator=gen(9)).cuda().bfloat16()
    got = []
    for turned in (False, True):
        p, c, g = base.clone(), base.bfloat16(), grad.clone()
        if turned:
            p, c, g = (q.t().contiguous().t() for q in (p, c, g))
            assert not p.is_contiguous()
        op = optimizer.AdamW([p, torch.ones(1, device="cuda")], [c, None], decay=0.1)
        op.step([g, torch.ones(1, device="cuda")], 0.1)
        got.append((p.clone(), c.clone()))
        with pytest.raises(ValueError, match="^gradient 0: the sizes and strides"):
            op.step([g.contiguous() if turned else g.t().contiguous().t(), None], 0.1)
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


def test_strides_of_single_elements_say_nothing():
    """The stride of a dimension of one element may change: no element is elsewhere."""
    from paper_2011_05630_amd import optimizer
    p, c = torch.zeros(1, 300).cuda(), torch.zeros(1, 300).cuda().bfloat16()
    op = optimizer.AdamW([p], [c])
    p.data = p.data.as_strided((1, 300), (7, 1))
    c.data = c.data.as_strided((1, 300), (5, 1))
    op.step([torch.ones(1, 300).cuda()], 0.5)
    assert (p == -0.5).all() and (c == -0.5).all()


@pytest.mark.parametrize("factor", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("state", ["fp32", "8bit"])
def test_a_factor_that_is_not_finite_leaves_everything(state, factor):
    op, params, _ = run_steps([100, 5000], "bf16", "fp32", "bf16", state, 10, steps=1)
    kept = {n: t.clone() for n, t in op.save_state().items()}
    before = [p.clone() for p in params]
    g = [torch.randn(100).cuda(), torch.randn(5000).cuda()]
    op.step(g, 0.1, factor=torch.full((1,), factor).cuda())
    for n, t in op.save_state().items():
        assert torch.equal(t.view(torch.uint8) if t.dtype != torch.int64 else t, kept[n].view(torch.uint8) if t.dtype != torch.int64 else kept[n])
    assert all(torch.equal(a, b) for a, b in zip(before, params))
    op.step(g, 0.1, factor=torch.full((1,), 1.0).cuda())
    assert int(op.count) == 2


@pytest.mark.parametrize("state", ["fp32", "8bit"])
def test_states_are_saved_and_loaded(state):
    """A run that is continued elsewhere is the same bit for bit, at any alignment of its tensors."""
    from paper_2011_05630_amd import optimizer
    op, params, _ = run_steps([65, 3000, 1], "bf16", "fp32", "fp16", state, 11)
    other = tensors([65, 3000, 1], torch.float32, 12, offset=5)
    for a, b in zip(other, params):
        a.copy_(b)
    second = optimizer.AdamW(other, decay=[0.0, 0.1, 0.2], state=state, seed=77)
    saved = op.save_state()
    second.load_state(saved)
    assert int(second.count) == 3
    g = tensors([65, 3000, 1], torch.bfloat16, 13)
    for o in (op, second):
        o.step(g, 0.01)
    for a, b in zip(other, params):
        assert torch.equal(a, b)
    third = op.save_state()
    assert all(torch.equal(bits_of(third[n]), bits_of(getattr(second, n))) for n in third if n != "count")
    second.load_state(dict(saved, count=3))
    assert int(second.count) == 3
    for bad in (dict(saved, count=-1), dict(saved, count=1.0), {n: t for n, t in saved.items() if n != "m"}, dict(saved, m=saved["m"][:64])):
        with pytest.raises(ValueError):
            second.load_state(bad)


@pytest.mark.parametrize("state", ["fp32", "8bit"])
def test_a_run_of_many_steps_goes_on_with_its_powers(state):
    """The betas' powers are a product of as many factors as steps were done, which one power of the count is not bit for bit."""
    from paper_2011_05630_amd import optimizer
    params = tensors([300], torch.float32, 17)
    op = optimizer.AdamW(params, betas=(0.9, 0.999), state=state)
    for s in range(70):
        op.step(tensors([300], torch.bfloat16, 18 + s % 3), 0.01)
    saved = op.save_state()
    assert saved["powers"].tolist()[:3] == [70.0, 0.9, 0.999] and torch.equal(saved["powers"], op.powers)
    second = optimizer.AdamW([p.clone() for p in params], betas=(0.9, 0.999), state=state)
    second.load_state(saved)
    assert torch.equal(second.powers, op.powers)
    # where they are not there, or belong to another count or other betas, they are formed anew
    other = optimizer.AdamW([p.clone() for p in params], betas=(0.8, 0.99), state=state)
    other.load_state(saved)
    first = {n: t for n, t in saved.items() if n != "powers"}
    for o, given, want in ((other, saved, (70, 0.8, 0.99)), (other, first, (70, 0.8, 0.99)), (other, dict(saved, count=3), (3, 0.8, 0.99)),
                           (second, first, (70, 0.9, 0.999)), (second, dict(saved, count=5), (5, 0.9, 0.999))):
        o.load_state(given)
        n, b1, b2 = want
        got = o.powers.tolist()
        assert got[:3] == [n, b1, b2] and int(o.count) == n
        for a, b in zip(got[3:], (b1 ** n, b2 ** n)):
            assert abs(a - b) <= 4 * 2.0 ** -52 * b
    for bad in (saved["powers"][:4], saved["powers"].float(), 1.0):
        with pytest.raises(ValueError, match="^powers: "):
            second.load_state(dict(saved, powers=bad))
    with pytest.raises(ValueError, match="^state: "):
        second.load_state(dict(saved, power=1.0))


def bits_of(t):
    return t.view(torch.uint8)


@pytest.mark.parametrize("state", ["fp32", "8bit"])
def test_a_captured_step_goes_on_counting(state):
    from paper_2011_05630_amd import optimizer
    sizes = [100, 4097, 50]
    made = []
    for _ in range(2):
        params, copies = tensors(sizes, torch.float32, 14), tensors(sizes, torch.bfloat16, 15)
        made.append((params, copies, optimizer.AdamW(params, copies, decay=0.1, state=state, seed=3)))
    grads = tensors(sizes, torch.bfloat16, 16)
    rate = torch.full((1,), 0.01).cuda()
    (params, copies, op), (params2, copies2, op2) = made

    def once(o):
        norm, factor = optimizer.gradient_norm(grads, most=1.0)
        o.step(grads, rate, factor=factor)
        return norm

    for o in (op, op2):                                     # (one eager step each)
        once(o)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm = once(op)
    for s in range(4):
        for g in grads:
            g.mul_(0.5 if s % 2 else 3.0)
        rate.mul_(0.7)
        graph.replay()
        torch.cuda.synchronize()
        want = once(op2)
        assert float(want) == float(norm) and int(op.count) == int(op2.count) == s + 2
        for a, b in zip(params + copies, params2 + copies2):
            assert torch.equal(a, b)
        for n in ("m", "v"):
            assert torch.equal(bits_of(getattr(op, n)), bits_of(getattr(op2, n)))


def test_a_parameter_of_a_module():
    """Leaves that require gradients are updated as under no_grad, and raise their version: a backward pass over old values is noticed."""
    from paper_2011_05630_amd import optimizer
    net = torch.nn.Linear(40, 30).cuda()
    op = optimizer.AdamW(list(net.parameters()))
    y = (net(torch.randn(5, 40).cuda()) ** 2).sum()
    y.backward(retain_graph=True)
    before = [p.detach().clone() for p in net.parameters()]
    versions = [p._version for p in net.parameters()]
    op.step([p.grad for p in net.parameters()], 0.1)
    assert all(p._version > v for p, v in zip(net.parameters(), versions))
    # the first step moves by the rate, against the gradient
    for p, b in zip(net.parameters(), before):
        moved = p.detach() - b
        assert torch.equal(moved.sign(), -p.grad.sign()) and float((moved.abs() - 0.1)[p.grad != 0].abs().max()) < 1e-3


# ---- the norm --------------------------------------------------------------------------------

def want_norm(grads):
    return math.sqrt(sum(float(g.double().square().sum()) for g in grads))


@pytest.mark.parametrize("t", ["bf16", "fp16", "fp32"])
def test_norm(t):
    from paper_2011_05630_amd import optimizer
    for sizes, offset in ((SIZES, 0), (SIZES, 3), ([1], 0), ([0], 0), ([0, 5, 0], 1), ([3 * 1000 * 1000 + 7], 0), ([10] * 500, 1)):
        announce(t, sizes[:3], offset)
        grads = tensors(sizes, T[t], 20, 0.1, offset)
        for most, scale in ((1e9, 1.0), (0.5, 1.0), (0.5, 0.25), (0.0, 1.0), (float("inf"), -2.0)):
            norm, factor = optimizer.gradient_norm(grads, most=most, scale=scale)
            want = want_norm(grads) * abs(scale)
            by = scale * min(1.0, most / want) if want > 0 else scale
            assert norm.dtype == factor.dtype == torch.float32 and norm.shape == factor.shape == ()
            # summed in 64 bits: a rounding to 32 bits, and the products' on the way
            assert abs(float(norm) - want) <= 2.0 ** -24 * want * 1.001
            assert abs(float(factor) - by) <= 2.0 ** -24 * abs(by) * 1.001
        same = optimizer.gradient_norm(grads, most=most, scale=scale)
        assert float(same[0]) == float(norm)


def test_norm_of_values_of_any_size():
    from paper_2011_05630_amd import optimizer
    for v in (1e-30, 1e-44, 1e30, 3e38):
        g = [torch.full((1000,), v).cuda(), torch.full((3,), v).cuda()]
        norm, factor = optimizer.gradient_norm(g, most=1.0)
        want = want_norm(g)
        if want > 3.4028235e38:
            assert norm.isinf() and factor.isnan()
        else:
            assert abs(float(norm) - want) <= 2.0 ** -24 * want * 1.001 + 2.0 ** -150 and torch.isfinite(factor)
    for bad in (float("nan"), float("inf"), float("-inf")):
        for at in (0, 999, 5000):
            g = torch.ones(5001).cuda()
            g[at] = bad
            norm, factor = optimizer.gradient_norm([g], most=1.0)
            assert not torch.isfinite(norm) and factor.isnan()


def test_norm_passes_over_none():
    from paper_2011_05630_amd import optimizer
    g = torch.randn(100, generator=gen(21)).cuda()
    assert float(optimizer.gradient_norm([None, g, None])[0]) == float(optimizer.gradient_norm([g])[0])
    assert float(optimizer.gradient_norm((q for q in [g, None]))[0]) == float(optimizer.gradient_norm([g])[0])
