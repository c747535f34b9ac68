"""GPU parity of the AdamW step on the adapters.  The operator is defined by fp32 roundings operation by operation, so the moments are
compared bit for bit; the parameters as well, as IEEE division and square root leave no freedom."""
import numpy as np
import pytest
import torch

import paper_2510_11696_amd as qerl
from oracle import update_oracle as uo

pytestmark = pytest.mark.gpu
HYPER = dict(lr=2e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.05)
LISTS = {"one": [1], "seven": [7], "block": [32], "ragged": [33, 8, 1, 2047, 2048, 2049, 0, 4096 + 17], "odd": [5005, 31, 100003], "many": [64 + i for i in range(200)]}


class _Set:
    """The tensors of a step on the GPU and the same in numpy."""

    def __init__(self, sizes, bits, seed, copies=True):
        rng = np.random.default_rng(seed)
        self.sizes, self.bits = sizes, bits
        self.starts, self.total = uo.state_starts(sizes)
        self.p = [rng.normal(size=n).astype(np.float32) * 0.1 for n in sizes]
        self.gp = [torch.from_numpy(a.copy()).cuda() for a in self.p]
        self.gc = [torch.empty((n,), dtype=torch.bfloat16, device="cuda") for n in sizes] if copies else None
        self.gg = [torch.empty((n,), device="cuda") for n in sizes]
        self.plan = qerl.lora_adamw_plan(self.gp, self.gg, self.gc, state_bits=bits)
        self.m, self.v = np.zeros(self.total, np.float32), np.zeros(self.total, np.float32)
        self.rng = rng

    def gradients(self, scale=1e-2):
        self.g = [(self.rng.normal(size=n) * scale * np.exp(self.rng.normal(size=n) * 2)).astype(np.float32) for n in self.sizes]
        for t, a in zip(self.gg, self.g):
            t.copy_(torch.from_numpy(a))

    def flat(self, parts):
        out = np.zeros(self.total, np.float32)
        for a, at in zip(parts, self.starts):
            out[at:at + len(a)] = a
        return out

    def reference(self, step, seed, grad_scale=None, **h):
        p, m, v = uo.adamw(self.flat(self.p), self.flat(self.g), self.m, self.v, step=step, grad_scale=grad_scale, **h)
        inside = self.flat([np.ones(n, np.float32) for n in self.sizes]) > 0
        m, v = np.where(inside, m, np.float32(0)), np.where(inside, v, np.float32(0))
        self.p = [p[at:at + n] for at, n in zip(self.starts, self.sizes)]
        if self.bits == 8:
            u = uo.random_fractions(self.total, step, seed)
            m, v = uo.decode(*uo.encode_first(m, u), 4), uo.decode(*uo.encode_second(v, u), 5)
        self.m, self.v = m, v

    def check(self):
        gm, gv = qerl.lora_adamw_moments(self.plan) if self.bits == 8 else (self.plan.m, self.plan.v)
        torch.cuda.synchronize()
        for name, a, b in (("m", gm, self.m), ("v", gv, self.v)):
            a = a.cpu().numpy()
            assert np.array_equal(a, b), (name, np.argwhere(a != b)[:4].tolist(), a[a != b][:4], b[a != b][:4])
        for i, (t, a) in enumerate(zip(self.gp, self.p)):
            assert np.array_equal(t.cpu().numpy(), a), (i, float(np.abs(t.cpu().numpy() - a).max()))
            if self.gc is not None:
                assert torch.equal(self.gc[i].cpu(), torch.from_numpy(a).to(torch.bfloat16))


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("sizes", list(LISTS), ids=list(LISTS))
def test_steps_equal_the_oracle(bits, sizes):
    print("adamw case", bits, sizes, flush=True)
    s = _Set(LISTS[sizes], bits, 5 + bits)
    for step in range(1, 6):
        s.gradients()
        qerl.lora_adamw_step(s.plan, step=step, seed=0x1234_5678_9ABC_DEF0 + step, **HYPER)
        s.reference(step, 0x1234_5678_9ABC_DEF0 + step, **HYPER)
        s.check()


@pytest.mark.parametrize("bits", [8, 32])
def test_without_copies_far_steps_and_other_factors(bits):
    s = _Set([1000, 77], bits, 3, copies=False)
    h = dict(lr=1e-4, beta1=0.0, beta2=0.95, eps=1e-6, weight_decay=0.0)
    for step in (1, 2, 1000003, 2 ** 33 + 5):
        s.gradients(1e-6)
        qerl.lora_adamw_step(s.plan, step=step, seed=9, **h)
        s.reference(step, 9, **h)
        s.check()


@pytest.mark.parametrize("bits", [8, 32])
def test_clipping(bits):
    s = _Set([5000, 33, 2048], bits, 8)
    for step, max_norm in ((1, 0.5), (2, 1e9), (3, float("inf"))):
        s.gradients(0.1)
        norm, scale = qerl.lora_adamw_grad_norm(s.plan, max_norm)
        want = np.sqrt(sum((a.astype(np.float64) ** 2).sum() for a in s.g))
        # an fp64 sum of exact squares, rounded once to fp32: 2^-24, and the fp64 sum's own error far below
        assert abs(norm.item() - want) <= 2.0 ** -23 * want
        f = np.float32(min(1.0, max_norm / (want + 1e-6)))
        assert abs(scale.item() - f) <= 2.0 ** -23 * f
        qerl.lora_adamw_step(s.plan, step=step, seed=1, grad_scale=scale, **HYPER)
        s.reference(step, 1, grad_scale=scale.item(), **HYPER)
        s.check()


@pytest.mark.parametrize("bits", [8, 32])
def test_a_gradient_that_is_not_finite_leaves_everything(bits):
    s = _Set([3000, 40], bits, 4)
    s.gradients()
    qerl.lora_adamw_step(s.plan, step=1, seed=1, **HYPER)
    s.reference(1, 1, **HYPER)
    for bad in (float("inf"), float("nan")):
        s.gg[0][17] = bad
        norm, scale = qerl.lora_adamw_grad_norm(s.plan, 1.0)
        assert not np.isfinite(norm.item()) and np.isnan(scale.item())
        qerl.lora_adamw_step(s.plan, step=2, seed=1, grad_scale=scale, **HYPER)
        s.check()
    # without the factor: the element, with 8 bits its block of 32, is NaN from then on, the rest is not
    qerl.lora_adamw_step(s.plan, step=2, seed=1, **HYPER)
    m, v = qerl.lora_adamw_moments(s.plan) if bits == 8 else (s.plan.m, s.plan.v)
    nan = torch.isnan(m).cpu().numpy() & torch.isnan(v).cpu().numpy()
    assert np.array_equal(np.flatnonzero(nan), np.arange(0, 32) if bits == 8 else [17])


@pytest.mark.parametrize("bits", [8, 32])
def test_zeros_tiny_and_huge_gradients(bits):
    s = _Set([256], bits, 6)
    for step, a in enumerate(([0.0] * 256, [1e-30] * 100 + [0.0] * 156, [1e15, -1e15] * 128, [3e-20 * 2.0 ** (i % 40) for i in range(256)]), 1):
        s.g = [np.array(a, np.float32)]
        s.gg[0].copy_(torch.from_numpy(s.g[0]))
        qerl.lora_adamw_step(s.plan, step=step, seed=3, **HYPER)
        s.reference(step, 3, **HYPER)
        s.check()
        assert np.all(np.isfinite(s.p[0]))


def test_moments_in_8_bits_follow_a_steady_gradient():
    """g = 1 for 3000 steps: m goes to 1, v to 1 - 0.999^t.  A rounding is unbiased and off by less than a step, 2^-3 of the value at most, so
    by 2^-4 of it in the root mean square.  m remembers ten steps: sqrt(10 / 2) 2^-4 = 0.14 per element at most, over 4096 elements 0.22 %.  v
    remembers 1000, but in a step of 0.001 of its value it rounds the other way only once in 125 steps or more: 2^-3 sqrt(500 / 125) = 0.25
    per element at most, 0.4 % over 4096.  Five of those are allowed.  To nearest, m would stand at 0.75 and v below 0.03."""
    n = 4096
    g = torch.ones((n,), device="cuda")
    p = torch.zeros((n,), device="cuda")
    plan = qerl.lora_adamw_plan([p], [g], state_bits=8)
    for t in range(1, 3001):
        qerl.lora_adamw_step(plan, lr=0.0, step=t, seed=11)
    m, v = qerl.lora_adamw_moments(plan)
    assert abs(v.mean().item() / (1 - 0.999 ** 3000) - 1) < 0.02, v.mean().item()
    assert abs(m.mean().item() - 1) < 0.011, m.mean().item()


@pytest.mark.parametrize("bits", [8, 32])
def test_captured_step_with_rate_and_count_on_the_device(bits):
    a, b = _Set([3001, 64], bits, 20), _Set([3001, 64], bits, 20)
    lr, step = torch.tensor([0.0], device="cuda"), torch.tensor([0], device="cuda")
    out = (torch.empty((1,), device="cuda"), torch.empty((1,), device="cuda"))
    h = {k: v for k, v in HYPER.items() if k != "lr"}

    def work():
        step.add_(1)
        qerl.lora_adamw_grad_norm(a.plan, 0.3, out=out)
        qerl.lora_adamw_step(a.plan, lr_device=lr, step_device=step, seed=5, grad_scale=out[1], **h)
    graph = torch.cuda.CUDAGraph()
    a.gradients()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        work()
    a.rng, b.rng = np.random.default_rng(1), np.random.default_rng(1)
    for t in range(1, 5):
        a.gradients()
        b.gradients()
        rate = np.float32(1e-3 * t).item()
        lr.fill_(rate)
        graph.replay()
        torch.cuda.synchronize()
        _, scale = qerl.lora_adamw_grad_norm(b.plan, 0.3)
        qerl.lora_adamw_step(b.plan, lr=rate, step=t, seed=5, grad_scale=scale, **h)
        for x, y in zip((*a.gp, *a.gc, a.plan.m, a.plan.v), (*b.gp, *b.gc, b.plan.m, b.plan.v)):
            assert torch.equal(x, y)
    assert step.item() == 4


def test_state_given_by_the_caller_and_its_gaps():
    sizes = [33, 40]
    starts, total = uo.state_starts(sizes)
    m, v = torch.full((total,), 3.0, device="cuda"), torch.full((total,), 2.0, device="cuda")
    p, g = [torch.ones((n,), device="cuda") for n in sizes], [torch.ones((n,), device="cuda") for n in sizes]
    plan = qerl.lora_adamw_plan(p, g, state_bits=32, state=(m, v))
    qerl.lora_adamw_step(plan, lr=1e-3, step=5)
    inside = torch.zeros((total,), dtype=torch.bool)
    for n, at in zip(sizes, starts):
        inside[at:at + n] = True
    assert not bool(m.cpu()[~inside].any()) and not bool(v.cpu()[~inside].any()) and bool((m.cpu()[inside] > 2).all())


@pytest.mark.parametrize("bits", [8, 32])
def test_captured_values_that_the_host_would_refuse_change_nothing(bits):
    s = _Set([500], bits, 2, copies=False)
    s.gradients()
    lr, step = torch.tensor([1e-3], device="cuda"), torch.tensor([1], device="cuda")
    h = {k: v for k, v in HYPER.items() if k != "lr"}
    for bad_lr, bad_step in ((1e-3, 0), (1e-3, -5), (-1.0, 1), (float("nan"), 1), (float("inf"), 1)):
        lr.fill_(bad_lr)
        step.fill_(bad_step)
        qerl.lora_adamw_step(s.plan, lr_device=lr, step_device=step, **h)
        s.check()


def test_nothing_to_do():
    e = lambda: torch.empty((0,), device="cuda")
    for bits in (8, 32):
        plan = qerl.lora_adamw_plan([e(), e()], [e(), e()], state_bits=bits)
        qerl.lora_adamw_step(plan, lr=1e-3, step=1)
        norm, scale = qerl.lora_adamw_grad_norm(plan, 1.0)
        assert norm.item() == 0 and scale.item() == 1
    plan = qerl.lora_adamw_plan([e()], [e()])
    assert qerl.lora_adamw_moments(plan)[0].numel() == 0


def test_more_elements_than_32_bits_count():
    """2^31 + 40 elements of one tensor and a few of another behind it, constant but for marked places."""
    n = 2 ** 31 + 40
    p, g = torch.zeros((n,), device="cuda"), torch.full((n,), 2.0 ** -10, device="cuda")
    at = torch.tensor([0, 1, 2 ** 31 - 1, 2 ** 31, n - 1], device="cuda")
    g[at] = torch.tensor([0.5, -0.25, 0.125, -1.0, 0.75], device="cuda")
    p2, g2 = torch.ones((5,), device="cuda"), torch.full((5,), 0.5, device="cuda")
    plan = qerl.lora_adamw_plan([p, p2], [g, g2], state_bits=8)
    norm, scale = qerl.lora_adamw_grad_norm(plan, 1e9)
    want = ((n - 5) * 2.0 ** -20 + sum(x * x for x in (0.5, 0.25, 0.125, 1.0, 0.75)) + 5 * 0.25) ** 0.5
    assert abs(norm.item() - want) <= 2.0 ** -23 * want and scale.item() == 1
    qerl.lora_adamw_step(plan, step=1, seed=3, **HYPER)
    idx = torch.cat([at, torch.tensor([12345, 2 ** 31 + 7], device="cuda")])
    ref, m, v = uo.adamw(np.zeros(7), g[idx].cpu().numpy(), np.zeros(7), np.zeros(7), step=1, **HYPER)
    assert np.array_equal(p[idx].cpu().numpy(), ref)
    ref2, _, _ = uo.adamw(np.ones(5), g2.cpu().numpy(), np.zeros(5), np.zeros(5), step=1, **HYPER)
    assert np.array_equal(p2.cpu().numpy(), ref2)
    # moments: within one rounding up of a step of 2^-3, and the first block against the oracle with its random bits
    u = uo.random_fractions(32, 1, 3)
    first = np.full(32, 2.0 ** -10, np.float32)
    first[:2] = 0.5, -0.25
    _, m, v = uo.adamw(np.zeros(32), first, np.zeros(32), np.zeros(32), step=1, **HYPER)
    c, f = uo.encode_first(m, u)
    assert np.array_equal(plan.m[:32].cpu().numpy(), c) and plan.m_scale[0].item() == f[0]
    last = 2 ** 31 // 32                                                    # the block that begins at 2^31
    assert plan.m_scale[last].item() == int(np.float32(np.float32(0.1) * np.float32(1.0)).view(np.uint32) >> 23)
    assert bool((plan.m[n:2 ** 31 + 64] == 0).all())


def test_binding_refusals():
    t = lambda n=8, dt=torch.float32: torch.zeros((n,), dtype=dt, device="cuda")
    for bad in (lambda: qerl.lora_adamw_plan([t()], [t(9)]), lambda: qerl.lora_adamw_plan([t(), t()], [t()]), lambda: qerl.lora_adamw_plan([t()], [t()], state_bits=16),
                lambda: qerl.lora_adamw_plan([t()], [t()], [t(4, torch.bfloat16)]), lambda: qerl.lora_adamw_plan([t(16)[::2]], [t()]),
                lambda: qerl.lora_adamw_plan([t()], [t()], state_bits=8, state=(t(32), t(32))),
                lambda: qerl.lora_adamw_step(qerl.lora_adamw_plan([t()], [t()]), step=1), lambda: qerl.lora_adamw_step(qerl.lora_adamw_plan([t()], [t()]), lr=1.0)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: qerl.lora_adamw_plan([t(8, torch.bfloat16)], [t()]), lambda: qerl.lora_adamw_plan([t()], [t(8, torch.float64)]),
                lambda: qerl.lora_adamw_plan([t()], [t()], state_bits=32, state=(t(32, torch.uint8), t(32)))):
        with pytest.raises(TypeError):
            bad()
    p = t()
    for bad in (lambda: qerl.lora_adamw_plan([p, p], [t(), t()]), lambda: qerl.lora_adamw_plan([p], [p]),
                lambda: qerl.lora_adamw_step(qerl.lora_adamw_plan([t()], [t()]), lr=1e-3, step=0), lambda: qerl.lora_adamw_grad_norm(qerl.lora_adamw_plan([t()], [t()]), 0.0)):
        with pytest.raises(qerl.QerlError):
            bad()


def test_update_of_a_policy_with_the_operators_around_its_linears():
    """One update as a program makes it: log-probabilities and slope of the head, their gradient through an NVFP4 + LoRA linear, clipping,
    AdamW on A and B, whose bf16 copies the next forward pass reads.  The gradients against an fp64 evaluation of the same chain (the
    linear's output is rounded to bf16 between the two), the step against the oracle on the gradients of the GPU."""
    import qerl_synth as qs
    from oracle import nvfp4_oracle as oracle
    M, K, H, V, r, scale = 70, 256, 128, 1500, 8, 2.0
    codes, scales, ts = oracle.nvfp4_quantize(qs.weights(H, K, 1).float().numpy())
    g = lambda a: torch.from_numpy(a).cuda()
    w, wt = (f(g(codes), g(scales), torch.tensor([ts], device="cuda")) for f in (qerl.nvfp4_prepack, qerl.nvfp4_prepack_t))
    A0, B0 = qs.lora_pair(H, K, r, 2, b_std=0.05)
    A, B = A0.cuda(), B0.cuda()
    x = qs.activations(M, K, 3).cuda()
    head = qerl.lm_head_prepack((torch.randn((V, H), generator=torch.Generator().manual_seed(4)) * 0.1).to(torch.bfloat16).cuda())
    t = torch.randint(0, V, (M,), generator=torch.Generator().manual_seed(5))
    weight = torch.randn((M,), generator=torch.Generator().manual_seed(6))
    master = [A.float().flatten(), B.float().flatten()]
    dA, dB = torch.empty((r, K), device="cuda"), torch.empty((H, r), device="cuda")
    plan = qerl.lora_adamw_plan(master, [dA.flatten(), dB.flatten()], [A.flatten(), B.flatten()], state_bits=8)
    y = qerl.nvfp4_lora_linear_packed(x, w, A, B, scale)
    lp, _, _, slope = qerl.lm_head_logprob_grad(y, head, t.cuda())
    dy = qerl.lm_head_logprob_backward(weight.cuda(), slope)
    dx, _, _ = qerl.nvfp4_lora_linear_backward(x, dy, wt, A, B, scale, dA=dA, dB=dB)
    # gradients from the definitions in fp64
    slope64 = uo.head_logprob(y.float().cpu().numpy(), head.weight.float().cpu().numpy(), t.numpy())[3]
    dy64 = weight.double().numpy()[:, None] * slope64
    _, dA64, dB64 = oracle.nvfp4_lora_linear_backward(x.float().cpu().numpy(), dy64, codes, scales, ts, A0.float().numpy(), B0.float().numpy(), scale)
    # dy is off by 2^-8 of itself twice (its own rounding, the weights'), so are sums over its elements at most: 2^-7 of the sums of magnitudes
    magA = scale * np.abs(np.abs(dy64) @ np.abs(B0.double().numpy())).T @ np.abs(x.double().cpu().numpy())
    magB = scale * np.abs(dy64).T @ np.abs(x.double().cpu().numpy() @ A0.double().numpy().T)
    E = np.abs(weight.double().numpy())[:, None] * (np.abs(slope64) + np.abs(head.weight.double().cpu().numpy()).max())
    magA += scale * (E @ np.abs(B0.double().numpy())).T @ np.abs(x.double().cpu().numpy())
    magB += scale * E.T @ np.abs(x.double().cpu().numpy() @ A0.double().numpy().T)
    assert np.all(np.abs(dA.double().cpu().numpy() - dA64) <= 2.0 ** -7 * magA)
    assert np.all(np.abs(dB.double().cpu().numpy() - dB64) <= 2.0 ** -7 * magB)
    assert np.linalg.norm(dA.double().cpu().numpy() - dA64) <= 2.0 ** -7 * np.linalg.norm(dA64)
    assert np.linalg.norm(dB.double().cpu().numpy() - dB64) <= 2.0 ** -7 * np.linalg.norm(dB64)
    # the step
    before = [m.cpu().numpy().copy() for m in master]
    norm, factor = qerl.lora_adamw_grad_norm(plan, 0.5)
    qerl.lora_adamw_step(plan, step=1, seed=7, grad_scale=factor, **HYPER)
    for p0, d, m, c in zip(before, (dA, dB), master, (A, B)):
        want, _, _ = uo.adamw(p0, d.flatten().cpu().numpy(), np.zeros_like(p0), np.zeros_like(p0), step=1, grad_scale=factor.item(), **HYPER)
        assert np.array_equal(m.cpu().numpy(), want) and torch.equal(c.flatten().cpu(), torch.from_numpy(want).to(torch.bfloat16))
    # the next forward pass reads the updated copies
    y2 = qerl.nvfp4_lora_linear_packed(x, w, A, B, scale)
    ref = oracle.nvfp4_lora_linear(x.float().cpu().numpy(), codes, scales, ts, A.float().cpu().numpy(), B.float().cpu().numpy(), scale)
    from tests.gpu_util import check_linear
    check_linear(y2, ref, "after the step")


@pytest.mark.parametrize("bits", [8, 32])
def test_captured_values_whose_factors_fp32_does_not_hold_change_nothing(bits):
    s = _Set([500], bits, 2, copies=False)
    s.gradients()
    lr, step = torch.tensor([3e38], device="cuda"), torch.tensor([1], device="cuda")
    for kw in (dict(beta1=0.9), dict(beta1=0.0, weight_decay=10.0)):                     # lr / (1 - b1^t), 1 - lr wd
        qerl.lora_adamw_step(s.plan, lr_device=lr, step_device=step, **kw)
        s.check()
    lr.fill_(HYPER["lr"])                                                                # the same step counts once they can be held
    s.reference(1, 0, **{**HYPER, "lr": lr.item()})
    qerl.lora_adamw_step(s.plan, lr_device=lr, step_device=step, **{k: v for k, v in HYPER.items() if k != "lr"})
    s.check()


@pytest.mark.parametrize("bits", [8, 32])
def test_the_smallest_eps_leaves_elements_without_a_gradient(bits):
    s = _Set([300], bits, 3)
    s.g = [np.zeros(300, np.float32)]
    s.gg[0].zero_()
    h = {**HYPER, "eps": 1e-45}
    qerl.lora_adamw_step(s.plan, step=1, seed=1, **h)
    s.reference(1, 1, **h)
    s.check()
    assert np.all(np.isfinite(s.p[0]))
    with pytest.raises(qerl.QerlError):
        qerl.lora_adamw_step(s.plan, step=2, seed=1, **{**HYPER, "eps": 1e-46})


def test_a_state_on_memory_of_the_tensors_is_refused():
    flat = torch.zeros((4096,), device="cuda")
    cut = lambda a, n: flat[a:a + n]
    other = lambda n, dt=torch.float32: torch.zeros((n,), dtype=dt, device="cuda")
    p, g, c = cut(0, 64), cut(64, 64), other(64, torch.bfloat16)
    byte = flat.view(torch.uint8)
    for state in ((cut(0, 64), other(64)), (other(64), cut(0, 64)), (cut(64, 64), other(64)), (other(64), cut(100, 64)), (cut(60, 64), other(64))):
        with pytest.raises(qerl.QerlError):
            qerl.lora_adamw_plan([p], [g], [c], state_bits=32, state=state)
    e = lambda n: other(n, torch.uint8)
    for state in ((byte[240:304], e(64), e(2), e(2)), (e(64), byte[256:320], e(2), e(2)), (e(64), e(64), byte[255:257], e(2)), (e(64), e(64), e(2), byte[511:513]),
                  (e(64), e(64), e(2), c.view(torch.uint8)[126:128])):
        with pytest.raises(qerl.QerlError):
            qerl.lora_adamw_plan([p], [g], [c], state_bits=8, state=state)
    assert not bool(flat.any())
    # beside them it works: everything in one buffer
    g.fill_(1.0)
    plan = qerl.lora_adamw_plan([p], [g], [c], state_bits=32, state=(cut(128, 64), cut(192, 64)))
    qerl.lora_adamw_step(plan, lr=1e-3, step=1)
    assert bool((flat[:64] < 0).all()) and bool((flat[128:256] > 0).all()) and not bool(flat[256:].any())


def test_moments_in_8_bits_at_the_end_of_the_range_stay_finite():
    """Moments between 1.875 2^127 and 2^128, over seeds that round most of them up: with beta2 = 0 the second is g^2, with beta1 = 0 the first g."""
    h = dict(lr=0.0, eps=1e-8, weight_decay=0.0, step=1)
    edge = np.float32(1.875 * 2.0 ** 127)
    for seed in range(3):
        s = _Set([256], 8, 9)
        s.g = [np.sqrt(np.linspace(0.90, 0.9999, 256) * np.float64(np.finfo(np.float32).max)).astype(np.float32) * (np.arange(256) % 2 * 2 - 1).astype(np.float32)]
        s.gg[0].copy_(torch.from_numpy(s.g[0]))
        b = dict(h, beta1=0.9, beta2=0.0, seed=seed)
        qerl.lora_adamw_step(s.plan, **b)
        s.reference(**b)
        s.check()
        assert s.v.max() == edge and (s.v == edge).sum() > 100
        # the first (g^2 is infinite then, so the second and the parameters are not of this world)
        s = _Set([256], 8, 9, copies=False)
        g = (np.linspace(1.75, 1.99, 256) * 2.0 ** 127).astype(np.float32) * (np.arange(256) % 2 * 2 - 1).astype(np.float32)
        s.gg[0].copy_(torch.from_numpy(g))
        qerl.lora_adamw_step(s.plan, beta1=0.0, beta2=0.9, seed=seed, **h)
        want = uo.decode(*uo.encode_first(g, uo.random_fractions(256, 1, seed)), 4)
        got = qerl.lora_adamw_moments(s.plan)[0].cpu().numpy()
        assert np.array_equal(got, want) and np.abs(got).max() == edge
