"""Cases for the operators at the two ends of a policy update: the head's log-probabilities with their gradient, and the
AdamW step on the adapters.

A case is a dict of plain values; `prepare` makes what a program holds before the call, `run` is one pass: in elementary torch
operations where `own` is false, through the library's entry points where it is true.  `exact` computes the same results in
64 bits from the definitions.

Kinds
    logprob   log-probability of one token per row under the language-model head, log-sum-exp and entropy
    train     the same with the gradient with respect to the hidden states for a given upstream gradient
    adamw     one optimizer step over the LoRA matrices of a stack of decoder layers: clipping norm, then the update of fp32
              master weights, their bf16 copies and the moments (32 bits, or 8 bits with a scale per block of 32)
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

VOCAB = 152064                                   # the vocabulary of the benchmark's models
# widths of the 7B and 14B shapes of the benchmark: hidden, k/v, intermediate
SHAPE_7B = dict(hidden=3584, kv=512, inter=18944)
SHAPE_14B = dict(hidden=5120, kv=1024, inter=13824)


def listed():
    return [
        # scoring one sampled token while a single sequence is decoded: nothing but the head's bytes
        dict(name="logprob 7b m1", kind="logprob", M=1, V=VOCAB, H=3584, entropy=False, masked=0.0, inv_t=1.0),
        # a decode batch of 16, with the entropy that the exploration study records
        dict(name="logprob 7b m16", kind="logprob", M=16, V=VOCAB, H=3584, entropy=True, masked=0.0, inv_t=1.0),
        # a vocabulary and a batch that no tile divides
        dict(name="logprob odd m77", kind="logprob", M=77, V=50257, H=2048, entropy=True, masked=0.1, inv_t=1.25),
        # old-policy log-probabilities of a full batch on the largest shapes
        dict(name="logprob 32b m4096", kind="logprob", M=4096, V=VOCAB, H=5120, entropy=True, masked=0.0, inv_t=1.0),
        # a small model's update: few tokens, an odd vocabulary
        dict(name="train small m200", kind="train", M=200, V=32001, H=1024, entropy=False, masked=0.0, inv_t=1.0),
        # a few uneven completions packed together, a quarter of the rows prompt or padding
        dict(name="train 7b m777", kind="train", M=777, V=VOCAB, H=3584, entropy=True, masked=0.25, inv_t=1.0),
        # the policy update on the largest shapes
        dict(name="train 32b m4096", kind="train", M=4096, V=VOCAB, H=5120, entropy=True, masked=0.0, inv_t=1.0),
        # a toy stack whose tensors have odd sizes: launch latency
        dict(name="adamw8 small", kind="adamw", bits=8, layers=2, r=5, clip=True, hidden=1001, kv=130, inter=2717),
        # adapters of rank 32 on all 28 layers, 8-bit moments, clipped
        dict(name="adamw8 7b r32", kind="adamw", bits=8, layers=28, r=32, clip=True, **SHAPE_7B),
        # one layer's adapters, 32-bit moments, without clipping
        dict(name="adamw32 layer r16", kind="adamw", bits=32, layers=1, r=16, clip=False, **SHAPE_7B),
        # rank 16 on 48 layers, 32-bit moments, clipped
        dict(name="adamw32 14b r16", kind="adamw", bits=32, layers=48, r=16, clip=True, **SHAPE_14B),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, round(lo * (hi / lo) ** rng.random())))


def draw(rng):
    kind = rng.choice(["logprob", "logprob", "logprob", "train", "train", "adamw", "adamw"])
    if kind == "adamw":
        h = rng.randint(128, 4096)
        return dict(kind=kind, bits=rng.choice([8, 32]), layers=_log_int(rng, 1, 16), r=rng.choice([3, 8, 16, 32, 64]), clip=rng.random() < 0.5,
                    hidden=h, kv=rng.randint(32, max(32, h // 4)), inter=round(h * rng.uniform(2.6, 5.4)))
    return dict(kind=kind, M=_log_int(rng, 1, 4096), V=_log_int(rng, 2000, VOCAB), H=8 * rng.randint(32, 640),
                entropy=rng.random() < 0.5, masked=rng.choice([0.0, 0.0, 0.2, 0.6]), inv_t=rng.choice([1.0, 1.0, 1.25, 0.7]))


def _tensors(case):
    """Sizes of the adapters' matrices, A [r, K] and B [N, r] of the seven linears of each layer."""
    h, kv, i, r = case["hidden"], case["kv"], case["inter"], case["r"]
    lin = [(h, h), (kv, h), (kv, h), (h, h), (i, h), (i, h), (h, i)]
    return [n for _ in range(case["layers"]) for N, K in lin for n in (r * K, r * N)]


class _State:
    pass


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = _State()
    s.case, s.seed = case, seed
    if case["kind"] == "adamw":
        return _prepare_adamw(s, gen)
    M, V, H = case["M"], case["V"], case["H"]
    s.W = torch.empty((V, H), dtype=torch.bfloat16, device="cuda")
    s.W.copy_(torch.randn((V, H), generator=gen, device="cuda") * 0.02)
    s.targets = torch.randint(0, V, (M,), generator=gen, device="cuda")
    # normalised hidden states that point towards their token's row by different amounts: its logit rises by up to 18, from a token that
    # the policy would hardly sample to one that it is sure of
    sure = 900.0 / H * torch.rand((M, 1), generator=gen, device="cuda")
    x = torch.randn((M, H), generator=gen, device="cuda") + sure * s.W[s.targets].float() / 0.02
    s.x = x.to(torch.bfloat16)
    s.targets = torch.where(torch.rand((M,), generator=gen, device="cuda") < case["masked"], torch.full_like(s.targets, -100), s.targets)
    s.grad = torch.randn((M,), generator=gen, device="cuda") / M           # of the loss with respect to each log-probability
    if own:
        import paper_2510_11696_amd as qerl
        s.head = qerl.lm_head_prepack(s.W, gradient=case["kind"] == "train")
        s.ws = qerl.lm_head_workspace(M, V, H, gradient=case["kind"] == "train")
    return s


def _prepare_adamw(s, gen):
    case = s.case
    sizes = _tensors(case)
    starts, total = [], 0
    for n in sizes:
        starts.append(total)
        total += -(-n // 32) * 32
    # every flat buffer holds the tensors one after the other, each from a multiple of 32 elements; the gaps stay zero
    ends = torch.tensor([a + n for a, n in zip(starts, sizes)], device="cuda")
    at = torch.arange(total, device="cuda")
    owner = torch.bucketize(at, torch.tensor(starts, device="cuda"), right=True) - 1
    inside = (at < ends[owner]).float()
    scale = torch.exp(torch.randn((len(sizes),), generator=gen, device="cuda"))[owner] * 1e-3 * inside
    del at, owner
    s.p = torch.randn((total,), generator=gen, device="cuda") * 0.05 * inside
    s.copy = s.p.to(torch.bfloat16)
    spread = torch.exp(torch.randn((total,), generator=gen, device="cuda"))
    s.g = torch.randn((total,), generator=gen, device="cuda") * scale * spread
    m = torch.randn((total,), generator=gen, device="cuda") * 0.3 * scale * spread
    v = (scale * spread).square() * (0.5 + torch.rand((total,), generator=gen, device="cuda"))
    s.total, s.step = total, 100
    s.hyper = dict(lr=1e-5, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01)
    s.max_norm = 1.0
    if case["bits"] == 8:
        half = torch.full((total,), 32768, device="cuda")
        (s.m, s.m_scale), (s.v, s.v_scale) = _encode(m, half, True), _encode(v, half, False)
    else:
        s.m, s.v, s.m_scale, s.v_scale = m, v, None, None
    if own:
        import paper_2510_11696_amd as qerl
        cut = lambda flat: [flat[a:a + n] for a, n in zip(starts, sizes)]
        s.plan = qerl.lora_adamw_plan(cut(s.p), cut(s.g), cut(s.copy), state_bits=case["bits"],
                                      state=(s.m, s.v, s.m_scale, s.v_scale) if case["bits"] == 8 else (s.m, s.v))
    return s


def run(s):
    return {"logprob": _logprob, "train": _train, "adamw": _adamw}[s.case["kind"]](s)


# ---- the head ------------------------------------------------------------------------------------------------------------
def _softmax_rows(s):
    """Logits, row maxima, e^(z - max), and in 64 bits their sums over the row and over what is not the row's own token (next to
    which the rest of a sure row would be lost in 32)."""
    z = (s.x.float() @ s.W.float().t()) * s.case["inv_t"]
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    at = s.targets.clamp(min=0)[:, None]
    rest = e.scatter(1, at, 0.0).sum(1, keepdim=True, dtype=torch.float64)
    return z, top, e, rest, rest + e.gather(1, at)


def _row_results(s, z, top, e, rest, total):
    taken = s.targets >= 0
    zt = z.gather(1, s.targets.clamp(min=0)[:, None])
    got = [-torch.log1p(rest * torch.exp(top - zt)), torch.log(total) + top]
    if s.case["entropy"]:
        got.append(torch.log(total) - (e * (z - top)).sum(1, keepdim=True, dtype=torch.float64) / total)
    return [(g[:, 0] * taken).to(torch.float32) for g in got]


def _logprob(s):
    if own:
        import paper_2510_11696_amd as qerl
        logp, lse, ent = qerl.lm_head_logprob(s.x, s.head, s.targets, inv_temperature=s.case["inv_t"], entropy=s.case["entropy"], workspace=s.ws)
        return [logp, lse] + ([ent] if s.case["entropy"] else [])
    return _row_results(s, *_softmax_rows(s))


def _train(s):
    if own:
        import paper_2510_11696_amd as qerl
        logp, lse, ent, slope = qerl.lm_head_logprob_grad(s.x, s.head, s.targets, inv_temperature=s.case["inv_t"], entropy=s.case["entropy"], workspace=s.ws)
        return [logp, lse] + ([ent] if s.case["entropy"] else []) + [qerl.lm_head_logprob_backward(s.grad, slope)]
    z, top, e, rest, total = _softmax_rows(s)
    got = _row_results(s, z, top, e, rest, total)
    d = e.div_(-total.to(torch.float32))
    d.scatter_(1, s.targets.clamp(min=0)[:, None], (rest / total).to(torch.float32))
    d *= (s.grad * (s.targets >= 0) * s.case["inv_t"])[:, None]
    return got + [(d @ s.W.float()).to(torch.bfloat16)]


# ---- the optimizer -------------------------------------------------------------------------------------------------------
# Moments in 8 bits: blocks of 32 elements share a scale byte, the exponent field of the block's largest magnitude as fp32 (at
# least 1; 255 for a block that is not finite).  The first moment has a sign, four exponent and three mantissa bits, the second five and
# three and never becomes 0; both are rounded up with the probability of what is cut off (16 random bits per element, for both).
# What is rounded is the moment in fp32, every operation of its update rounded by itself.
def _encode(x, random16, first):
    mag = x.abs().view(-1, 32)
    field = (mag.amax(1).view(torch.int32) >> 23).clamp(min=1)
    lift = ((14 if first else 30) - field).double()[:, None]
    bits = (mag.double() * torch.exp2(lift)).to(torch.float32).view(torch.int32)
    code = (bits + (random16.view(-1, 32).to(torch.int32) << 4)) >> 20
    if first:
        code = code | ((x.view(-1, 32) < 0).to(torch.int32) << 7)
    else:
        code = torch.where(mag > 0, code.clamp(min=1), torch.zeros_like(bits))
    return code.to(torch.uint8).view(-1), field.to(torch.uint8)


def _decode(code, field, first):
    c = code.view(-1, 32).to(torch.int32)
    drop = (field.to(torch.int32) - (14 if first else 30)).double()[:, None]
    mag = ((c & 127 if first else c) << 20).view(torch.float32).double() * torch.exp2(drop)
    mag = torch.where(c > 127, -mag, mag) if first else mag
    return mag.to(torch.float32).view(-1)


def _round_keys(c0, c1, c2, c3, k0, k1):
    """One round of Philox4x32 on 32-bit words held in int64."""
    a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
    return ((b >> 32) & 0xFFFFFFFF) ^ c1 ^ k0, b & 0xFFFFFFFF, ((a >> 32) & 0xFFFFFFFF) ^ c3 ^ k1, a & 0xFFFFFFFF


def _random16(total, step, seed):
    """16 random bits per element: group b of eight elements takes the four words of the counter (b, step) under the key `seed`."""
    b = torch.arange(total // 8, device="cuda")
    c = (b & 0xFFFFFFFF, b >> 32, torch.full_like(b, step & 0xFFFFFFFF), torch.full_like(b, step >> 32))
    for i in range(10):
        c = _round_keys(*c, ((seed & 0xFFFFFFFF) + i * 0x9E3779B9) & 0xFFFFFFFF, ((seed >> 32) + i * 0xBB67AE85) & 0xFFFFFFFF)
    words = torch.stack(c, 1)
    return torch.stack((words & 0xFFFF, words >> 16), 2).view(-1)


def _adamw(s):
    h, case = s.hyper, s.case
    s.step += 1
    if own:
        import paper_2510_11696_amd as qerl
        norm, factor = qerl.lora_adamw_grad_norm(s.plan, s.max_norm) if case["clip"] else (None, None)
        qerl.lora_adamw_step(s.plan, step=s.step, seed=s.seed, grad_scale=factor, **h)
        m, v = qerl.lora_adamw_moments(s.plan) if case["bits"] == 8 else (s.m, s.v)
        return [s.p, s.copy, m, v] + ([norm] if case["clip"] else [])
    m, v, g = s.m, s.v, s.g
    if case["bits"] == 8:
        m, v = _decode(s.m, s.m_scale, True), _decode(s.v, s.v_scale, False)
    norm = None
    if case["clip"]:
        long = s.g.double().square().sum().sqrt()
        norm = long.to(torch.float32).view(1)
        g = g * (s.max_norm / (long + 1e-6)).clamp(max=1.0).to(torch.float32)
    m = h["beta1"] * m + (1.0 - h["beta1"]) * g
    v = h["beta2"] * v + (1.0 - h["beta2"]) * (g * g)
    root = torch.sqrt(v) * (1.0 / math.sqrt(1.0 - h["beta2"] ** s.step)) + h["eps"]
    s.p.copy_(s.p * (1.0 - h["lr"] * h["weight_decay"]) - (h["lr"] / (1.0 - h["beta1"] ** s.step)) * m / root)
    s.copy.copy_(s.p)
    if case["bits"] == 8:
        random16 = _random16(s.total, s.step, s.seed)
        (s.m, s.m_scale), (s.v, s.v_scale) = _encode(m, random16, True), _encode(v, random16, False)
        m, v = _decode(s.m, s.m_scale, True), _decode(s.v, s.v_scale, False)
    else:
        s.m.copy_(m)
        s.v.copy_(v)
    return [s.p, s.copy, m, v] + ([norm] if case["clip"] else [])


# ---- what a pass cannot do without -----------------------------------------------------------------------------------------
def work(case):
    if case["kind"] == "adamw":
        n = sum(_tensors(case))
        # gradient, master weight in and out, copy out; moments in and out; the moments as values where they are held in 8 bits
        per = 4 + 8 + 2 + (16 if case["bits"] == 32 else 4 + 4 / 32 + 8)
        return {"bytes": n * (per + (4 if case["clip"] else 0)), "flops": 15 * n}
    M, V, H = case["M"], case["V"], case["H"]
    rows = M * (8 + 8 + (4 if case["entropy"] else 0))
    if case["kind"] == "logprob":
        return {"bytes": 2 * V * H + 2 * M * H + rows, "flops": 2 * M * V * H}
    return {"bytes": 2 * V * H + 2 * M * H + 2 * M * H + rows + 4 * M, "flops": 4 * M * V * H}


# ---- 64 bits ---------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "adamw":
        return _exact_adamw(s)
    W = s.W.double()
    logp, lse, ent, dx = [], [], [], []
    for x, t, g in zip(s.x.split(512), s.targets.split(512), s.grad.split(512)):
        z = torch.matmul(x.double(), W.t()) * case["inv_t"]
        n = torch.logsumexp(z, 1)
        p = torch.exp(z - n[:, None])
        keep, row = t >= 0, torch.arange(len(t), device="cuda")
        lse.append(n * keep)
        logp.append((z[row, t.clamp(min=0)] - n) * keep)
        ent.append((n - (p * z).sum(1)) * keep)
        if case["kind"] == "train":
            want = s.W[t.clamp(min=0)].double() - torch.matmul(p, W)
            dx.append(want * (case["inv_t"] * g.double() * keep)[:, None])
    got = [torch.cat(logp), torch.cat(lse)] + ([torch.cat(ent)] if case["entropy"] else [])
    return got + ([torch.cat(dx)] if dx else [])


def _exact_adamw(s):
    h, eight, t = s.hyper, s.case["bits"] == 8, s.step + 1

    def grid(x, low):
        """Exponent of each block of 32, and the spacing of the 8-bit values around each element."""
        _, top = torch.frexp(x.abs().view(-1, 32).amax(1, keepdim=True))
        _, here = torch.frexp(x.abs().view(-1, 32))
        top = torch.where(x.abs().view(-1, 32).amax(1, keepdim=True) > 0, top, torch.full_like(top, -200))
        return torch.exp2(torch.maximum(here - 1, top - 1 - low).double() - 3).view(-1)

    def value(code, field, exponent_bits):
        top, signed = 2 ** exponent_bits - 2, exponent_bits == 4
        table = []
        for c in range(256):
            e, frac = (c & 127 if signed else c) >> 3, (c & 7) / 8.0
            mag = (1 + frac) * 2.0 ** (e - top) if e else frac * 2.0 ** (1 - top)
            table.append(-mag if signed and c > 127 else mag)
        one = torch.tensor(table, dtype=torch.float64, device="cuda")[code.long()]
        return (one.view(-1, 32) * torch.exp2(field.double() - 127)[:, None]).view(-1)

    m, v = (value(s.m, s.m_scale, 4), value(s.v, s.v_scale, 5)) if eight else (s.m.double(), s.v.double())
    # 8-bit moments are defined by the roundings of their update to fp32; everything else is left unrounded
    f32 = (lambda x: x.to(torch.float32).double()) if eight else (lambda x: x)
    const = (lambda x: float(np.float32(x))) if eight else (lambda x: x)
    g = s.g.double()
    norm = torch.sqrt(torch.dot(g, g)).view(1)
    if s.case["clip"]:
        g = f32(g * f32(torch.clamp(s.max_norm / (norm + 1e-6), max=1.0)))
    m = f32(f32(const(h["beta1"]) * m) + f32(const(1 - h["beta1"]) * g))
    v = f32(f32(const(h["beta2"]) * v) + f32(const(1 - h["beta2"]) * f32(g * g)))
    p = s.p.double()
    p = p - h["lr"] * h["weight_decay"] * p - h["lr"] * (m / (1 - h["beta1"] ** t)) / (torch.sqrt(v / (1 - h["beta2"] ** t)) + h["eps"])
    if eight:
        fraction = torch.from_numpy(_uniform(s.total, t, s.seed)).cuda()
        step = grid(m, 13)
        m = torch.floor(m.abs() / step + fraction) * step * torch.sign(m)
        step = grid(v, 29)
        up = torch.floor(v / step + fraction)
        v = torch.where(v > 0, up.clamp(min=1) * step, torch.zeros_like(v))
    return [p, p, m, v] + ([norm] if s.case["clip"] else [])


def _uniform(total, step, seed):
    """The random fractions as multiples of 2^-16, from the generator's definition on unsigned words."""
    word = lambda v: np.uint64(v & 0xFFFFFFFF)
    at = np.arange(total // 8, dtype=np.uint64)
    x = [at & word(-1), at >> np.uint64(32), np.full_like(at, word(step)), np.full_like(at, word(step >> 32))]
    key = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        p, q = x[0] * word(0xD2511F53), x[2] * word(0xCD9E8D57)
        x = [(q >> np.uint64(32)) ^ x[1] ^ word(key[0]), q & word(-1), (p >> np.uint64(32)) ^ x[3] ^ word(key[1]), p & word(-1)]
        key = [(key[0] + 0x9E3779B9) & 0xFFFFFFFF, (key[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack([half for w in x for half in (w & np.uint64(0xFFFF), w >> np.uint64(16))], 1).reshape(-1).astype(np.float64) / 65536.0
