"""GPU parity of the head's log-probabilities, their slope and the backward, against the fp64 oracle.

Tolerances, derived from the arithmetic.  With u = 2^-24 and B = the most that a logit can be off:
  a logit is a sum of H exact products in fp32, taken 16 at a time over at most H / 16 steps (and a few more that join parts): every
  product passes at most H / 16 + 24 roundings, so B <= (H / 16 + 24) u (T^-1 max_v sum_k |x_k W_vk|); the scaling to powers of two adds
  4 u max |z|;
  D = 2 (B + 4 u max |z|) bounds the error of a difference of logits, 2^-17 the relative error of a sum of exponentials (at most
  128 roundings of positive terms, exp2 among them);
  logprob = -ln(1 + o): d ln(1 + o) = (1 - p) d ln o, so |error| <= (D + 2^-17) min(1, |logprob|) + 2^-22 |logprob|;
  lse <= D + 2^-17 + 2^-22 |lse|;  entropy: both terms' errors, weights off by D + 2^-17 each: (D + 2^-16) (2 + max |z - lse|);
  slope: (1 - p_t) and the weights p_v off by D + 2^-16, the weights rounded to bf16 (2^-8) besides, and the sum over v in fp32
  with at most V / 16 + 64 roundings: T^-1 [ (D + 2^-16) (1 - p_t) |W_t| + (2^-8 + D + 2^-16 + (V / 16 + 64) u) sum p_v |W_v| ];
  dx: one more rounding to bf16, 2^-8 |dx|."""
import numpy as np
import pytest
import torch

import paper_2510_11696_amd as qerl
from oracle import update_oracle as uo

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _inputs(M, V, H, seed, sure=12.0, ldx=0, ldw=0):
    g = torch.Generator().manual_seed(seed)
    W = (torch.randn((V, H), generator=g) * 0.02 * (4096.0 / H) ** 0.5).to(torch.bfloat16)
    t = torch.randint(0, V, (M,), generator=g)
    pull = sure / (0.02 * (4096.0 / H) ** 0.5 * H) * torch.rand((M, 1), generator=g)
    x = (torch.randn((M, H), generator=g) + pull * W[t].float() / (0.02 * (4096.0 / H) ** 0.5)).to(torch.bfloat16)

    def strided(a, ld):
        if not ld:
            return a.cuda()
        buf = torch.full((a.shape[0], ld), float("nan"), dtype=torch.bfloat16)        # what lies between the rows is never used
        buf[:, :a.shape[1]] = a
        return buf.cuda()[:, :a.shape[1]]
    return strided(x, ldx), strided(W, ldw), t


def _bounds(x, W, t, inv_t, H, V):
    x, W = x.double().cpu().numpy(), W.double().cpu().numpy()
    z = inv_t * (x @ W.T)
    B = (H / 16 + 24) * U * inv_t * (np.abs(x) @ np.abs(W).T).max(1)
    D = 2 * (B + 4 * U * np.abs(z).max(1))
    lp, lse, ent, slope = uo.head_logprob(x, W, t, inv_t)
    tol_lp = (D + 2.0 ** -17) * np.minimum(1, np.abs(lp)) + 2.0 ** -22 * np.abs(lp)
    tol_lse = D + 2.0 ** -17 + 2.0 ** -22 * np.abs(lse)
    tol_ent = (D + 2.0 ** -16) * (2 + np.abs(z - lse[:, None]).max(1))
    p = np.exp(z - lse[:, None])
    at = np.clip(t, 0, V - 1)
    p[np.arange(len(t)), at] = 0
    D = D[:, None]
    tol_slope = inv_t * ((D + 2.0 ** -16) * p.sum(1, keepdims=True) * np.abs(W[at]) + (2.0 ** -8 + D + 2.0 ** -16 + (V / 16 + 64) * U) * (p @ np.abs(W)))
    return (lp, lse, ent, slope), (tol_lp, tol_lse, tol_ent, tol_slope)


def _check(got, ref, tol, keep, what):
    for name, a, r, e in zip(("logprob", "lse", "entropy", "slope"), got, ref, tol):
        if a is None:
            continue
        a = a.double().cpu().numpy()[keep]
        off = np.abs(a - r[keep]) - e[keep]
        assert np.all(np.isfinite(a)) and np.all(off <= 0), (what, name, float(off.max()), np.argwhere(~(off <= 0))[:4].tolist())


SHAPES = [(1, 1, 8), (1, 2, 64), (3, 63, 72), (16, 64, 64), (17, 65, 128), (31, 1000, 256), (33, 2049, 520), (64, 257, 1024), (65, 4097, 64), (100, 3001, 136),
          (129, 1500, 264), (200, 777, 96), (255, 5001, 64), (256, 256, 512), (257, 511, 64), (300, 2000, 1032), (513, 1300, 192), (700, 130, 2048)]


@pytest.mark.parametrize("M,V,H", SHAPES)
@pytest.mark.parametrize("inv_t", [1.0, 0.7])
def test_logprob_and_slope(M, V, H, inv_t):
    print("head case", M, V, H, inv_t, flush=True)
    x, W, t = _inputs(M, V, H, 7000 + M + V + H)
    head = qerl.lm_head_prepack(W)
    ref, tol = _bounds(x, W, t.numpy(), inv_t, H, V)
    td = t.cuda()
    lp, lse, ent = qerl.lm_head_logprob(x, head, td, inv_t, entropy=True)
    _check((lp, lse, ent), ref, tol, slice(None), ("logprob", M, V, H))
    got = qerl.lm_head_logprob_grad(x, head, td, inv_t, entropy=True)
    _check(got, ref, tol, slice(None), ("grad", M, V, H))
    g = torch.randn((M,), generator=torch.Generator().manual_seed(M))
    dx = qerl.lm_head_logprob_backward(g.cuda(), got[3])
    want, e = g.double().numpy()[:, None] * ref[3], np.abs(g.double().numpy())[:, None] * tol[3]
    off = np.abs(dx.double().cpu().numpy() - want) - (e + 2.0 ** -8 * (np.abs(want) + e))
    assert np.all(off <= 1e-38), float(off.max())
    # bit for bit the same again, and without entropy
    again = qerl.lm_head_logprob_grad(x, head, td, inv_t)
    assert again[2] is None and all(torch.equal(a, b) for a, b in zip((again[0], again[1], again[3]), (got[0], got[1], got[3])))
    assert torch.equal(qerl.lm_head_logprob(x, head, td, inv_t)[0], lp)


def _check_on_gpu(x, head, t, inv_t, got, what, chunk=16384):
    """The same bounds with the fp64 reference on the GPU, the vocabulary in chunks; got: (logprob, lse, entropy[, slope])."""
    M, H = x.shape
    V = head.V
    xd, row = x.double(), torch.arange(M, device="cuda")
    pieces = [slice(a, min(a + chunk, V)) for a in range(0, V, chunk)]
    z = torch.cat([torch.matmul(xd, head.weight[c].double().t()) for c in pieces], 1) * inv_t
    size = torch.stack([torch.matmul(xd.abs(), head.weight[c].double().abs().t()).amax(1) for c in pieces]).amax(0) * inv_t
    lse = torch.logsumexp(z, 1)
    p = torch.exp(z - lse[:, None])
    ent = lse - (p * z).sum(1)
    zt = z[row, t]
    z[row, t] = -float("inf")
    lp = -torch.log1p(torch.exp(z - zt[:, None]).sum(1))
    z[row, t] = zt
    D = 2 * ((H / 16 + 24) * U * size + 4 * U * z.abs().amax(1))
    tol = [(D + 2.0 ** -17) * lp.abs().clamp(max=1) + 2.0 ** -22 * lp.abs(), D + 2.0 ** -17 + 2.0 ** -22 * lse.abs(),
           (D + 2.0 ** -16) * (2 + (z - lse[:, None]).abs().amax(1))]
    ref = [lp, lse, ent]
    if len(got) == 4:
        p[row, t] = 0
        Wt = head.weight[t].double()
        rest, D = p.sum(1, keepdim=True), D[:, None]
        slope, mag = rest * Wt, torch.zeros((M, H), dtype=torch.float64, device="cuda")
        for c in pieces:
            w = head.weight[c].double()
            slope -= torch.matmul(p[:, c], w)
            mag += torch.matmul(p[:, c], w.abs())
        ref.append(inv_t * slope)
        tol.append(inv_t * ((D + 2.0 ** -16) * rest * Wt.abs() + (2.0 ** -8 + D + 2.0 ** -16 + (V / 16 + 64) * U) * mag))
    for name, a, r, e in zip(("logprob", "lse", "entropy", "slope"), got, ref, tol):
        off = (a.double() - r).abs() - e
        assert bool(torch.isfinite(a).all()) and bool((off <= 0).all()), (what, name, float(off.max()))


# sizes at which whole tiles fill the chip (256 rows x 256 rows of the vocabulary), with every kind of remainder; 4096 x 5120 takes the sums'
# tiles of 320; 8192 rows take the vocabulary in pieces
LARGE = [(257, 16640, 64), (300, 17001, 72), (511, 16577, 136), (700, 12007, 1000), (1025, 8193, 328), (2049, 4097, 192), (3000, 3001, 520), (4096, 1500, 5120),
         (8192, 25000, 264)]


@pytest.mark.parametrize("M,V,H", LARGE)
def test_whole_tiles(M, V, H):
    print("large case", M, V, H, flush=True)
    x, W, t = _inputs(M, V, H, 300 + M)
    head, td = qerl.lm_head_prepack(W), t.cuda()
    wt = head.weight_t
    assert torch.equal(wt[:, :V], W.t()) and not bool(wt[:, V:].any())
    pick = torch.randperm(M, generator=torch.Generator().manual_seed(M))[:700].cuda()
    for got in (qerl.lm_head_logprob(x, head, td, 0.8, entropy=True), qerl.lm_head_logprob_grad(x, head, td, 0.8, entropy=True)):
        _check_on_gpu(x[pick], head, td[pick], 0.8, [a[pick] for a in got], (M, V, H))
    # half of the rows without a loss: the others as they were, up to the order of sums
    some = td.clone()
    some[::2] = -1
    part = qerl.lm_head_logprob_grad(x, head, some, 0.8, entropy=True)
    keep = pick[pick % 2 == 1]
    _check_on_gpu(x[keep], head, td[keep], 0.8, [a[keep] for a in part], ("half", M, V, H))
    assert all(not bool(a[::2].any()) for a in part)


@pytest.mark.parametrize("M", [3, 70, 300])
def test_a_head_of_more_than_4_gib(M):
    V, H = 140000, 16384
    gen = torch.Generator(device="cuda").manual_seed(M)
    W = torch.empty((V, H), dtype=torch.bfloat16, device="cuda")
    for a in range(0, V, 20000):
        W[a:a + 20000] = torch.randn((min(20000, V - a), H), generator=gen, device="cuda") * 0.01
    t = torch.randint(0, V, (M,), generator=gen, device="cuda")
    t[0] = V - 1
    x = (torch.randn((M, H), generator=gen, device="cuda") + 0.06 * torch.rand((M, 1), generator=gen, device="cuda") * W[t].float() / 0.01).to(torch.bfloat16)
    head = qerl.lm_head_prepack(W)
    _check_on_gpu(x, head, t, 1.0, qerl.lm_head_logprob(x, head, t, entropy=True), ("4 GiB", M))
    _check_on_gpu(x, head, t, 1.0, qerl.lm_head_logprob_grad(x, head, t, entropy=True), ("4 GiB", M))


@pytest.mark.parametrize("M", [5, 40, 150, 600])
@pytest.mark.parametrize("masked", [0.3, 1.0])
def test_rows_without_a_loss_and_bad_targets(M, masked):
    V, H = 1234, 128
    print("mask case", M, masked, flush=True)
    x, W, t = _inputs(M, V, H, 99 + M)
    g = torch.Generator().manual_seed(M)
    t[torch.rand((M,), generator=g) < masked] = -100
    if masked < 1:
        t[M // 2], t[M // 3] = V, 2 ** 40                  # beyond the vocabulary
    x[t.cuda() < 0] = float("nan")                         # what rows without a loss hold does not matter
    head = qerl.lm_head_prepack(W)
    xz = torch.where((t >= 0).cuda()[:, None], x, torch.zeros_like(x))
    ref, tol = _bounds(xz, W, t.numpy(), 1.0, H, V)
    keep = ((t >= 0) & (t < V)).numpy()
    for got in (qerl.lm_head_logprob(x, head, t.cuda(), entropy=True), qerl.lm_head_logprob_grad(x, head, t.cuda(), entropy=True)):
        if keep.any():
            _check(got, ref, tol, keep, ("masked", M))
        for a in got:
            a = a.cpu()
            assert not a[t < 0].any() and bool(torch.isnan(a[t >= V]).all())
    dx = qerl.lm_head_logprob_backward(torch.ones((M,), device="cuda"), got[3]).cpu()
    assert not dx[t < 0].any() and bool(torch.isnan(dx[t >= V].float()).all()) and bool(torch.isfinite(dx[torch.from_numpy(keep)].float()).all())


@pytest.mark.parametrize("M,V,H", [(7, 300, 72), (150, 700, 200), (520, 300, 64)])
def test_strides_and_what_lies_between_rows(M, V, H):
    print("stride case", M, V, H, flush=True)
    x, W, t = _inputs(M, V, H, 5, ldx=H + 24, ldw=H + 8)
    head = qerl.lm_head_prepack(W)
    ref, tol = _bounds(x, W, t.numpy(), 1.0, H, V)
    slope = torch.full((M + 2, H + 12), 7.0, device="cuda")
    out = [torch.full((M + 2,), 7.0, device="cuda") for _ in range(3)]
    got = [o[:M] for o in out] + [slope[:M, :H]]
    qerl.lm_head_logprob_grad(x, head, t.cuda(), entropy=True, out=got)
    _check(got, ref, tol, slice(None), ("strided", M))
    assert all(bool((o[M:] == 7).all()) for o in out) and bool((slope[M:] == 7).all()) and bool((slope[:, H:] == 7).all())
    dx = torch.full((M + 2, H + 16), 7.0, dtype=torch.bfloat16, device="cuda")
    g = torch.randn((M,), device="cuda")
    qerl.lm_head_logprob_backward(g, slope[:M, :H], out=dx[:M, :H])
    assert bool((dx[M:] == 7).all()) and bool((dx[:, H:] == 7).all())
    assert torch.equal(dx[:M, :H], (g[:, None] * slope[:M, :H]).to(torch.bfloat16))
    # written over memory full of NaN, and by a workspace full of NaN
    ws = qerl.lm_head_workspace(M, V, H)
    ws.fill_(255)
    again = qerl.lm_head_logprob_grad(x, head, t.cuda(), entropy=True, workspace=ws)
    assert all(torch.equal(a, b) for a, b in zip(again, got))


@pytest.mark.parametrize("M", [3, 90, 300])
def test_logits_far_apart(M):
    """Logits up to hundreds of powers of two above the row's own token: references are raised, nothing overflows."""
    V, H = 900, 64
    x, W, t = _inputs(M, V, H, 31 + M, sure=0.0)
    W[450:460] *= 40
    W[850] *= 120
    t[:] = torch.arange(M) % 400
    t[0] = 850
    head = qerl.lm_head_prepack(W)
    ref, tol = _bounds(x, W, t.numpy(), 1.0, H, V)
    assert np.ptp(ref[0]) > 50
    for got in (qerl.lm_head_logprob(x, head, t.cuda(), entropy=True), qerl.lm_head_logprob_grad(x, head, t.cuda(), entropy=True)):
        _check(got, ref, tol, slice(None), ("far", M))


def test_references_raised_between_pieces():
    """8192 rows take the vocabulary in several pieces; later pieces hold the largest logits, in steps, so that sums of earlier ones are
    scaled down to nothing or nearly."""
    M, V, H = 8200, 30000, 64
    x, W, t = _inputs(M, V, H, 77, sure=6.0)
    W[13000:13010] *= 12
    W[29990:] *= 30
    t = t % 12000
    head = qerl.lm_head_prepack(W)
    got = qerl.lm_head_logprob_grad(x, head, t.cuda(), entropy=True)
    ref_only = qerl.lm_head_logprob(x, head, t.cuda(), entropy=True)
    rows = np.r_[0:40, 4000:4040, 8150:8200]
    ref, tol = _bounds(x[rows], W, t.numpy()[rows], 1.0, H, V)
    _check([a[rows] for a in got], ref, tol, slice(None), "pieces")
    _check([a[rows] for a in ref_only], ref, tol, slice(None), "rows only")


def test_a_row_with_nan_or_infinity_stays_alone():
    M, V, H = 300, 500, 64
    for m in (M, 20):
        x, W, t = _inputs(m, V, H, 12)
        head = qerl.lm_head_prepack(W)
        good = qerl.lm_head_logprob_grad(x, head, t.cuda(), entropy=True)
        x[3, 5], x[7, 1] = float("nan"), float("inf")
        rest = [i for i in range(m) if i not in (3, 7)]
        for got in (qerl.lm_head_logprob(x, head, t.cuda(), entropy=True), qerl.lm_head_logprob_grad(x, head, t.cuda(), entropy=True)):
            for a, b in zip(got, good):
                if len(got) == 4:
                    assert torch.equal(a[rest], b[rest])
                assert not bool(torch.isfinite(a[3]).any())
            assert bool(torch.isnan(got[0][7]))


def test_gradient_by_differences():
    """The slope along a direction against differences of the log-probability over a step that shows in bf16."""
    M, V, H = 64, 2000, 256
    x, W, t = _inputs(M, V, H, 21, sure=6.0)
    head = qerl.lm_head_prepack(W)
    lp, _, _, slope = qerl.lm_head_logprob_grad(x, head, t.cuda())
    step = (torch.randint(0, 2, (M, H), generator=torch.Generator().manual_seed(3)).cuda() * 2 - 1) * 2.0 ** -5
    up, down = (x.float() + step).to(torch.bfloat16), (x.float() - step).to(torch.bfloat16)
    change = qerl.lm_head_logprob(up, head, t.cuda())[0].double() - qerl.lm_head_logprob(down, head, t.cuda())[0].double()
    d = up.double() - down.double()
    want = (d * slope.double()).sum(1)
    # central differences leave the third derivative: |d . W|^3 / 24 at most over the spread of the logits of one step, and bf16 weights
    spread = (d @ W.double().T)
    size = spread.abs().amax(1)
    tol = size ** 3 / 24 * 6 + 2.0 ** -8 * size + 1e-4
    # x +- step are not centred on x exactly where their roundings differ: second derivative times the offset of the middle
    off = ((up.double() + down.double()) / 2 - x.double()) @ W.double().T
    tol = tol + size * off.abs().amax(1) * 2
    assert bool(((change - want).abs() <= tol).all()), float(((change - want).abs() / tol).max())
    assert float((change - want).abs().mean()) < 0.1 * float(want.abs().mean())


@pytest.mark.parametrize("M", [8, 300])
def test_captured_and_replayed(M):
    V, H = 3000, 128
    x, W, t = _inputs(M, V, H, 55)
    head, td, g = qerl.lm_head_prepack(W), t.cuda(), torch.randn((M,), device="cuda")
    ws = qerl.lm_head_workspace(M, V, H)
    out = [torch.empty((M,), device="cuda") for _ in range(3)] + [torch.empty((M, H), device="cuda")]
    dx = torch.empty((M, H), dtype=torch.bfloat16, device="cuda")

    def step():
        qerl.lm_head_logprob_grad(x, head, td, entropy=True, workspace=ws, out=out)
        qerl.lm_head_logprob_backward(g, out[3], out=dx)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        x2, _, t2 = _inputs(M, V, H, 60 + i)
        x.copy_(x2)
        td.copy_(t2)
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in out] + [dx.clone()]
        eager = qerl.lm_head_logprob_grad(x, head, td, entropy=True)
        assert all(torch.equal(a, b) for a, b in zip(got, (*eager, qerl.lm_head_logprob_backward(g, eager[3]))))


def test_on_another_stream():
    M, V, H = 100, 2000, 128
    x, W, t = _inputs(M, V, H, 3)
    head, td = qerl.lm_head_prepack(W), t.cuda()
    want = qerl.lm_head_logprob_grad(x, head, td)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = qerl.lm_head_logprob_grad(x, head, td)
    s.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[3], want[3])


def test_binding_refusals():
    x, W, t = _inputs(4, 100, 64, 1)
    head = qerl.lm_head_prepack(W, gradient=False)
    td = t.cuda()
    for bad in (lambda: qerl.lm_head_logprob_grad(x, head, td), lambda: qerl.lm_head_logprob(x[:, :32], head, td), lambda: qerl.lm_head_logprob(x, head, td[:3]),
                lambda: qerl.lm_head_logprob(x.t(), head, td), lambda: qerl.lm_head_prepack(W.t()),
                lambda: qerl.lm_head_logprob(x, head, td, entropy=True, out=(torch.empty(4, device="cuda"), None, None))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: qerl.lm_head_logprob(x, head, td.int()), lambda: qerl.lm_head_logprob(x.float(), head, td), lambda: qerl.lm_head_logprob(x, head, t),
                lambda: qerl.lm_head_logprob(x, head, td, workspace=torch.empty(1 << 20, dtype=torch.uint8))):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises(qerl.QerlError):
        qerl.lm_head_logprob(x, head, td, inv_temperature=0.0)
    with pytest.raises(qerl.QerlError):
        qerl.lm_head_logprob(x, head, td, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    e = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    got = qerl.lm_head_logprob(e, head, td[:0], entropy=True)
    assert got[0].shape == (0,)


def _slope_bound(x, W, t, inv_t):
    """(slope, tolerance) where a probability of 1/32 or more of what all but the row's own token hold enters the sum in fp32: only the others carry the
    2^-8 of bf16 in the bound at the top of this file."""
    x, W = x.double().cpu().numpy(), W.double().cpu().numpy()
    (M, H), V = x.shape, W.shape[0]
    z = inv_t * (x @ W.T)
    D = (2 * ((H / 16 + 24) * U * inv_t * (np.abs(x) @ np.abs(W).T).max(1) + 4 * U * np.abs(z).max(1)))[:, None]
    _, lse, _, slope = uo.head_logprob(x, W, t, inv_t)
    p = np.exp(z - lse[:, None])
    p[np.arange(M), t] = 0
    rest = p.sum(1, keepdims=True)
    small = np.where(p >= rest / 32, 0, p)
    return slope, inv_t * ((D + 2.0 ** -16) * rest * np.abs(W[t]) + (D + 2.0 ** -16 + (V / 16 + 64) * U) * (p @ np.abs(W)) + 2.0 ** -8 * (small @ np.abs(W)))


def _check_slope(slope, x, W, t, inv_t, what):
    want, tol = _slope_bound(x, W, t, inv_t)
    off = np.abs(slope.double().cpu().numpy() - want) - tol
    assert np.all(off <= 0), (what, float((off + tol).max()), float((off / tol).max()), np.argwhere(~(off <= 0))[:4].tolist())
    return want, tol


@pytest.mark.parametrize("together", [1, 2, 5])
@pytest.mark.parametrize("M,V,H,inv_t", [(1, 300, 64, 1.0), (40, 5000, 256, 1.0), (100, 3001, 136, 0.7), (300, 2000, 264, 1.0), (700, 4099, 128, 1.25)])
def test_rows_whose_mass_is_on_other_tokens(M, V, H, inv_t, together):
    """An unlikely token was sampled: one, two or five neighbouring others hold nearly all of the mass, at the vocabulary's ends and across the
    borders of tiles among them.  The slope there is little but a few rows of W, so that nothing averages a rounding of their probabilities."""
    print("dominated case", M, V, H, inv_t, together, flush=True)
    x, W, t = _inputs(M, V, H, 500 + M, sure=0.0)
    g = torch.Generator().manual_seed(M + together)
    u = torch.randint(0, V - together, (M,), generator=g)
    u[: min(M, 6)] = torch.tensor([V - together, 0, 62, 126, 254, 1022 % (V - together)])[: min(M, 6)]
    t = torch.where((t >= u) & (t < u + together), (u + together + 1) % V, t)
    Wf = W.float().cpu()
    xf = x.float().cpu()
    for i in range(together):
        w = Wf[u + i]
        xf += (11.0 + 3 * torch.rand((M, 1), generator=g)) / inv_t * w / (w * w).sum(1, keepdim=True)
    x.copy_(xf.to(torch.bfloat16))
    head = qerl.lm_head_prepack(W)
    got = qerl.lm_head_logprob_grad(x, head, t.cuda(), inv_t, entropy=True)
    want, tol = _check_slope(got[3], x, W, t.numpy(), inv_t, (M, V, H, together))
    # the bound is one that a rounding of the large ones to bf16 (2^-10 of the slope in the mean) would not meet
    assert np.median(np.linalg.norm(tol, axis=1) / np.linalg.norm(want, axis=1)) < 2.0 ** -10
    ref, all_tol = _bounds(x, W, t.numpy(), inv_t, H, V)
    _check(got, ref, all_tol, slice(None), ("dominated", M, V, H))
    # some rows without a loss among them; the others bit for bit, up to the order of sums where rows are left out
    some = t.clone()
    some[::3] = -1
    part = qerl.lm_head_logprob_grad(x, head, some.cuda(), inv_t)[3]
    keep = np.arange(M) % 3 != 0
    if keep.any():
        _check_slope(part[torch.from_numpy(keep)], x[torch.from_numpy(keep)], W, t.numpy()[keep], inv_t, ("masked", M, V, H, together))
    assert not bool(part[::3].any())


@pytest.mark.parametrize("levels", [(0, 0, 0, 0, 0), (0, 3, 6, 9, 12), (12, 9, 6, 3, 0), (0, 3, 80, 83, 90)])
def test_large_probabilities_of_several_pieces(levels):
    """8200 rows take the vocabulary in five pieces.  25 tokens in nearly equal parts stand out in each of the first four, three in the last, `levels`
    above one another: where the levels rise, more are large on the way than are kept, and the three have to stay; with a step of 77 references
    are raised in between."""
    M, V, H = 8200, 60000, 64
    g = torch.Generator().manual_seed(levels[0] + levels[4])
    d = torch.randn((H,), generator=g)
    d /= d.norm()
    W = torch.randn((V, H), generator=g) * 0.05
    for a, n, level in zip((100, 14000, 26000, 40000, V - 3), (25, 25, 25, 25, 3), levels):
        apart = torch.randn((n, H), generator=g) * 0.3
        W[a:a + n] = d * (12 + level) / 8 + apart - (apart @ d)[:, None] * d
    W = W.to(torch.bfloat16).cuda()
    x = (8 * d + torch.randn((M, H), generator=g) * 0.02).to(torch.bfloat16).cuda()
    t = torch.randint(200, 13000, (M,), generator=g)
    slope = qerl.lm_head_logprob_grad(x, qerl.lm_head_prepack(W), t.cuda())[3]
    rows = np.r_[0:30, 4000:4030, 8170:8200]
    _check_slope(slope[rows], x[rows], W, t.numpy()[rows], 1.0, levels)


def test_a_large_probability_beside_a_token_that_is_nearly_certain():
    """1 - p_t is small and one other token holds nearly all of it: the slope, small as a whole, keeps its relative precision."""
    M, V, H = 90, 2500, 256
    x, W, t = _inputs(M, V, H, 41, sure=0.0)
    u = (t + 700) % V
    Wf, xf = W.float().cpu(), x.float().cpu()
    for at, z in ((t, 30.0), (u, 14.0)):
        w = Wf[at]
        xf += z * w / (w * w).sum(1, keepdim=True)
    x.copy_(xf.to(torch.bfloat16))
    got = qerl.lm_head_logprob_grad(x, qerl.lm_head_prepack(W), t.cuda())
    assert float(got[0].median()) > -1e-3
    _check_slope(got[3], x, W, t.numpy(), 1.0, "sure")


@pytest.mark.parametrize("m", [20, 50, 100, 200, 300])
def test_rows_beside_one_that_is_not_finite_are_as_without_it(m):
    """Both calls on every tile for few and for many rows, against the same call on clean rows, bit for bit."""
    V, H = 500, 64
    x, W, t = _inputs(m, V, H, 12)
    head, td = qerl.lm_head_prepack(W), t.cuda()
    calls = (lambda: qerl.lm_head_logprob(x, head, td, entropy=True), lambda: qerl.lm_head_logprob_grad(x, head, td, entropy=True))
    clean = [call() for call in calls]
    x[3, 5], x[7, 1], x[m - 1, 63] = float("nan"), float("inf"), -float("inf")
    rest = [i for i in range(m) if i not in (3, 7, m - 1)]
    for call, good in zip(calls, clean):
        for a, b in zip(call(), good):
            assert torch.equal(a[rest], b[rest])
            assert not bool(torch.isfinite(a[3]).any())


@pytest.mark.parametrize("M,V", [(300, 4099), (2100, 60000)])
def test_large_probabilities_in_a_used_workspace_and_on_replay(M, V):
    """One and several pieces: the same bits whatever the workspace holds, again, and on every replay with other rows, some of them with a large
    probability, some without, some without a loss."""
    H = 64
    x, W, t = _inputs(M, V, H, 900 + M, sure=0.0)
    head, g = qerl.lm_head_prepack(W), torch.Generator().manual_seed(M)
    Wf = W.float().cpu()

    def rows(i):
        u, z = torch.randint(0, V, (M,), generator=g), torch.tensor([0.0, 9.0, 13.0])[torch.randint(0, 3, (M,), generator=g)][:, None]
        w = Wf[u]
        x.copy_((torch.randn((M, H), generator=g) * 0.5 + z * w / (w * w).sum(1, keepdim=True)).to(torch.bfloat16))
        td.copy_(torch.where(torch.rand((M,), generator=g) < 0.2 * i, torch.full_like(t, -1), t))
    td = t.cuda()
    rows(1)
    ws = qerl.lm_head_workspace(M, V, H)
    out = [torch.empty((M,), device="cuda") for _ in range(3)] + [torch.empty((M, H), device="cuda")]
    call = lambda: qerl.lm_head_logprob_grad(x, head, td, entropy=True, workspace=ws, out=out)
    for byte in (0, 255, 0x7F):
        ws.fill_(byte)
        call()
        first = [o.clone() for o in out] if byte == 0 else first
        assert all(torch.equal(a, b) for a, b in zip(first, out)), byte
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        rows(i)
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in out]
        assert all(torch.equal(a, b) for a, b in zip(got, qerl.lm_head_logprob_grad(x, head, td, entropy=True)))
        keep = torch.nonzero(td.cpu() >= 0)[:200, 0]
        _check_slope(got[3][keep.cuda()], x[keep.cuda()], W, t.numpy()[keep.numpy()], 1.0, (M, V, i))
