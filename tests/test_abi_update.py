"""CPU: the operators around a policy update refuse misuse on the host, before anything could be launched (no pointer below is ever
dereferenced), and their sizes are consistent."""
import ctypes

import pytest

import paper_2510_11696_amd as qerl
from paper_2510_11696_amd.binding import _AdamWHyper, _AdamWPlanStruct, _AdamWState, _AdamWTensor

FAKE = 0x10000
BIG = 1 << 40
p = ctypes.c_void_p
NULL, SHAPE, ALIGN, WORKSPACE = -1, -2, -3, -4


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(qerl.LIB_PATH):
        from paper_2510_11696_amd import build
        build.build(verbose=False)
    return qerl.load_library()


def _logprob(lib, gradient, **kw):
    a = dict(x=FAKE, M=4, H=64, ldx=64, W=FAKE, V=100, ldw=64, Wt=FAKE, targets=FAKE, it=1.0, lp=FAKE, lse=FAKE, ent=FAKE, slope=FAKE, lds=64,
             ws=FAKE, wsb=BIG)
    a.update(kw)
    head = [a["x"], a["M"], a["H"], a["ldx"], a["W"], a["V"], a["ldw"]]
    rows = [a["targets"], a["it"], a["lp"], a["lse"], a["ent"]]
    if gradient:
        return lib.lm_head_logprob_grad(*head, a["Wt"], *rows, a["slope"], a["lds"], a["ws"], a["wsb"], None)
    return lib.lm_head_logprob(*head, *rows, a["ws"], a["wsb"], None)


@pytest.mark.parametrize("gradient", [False, True])
def test_logprob_refusals(lib, gradient):
    call = lambda **kw: _logprob(lib, gradient, **kw)
    assert call(M=0) == 0 and call(M=0, x=None, W=None) == 0
    for kw in (dict(M=-1), dict(V=0), dict(H=0), dict(H=60, ldx=64), dict(H=4), dict(ldx=56), dict(ldw=56), dict(V=(1 << 22) + 1), dict(M=1 << 31), dict(ldx=1 << 18), dict(ldw=1 << 18),
               dict(it=0.0), dict(it=-1.0), dict(it=float("inf")), dict(it=float("nan")), dict(it=3e38)):
        assert call(**kw) == SHAPE, kw
    for k in ("x", "W", "targets", "lp"):
        assert call(**{k: None}) == NULL, k
    for kw in (dict(x=FAKE + 8), dict(W=FAKE + 2), dict(ldx=68), dict(ldw=66), dict(targets=FAKE + 4), dict(lp=FAKE + 2), dict(lse=FAKE + 1), dict(ent=FAKE + 2)):
        assert call(**kw) == ALIGN, kw
    need = lib.lm_head_logprob_workspace_bytes(4, 100, 64, int(gradient))
    assert need > 0
    for kw in (dict(ws=None), dict(ws=FAKE + 64), dict(wsb=need - 1)):
        assert call(**kw) == WORKSPACE, kw
    if gradient:
        assert call(lds=60) == SHAPE and call(lds=66) == ALIGN and call(slope=FAKE + 4) == ALIGN and call(Wt=FAKE + 8) == ALIGN
        assert call(slope=None) == NULL and call(Wt=None) == NULL


def test_logprob_sizes(lib):
    size = lib.lm_head_logprob_workspace_bytes
    assert size(-1, 100, 64, 0) == 0 and size(4, 0, 64, 0) == 0 and size(4, 100, 4, 1) == 0 and size(0, 100, 64, 1) > 0
    for g in (0, 1):
        for V in (1, 63, 50257, 152064):
            for H in (64, 3584, 5120):
                got = [size(M, V, H, g) for M in (1, 15, 16, 17, 32, 33, 64, 65, 100, 128, 129, 200, 256, 257, 500, 512, 777, 1024, 2048, 4096, 8192, 8193, 100000)]
                assert got == sorted(got) and got[-1] == got[-2] == got[-3] and got[-1] < 2 << 30, (V, H, g, got)
    assert lib.lm_head_prepack_t_bytes(50257, 64) == 50304 * 64 * 2 and lib.lm_head_prepack_t_bytes(0, 64) == 0
    t = lib.lm_head_prepack_t
    assert t(FAKE, 10, 60, 64, FAKE, None) == SHAPE and t(FAKE, -1, 64, 64, FAKE, None) == SHAPE and t(FAKE, 10, 64, 56, FAKE, None) == SHAPE
    assert t(None, 10, 64, 64, FAKE, None) == NULL and t(FAKE, 10, 64, 64, None, None) == NULL
    assert t(FAKE + 2, 10, 64, 64, FAKE, None) == ALIGN and t(FAKE, 10, 64, 68, FAKE, None) == ALIGN and t(FAKE, 10, 64, 64, FAKE + 8, None) == ALIGN
    assert t(FAKE, 0, 64, 64, FAKE, None) == 0
    b = lib.lm_head_logprob_backward
    assert b(FAKE, FAKE, 64, 0, 64, FAKE, 64, None) == 0
    assert b(FAKE, FAKE, 56, 4, 64, FAKE, 64, None) == SHAPE and b(FAKE, FAKE, 64, 4, 60, FAKE, 64, None) == SHAPE
    assert b(FAKE, FAKE, 64, 4, 64, FAKE, 56, None) == SHAPE and b(FAKE, FAKE, 64, -1, 64, FAKE, 64, None) == SHAPE
    assert b(None, FAKE, 64, 4, 64, FAKE, 64, None) == NULL and b(FAKE, None, 64, 4, 64, FAKE, 64, None) == NULL and b(FAKE, FAKE, 64, 4, 64, None, 64, None) == NULL
    assert b(FAKE, FAKE, 66, 4, 64, FAKE, 64, None) == ALIGN and b(FAKE, FAKE, 64, 4, 64, FAKE, 68, None) == ALIGN and b(FAKE + 2, FAKE, 64, 4, 64, FAKE, 64, None) == ALIGN


def _tensors(spec):
    """spec: (param, copy, grad, n) each."""
    arr = (_AdamWTensor * len(spec))()
    for i, s in enumerate(spec):
        arr[i] = _AdamWTensor(*s)
    return arr


def _make(lib, spec, n=None, table=FAKE, nbytes=BIG):
    arr = _tensors(spec)
    plan = _AdamWPlanStruct()
    return lib.lora_adamw_make_plan(ctypes.cast(arr, p), len(spec) if n is None else n, table, nbytes, ctypes.byref(plan), None)


def test_adamw_plan_refusals(lib):
    G = 0x100000
    ok = [(G, 2 * G, 3 * G, 1000), (4 * G, None, 5 * G, 7)]
    arr = ctypes.cast(_tensors(ok), p)
    need = lib.lora_adamw_plan_bytes(arr, 2)
    assert need > 0 and lib.lora_adamw_state_elements(arr, 2) == 1024 + 32
    assert lib.lora_adamw_plan_bytes(arr, 0) == 0 and lib.lora_adamw_state_elements(arr, 0) == -1
    assert lib.lora_adamw_plan_bytes(None, 2) == 0 and lib.lora_adamw_state_elements(None, 2) == -1
    assert lib.lora_adamw_make_plan(None, 2, FAKE, BIG, ctypes.byref(_AdamWPlanStruct()), None) == NULL
    assert lib.lora_adamw_make_plan(arr, 2, FAKE, BIG, None, None) == NULL
    assert _make(lib, ok, n=0) == SHAPE and _make(lib, ok, n=-1) == SHAPE
    assert _make(lib, [(G, None, 2 * G, -1)]) == SHAPE and _make(lib, [(G, None, 2 * G, 1 << 50)]) == SHAPE
    assert _make(lib, [(None, None, 2 * G, 8)]) == NULL and _make(lib, [(G, None, None, 8)]) == NULL
    assert _make(lib, [(G + 4, None, 2 * G, 8)]) == ALIGN and _make(lib, [(G, None, 2 * G + 8, 8)]) == ALIGN and _make(lib, [(G, 3 * G + 2, 2 * G, 8)]) == ALIGN
    # memory that a step writes, named twice
    assert _make(lib, [(G, None, 2 * G, 8), (G, None, 3 * G, 8)]) == SHAPE
    assert _make(lib, [(G, None, 2 * G, 8), (G + 16, None, 3 * G, 8)]) == SHAPE
    assert _make(lib, [(G, G + 16, 2 * G, 8)]) == SHAPE
    assert _make(lib, [(G, None, G, 8)]) == SHAPE and _make(lib, [(G, None, 2 * G, 8), (3 * G, None, G + 16, 8)]) == SHAPE
    assert _make(lib, [(G, 3 * G, 2 * G, 8), (4 * G, 3 * G, 5 * G, 8)]) == SHAPE
    assert _make(lib, ok, nbytes=need - 1) == WORKSPACE and _make(lib, ok, table=None) == WORKSPACE and _make(lib, ok, table=FAKE + 16) == WORKSPACE


def test_adamw_step_norm_and_moments_refusals(lib):
    def step(plan=None, state=None, **kw):
        pl = _AdamWPlanStruct(FAKE, 1024, 1, 1)
        st = _AdamWState(8, 2 * FAKE, 3 * FAKE, 4 * FAKE, 5 * FAKE)
        for d, src in ((pl, plan), (st, state)):
            for k, v in (src or {}).items():
                setattr(d, k, v)
        h = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, step=1, seed=0, lr_device=None, step_device=None, grad_scale=None)
        h.update(kw)
        return lib.lora_adamw_step(ctypes.byref(pl), ctypes.byref(st), ctypes.byref(_AdamWHyper(*h.values())), None)
    nan, inf = float("nan"), float("inf")
    assert step(plan=dict(chunks=0)) == 0
    for kw in (dict(lr=-1.0), dict(lr=nan), dict(lr=inf), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=nan), dict(eps=0.0), dict(eps=nan),
               dict(weight_decay=-1.0), dict(weight_decay=inf), dict(step=0), dict(step=-3)):
        assert step(**kw) == SHAPE, kw
    assert step(lr=nan, lr_device=FAKE + 2) == ALIGN and step(step=0, step_device=FAKE + 4) == ALIGN and step(grad_scale=FAKE + 1) == ALIGN
    assert step(state=dict(bits=16)) == SHAPE and step(state=dict(m=None)) == NULL and step(state=dict(v_scale=None)) == NULL
    for kw in (dict(v=2 * FAKE), dict(v=2 * FAKE + 1008), dict(m_scale=2 * FAKE), dict(v_scale=3 * FAKE + 16), dict(v_scale=4 * FAKE + 31),
               dict(bits=32, v=2 * FAKE + 4080)):                                # parts of the state that share memory
        assert step(state=kw) == SHAPE, kw
    assert step(plan=dict(elements=0, chunks=0), state=dict(m=None, v=None)) == 0
    assert step(state=dict(m=2 * FAKE + 8)) == ALIGN and step(plan=dict(table=None)) == NULL and step(plan=dict(chunks=-1)) == SHAPE
    pl, st = _AdamWPlanStruct(FAKE, 1024, 1, 1), _AdamWState(8, 2 * FAKE, 3 * FAKE, 4 * FAKE, 5 * FAKE)
    pb, sb = ctypes.byref(pl), ctypes.byref(st)
    assert lib.lora_adamw_step(None, sb, ctypes.byref(_AdamWHyper()), None) == NULL and lib.lora_adamw_step(pb, None, ctypes.byref(_AdamWHyper()), None) == NULL
    assert lib.lora_adamw_step(pb, sb, None, None) == NULL
    norm = lib.lora_adamw_grad_norm
    assert norm(None, 1.0, FAKE, FAKE, None) == NULL and norm(pb, 1.0, FAKE, None, None) == NULL
    assert norm(pb, 0.0, FAKE, FAKE, None) == SHAPE and norm(pb, nan, FAKE, FAKE, None) == SHAPE
    assert norm(pb, 1.0, FAKE + 2, FAKE, None) == ALIGN and norm(pb, 1.0, FAKE, FAKE + 2, None) == ALIGN
    mom = lib.lora_adamw_moments
    assert mom(pb, sb, None, FAKE, None) == NULL and mom(pb, sb, FAKE + 4, FAKE, None) == ALIGN
    st.bits = 32
    assert mom(pb, sb, FAKE, FAKE, None) == SHAPE


def test_binding_refuses_cpu_tensors():
    import torch
    with pytest.raises(TypeError):
        qerl.lm_head_prepack(torch.zeros((8, 64), dtype=torch.bfloat16))
    with pytest.raises(TypeError):
        qerl.lora_adamw_plan([torch.zeros(8)], [torch.zeros(8)])
    with pytest.raises(TypeError):
        qerl.lm_head_logprob_backward(torch.zeros(4), torch.zeros((4, 64)))
    with pytest.raises(ValueError):
        qerl.lora_adamw_plan([], [])


def _step(lib, **kw):
    h = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, step=1, seed=0, lr_device=None, step_device=None, grad_scale=None)
    h.update(kw)
    pl, st = _AdamWPlanStruct(FAKE, 1024, 0, 1), _AdamWState(8, 2 * FAKE, 3 * FAKE, 4 * FAKE, 5 * FAKE)      # no pieces: nothing is launched
    return lib.lora_adamw_step(ctypes.byref(pl), ctypes.byref(st), ctypes.byref(_AdamWHyper(*h.values())), None)


def test_adamw_numbers_that_fp32_does_not_hold(lib):
    """What the kernel computes with are the numbers as fp32: an eps that rounds to 0 would leave 0 / 0 wherever there has been no gradient."""
    for kw in (dict(eps=1e-46), dict(eps=1e300), dict(lr=1e39), dict(lr=1e38, beta1=0.9), dict(lr=1e20, weight_decay=1e30), dict(lr=1e300, weight_decay=1e300)):
        assert _step(lib, **kw) == SHAPE, kw
    for kw in (dict(eps=1e-45), dict(eps=3e38), dict(lr=3e37), dict(lr=0.0, weight_decay=1e30), dict(lr=1e8, weight_decay=1e30),
               dict(beta1=1 - 2.0 ** -53, beta2=1 - 2.0 ** -53), dict(lr=1e-3, beta1=0.0, step=2 ** 62)):
        assert _step(lib, **kw) == 0, kw


def test_adamw_state_must_be_apart_from_the_tensors(lib):
    G = 0x100000
    tensors = [(G, 2 * G, 3 * G, 1000), (4 * G, None, 5 * G, 7), (None, None, None, 0)]     # 1056 state elements
    arr, table = ctypes.cast(_tensors(tensors), p), 20 * G
    nbytes = lib.lora_adamw_plan_bytes(arr, 3)

    def check(bits=8, m=10 * G, v=11 * G, ms=12 * G, vs=13 * G, table=table):
        st = _AdamWState(bits, m, v, ms, vs)
        return lib.lora_adamw_check_state(arr, 3, table, ctypes.byref(st))
    assert check() == 0 and check(bits=32) == 0 and check(table=None) == 0
    for bits in (8, 32):
        size = 1056 * bits // 8
        for part in ("m", "v"):
            # on a parameter, a copy or a gradient: at its start, over its last element, from before into its first
            for start, length in ((G, 4000), (2 * G, 2000), (3 * G, 4000), (4 * G, 28), (5 * G, 28)):
                for at in (start, (start + length - 1) // 16 * 16, start - size + 16):
                    assert check(bits, **{part: at}) == SHAPE, (bits, part, hex(at))
                assert check(bits, **{part: (start + length + 15) // 16 * 16}) == 0 and check(bits, **{part: (start - size) // 16 * 16}) == 0
            assert check(bits, **{part: table}) == SHAPE and check(bits, **{part: table + nbytes - 16}) == SHAPE and check(bits, **{part: table + nbytes}) == 0
            assert check(bits, **{part: table + 16}, table=None) == 0
    for part in ("ms", "vs"):
        for at in (G + 3999, 2 * G - 32, 3 * G, table):
            assert check(**{part: at}) == SHAPE, (part, hex(at))
        assert check(**{part: G - 33}) == 0 and check(**{part: G + 4000}) == 0 and check(bits=32, **{part: G}) == 0
    assert check(v=10 * G + 16) == SHAPE and check(bits=16) == SHAPE and check(m=None) == NULL and check(ms=None) == NULL and check(m=10 * G + 8) == ALIGN
    empty = ctypes.cast(_tensors([(None, None, None, 0)]), p)
    assert lib.lora_adamw_check_state(empty, 1, table, ctypes.byref(_AdamWState(8, None, None, None, None))) == 0
    assert lib.lora_adamw_check_state(arr, 0, table, ctypes.byref(_AdamWState(8))) == SHAPE
    assert lib.lora_adamw_check_state(None, 1, table, ctypes.byref(_AdamWState(8))) == NULL and lib.lora_adamw_check_state(arr, 3, table, None) == NULL
    # the table of a plan
    assert _make(lib, tensors, table=3 * G + 3840) == SHAPE and _make(lib, tensors, table=G - 256) == SHAPE


def test_gradients_of_a_backward_call_must_be_apart(lib):
    """dA and dB are written by one launch.  The other refusals keep their order: these calls have everything else right, and none is launched."""
    from paper_2510_11696_amd.binding import _BackwardDesc
    G, M, K, N, r = 0x100000, 4, 64, 32, 8
    size_a, size_b = 4 * r * K, 4 * r * N

    def single(dA, dB):
        return lib.nvfp4_lora_linear_backward(FAKE, FAKE, M, K, N, K, N, FAKE, FAKE, FAKE, FAKE, r, 1.0, FAKE, K, dA, dB, FAKE, BIG, None)

    def group(*grads):
        d = (_BackwardDesc * len(grads))()
        for m, g in zip(d, grads):
            m.dy, m.lddy, m.N, m.packed_t, m.tensor_scale = FAKE, N, N, FAKE, FAKE
            if g is not None:
                m.A, m.B, m.r, m.lora_scale, m.dA, m.dB = FAKE, FAKE, r, 1.0, *g
        return lib.nvfp4_lora_linear_backward_group(FAKE, M, K, K, ctypes.cast(d, p), len(grads), FAKE, K, FAKE, BIG, None)
    for call in (single, lambda *g: group(g), lambda *g: group(None, g), lambda *g: group((8 * G, 9 * G), g)):
        for dA, dB in ((G, G), (G, G + size_a - 4), (G + size_b - 4, G)):
            assert call(dA, dB) == SHAPE, (dA, dB)
    ok = (G, 2 * G)
    for bad in (ok, (G + size_a - 4, 3 * G), (3 * G, G + size_a - 4), (2 * G, 3 * G), (3 * G, 2 * G - size_b + 4), (3 * G, 2 * G)):
        assert group(ok, bad) == SHAPE and group(ok, None, bad) == SHAPE and group(bad, None, (5 * G, 6 * G), ok) == SHAPE, bad


def test_logprob_workspace_is_0_for_every_size_that_is_refused(lib):
    size = lib.lm_head_logprob_workspace_bytes
    for g in (0, 1):
        for M, V, H in ((4, 100, 9), (4, 100, 60), (4, 100, 4), (4, 100, 0), (4, 100, 1 << 18), (-1, 100, 64), (1 << 31, 100, 64), (4, 0, 64), (4, (1 << 22) + 1, 64)):
            assert size(M, V, H, g) == 0, (M, V, H)
            if M > 0:
                assert _logprob(lib, bool(g), M=M, V=V, H=H, ldx=1 << 18 if H >= 1 << 18 else 64, ldw=1 << 18 if H >= 1 << 18 else 64) == SHAPE, (M, V, H)
        for M, V, H in ((4, 100, 8), (4, 100, (1 << 18) - 8), (1, 1 << 22, 64)):
            assert size(M, V, H, g) > 0, (M, V, H)
    with pytest.raises(ValueError):
        qerl.lm_head_workspace(4, 100, 60)


def test_adamw_pieces_that_one_launch_has_no_threads_for(lib):
    """A workgroup of 256 threads per piece of 2048 elements, fewer than 2^32 threads in a launch."""
    most = 2048 * (2 ** 24 - 1)
    one = lambda *ns: ctypes.cast(_tensors([(FAKE, None, FAKE, n) for n in ns]), p)
    assert lib.lora_adamw_state_elements(one(most), 1) == most and lib.lora_adamw_plan_bytes(one(most), 1) > 4 * (2 ** 24 - 1)
    for ns in ((most + 1,), (most, 1), (most // 2, most // 2, 4096)):
        assert lib.lora_adamw_state_elements(one(*ns), len(ns)) == -1 and lib.lora_adamw_plan_bytes(one(*ns), len(ns)) == 0, ns
    assert lib.lora_adamw_state_elements(one(most - 2048, 1, 0), 3) == most - 2048 + 32
    st, h = _AdamWState(8, FAKE, FAKE, FAKE, FAKE), _AdamWHyper(1e-3, 0.9, 0.999, 1e-8, 0.0, 1)
    assert lib.lora_adamw_step(ctypes.byref(_AdamWPlanStruct(FAKE, most + 2048, 2 ** 24, 1)), ctypes.byref(st), ctypes.byref(h), None) == SHAPE
