"""Pins of the update oracle (CPU): closed forms, differences, and the 8-bit formats by exhaustion."""
import numpy as np
import pytest

from oracle import update_oracle as uo


def test_head_closed_forms():
    # two tokens of equal logits: ln 1/2 each, entropy ln 2; slope (W_0 - W_1) / 2
    x = np.array([[1.0, 2.0]])
    W = np.array([[3.0, 1.0], [1.0, 2.0]])
    lp, lse, ent, slope = uo.head_logprob(x, W, [0])
    assert np.allclose([lp[0], lse[0], ent[0]], [-np.log(2), 5 + np.log(2), np.log(2)], atol=1e-15)
    assert np.allclose(slope, [(W[0] - W[1]) / 2], atol=1e-15)
    # one token: certain
    lp, lse, ent, slope = uo.head_logprob(x, W[:1], [0])
    assert lp[0] == 0 and lse[0] == 5 and ent[0] == 0 and not slope.any()


def test_head_slope_is_the_derivative():
    rng = np.random.default_rng(3)
    x, W, t = rng.normal(size=(5, 7)), rng.normal(size=(11, 7)), np.array([0, 10, 3, -1, 11])
    _, _, _, slope = uo.head_logprob(x, W, t, 0.7)
    for k in range(7):
        d = np.zeros_like(x)
        d[:, k] = 1e-5
        num = (uo.head_logprob(x + d, W, t, 0.7)[0] - uo.head_logprob(x - d, W, t, 0.7)[0]) / 2e-5
        assert np.allclose(num[:3], slope[:3, k], atol=1e-8)
    assert not slope[3].any() and np.isnan(slope[4]).all()


def test_eight_bit_values_are_a_strictly_rising_grid():
    for bits, top in ((4, 14), (5, 30)):
        g = uo.grid_values(bits)
        assert g[0] == 0 and np.all(np.diff(g) > 0)
        assert g[top * 8] == 1.0 and g[1] == 2.0 ** (-top - 2)
        c = np.arange(256, dtype=np.uint8)
        f = np.full(8, 127, np.uint8)
        v = uo.decode(c, f, bits)
        assert np.array_equal(np.abs(v[:128]), g[:128].astype(np.float32))


@pytest.mark.parametrize("field", [30, 127, 254])
def test_values_of_the_grid_stay_and_others_go_up_by_their_fraction(field):
    base = 2.0 ** (field - 127)
    for bits, encode in ((4, uo.encode_first), (5, uo.encode_second)):
        g = uo.grid_values(bits)
        x = np.zeros(64, np.float32)
        x[0::32] = 1.5 * base                               # fixes the blocks' exponent
        lo = np.arange(40, 71) if bits == 4 else np.arange(100, 131)
        x[1:32] = (g[lo] * base).astype(np.float32)
        x[33:64] = (0.25 * g[lo] + 0.75 * g[lo + 1]) * base * (-1 if bits == 4 else 1)
        for u, up in ((0.0, 0), (0.25 - 2.0 ** -16, 0), (0.25, 1), (1 - 2.0 ** -16, 1)):
            codes, f = encode(x, np.full(64, u))
            assert np.all(f == field) and np.array_equal(codes[1:32], lo)
            assert np.array_equal(codes[33:64], lo + up + (128 if bits == 4 else 0))


def test_second_moment_rounding_is_unbiased_and_never_reaches_zero():
    x = np.zeros(32, np.float32)
    x[0], x[1], x[2] = 1.0, 1.0625 * 2 ** -9, 1e-30
    n = 4096
    total = np.zeros(32)
    for s in range(n // 16):
        u = (np.arange(32) * 2048 + s * 256) % 65536 / 65536.0            # 256 steps of 256: every element walks once through all fractions
        codes, f = uo.encode_second(x, u)
        total += uo.decode(codes, f, 5)
        assert codes[2] == 1 and codes[3] == 0
    assert total[0] == n // 16
    assert abs(total[1] / (n // 16) / x[1] - 1) < 2 ** -3 / 64


def test_adamw_first_step_moves_by_the_rate():
    g = np.array([0.3, -2.0, 1e-4], np.float32)
    p, m, v = uo.adamw(np.zeros(3), g, np.zeros(3), np.zeros(3), 1e-3, 0.9, 0.999, 1e-8, 0.0, 1)
    assert np.allclose(p, -1e-3 * np.sign(g), rtol=2e-4)
    p2, _, _ = uo.adamw(np.ones(3), g * 4, np.zeros(3), np.zeros(3), 1e-3, 0.9, 0.999, 1e-8, 0.1, 1, grad_scale=0.25)
    assert np.allclose(p2, 1 - 1e-4 - 1e-3 * np.sign(g), rtol=1e-6)


def test_the_largest_values_stay_finite():
    x = np.full(32, np.finfo(np.float32).max, np.float32)
    x[1::2] = 1.875 * 2.0 ** 127
    for u in (0.0, 0.5, 1 - 2.0 ** -16):
        for sign in (1, -1):
            codes, field = uo.encode_first(sign * x, np.full(32, u))
            assert np.all(field == 254) and np.array_equal(uo.decode(codes, field, 4), np.full(32, sign * 1.875 * 2.0 ** 127, np.float32))
        codes, field = uo.encode_second(x, np.full(32, u))
        assert np.all(field == 254) and np.array_equal(uo.decode(codes, field, 5), np.full(32, 1.875 * 2.0 ** 127, np.float32))
    # one power of two lower the next value exists, and is reached
    codes, field = uo.encode_first(x / 2, np.full(32, 1 - 2.0 ** -16))
    assert np.all(field == 253) and np.array_equal(uo.decode(codes, field, 4)[:2], [2.0 ** 127, 1.875 * 2.0 ** 126])
