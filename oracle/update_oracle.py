"""References of the operators around a policy update: the head's log-probabilities with their gradient (fp64), and the AdamW step on
the adapters (IEEE fp32 operation by operation, as the operator defines it, and its 8-bit moments).

Plain numpy; nothing here is shared with the GPU code.
"""
from __future__ import annotations

import numpy as np

from .nvfp4_oracle import philox4x32_10

BLOCK = 32          # state elements that share a scale byte


# ---- the head --------------------------------------------------------------------------------------------------------
def head_logprob(x, W, targets, inv_temperature=1.0):
    """(logprob, lse, entropy, slope) in fp64; rows whose target is below 0 are zero, beyond the vocabulary NaN."""
    x, W = np.asarray(x, np.float64), np.asarray(W, np.float64)
    t = np.asarray(targets)
    M, V = x.shape[0], W.shape[0]
    z = inv_temperature * (x @ W.T)
    with np.errstate(all="ignore"):
        top = z.max(1, keepdims=True)
        e = np.exp(z - top)
        lse = np.log(e.sum(1)) + top[:, 0]
        p = e / e.sum(1, keepdims=True)
        entropy = lse - (p * z).sum(1)
        at = np.clip(t, 0, V - 1)
        zt = z[np.arange(M), at]
        others = z.copy()
        others[np.arange(M), at] = -np.inf
        logprob = -np.log1p(np.exp(others - zt[:, None]).sum(1))
        q = p.copy()
        q[np.arange(M), at] = 0.0
        slope = inv_temperature * (q.sum(1, keepdims=True) * W[at] - q @ W)
    for out in (logprob, lse, entropy, slope):
        out[t < 0] = 0.0
        out[t >= V] = np.nan
    return logprob, lse, entropy, slope


# ---- the optimizer ---------------------------------------------------------------------------------------------------
def state_starts(sizes):
    """First state element of every tensor, and the state's length."""
    starts, at = [], 0
    for n in sizes:
        starts.append(at)
        at += -(-n // BLOCK) * BLOCK
    return starts, at


def grid_values(exponent_bits):
    """The non-negative 8-bit values relative to the block's exponent: ascending, value of code c at index c."""
    top = 14 if exponent_bits == 4 else 30
    return np.array([(8 + (c & 7)) * 2.0 ** ((c >> 3) - top - 3) if c >> 3 else (c & 7) * 2.0 ** (1 - top - 3)
                     for c in range(128 if exponent_bits == 4 else 256)])


def block_field(x):
    """fp32 exponent field of each block's largest magnitude, at least 1."""
    mag = np.abs(np.asarray(x, np.float32)).reshape(-1, BLOCK)
    return np.maximum(mag.max(1).view(np.uint32) >> 23, 1).astype(np.uint8)


def decode(codes, field, exponent_bits):
    c = np.asarray(codes, np.uint8).reshape(-1, BLOCK).astype(np.int64)
    body = c & 127 if exponent_bits == 4 else c
    v = grid_values(exponent_bits)[body] * np.exp2(field.astype(np.float64) - 127)[:, None]
    v = np.where(c > 127, -v, v) if exponent_bits == 4 else v
    v = np.where(field[:, None] == 255, np.nan, v)
    return v.astype(np.float32).reshape(-1)


def _encode(x, fractions, exponent_bits):
    """(codes of the magnitudes, field): rounded up where the distance from the value below, in steps, plus the fraction (a multiple of 2^-16)
    reaches 1; where that would be 2^128, the value below stays.  Distances are taken to 20 bits of a step, as an fp32 near the bottom of its range holds them (only magnitudes below the
    format's smallest normal value have more)."""
    x = np.asarray(x, np.float32)
    field = block_field(x)
    q = np.abs(x.astype(np.float64)).reshape(-1, BLOCK) * np.exp2(127.0 - field)[:, None]
    grid = grid_values(exponent_bits)
    lo = np.clip(np.searchsorted(grid, q, side="right") - 1, 0, len(grid) - 2)
    part = (q - grid[lo]) / (grid[lo + 1] - grid[lo])
    part = np.rint(part * 2.0 ** 20) / 2.0 ** 20
    code = lo + (part + np.asarray(fractions).reshape(-1, BLOCK) >= 1.0)
    top = 14 if exponent_bits == 4 else 30
    return np.where(field[:, None] == 254, np.minimum(code, 8 * top + 7), code), field


def encode_first(x, fractions):
    """(codes, field): sign, 4 + 3 bits."""
    code, field = _encode(x, fractions, 4)
    return (code + 128 * (np.asarray(x).reshape(-1, BLOCK) < 0)).astype(np.uint8).reshape(-1), field


def encode_second(x, fractions):
    """(codes, field): 5 + 3 bits; a value above zero gets at least code 1."""
    code, field = _encode(x, fractions, 5)
    return np.where(np.asarray(x).reshape(-1, BLOCK) > 0, np.maximum(code, 1), 0).astype(np.uint8).reshape(-1), field


def random_fractions(elements, step, seed):
    """Multiples of 2^-16 in [0, 1): element j of group b of eight takes half j % 2 of word j / 2 of Philox(counter (b, step), key seed)."""
    b = np.arange(elements // 8, dtype=np.uint64)
    words = lambda v: (v & 0xFFFFFFFF, v >> 32)
    ctr = np.stack([b & np.uint64(0xFFFFFFFF), b >> np.uint64(32)] + [np.full_like(b, w) for w in words(step)], axis=1)
    r = philox4x32_10(ctr, words(seed & (2 ** 64 - 1)))
    return np.stack([r & 0xFFFF, r >> 16], axis=2).reshape(-1) / 65536.0


def adamw(p, g, m, v, lr, beta1, beta2, eps, weight_decay, step, grad_scale=None):
    """(p', m', v'), each operation an fp32 rounding, the factors formed in fp64."""
    f = np.float32
    p, g, m, v = (np.asarray(a, f) for a in (p, g, m, v))
    if grad_scale is not None:
        g = g * f(grad_scale)
    m = f(beta1) * m + f(1.0 - beta1) * g
    v = f(beta2) * v + f(1.0 - beta2) * (g * g)
    root = np.sqrt(v) * f(1.0 / np.sqrt(1.0 - beta2 ** step)) + f(eps)
    p = p * f(1.0 - lr * weight_decay) - f(lr / (1.0 - beta1 ** step)) * m / root
    return p, m, v
