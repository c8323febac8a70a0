"""Oracle for the operators beside the chunk loop: the root-mean-square norm with
its gradients, 8-bit block quantisation and product, and rotary positions.

TEST INFRASTRUCTURE ONLY.  Everything is float64 on the stored input values, from
the definitions in ``include/hcms.h``; this module never imports the product path.
"""
from __future__ import annotations

import math

import numpy as np

BLOCK = 128


# ---------------------------------------------------------------------------
# Norm
# ---------------------------------------------------------------------------
def rms_norm(x, weight, eps, residual=None):
    """(y, h) of rows: h = x + residual, y = h / sqrt(mean(h^2) + eps) weight."""
    h = x if residual is None else x + residual
    return h / np.sqrt((h * h).mean(axis=1, keepdims=True) + eps) * weight, h


def rms_norm_backward(dy, x, weight, eps, residual=None, dh=None):
    """(dx, dw): the gradients of sum(dy y) + sum(dh h)."""
    h = x if residual is None else x + residual
    r = 1.0 / np.sqrt((h * h).mean(axis=1, keepdims=True) + eps)
    n, g = h * r, dy * weight
    dx = r * (g - n * (g * n).mean(axis=1, keepdims=True))
    return dx if dh is None else dx + dh, (dy * n).sum(axis=0)


# ---------------------------------------------------------------------------
# 8 bits
# ---------------------------------------------------------------------------
def e4m3(x):
    """Nearest e4m3 value, ties to the even one: 3 bits behind the leading one
    down to 2^-6, steps of 2^-9 below; |x| <= 448 is taken for granted."""
    x = np.asarray(x, dtype=np.float64)
    _, e = np.frexp(x)
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    return np.rint(x / step) * step


def scale_exponent(amax: float) -> int:
    """The smallest e >= -126 with amax <= 448 * 2^e; 128 (NaN) if amax is not finite."""
    if not math.isfinite(amax):
        return 128
    e = -126
    while amax > math.ldexp(448.0, e):
        e += 1
    return e


def quantize(x, rows: int):
    """(values on the e4m3 grid, exponents [blocks of rows][blocks of 128]) of x
    [M][K], blocks of ``rows`` x 128.  Exponents as :func:`scale_exponent`, with 448
    as 0.875 * 2^9; values of a block with an infinity or a NaN are NaN."""
    M, K = x.shape
    R, B = -(-M // rows), -(-K // BLOCK)
    pad = np.zeros((R * rows, B * BLOCK))
    pad[:M, :K] = np.where(np.isfinite(x), x, np.nan)
    blocks = pad.reshape(R, rows, B, BLOCK)
    amax = np.abs(blocks).max(axis=(1, 3))
    bad = np.isnan(amax)
    m, e = np.frexp(np.where(bad, 0.0, amax))
    exps = np.where(bad, 128, np.maximum(e - 9 + (m > 0.875), -126)).astype(np.int64)
    exps[amax == 0] = -126
    q = e4m3(np.where(bad[:, None, :, None], 0.0, np.ldexp(np.nan_to_num(blocks), -np.where(bad, 0, exps)[:, None, :, None])))
    q = np.where(bad[:, None, :, None], np.nan, q)
    return q.reshape(R * rows, B * BLOCK)[:M, :K], exps


def held(x, rows: int, least: float = 0.0):
    """The values that x's 8-bit form stands for; with ``least``, the magnitudes of
    those that are not zero, taken to be at least ``least`` of their scale."""
    q, e = quantize(x, rows)
    if least:
        q = np.where(q != 0, np.maximum(np.abs(q), least), 0.0)
    s = np.repeat(np.repeat(np.where(e < 128, np.ldexp(1.0, np.minimum(e, 127)), np.nan), rows, 0),
                  BLOCK, 1)
    return q * s[:x.shape[0], :x.shape[1]]


def scale_bytes(exps):
    """Exponents [rows][blocks] as the bytes [groups of four][rows][4], the fill of
    the last group being the scale of a block of zeros."""
    rows, blocks = exps.shape
    out = np.ones((-(-blocks // 4), rows, 4), dtype=np.uint8)
    for b in range(blocks):
        out[b // 4, :, b % 4] = exps[:, b] + 127
    return out


# ---------------------------------------------------------------------------
# Rotary positions
# ---------------------------------------------------------------------------
def frequencies(pairs, base=10000.0, scaling="none", factor=1.0, original_length=0.0,
                beta_fast=32.0, beta_slow=1.0):
    """(frequencies, magnitude) from the wavelengths: pair i turns
    original_length * f_i / (2 pi) times over the original length."""
    i = np.arange(pairs, dtype=np.float64)
    f = base ** (-i / pairs)
    if scaling == "linear":
        return f / factor, 1.0
    if scaling == "ntk":
        return (f if pairs == 1 else (base * factor ** (pairs / (pairs - 1))) ** (-i / pairs)), 1.0
    if scaling == "none":
        return f, 1.0
    # Turns over the original length, of twice as many pairs as there are: the mixture
    # starts at the last pair that turns beta_fast times and ends at the first one that
    # turns no more than beta_slow times, past the pairs or not.
    turns = original_length / (2 * math.pi) * base ** (-np.arange(2 * pairs) / pairs)
    lo, hi = max(int((turns >= beta_fast).sum()) - 1, 0), min(int((turns > beta_slow).sum()), 2 * pairs - 1)
    slow = np.interp(i, [lo, hi], [0.0, 1.0]) if hi > lo else np.ones(pairs)
    slow = np.where(turns[:pairs] >= beta_fast, 0.0, np.where(turns[:pairs] <= beta_slow, 1.0, slow))
    return f * (1 - slow) + f / factor * slow, 0.1 * math.log(factor) + 1.0


def rotate(x, angles, magnitude=1.0, layout="interleaved", inverse=False):
    """x [S][H][d] with its first 2 * angles.shape[1] elements turned by angles
    [S][pairs], by complex multiplication."""
    x = np.array(x, dtype=np.float64)
    P = angles.shape[1]
    a, b = (slice(0, 2 * P, 2), slice(1, 2 * P, 2)) if layout == "interleaved" else (slice(0, P), slice(P, 2 * P))
    z = (x[..., a] + 1j * x[..., b]) * (magnitude * np.exp((-1j if inverse else 1j) * angles))[:, None, :]
    x[..., a], x[..., b] = z.real, z.imag
    return x
