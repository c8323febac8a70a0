"""Oracle for the norm and rotation of head vectors in one pass, the paged cache of
keys and values in 4 bits, and attention over it.

TEST INFRASTRUCTURE ONLY.  Everything is float64 on the stored input values, from the
definitions in ``include/hcms.h``; this module never imports the product path.
"""
from __future__ import annotations

import math

import numpy as np

from . import operators as op

BLOCK, CHUNK = 32, 64
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


# ---------------------------------------------------------------------------
# Norm and rotation
# ---------------------------------------------------------------------------
def coordinates(grid, places):
    """[n][axes] of places on the row-major grid."""
    return np.stack(np.unravel_index(np.asarray(places), tuple(grid)), 1)


def factors(table, grid, axis_pairs, coords):
    """Complex factors [n][pairs] of a rotation table's entries [E][2] at coordinates
    [n][axes]; NaN outside the grid."""
    out, first = [], 0
    for a, (size, p) in enumerate(zip(grid, axis_pairs)):
        z = table[first:first + size * p].reshape(size, p, 2)
        c = coords[:, a]
        out.append(z[np.clip(c, 0, size - 1)])
        first += size * p
    z = np.concatenate(out, 1)
    z = z[..., 0] + 1j * z[..., 1]
    bad = ((coords < 0) | (coords >= np.array(grid))).any(1)
    z[bad] = np.nan + 1j * np.nan
    return z


def turn(x, z, layout="interleaved"):
    """x [T][H][d] with its first elements turned by z [T][pairs]."""
    x = np.array(x, dtype=np.float64)
    P = z.shape[1]
    a, b = (slice(0, 2 * P, 2), slice(1, 2 * P, 2)) if layout == "interleaved" else (slice(0, P), slice(P, 2 * P))
    c, s = z.real[:, None], z.imag[:, None]
    u, v = x[..., a].copy(), x[..., b].copy()
    x[..., a], x[..., b] = u * c - v * s, u * s + v * c
    return x


def head_norm(x, w, eps, z, layout="interleaved"):
    """Each head vector normed, weighted and turned."""
    return turn(x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w, z, layout)


def head_norm_backward(dy, x, w, eps, z, layout="interleaved"):
    """(dx, dw): the gradients of sum(dy y)."""
    S, H, d = x.shape
    g = turn(dy, z.conj(), layout)
    dx, dw = op.rms_norm_backward(g.reshape(S * H, d), x.reshape(S * H, d), w, eps)
    return dx.reshape(S, H, d), dw


# ---------------------------------------------------------------------------
# 4 bits
# ---------------------------------------------------------------------------
def e2m1(x):
    """Codes of the nearest e2m1 values, ties to the even code; |x| <= 6."""
    a = np.abs(x)
    near = np.abs(a[..., None] - GRID)
    best = near.min(-1, keepdims=True)
    tied = near == best
    even = tied & (np.arange(8) % 2 == 0)
    pick = np.where(even.any(-1, keepdims=True), even, tied)
    return np.argmax(pick, -1) + 8 * np.signbit(x)


def scale_exponent(amax: float) -> int:
    """The smallest e >= -126 with amax <= 6 * 2^e; 128 (NaN) if amax is not finite."""
    if not math.isfinite(amax):
        return 128
    e = -126
    while amax > math.ldexp(6.0, e):
        e += 1
    return e


def quantize(x):
    """(codes, exponents) of x [..., d], a block for each 32 elements; an infinity or a
    NaN makes its block's exponent 128 and its codes 0."""
    b = np.asarray(x, dtype=np.float64).reshape(*x.shape[:-1], -1, BLOCK)
    amax = np.abs(np.where(np.isfinite(b), b, np.nan)).max(-1)
    e = np.vectorize(scale_exponent)(amax)
    ok = e < 128
    q = e2m1(np.ldexp(np.where(ok[..., None], b, 0.0), np.where(ok, -e, 0)[..., None]))
    return q.reshape(x.shape), e


def values(codes, e):
    """What codes [..., d] with exponents [..., d / 32] stand for."""
    v = np.where(codes >= 8, -1.0, 1.0) * GRID[codes % 8]
    s = np.where(e < 128, np.ldexp(1.0, np.minimum(e, 127)), np.nan)
    return v * np.repeat(s, BLOCK, -1)


def held(x):
    return values(*quantize(x))


def key_scale_place(t):
    return 4 * (t % 16) + t // 16


def value_place(t):
    return 16 * (t // 4 % 4) + 4 * (t // 16) + t % 4


def store(cache, page, slot, head, k, v):
    """Writes one token's key and value [d] (float64) into numpy arrays ``cache`` =
    (k, v, k_scale, v_scale) of the layout in hcms.h."""
    ck, cv, sk, sv = cache
    chunk, t = divmod(slot, CHUNK)
    q, e = quantize(k)
    ck[page, head, slot] = q[0::2] + 16 * q[1::2]
    sk[page, head, chunk, :, key_scale_place(t)] = e + 127
    q, e = quantize(v)
    cv[page, head, chunk, :, value_place(t)] = q[0::2] + 16 * q[1::2]
    sv[page, head, chunk, :, value_place(t)] = e + 127


def read(cache, pages, length):
    """Keys and values [length][heads][d] of a sequence with these pages."""
    ck, cv, sk, sv = cache
    heads, page, half = ck.shape[1:]
    K, V = np.empty((2, length, heads, 2 * half))
    for p in range(length):
        g, slot = pages[p // page], p % page
        chunk, t = divmod(slot, CHUNK)
        for out, byte, e in ((K, ck[g, :, slot], sk[g, :, chunk, :, key_scale_place(t)]),
                             (V, cv[g, :, chunk, :, value_place(t)], sv[g, :, chunk, :, value_place(t)])):
            code = np.stack((byte & 15, byte >> 4), -1).reshape(heads, -1)
            out[p] = values(code.astype(int), e.astype(int) - 127)
    return K, V


# ---------------------------------------------------------------------------
# Attention
# ---------------------------------------------------------------------------
def sees(n, length, causal, window):
    """[begin, end) of the tokens that each of a sequence's n rows sees."""
    end = np.maximum(length - n + np.arange(n) + 1 if causal else np.full(n, length), 0)
    return np.maximum(end - window, 0) if window else np.zeros(n, int), end


def attention(q, K, V, scale, causal=False, window=0):
    """(out, sum of p |v| / sum of p, largest sum of |q k| of a row) for rows q
    [n][H][d] that are the last ones of a sequence of K and V [length][heads][d]."""
    n, H, d = q.shape
    length, heads = K.shape[:2]
    out, mass, most = np.zeros_like(q), np.zeros_like(q), np.zeros((n, H))
    begin, end = sees(n, length, causal, window)
    for i in range(n):
        a, b = begin[i], end[i]
        if a >= b:
            continue
        for h in range(H):
            k, v = K[a:b, h * heads // H], V[a:b, h * heads // H]
            s = scale * (k @ q[i, h])
            p = np.exp(s - s.max())
            out[i, h], mass[i, h] = p @ v / p.sum(), p @ np.abs(v) / p.sum()
            most[i, h] = (np.abs(k) @ np.abs(q[i, h])).max()
    return out, mass, most
