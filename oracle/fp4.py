"""The 4-bit calls in float64, by definition: e2m1 codes, the scales of a KV
cache, its append and its rows, and the norms and rotation of queries and keys.

e2m1: sign, two exponent bits (bias 1), one fraction bit; exponent 0 is subnormal;
there are no infinities and no NaN.  A key's 32 columns share an exponent byte,
2^(byte - 127), or NaN (255); a value's row shares a bfloat16.  The paper says
nothing of storage in 4 bits; layouts and scales are those of
include/sdverify_fp4.h.
"""

from __future__ import annotations

from fractions import Fraction

import numpy as np

BLOCK = 64
GROUP = 32
LOWEST = -100
# The largest scales with which 6, the largest code, stands for a finite float32: 2^125, and the bits of 170 * 2^118.
HIGHEST = 125
HIGHEST_VALUE = 0x7e2a
VALUES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6])


def encode(x):
    """Nearest codes of x, ties to the even code; magnitudes past 6 are 6."""
    x = np.asarray(x, dtype=np.float64)
    d = np.abs(np.abs(x)[..., None] - VALUES[:8])
    near = d == d.min(axis=-1, keepdims=True)
    even = near & (np.arange(8) % 2 == 0)
    code = np.where(even.any(-1), even.argmax(-1), near.argmax(-1))
    return (code | np.where(np.signbit(x), 8, 0)).astype(np.uint8)


def scale_exponent(most):
    """Smallest e >= LOWEST with most <= 6 * 2^e."""
    e = LOWEST
    while most > 6 * 2.0 ** e:
        e += 1
    return e


def bf16_value(bits):
    with np.errstate(invalid="ignore"):  # signalling NaN
        return np.asarray(np.asarray(bits, dtype=np.uint32) << 16, dtype=np.uint32).view(np.float32).astype(np.float64)


def value_scale(most):
    """Bits of the smallest bfloat16 s >= 2^LOWEST with most <= 6 s."""
    bits = (LOWEST + 127) << 7
    up = 0x7f7f
    while bits < up:  # positive bfloat16 are ordered by their bits
        mid = (bits + up) // 2
        if Fraction(float(most)) <= 6 * Fraction(float(bf16_value(mid))):
            up = mid
        else:
            bits = mid + 1
    return bits


# ---- the cache ----------------------------------------------------------------

def k_index(dim):
    """[64][dim]: half byte (twice the byte, one more for the high half) of a K block."""
    n, d = np.meshgrid(np.arange(BLOCK), np.arange(dim), indexing="ij")
    byte = ((n // 16 * 4 + d // (dim // 4)) * 16 + n % 16) * (dim // 8) + d % (dim // 4) // 2
    return 2 * byte + d % 2


def v_index(dim):
    """[64][dim]: the same of a V block."""
    n, d = np.meshgrid(np.arange(BLOCK), np.arange(dim), indexing="ij")
    return 2 * ((d // 16 * 64 + n) * 8 + d % 16 // 2) + d % 2


def k_scale_index(dim):
    """[64][dim/32]: where the scale of a key's columns lies among a block's."""
    n, g = np.meshgrid(np.arange(BLOCK), np.arange(dim // GROUP), indexing="ij")
    return (g * 16 + n % 16) * 4 + n // 16


def unpack(block):
    """Bytes [...] as half bytes, twice as many."""
    return np.stack([block & 15, block >> 4], axis=-1).reshape(*block.shape[:-1], -1)


def pack(codes):
    return (codes[..., 0::2] | codes[..., 1::2] << 4).astype(np.uint8)


def key_scales(scales, dim):
    """Scale bytes of a K block as values [64][dim]."""
    e = scales[k_scale_index(dim)].astype(np.float64) - 127
    return np.repeat(np.where(e == 128, np.nan, 2.0 ** e), GROUP, axis=1)


def rows(k, v, k_scale, v_scale, table_row, first, count, head):
    """Keys and values first .. first + count - 1 of one request and head, float64 [count][D].

    k, v [pages][Hkv][blocks][32 D] bytes, k_scale [pages][Hkv][blocks][2 D] bytes, v_scale
    [pages][Hkv][blocks][64] bits of bfloat16."""
    blocks, dim = k.shape[2], k.shape[3] // 32
    out = np.empty((2, count, dim))
    for n in range(first, first + count):
        at = int(table_row[n // BLOCK // blocks]), head, n // BLOCK % blocks
        out[0, n - first] = (VALUES[unpack(k[at])[k_index(dim)]] * key_scales(k_scale[at], dim))[n % BLOCK]
        out[1, n - first] = (VALUES[unpack(v[at])[v_index(dim)]] * bf16_value(v_scale[at])[:, None])[n % BLOCK]
    return out[0], out[1]


def append(k, v, k_scale, v_scale, table, k_new, v_new, new_off, new_len, kv_len):
    """The four pools after an append (copies).  New rows [T][Hkv][D]; request b's keys
    kv_len - new_len .. are its rows new_off .. .  Elements past 6 of the largest scale become 6 of it."""
    k, v, k_scale, v_scale = k.copy(), v.copy(), k_scale.copy(), v_scale.copy()
    heads, blocks, dim = k.shape[1], k.shape[2], k.shape[3] // 32
    ki, vi, si = k_index(dim), v_index(dim), k_scale_index(dim)
    for b in range(len(kv_len)):
        for j in range(int(new_len[b])):
            n = int(kv_len[b]) - int(new_len[b]) + j
            for h in range(heads):
                at = int(table[b][n // BLOCK // blocks]), h, n // BLOCK % blocks
                x = np.asarray(k_new[int(new_off[b]) + j, h], dtype=np.float64).reshape(-1, GROUP)
                codes = unpack(k[at])
                for g in range(dim // GROUP):
                    number = np.isfinite(x[g]).all()
                    e = min(scale_exponent(np.abs(x[g]).max()), HIGHEST) if number else 128
                    codes[ki[n % BLOCK, g * GROUP:(g + 1) * GROUP]] = encode(x[g] * 2.0 ** -e) if number else 0
                    k_scale[at][si[n % BLOCK, g]] = e + 127
                k[at] = pack(codes)
                x = np.asarray(v_new[int(new_off[b]) + j, h], dtype=np.float64)
                number = np.isfinite(x).all()
                s = min(value_scale(np.abs(x).max()), HIGHEST_VALUE) if number else 0x7fc0
                codes = unpack(v[at])
                # float64 quotients of float32 by bfloat16 fall on a border of codes only where the true ones do
                codes[vi[n % BLOCK]] = encode(x / bf16_value(s)) if number else 0
                v[at], v_scale[at][n % BLOCK] = pack(codes), s
    return k, v, k_scale, v_scale


def kv4_segments(k, v, k_scale, v_scale, table, kv_len):
    """The caches as contiguous segments (k_pool, v_pool, kv_off), the layout
    that verify_attention and tree_attention take."""
    heads, blocks, dim = k.shape[1], k.shape[2], k.shape[3] // 32
    ki, vi = k_index(dim), v_index(dim)
    parts, off, at = ([], []), [], 0
    for b, n in enumerate(kv_len):
        off.append(at)
        for h in range(heads):
            kk, vv = np.empty((-(-int(n) // BLOCK) * BLOCK, dim)), np.empty((-(-int(n) // BLOCK) * BLOCK, dim))
            for n0 in range(0, int(n), BLOCK):
                p = int(table[b][n0 // BLOCK // blocks]), h, n0 // BLOCK % blocks
                kk[n0:n0 + BLOCK] = VALUES[unpack(k[p])[ki]] * key_scales(k_scale[p], dim)
                with np.errstate(invalid="ignore"):  # 0 times infinity, past the last key
                    vv[n0:n0 + BLOCK] = VALUES[unpack(v[p])[vi]] * bf16_value(v_scale[p])[:, None]
            parts[0].append(kk[:int(n)].reshape(-1))
            parts[1].append(vv[:int(n)].reshape(-1))
        at += heads * int(n) * dim
    return np.concatenate(parts[0]), np.concatenate(parts[1]), np.array(off)


# ---- norms and rotation ------------------------------------------------------------

def norm_rope(x, weight, positions, inv_freq, eps, interleaved):
    """Rows [T][H][D] normed head by head (weight None: as they are) and turned; also
    the magnitudes that each element's two terms add up to, for error bounds."""
    x = np.asarray(x, dtype=np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps) * np.asarray(weight, dtype=np.float64)
    half = len(inv_freq)
    t = np.asarray(positions, dtype=np.float64)[:, None] * np.asarray(inv_freq, dtype=np.float64)
    c, s = np.cos(t)[:, None], np.sin(t)[:, None]
    a = slice(0, 2 * half, 2) if interleaved else slice(0, half)
    b = slice(1, 2 * half, 2) if interleaved else slice(half, 2 * half)
    y, mag = x.copy(), np.abs(x)
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    mag[..., a] = mag[..., b] = np.hypot(x[..., a], x[..., b])
    return y, mag
