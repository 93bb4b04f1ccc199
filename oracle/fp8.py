"""The 8-bit calls in float64, by definition: e4m3 codes, power-of-two block
scales of a KV cache, its append and its rows, the normed 8-bit rows, and the
vocabulary projection with a scale for each block of 128.

e4m3: sign, four exponent bits (bias 7), three fraction bits; exponent 0 is
subnormal; 0x7f and 0xff are NaN and there are no infinities.  A cache scale is
an exponent byte, 2^(byte - 127).  The paper says nothing of storage in 8 bits;
layouts and scales are those of include/sdverify_fp8.h.
"""

from __future__ import annotations

import numpy as np

BLOCK = 64
COLS = 128
LOWEST = -100


def e4m3_values():
    """The value of every code, [256]."""
    v = np.empty(256)
    for c in range(256):
        e, f = (c >> 3) & 15, c & 7
        x = np.ldexp(1 + f / 8, e - 7) if e else np.ldexp(f / 8, -6)
        v[c] = np.nan if c & 127 == 127 else -x if c & 128 else x
    return v


VALUES = e4m3_values()
_POSITIVE = VALUES[:127]  # 0 .. 448, ascending


def encode(x):
    """Nearest codes of x, ties to the even code; NaN (0x7f) for NaN, infinities
    and magnitudes that round past 448."""
    x = np.asarray(x, dtype=np.float64)
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    hi = np.clip(np.searchsorted(_POSITIVE, a), 1, 126)
    lo = hi - 1
    dl, dh = a - _POSITIVE[lo], _POSITIVE[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    code = np.where(a > 464, 127, code)  # halfway to the next step, which does not exist
    code = np.where(np.isfinite(x), code, 127)
    return (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def decode(c):
    return VALUES[np.asarray(c)]


def scale_exponent(most):
    """Smallest e >= LOWEST with most <= 448 * 2^e."""
    e = LOWEST
    while most > 448 * 2.0 ** e:
        e += 1
    return e


# ---- the cache ----------------------------------------------------------------

def k_index(dim):
    """[64][dim]: where key and column lie among a K block's codes."""
    n, d = np.meshgrid(np.arange(BLOCK), np.arange(dim), indexing="ij")
    t, r = n // 16, n % 16
    i, g, b = d // 64, d % 64 // 16, d % 16
    return (((i * 4 + t) * 4 + g) * 16 + r) * 16 + b


def v_index(dim):
    """[64][dim]: where key and column lie among a V block's codes."""
    n, d = np.meshgrid(np.arange(BLOCK), np.arange(dim), indexing="ij")
    t, g, r = n // 16, n % 16 // 4, n % 4
    return (((d // 16 * 4 + g) * 16 + d % 16) * 4 + t) * 4 + r


def cache_rows(pool, scales, table_row, length, head, index):
    """Keys 0 .. length - 1 of one request and head as float64 [length][D].

    pool [pages][Hkv][blocks][64 D] codes, scales [pages][Hkv][blocks] bytes."""
    blocks = scales.shape[2]
    rows = np.empty((length, index.shape[1]))
    for n0 in range(0, length, BLOCK):
        page, blk = int(table_row[n0 // BLOCK // blocks]), n0 // BLOCK % blocks
        v = decode(pool[page, head, blk][index]) * 2.0 ** (int(scales[page, head, blk]) - 127)
        m = min(BLOCK, length - n0)
        rows[n0:n0 + m] = v[:m]
    return rows


def append(pool, scales, table, new, new_off, new_len, kv_len, index):
    """The pool's codes and scale bytes after an append (copies).  new
    [T][Hkv][D]; request b's keys kv_len - new_len .. are its rows new_off .. ."""
    pool, scales = pool.copy(), scales.copy()
    blocks, heads = scales.shape[2], scales.shape[1]
    for b in range(len(kv_len)):
        end, begin = int(kv_len[b]), int(kv_len[b]) - int(new_len[b])
        for n0 in range(begin // BLOCK * BLOCK, end if new_len[b] else 0, BLOCK):
            page, blk = int(table[b][n0 // BLOCK // blocks]), n0 // BLOCK % blocks
            lo, hi = max(begin, n0), min(end, n0 + BLOCK)
            for h in range(heads):
                x = np.asarray(new[int(new_off[b]) + lo - begin:int(new_off[b]) + hi - begin, h], dtype=np.float64)
                finite = np.abs(x[np.isfinite(x)])
                e = scale_exponent(finite.max() if finite.size else 0.0)
                code = pool[page, h, blk].copy()
                if lo > n0:
                    was = int(scales[page, h, blk]) - 127
                    e = max(e, was)
                    if e > was:
                        code[index[:lo - n0]] = encode(decode(code[index[:lo - n0]]) * 2.0 ** (was - e))
                code[index[lo - n0:hi - n0]] = encode(x * 2.0 ** -e)
                pool[page, h, blk], scales[page, h, blk] = code, e + 127
    return pool, scales


def kv8_segments(k, v, k_scale, v_scale, table, kv_len):
    """The caches as contiguous segments (k_pool, v_pool, kv_off), the layout
    that verify_attention and tree_attention take."""
    heads = k_scale.shape[1]
    dim = k.shape[-1] // BLOCK
    ki, vi = k_index(dim), v_index(dim)
    parts, off, at = ([], []), [], 0
    for b, n in enumerate(kv_len):
        off.append(at)
        for h in range(heads):
            parts[0].append(cache_rows(k, k_scale, table[b], int(n), h, ki).reshape(-1))
            parts[1].append(cache_rows(v, v_scale, table[b], int(n), h, vi).reshape(-1))
        at += heads * int(n) * dim
    return np.concatenate(parts[0]), np.concatenate(parts[1]), np.array(off)


# ---- the projection's rows and product ----------------------------------------------

def residual_norm(x, residual, weight, eps):
    """(h, y, scales [ceil(W/128)][rows]) with codes encode(y / scale)."""
    h = np.asarray(x, dtype=np.float64) + (0.0 if residual is None else np.asarray(residual, dtype=np.float64))
    y = h / np.sqrt((h * h).mean(axis=1, keepdims=True) + eps) * np.asarray(weight, dtype=np.float64)
    scales = [np.maximum(np.abs(y[:, i:i + COLS]).max(axis=1) / 448, 2.0 ** -126) for i in range(0, y.shape[1], COLS)]
    return h, y, np.stack(scales)


def dequantised(codes, scales_by_row):
    """codes [R][K] times scales [R][ceil(K/128)], a scale for each 128 columns."""
    return decode(codes) * np.repeat(scales_by_row, COLS, axis=1)[:, :codes.shape[1]]


def logits_fp8(hidden, hidden_scale, w, w_scale):
    """(logits, sum of the terms' magnitudes), both [M][V]."""
    a = dequantised(hidden, np.asarray(hidden_scale, dtype=np.float64).T)
    b = dequantised(w, np.repeat(np.asarray(w_scale, dtype=np.float64), COLS, axis=0)[:w.shape[0]])
    return a @ b.T, np.abs(a) @ np.abs(b).T
