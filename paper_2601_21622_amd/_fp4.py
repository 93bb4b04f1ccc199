"""ctypes marshalling of the 4-bit calls (include/sdverify_fp4.h).

Argument conversion, and the checks that only tensors allow: element types,
sizes, and one device for all.  A call runs on that device (and, without a
``stream``, on its current stream), whichever device is current.
"""

from __future__ import annotations

import ctypes
import functools
import os
import re
from typing import Sequence

import numpy as np
import torch

from . import _binding as _b
from ._binding import SD_DTYPE_BF16, SD_DTYPE_F32, Dims
from ._fp8 import _device, _lengths, _new_rows, _passes, _run, _typed

SD_KV4_BLOCK = 64
SD_KV4_GROUP = 32

_HEADER = os.path.join(os.path.dirname(_b._HEADER), "sdverify_fp4.h")


_SCALES = (torch.bfloat16, torch.int16, torch.uint16)


class KV4Cache(ctypes.Structure):
    """sd_kv4_cache_t: a 4-bit paged cache.  Build it with KV4Cache.of(...),
    which checks the pools against each other and keeps them referenced as long as it
    lives: a captured graph's calls need it alive for as long as the graph is replayed."""
    _fields_ = [
        ("k", ctypes.c_void_p),
        ("v", ctypes.c_void_p),
        ("k_scale", ctypes.c_void_p),
        ("v_scale", ctypes.c_void_p),
        ("block_table", ctypes.c_void_p),
        ("max_pages", ctypes.c_int32),
        ("page_size", ctypes.c_int32),
        ("num_pages", ctypes.c_int32),
    ]

    @classmethod
    def of(cls, k, v, k_scale, v_scale, block_table, page_size: int) -> "KV4Cache":
        """Pools of bytes (two codes each), whose first dimension is the page and whose second
        the head, exponent bytes k_scale and bfloat16 (or 16-bit integer) v_scale likewise, and
        the int32 table [B][max_pages]."""
        page_size = int(page_size)
        for t in (k, v, k_scale, v_scale):
            if t.dim() < 3 or t.shape[:2] != k.shape[:2]:
                raise ValueError("pools must be [pages][heads] and what a page of a head holds")
        pages, heads = int(k.shape[0]), int(k.shape[1])
        keys = pages * heads * page_size
        if any(t.element_size() != 1 for t in (k, v, k_scale)) or v.numel() != k.numel():
            raise ValueError("k, v and k_scale must be bytes, k and v of one size")
        if v_scale.dtype not in _SCALES or v_scale.numel() != keys:
            raise ValueError("v_scale must be a bfloat16 for each key")
        dim = 2 * k.numel() // max(1, keys)
        if dim * keys != 2 * k.numel() or k_scale.numel() * SD_KV4_GROUP != dim * keys:
            raise ValueError("pool sizes are not pages * heads * page_size * head_dim / 2, and a scale byte for each key and 32 columns")
        if block_table.dtype != torch.int32 or block_table.dim() != 2:
            raise ValueError("need an int32 block table [B][max_pages]")
        c = cls(*(_b._ptr(t) for t in (k, v, k_scale, v_scale, block_table)), int(block_table.shape[1]), page_size, pages)
        c._tensors = (k, v, k_scale, v_scale, block_table)
        c._heads, c._dim, c._rows = heads, dim, int(block_table.shape[0])
        c._device = _device(c._tensors)
        return c

    def _fits(self, dims: Dims, dev: int) -> None:
        if dev != self._device:
            raise ValueError("device arguments must be on one device")
        if dims.n_kv_heads != self._heads or dims.head_dim != self._dim or dims.batch > self._rows:
            raise ValueError("the cache's heads, head dimension or table rows are not those of dims")


class Rope(ctypes.Structure):
    """sd_rope_t"""
    _fields_ = [(n, ctypes.c_int32) for n in ("rows", "n_q_heads", "n_kv_heads", "head_dim", "rotary_dim", "interleaved",
                                              "dtype")] + [("eps", ctypes.c_float)]


_ready = False


def _library() -> ctypes.CDLL:
    global _ready
    lib = _b.library()
    if not _ready:
        P, I32, I64, SZ, F = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float
        DP, CP = ctypes.POINTER(Dims), ctypes.POINTER(KV4Cache)
        lib.sd_kv4_workspace_bytes.argtypes = [DP, I32]
        lib.sd_kv4_workspace_bytes.restype = SZ
        for name, args in (("sd_qk_norm_rope", [ctypes.POINTER(Rope), P, I64, P, I64, P, P, P, P, P, I64, P, I64, P]),
                           ("sd_kv4_append", [DP, CP, P, I64, P, I64, P, P, P, P]),
                           ("sd_kv4_read", [DP, CP, P, P, P, P, I64, P, I64, P]),
                           ("sd_verify_attention_kv4", [DP, P, CP, P, P, F, P, P, SZ, P])):
            getattr(lib, name).argtypes = args
            getattr(lib, name).restype = ctypes.c_int
        _ready = True
    return lib


def exported_fp4_symbols() -> list:
    """Names of the functions include/sdverify_fp4.h declares."""
    with open(_HEADER) as f:
        return re.findall(r"SD_API\s+[\w\s\*]*?\b(sd_\w+)\s*\(", f.read())


# ---- the C calls ----------------------------------------------------------------

def sd_kv4_workspace_bytes(dims: Dims, max_kv_len: int) -> int:
    return int(_library().sd_kv4_workspace_bytes(ctypes.byref(dims), int(max_kv_len)))


def _head_rows(t, shape, dtype, what: str):
    """Address and row stride of [rows][heads][head_dim] (rows may be slices of wider ones)."""
    if t.dtype != dtype:
        raise ValueError(f"{what}: expected {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{what}: expected rows [{shape[0]}][{shape[1]}][{shape[2]}]")
    row, head, column = t.stride()
    if column != 1 or (head != shape[2] and shape[1] > 1):
        raise ValueError(f"{what}: a row must be contiguous")
    return t.data_ptr(), row if shape[0] > 1 else shape[1] * shape[2]


@functools.lru_cache(maxsize=64)
def _rope(*fields):
    rope = Rope(*fields)
    return rope, ctypes.byref(rope)


def sd_qk_norm_rope(q, k, positions, inv_freq, q_weight, k_weight, eps: float, q_out, k_out, interleaved: bool = False,
                    stream=None) -> None:
    """Rows, heads and columns are q's and k's: [rows][heads][head_dim], float32 or bfloat16;
    rotary_dim is twice inv_freq's length."""
    dev = _device((q, k, positions, inv_freq, q_weight, k_weight, q_out, k_out))
    t, qh, kh = q.dtype, q.shape, k.shape
    if len(qh) != 3 or len(kh) != 3 or (t != torch.bfloat16 and t != torch.float32):
        raise ValueError("q and k: expected float32 or bfloat16 rows [rows][heads][head_dim]")
    rows, heads, dim = qh
    if kh[0] != rows or kh[2] != dim:
        raise ValueError(f"k: expected rows [{rows}][heads][{dim}]")
    qp, qs = _head_rows(q, qh, t, "q")
    kp, ks = _head_rows(k, kh, t, "k")
    qo, qos = _head_rows(q_out, qh, t, "q_out")
    ko, kos = _head_rows(k_out, kh, t, "k_out")
    rope = _rope(rows, heads, kh[1], dim, 2 * inv_freq.numel(), 1 if interleaved else 0,
                 SD_DTYPE_F32 if t == torch.float32 else SD_DTYPE_BF16, eps)[1]
    _run(_library().sd_qk_norm_rope, "sd_qk_norm_rope", dev, stream, rope, qp, qs, kp, ks,
         _typed(positions, torch.int32, "positions", rows), _typed(inv_freq, torch.float32, "inv_freq", 0),
         None if q_weight is None else _typed(q_weight, t, "q_weight", dim),
         None if k_weight is None else _typed(k_weight, t, "k_weight", dim), qo, qos, ko, kos)


def sd_kv4_append(dims: Dims, cache: KV4Cache, k_new, v_new, new_off: Sequence[int], new_len: Sequence[int],
                  kv_len: Sequence[int], stream=None) -> None:
    dev = _device((k_new, v_new))
    cache._fits(dims, dev)
    B = dims.batch
    off, off_p = _lengths(new_off, np.int64, B, "new_off")
    new, new_p = _lengths(new_len, np.int32, B, "new_len")
    ln, len_p = _lengths(kv_len, np.int32, B, "kv_len")
    k, k_stride = _new_rows(k_new, dims, "k_new")
    v, v_stride = _new_rows(v_new, dims, "v_new")
    if _passes(off, new, min(k_new.shape[0], v_new.shape[0])):
        raise ValueError("new_off + new_len passes the last new row")
    if (k == 0 or v == 0) and not (new > 0).any():  # no rows at all: nothing to append
        return
    _run(_library().sd_kv4_append, "sd_kv4_append", dev, stream, ctypes.byref(dims), ctypes.byref(cache), k, k_stride,
         v, v_stride, off_p, new_p, len_p)


def sd_kv4_read(dims: Dims, cache: KV4Cache, first: Sequence[int], count: Sequence[int], out_off: Sequence[int], k_out,
                v_out, stream=None) -> None:
    """k_out and v_out: rows [T][n_kv_heads][head_dim] in dims.dtype; either may be None."""
    dev = _device((k_out, v_out))
    cache._fits(dims, dev)
    B = dims.batch
    at, at_p = _lengths(first, np.int32, B, "first")
    n, n_p = _lengths(count, np.int32, B, "count")
    off, off_p = _lengths(out_off, np.int64, B, "out_off")
    k, k_stride = (None, 0) if k_out is None else _new_rows(k_out, dims, "k_out")
    v, v_stride = (None, 0) if v_out is None else _new_rows(v_out, dims, "v_out")
    if _passes(off, n, min(len(t) for t in (k_out, v_out) if t is not None)):
        raise ValueError("out_off + count passes the last row")
    if not (k or v) and not (n > 0).any():  # no rows at all: nothing to read
        return
    _run(_library().sd_kv4_read, "sd_kv4_read", dev, stream, ctypes.byref(dims), ctypes.byref(cache), at_p, n_p,
         off_p, k, k_stride, v, v_stride)


def sd_verify_attention_kv4(dims: Dims, q, cache: KV4Cache, kv_len: Sequence[int], parent, scale: float, out, workspace,
                            stream=None) -> None:
    dev = _device((q, parent, out, workspace))
    cache._fits(dims, dev)
    n = dims.batch * (dims.gamma + 1) * dims.n_q_heads * dims.head_dim
    ln, len_p = _lengths(kv_len, np.int32, dims.batch, "kv_len")
    p = None if parent is None else _typed(parent, torch.int32, "parent", dims.batch * dims.gamma)
    _run(_library().sd_verify_attention_kv4, "sd_verify_attention_kv4", dev, stream, ctypes.byref(dims),
         _typed(q, torch.bfloat16, "q", n), ctypes.byref(cache), len_p, p, float(scale),
         _typed(out, torch.bfloat16, "out", n), _b._ptr(workspace), _b._nbytes(workspace))
