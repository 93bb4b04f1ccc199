"""ctypes marshalling of the 8-bit calls (include/sdverify_fp8.h).

Argument conversion, and the checks that only tensors allow: element types,
sizes, and one device for all.  A call runs on that device (and, without a
``stream``, on its current stream), whichever device is current.
"""

from __future__ import annotations

import ctypes
import os
import re
from typing import Sequence

import numpy as np
import torch

from . import _binding as _b
from ._binding import SD_DTYPE_BF16, SD_DTYPE_F32, Dims, _check

SD_KV8_BLOCK = 64
SD_FP8_BLOCK = 128

_HEADER = os.path.join(os.path.dirname(_b._HEADER), "sdverify_fp8.h")
_F8 = torch.float8_e4m3fn
_TYPES = {SD_DTYPE_F32: torch.float32, SD_DTYPE_BF16: torch.bfloat16}


class KV8Cache(ctypes.Structure):
    """sd_kv8_cache_t: an 8-bit paged cache.  Build it with KV8Cache.of(...),
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
    def of(cls, k, v, k_scale, v_scale, block_table, page_size: int) -> "KV8Cache":
        """Pools of e4m3 (or uint8) codes, whose first dimension is the page,
        scale pools [pages][Hkv][page_size / 64] of exponent bytes, and the
        int32 table [B][max_pages]."""
        page_size = int(page_size)
        for t in (k, v):
            if t.element_size() != 1 or t.shape[0] != k.shape[0] or t.numel() != k.numel():
                raise ValueError("k and v must be pools of one-byte codes of one size")
        for t in (k_scale, v_scale):
            if t.element_size() != 1 or t.dim() != 3 or t.shape[0] != k.shape[0] or t.shape[2] * SD_KV8_BLOCK != page_size:
                raise ValueError("scales must be bytes [pages][heads][page_size / 64]")
        if k_scale.shape != v_scale.shape or block_table.dtype != torch.int32 or block_table.dim() != 2:
            raise ValueError("need equal scale pools and an int32 block table [B][max_pages]")
        c = cls(*(_b._ptr(t) for t in (k, v, k_scale, v_scale, block_table)), int(block_table.shape[1]), page_size,
                int(k.shape[0]))
        c._tensors = (k, v, k_scale, v_scale, block_table)
        c._heads = int(k_scale.shape[1])
        c._rows = int(block_table.shape[0])
        rows = int(k.shape[0]) * c._heads * page_size
        c._dim = k.numel() // max(1, rows)
        if c._dim * rows != k.numel():
            raise ValueError("a pool's size is not pages * heads * page_size * head_dim")
        c._device = _device(c._tensors)
        return c

    def _fits(self, dims: Dims, dev: int) -> None:
        if dev != self._device:
            raise ValueError("device arguments must be on one device")
        if dims.n_kv_heads != self._heads or dims.head_dim != self._dim or dims.batch > self._rows:
            raise ValueError("the cache's heads, head dimension or table rows are not those of dims")


class Norm(ctypes.Structure):
    """sd_norm_t"""
    _fields_ = [("rows", ctypes.c_int32), ("width", ctypes.c_int32), ("dtype", ctypes.c_int32), ("eps", ctypes.c_float)]


_ready = False


def _library() -> ctypes.CDLL:
    global _ready
    lib = _b.library()
    if not _ready:
        P, I32, I64, SZ, F = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float
        DP, CP = ctypes.POINTER(Dims), ctypes.POINTER(KV8Cache)
        lib.sd_fp8_workspace_bytes.argtypes = [DP, I32]
        lib.sd_fp8_workspace_bytes.restype = SZ
        for name, args in (("sd_kv8_append", [DP, CP, P, I64, P, I64, P, P, P, P]),
                           ("sd_verify_attention_kv8", [DP, P, CP, P, P, F, P, P, SZ, P]),
                           ("sd_residual_norm_fp8", [ctypes.POINTER(Norm), P, P, P, P, P, P, P]),
                           ("sd_verify_logits_fp8", [DP, P, P, P, P, P, P, P, SZ, P])):
            getattr(lib, name).argtypes = args
            getattr(lib, name).restype = ctypes.c_int
        _ready = True
    return lib


def exported_fp8_symbols() -> list:
    """Names of the functions include/sdverify_fp8.h declares."""
    with open(_HEADER) as f:
        return re.findall(r"SD_API\s+[\w\s\*]*?\b(sd_\w+)\s*\(", f.read())


# ---- marshalling helpers ------------------------------------------------------

def _device(tensors) -> int:
    """The index of the one device of the tensors (None among them is left out)."""
    dev = -2  # none yet; a host tensor's is -1
    for t in tensors:
        if t is None:
            continue
        if not isinstance(t, torch.Tensor):
            raise TypeError(f"expected a torch device tensor, got {type(t).__name__}")
        d = t.get_device()
        if d != dev:
            if d < 0:
                raise ValueError("device arguments must be GPU tensors")
            if dev >= 0:
                raise ValueError("device arguments must be on one device")
            dev = d
    return dev


def _typed(t, dtype, what: str, elements: int) -> int:
    """The address of a contiguous tensor of this type with this many elements at least."""
    if t.dtype != dtype and not (dtype == _F8 and t.dtype == torch.uint8):
        raise ValueError(f"{what}: expected {dtype}, got {t.dtype}")
    if t.numel() < elements:
        raise ValueError(f"{what}: {t.numel()} elements, {elements} needed")
    if not t.is_contiguous():
        raise ValueError("device arguments must be contiguous")
    return t.data_ptr()


_address, _byte = ctypes.addressof, ctypes.c_char.from_buffer


def _lengths(a, dtype, batch: int, what: str):
    arr = np.ascontiguousarray(a, dtype=dtype)
    if arr.size != batch:
        raise ValueError(f"{what}: {arr.size} entries for {batch} requests")
    try:  # a third of the other way's time
        return arr, _address(_byte(arr))
    except (TypeError, ValueError):  # not writable, or empty
        return arr, arr.__array_interface__["data"][0]


def _passes(off, count, limit: int) -> bool:
    """Whether some request's rows end past `limit` (a request without rows has none)."""
    over = off > np.subtract(limit, count, dtype=np.int64)  # a sum could wrap
    return bool(over.any()) and bool((over & (count > 0)).any())


def _run(fn, where: str, dev: int, stream, *args) -> None:
    if stream is None:
        handle = torch._C._cuda_getCurrentRawStream(dev)
    elif isinstance(stream, torch.cuda.Stream):
        if stream.device.index != dev:
            raise ValueError("the stream belongs to another device than the tensors")
        handle = stream.cuda_stream
    else:
        handle = int(stream)
    if dev == torch._C._cuda_getDevice():
        st = fn(*args, handle)
    else:
        with torch.cuda.device(dev):
            st = fn(*args, handle)
    _check(st, where)


# ---- the C calls ----------------------------------------------------------------

def sd_fp8_workspace_bytes(dims: Dims, max_kv_len: int) -> int:
    return int(_library().sd_fp8_workspace_bytes(ctypes.byref(dims), int(max_kv_len)))


def _new_rows(t, dims: Dims, what: str):
    """Address and row stride of [T][Hkv][D] rows (rows may be slices of wider ones)."""
    if t.dtype != _TYPES.get(dims.dtype):
        raise ValueError(f"{what}: the type is not dims.dtype's")
    shape, heads, dim = t.shape, dims.n_kv_heads, dims.head_dim
    if len(shape) != 3 or shape[1] != heads or shape[2] != dim:
        raise ValueError(f"{what}: expected rows [T][n_kv_heads][head_dim]")
    row, head, column = t.stride()
    if column != 1 or (heads > 1 and head != dim):
        raise ValueError(f"{what}: a row must be contiguous")
    return t.data_ptr(), row if shape[0] > 1 else heads * dim


def sd_kv8_append(dims: Dims, cache: KV8Cache, k_new, v_new, new_off: Sequence[int], new_len: Sequence[int],
                  kv_len: Sequence[int], stream=None) -> None:
    dev = _device((k_new, v_new))
    cache._fits(dims, dev)
    off, off_p = _lengths(new_off, np.int64, dims.batch, "new_off")
    new, new_p = _lengths(new_len, np.int32, dims.batch, "new_len")
    ln, len_p = _lengths(kv_len, np.int32, dims.batch, "kv_len")
    k, k_stride = _new_rows(k_new, dims, "k_new")
    v, v_stride = _new_rows(v_new, dims, "v_new")
    if _passes(off, new, min(k_new.shape[0], v_new.shape[0])):
        raise ValueError("new_off + new_len passes the last new row")
    if k == 0 or v == 0:  # no rows at all: nothing to append
        if k_new.numel() == 0 and v_new.numel() == 0 and not (new > 0).any():
            return
    _run(_library().sd_kv8_append, "sd_kv8_append", dev, stream, ctypes.byref(dims), ctypes.byref(cache), k, k_stride,
         v, v_stride, off_p, new_p, len_p)


def sd_verify_attention_kv8(dims: Dims, q, cache: KV8Cache, kv_len: Sequence[int], parent, scale: float, out, workspace,
                            stream=None) -> None:
    dev = _device((q, parent, out, workspace))
    cache._fits(dims, dev)
    n = dims.batch * (dims.gamma + 1) * dims.n_q_heads * dims.head_dim
    ln, len_p = _lengths(kv_len, np.int32, dims.batch, "kv_len")
    p = None if parent is None else _typed(parent, torch.int32, "parent", dims.batch * dims.gamma)
    _run(_library().sd_verify_attention_kv8, "sd_verify_attention_kv8", dev, stream, ctypes.byref(dims),
         _typed(q, torch.bfloat16, "q", n), ctypes.byref(cache), len_p, p, float(scale),
         _typed(out, torch.bfloat16, "out", n), _b._ptr(workspace), _b._nbytes(workspace))


def sd_residual_norm_fp8(x, residual, weight, eps: float, new_residual, out, out_scale, stream=None) -> None:
    """Rows and columns are x's: [rows][width], float32 or bfloat16."""
    dev = _device((x, residual, weight, new_residual, out, out_scale))
    if x.dim() != 2 or x.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("x: expected float32 or bfloat16 rows [rows][width]")
    rows, width = x.shape
    n, t = rows * width, x.dtype
    norm = Norm(rows, width, SD_DTYPE_F32 if t == torch.float32 else SD_DTYPE_BF16, float(eps))
    _run(_library().sd_residual_norm_fp8, "sd_residual_norm_fp8", dev, stream, ctypes.byref(norm), _b._ptr(x),
         None if residual is None else _typed(residual, t, "residual", n), _typed(weight, t, "weight", width),
         None if new_residual is None else _typed(new_residual, t, "new_residual", n), _typed(out, _F8, "out", n),
         _typed(out_scale, torch.float32, "out_scale", -(-width // SD_FP8_BLOCK) * rows))


def sd_verify_logits_fp8(dims: Dims, hidden, hidden_scale, w, w_scale, logits, row_lse, workspace, stream=None) -> None:
    dev = _device((hidden, hidden_scale, w, w_scale, logits, row_lse, workspace))
    M, V, K = dims.batch * (dims.gamma + 1), dims.vocab, dims.hidden
    kb, vb = -(-K // SD_FP8_BLOCK), -(-V // SD_FP8_BLOCK)
    _run(_library().sd_verify_logits_fp8, "sd_verify_logits_fp8", dev, stream, ctypes.byref(dims),
         _typed(hidden, _F8, "hidden", M * K), _typed(hidden_scale, torch.float32, "hidden_scale", kb * M),
         _typed(w, _F8, "w", V * K), _typed(w_scale, torch.float32, "w_scale", vb * kb),
         _typed(logits, torch.float32, "logits", M * V), _typed(row_lse, torch.float32, "row_lse", M),
         _b._ptr(workspace), _b._nbytes(workspace))
