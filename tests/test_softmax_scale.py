"""Softmax scales of the calls over 8-bit and 4-bit caches, on the CPU: the kernels work with scale * log2 e, which
has to be a finite float32, or scores of zero would be NaN."""

import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2601_21622_amd as sd

P = 0x100000  # a fake, aligned address: every call below fails its host checks
FIRST = float(np.float32(np.finfo(np.float32).max / math.log2(math.e)))  # scale * log2 e rounds to float32's end about here


@pytest.mark.skipif(torch.cuda.is_available(), reason="host-validation tests use fake pointers")
@pytest.mark.parametrize("call,cache", [("sd_verify_attention_kv4", sd.KV4Cache), ("sd_verify_attention_kv8", sd.KV8Cache)])
@pytest.mark.parametrize("scale,status", [
    (0.1, sd.SD_ERR_WORKSPACE), (1e-45, sd.SD_ERR_WORKSPACE), (FIRST * 0.999, sd.SD_ERR_WORKSPACE),
    (FIRST * 1.001, sd.SD_ERR_INVALID_ARGUMENT), (3.4e38, sd.SD_ERR_INVALID_ARGUMENT), (math.inf, sd.SD_ERR_INVALID_ARGUMENT),
    (math.nan, sd.SD_ERR_INVALID_ARGUMENT), (0.0, sd.SD_ERR_INVALID_ARGUMENT), (-1.0, sd.SD_ERR_INVALID_ARGUMENT)])
def test_scales_are_finite_in_the_log2_domain(call, cache, scale, status):
    d = sd.Dims(batch=1, gamma=3, n_q_heads=8, n_kv_heads=2, head_dim=128, hidden=1024, vocab=1000, dtype=1)
    sd.sd_kv4_workspace_bytes(d, 10), sd.sd_fp8_workspace_bytes(d, 10)  # set the argument types
    c = cache(P, P, P, P, P, 2000, 64, 4000)
    lens = (ctypes.c_int32 * 1)(100000)  # cut into chunks, for which 64 bytes are no workspace
    assert getattr(sd.library(), call)(ctypes.byref(d), P, ctypes.byref(c), lens, None, scale, P, P, 64, None) == status
