"""Refusals of the 8-bit calls, on the CPU: bad arguments return the
documented status before anything is enqueued, and the binding refuses what
only tensors show."""

import ctypes

import pytest
import torch

import paper_2601_21622_amd as sd

P = 0x100000  # a fake, aligned address: every call below fails its host checks
cpu_only = pytest.mark.skipif(torch.cuda.is_available(), reason="host-validation tests use fake pointers")
BAD, UNSUPPORTED, WORKSPACE = sd.SD_ERR_INVALID_ARGUMENT, sd.SD_ERR_UNSUPPORTED, sd.SD_ERR_WORKSPACE


def dims(**kw):
    base = dict(batch=2, gamma=3, n_q_heads=8, n_kv_heads=2, head_dim=128, hidden=1024, vocab=1000, dtype=1)
    base.update(kw)
    return sd.Dims(**base)


def cache(**kw):
    base = dict(k=P, v=P, k_scale=P, v_scale=P, block_table=P, max_pages=4, page_size=64, num_pages=16)
    base.update(kw)
    return sd.KV8Cache(**base)


def ints(v, t=ctypes.c_int32):
    return (t * len(v))(*v)


def lib():
    sd.sd_fp8_workspace_bytes(dims(), 10)  # sets the argument types
    return sd.library()


def test_exports():
    names = sd.exported_fp8_symbols()
    assert set(names) == {"sd_fp8_workspace_bytes", "sd_kv8_append", "sd_verify_attention_kv8", "sd_residual_norm_fp8",
                          "sd_verify_logits_fp8"}
    for n in names:
        assert hasattr(sd.library(), n)


def test_workspace_bytes():
    a = sd.sd_fp8_workspace_bytes(dims(), 1000)
    assert 0 < a <= sd.sd_fp8_workspace_bytes(dims(), 1 << 20)
    assert sd.sd_fp8_workspace_bytes(dims(gamma=0), 1) > 0
    assert sd.sd_fp8_workspace_bytes(dims(head_dim=96, hidden=100), 1000) == 0
    assert sd.sd_fp8_workspace_bytes(dims(flags=1), 1000) == 0


@pytest.mark.parametrize("vocab", [100, 32000, 33000, 128256])
def test_projection_workspace_grows_with_rows(vocab):
    """A projection's workspace for a large batch serves every smaller one (heads none: the attention has no part)."""
    n = [sd.sd_fp8_workspace_bytes(dims(batch=b, gamma=0, n_q_heads=0, vocab=vocab), 1) for b in range(1, 700)]
    assert all(0 < a <= b for a, b in zip(n, n[1:]))


CACHES = [dict(k=None), dict(v=None), dict(k_scale=None), dict(v_scale=None), dict(block_table=None), dict(k=P + 8),
          dict(v=P + 4), dict(block_table=P + 2), dict(page_size=32), dict(page_size=96), dict(page_size=8192),
          dict(max_pages=0), dict(num_pages=0)]


@cpu_only
@pytest.mark.parametrize("bad", CACHES)
def test_bad_caches(bad):
    c = ctypes.byref(cache(**bad))
    assert lib().sd_verify_attention_kv8(ctypes.byref(dims()), P, c, ints([64, 64]), None, 0.1, P, P, 1 << 30, None) == BAD
    assert lib().sd_kv8_append(ctypes.byref(dims()), c, P, 256, P, 256, ints([0, 1], ctypes.c_int64), ints([1, 1]),
                               ints([5, 5]), None) == BAD


def attend(d=None, c=None, q=P, lens=(200, 64), parent=None, scale=0.1, out=P, ws=P, n=1 << 30):
    return lib().sd_verify_attention_kv8(ctypes.byref(d or dims()), q, ctypes.byref(c or cache()),
                                         None if lens is None else ints(lens), parent, scale, out, ws, n, None)


@cpu_only
@pytest.mark.parametrize("bad,status", [
    (dict(batch=0), BAD), (dict(gamma=-1), BAD), (dict(n_q_heads=7), BAD), (dict(n_kv_heads=0), BAD), (dict(dtype=7), BAD),
    (dict(flags=1), BAD), (dict(head_dim=96), UNSUPPORTED), (dict(dtype=0), UNSUPPORTED), (dict(gamma=64), UNSUPPORTED),
    (dict(n_q_heads=68), UNSUPPORTED), (dict(n_q_heads=140000, n_kv_heads=70000), UNSUPPORTED),
])
def test_attention_refuses_shapes(bad, status):
    assert attend(d=dims(**bad)) == status


@cpu_only
@pytest.mark.parametrize("kw,status", [
    (dict(q=None), BAD), (dict(q=P + 8), BAD), (dict(out=None), BAD), (dict(out=P + 2), BAD), (dict(ws=None), BAD),
    (dict(ws=P + 8), BAD), (dict(lens=None), BAD), (dict(lens=(3, 64)), BAD), (dict(lens=(0, 64)), BAD),
    (dict(lens=(257, 64)), BAD), (dict(parent=P + 2), BAD), (dict(scale=0.0), BAD), (dict(scale=-1.0), BAD),
    (dict(scale=float("nan")), BAD), (dict(scale=float("inf")), BAD), (dict(n=64), WORKSPACE),
])
def test_attention_refuses_arguments(kw, status):
    assert attend(**kw) == status


def append(d=None, k=P, ks=256, v=P, vs=256, off=(0, 1), new=(1, 1), lens=(5, 200)):
    return lib().sd_kv8_append(ctypes.byref(d or dims()), ctypes.byref(cache()), k, ks, v, vs,
                               None if off is None else ints(off, ctypes.c_int64), None if new is None else ints(new),
                               None if lens is None else ints(lens), None)


@cpu_only
@pytest.mark.parametrize("kw,status", [
    (dict(k=None), BAD), (dict(v=None), BAD), (dict(k=P + 8), BAD), (dict(ks=255), BAD), (dict(ks=128), BAD),
    (dict(ks=260), BAD), (dict(vs=0), BAD), (dict(off=None), BAD), (dict(off=(-1, 0)), BAD), (dict(new=None), BAD),
    (dict(new=(-1, 1)), BAD), (dict(new=(6, 1)), BAD), (dict(lens=None), BAD), (dict(lens=(5, 257)), BAD),
    (dict(d=dims(head_dim=32)), UNSUPPORTED), (dict(d=dims(batch=-1)), BAD), (dict(d=dims(dtype=0), ks=258), BAD),
])
def test_append_refuses(kw, status):
    assert append(**kw) == status


@cpu_only
def test_append_of_nothing_enqueues_nothing():
    assert append(new=(0, 0)) == sd.SD_OK


@cpu_only
@pytest.mark.parametrize("kw,ptr,status", [
    (dict(rows=0), {}, BAD), (dict(width=0), {}, BAD), (dict(width=100), {}, UNSUPPORTED), (dict(width=65536), {}, UNSUPPORTED),
    (dict(rows=1 << 25), {}, UNSUPPORTED), (dict(dtype=3), {}, BAD), (dict(eps=-1e-6), {}, BAD),
    (dict(eps=float("nan")), {}, BAD), (dict(eps=float("inf")), {}, BAD), ({}, dict(x=None), BAD), ({}, dict(x=P + 8), BAD),
    ({}, dict(r=P + 8), BAD), ({}, dict(w=None), BAD), ({}, dict(o=P + 4), BAD), ({}, dict(n=P + 4), BAD), ({}, dict(s=None), BAD),
    ({}, dict(s=P + 2), BAD),
])
def test_norm_refuses(kw, ptr, status):
    base = dict(rows=4, width=128, dtype=1, eps=1e-5)
    base.update(kw)
    p = dict(x=P, r=P, w=P, n=P, o=P, s=P)
    p.update(ptr)
    assert lib().sd_residual_norm_fp8(ctypes.byref(sd.Norm(**base)), p["x"], p["r"], p["w"], p["n"], p["o"], p["s"],
                                      None) == status
    assert lib().sd_residual_norm_fp8(None, P, P, P, P, P, P, None) == BAD


@cpu_only
@pytest.mark.parametrize("kw,ptr,status", [
    (dict(hidden=100), {}, UNSUPPORTED), (dict(vocab=0), {}, BAD), (dict(vocab=3_000_000), {}, UNSUPPORTED),
    (dict(hidden=2 ** 23 + 32), {}, UNSUPPORTED), (dict(batch=2 ** 22 + 1), {}, UNSUPPORTED),
    (dict(gamma=-1), {}, BAD), (dict(flags=1), {}, BAD), (dict(batch=1 << 24, gamma=1), {}, UNSUPPORTED), ({}, dict(h=None), BAD),
    ({}, dict(h=P + 8), BAD), ({}, dict(hs=P + 2), BAD), ({}, dict(w=P + 4), BAD), ({}, dict(ws=None), BAD),
    ({}, dict(lo=P + 4), BAD), ({}, dict(lse=None), BAD), ({}, dict(work=None), BAD), ({}, dict(n=8), WORKSPACE),
])
def test_logits_refuses(kw, ptr, status):
    p = dict(h=P, hs=P, w=P, ws=P, lo=P, lse=P, work=P, n=1 << 30)
    p.update(ptr)
    assert lib().sd_verify_logits_fp8(ctypes.byref(dims(**kw)), p["h"], p["hs"], p["w"], p["ws"], p["lo"], p["lse"],
                                      p["work"], p["n"], None) == status


def test_binding_refuses_host_tensors():
    t = torch.zeros(64, 64)
    with pytest.raises(ValueError):
        sd.sd_residual_norm_fp8(t, None, t, 1e-5, None, t, t)
    with pytest.raises(TypeError):
        sd.sd_residual_norm_fp8(3, None, t, 1e-5, None, t, t)
    with pytest.raises(ValueError):
        sd.sd_verify_logits_fp8(dims(), t, t, t, t, t, t, t)
