"""Refusals of the 4-bit calls, on the CPU: bad arguments return the
documented status before anything is enqueued, and the binding refuses what
only tensors show."""

import ctypes

import numpy as np
import pytest
import torch

import paper_2601_21622_amd as sd
from paper_2601_21622_amd import _fp8

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
    return sd.KV4Cache(**base)


def ints(v, t=ctypes.c_int32):
    return (t * len(v))(*v)


def lib():
    sd.sd_kv4_workspace_bytes(dims(), 10)  # sets the argument types
    return sd.library()


def test_exports():
    names = sd.exported_fp4_symbols()
    assert set(names) == {"sd_kv4_workspace_bytes", "sd_qk_norm_rope", "sd_kv4_append", "sd_kv4_read",
                          "sd_verify_attention_kv4"}
    for n in names:
        assert hasattr(sd.library(), n)


def test_workspace_bytes():
    a = sd.sd_kv4_workspace_bytes(dims(), 1000)
    assert 0 < a <= sd.sd_kv4_workspace_bytes(dims(), 1 << 20)
    assert sd.sd_kv4_workspace_bytes(dims(gamma=0), 1) > 0
    for bad in (dict(head_dim=96), dict(flags=1), dict(dtype=0), dict(gamma=64), dict(n_q_heads=7)):
        assert sd.sd_kv4_workspace_bytes(dims(**bad), 1000) == 0
    assert sd.sd_kv4_workspace_bytes(dims(), 3) == 0


CACHES = [dict(k=None), dict(v=None), dict(k_scale=None), dict(v_scale=None), dict(block_table=None), dict(k=P + 8),
          dict(v=P + 4), dict(k_scale=P + 1), dict(v_scale=P + 2), dict(block_table=P + 2), dict(page_size=32),
          dict(page_size=96), dict(page_size=8192), dict(max_pages=0), dict(num_pages=0)]


@cpu_only
@pytest.mark.parametrize("bad", CACHES)
def test_bad_caches(bad):
    c = ctypes.byref(cache(**bad))
    i64 = ints([0, 1], ctypes.c_int64)
    assert lib().sd_verify_attention_kv4(ctypes.byref(dims()), P, c, ints([64, 64]), None, 0.1, P, P, 1 << 30, None) == BAD
    assert lib().sd_kv4_append(ctypes.byref(dims()), c, P, 256, P, 256, i64, ints([1, 1]), ints([5, 5]), None) == BAD
    assert lib().sd_kv4_read(ctypes.byref(dims()), c, ints([1, 1]), ints([5, 5]), i64, P, 256, P, 256, None) == BAD


def attend(d=None, q=P, lens=(200, 64), parent=None, scale=0.1, out=P, ws=P, n=1 << 30):
    return lib().sd_verify_attention_kv4(ctypes.byref(d or dims()), q, ctypes.byref(cache()),
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


@cpu_only
@pytest.mark.parametrize("kw,status", [
    (dict(k=None), BAD), (dict(v=None), BAD), (dict(k=P + 8), BAD), (dict(ks=255), BAD), (dict(ks=128), BAD),
    (dict(ks=260), BAD), (dict(vs=0), BAD), (dict(off=None), BAD), (dict(off=(-1, 0)), BAD), (dict(new=None), BAD),
    (dict(new=(-1, 1)), BAD), (dict(new=(6, 1)), BAD), (dict(lens=None), BAD), (dict(lens=(5, 257)), BAD),
    (dict(d=dims(head_dim=32)), UNSUPPORTED), (dict(d=dims(batch=-1)), BAD), (dict(d=dims(dtype=0), ks=258), BAD),
    (dict(new=(0, 0)), sd.SD_OK),  # enqueues nothing
])
def test_append_refuses(kw, status):
    a = dict(d=dims(), k=P, ks=256, v=P, vs=256, off=(0, 1), new=(1, 1), lens=(5, 200))
    a.update(kw)
    assert lib().sd_kv4_append(ctypes.byref(a["d"]), ctypes.byref(cache()), a["k"], a["ks"], a["v"], a["vs"],
                               None if a["off"] is None else ints(a["off"], ctypes.c_int64),
                               None if a["new"] is None else ints(a["new"]),
                               None if a["lens"] is None else ints(a["lens"]), None) == status


@cpu_only
@pytest.mark.parametrize("kw,status", [
    (dict(k=None, v=None), BAD), (dict(k=P + 8), BAD), (dict(v=P + 4), BAD), (dict(ks=255), BAD), (dict(vs=128), BAD),
    (dict(first=None), BAD), (dict(first=(-1, 0)), BAD), (dict(first=(200, 0), count=(57, 1)), BAD),
    (dict(first=(2 ** 31 - 1, 0), count=(2 ** 31 - 1, 1)), BAD), (dict(count=None), BAD), (dict(count=(-1, 0)), BAD),
    (dict(off=None), BAD), (dict(off=(0, -1)), BAD), (dict(d=dims(head_dim=32)), UNSUPPORTED), (dict(d=dims(flags=1)), BAD),
    (dict(count=(0, 0)), sd.SD_OK), (dict(count=(0, 0), k=None, ks=0), sd.SD_OK),  # enqueue nothing
])
def test_read_refuses(kw, status):
    a = dict(d=dims(), k=P, ks=256, v=P, vs=256, off=(0, 1), first=(0, 3), count=(1, 1))
    a.update(kw)
    assert lib().sd_kv4_read(ctypes.byref(a["d"]), ctypes.byref(cache()), None if a["first"] is None else ints(a["first"]),
                             None if a["count"] is None else ints(a["count"]),
                             None if a["off"] is None else ints(a["off"], ctypes.c_int64), a["k"], a["ks"], a["v"],
                             a["vs"], None) == status


@cpu_only
@pytest.mark.parametrize("kw,arg,status", [
    (dict(rows=-1), {}, BAD), (dict(n_q_heads=0), {}, BAD), (dict(n_kv_heads=0), {}, BAD), (dict(head_dim=0), {}, BAD),
    (dict(rotary_dim=0), {}, BAD), (dict(rotary_dim=144), {}, BAD), (dict(interleaved=2), {}, BAD), (dict(dtype=5), {}, BAD),
    (dict(eps=-1e-6), {}, BAD), (dict(eps=float("nan")), {}, BAD), (dict(eps=float("inf")), {}, BAD),
    (dict(head_dim=256), {}, UNSUPPORTED), (dict(rotary_dim=24), {}, UNSUPPORTED), (dict(rows=1 << 24), {}, UNSUPPORTED),
    (dict(n_q_heads=65536), dict(qs=1 << 24, qos=1 << 24), UNSUPPORTED), ({}, dict(q=None), BAD), ({}, dict(k=P + 8), BAD),
    ({}, dict(pos=None), BAD), ({}, dict(pos=P + 2), BAD), ({}, dict(f=None), BAD), ({}, dict(qw=P + 8), BAD),
    ({}, dict(kw=P + 4), BAD), ({}, dict(qo=None), BAD), ({}, dict(ko=P + 2), BAD), ({}, dict(qs=1023), BAD),
    ({}, dict(ks=255), BAD), ({}, dict(qos=1028), BAD), ({}, dict(kos=128), BAD), (dict(dtype=0), dict(qs=1026), BAD),
    (dict(rows=0), dict(q=None, k=None, pos=None, qo=None, ko=None), sd.SD_OK),
])
def test_rope_refuses(kw, arg, status):
    base = dict(rows=4, n_q_heads=8, n_kv_heads=2, head_dim=128, rotary_dim=128, interleaved=0, dtype=1, eps=1e-6)
    base.update(kw)
    a = dict(q=P, qs=1024, k=P, ks=256, pos=P, f=P, qw=P, kw=P, qo=P, qos=1024, ko=P, kos=256)
    a.update(arg)
    f = lib().sd_qk_norm_rope
    assert f(ctypes.byref(sd.Rope(**base)), a["q"], a["qs"], a["k"], a["ks"], a["pos"], a["f"], a["qw"], a["kw"], a["qo"],
             a["qos"], a["ko"], a["kos"], None) == status
    assert f(None, P, 1024, P, 256, P, P, P, P, P, 1024, P, 256, None) == BAD


def test_binding_refuses_host_tensors():
    t = torch.zeros(4, 2, 64)
    with pytest.raises(ValueError):
        sd.sd_qk_norm_rope(t, t, t, t, None, None, 1e-6, t, t)
    with pytest.raises(TypeError):
        sd.sd_qk_norm_rope(t.numpy(), t, t, t, None, None, 1e-6, t, t)
    with pytest.raises(ValueError):
        sd.KV4Cache.of(t, t, t, t, torch.zeros(1, 1, dtype=torch.int32), 64)


class _OnGpu(torch.Tensor):
    """A tensor that says it lies on the first GPU."""

    def get_device(self):
        return 0


@pytest.mark.parametrize("order", ["host", "host first", "host last"])
def test_one_host_tensor_is_refused(order):
    host, gpu = torch.zeros(8), torch.zeros(8).as_subclass(_OnGpu)
    tensors = {"host": [host, None, host], "host first": [None, host, gpu], "host last": [gpu, None, host]}[order]
    with pytest.raises(ValueError, match="GPU tensors"):
        _fp8._device(tensors)
    assert _fp8._device([None, gpu, gpu]) == 0


def test_binding_refuses_well_formed_host_tensors():
    q, f, pos = torch.zeros(4, 2, 64), torch.zeros(32), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU tensors"):
        sd.sd_qk_norm_rope(q, q, pos, f, None, None, 1e-6, q, q)


@pytest.mark.parametrize("off,count,over", [
    ([0, 6], [4, 4], False), ([0, 7], [4, 4], True), ([0, 99], [10, 0], False), ([0, 0], [11, 0], True), ([10], [0], False),
    ([2 ** 63 - 1], [1], True), ([2 ** 63 - 1], [2 ** 31 - 1], True), ([2 ** 63 - 1], [0], False), ([0], [-2 ** 31], False)])
def test_rows_past_the_last_are_noticed(off, count, over):
    """Negative counts and offsets are the call's own to refuse; sums do not wrap."""
    assert _fp8._passes(np.array(off), np.array(count, dtype=np.int32), 10) == over
