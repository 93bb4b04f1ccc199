"""Handles of the quantised caches hold their pools as long as they live, and no longer."""

import gc
import weakref

import pytest
import torch

import paper_2601_21622_amd as sd
from paper_2601_21622_amd import _binding


class _OnGpu(torch.Tensor):
    """A tensor that says it lies on the first GPU."""

    def get_device(self):
        return 0


def kv4(device, pages=3, heads=2, dim=64, page=128):
    byte = dict(dtype=torch.uint8, device=device)
    shape = (pages, heads, page // 64)
    return sd.KV4Cache, [torch.zeros((*shape, 32 * dim), **byte), torch.zeros((*shape, 32 * dim), **byte),
                         torch.zeros((*shape, 2 * dim), **byte), torch.zeros((*shape, 64), dtype=torch.bfloat16, device=device),
                         torch.zeros((1, pages), dtype=torch.int32, device=device)], page


def kv8(device, pages=3, heads=2, dim=64, page=128):
    byte = dict(dtype=torch.uint8, device=device)
    shape = (pages, heads, page // 64)
    return sd.KV8Cache, [torch.zeros((*shape, 64 * dim), **byte), torch.zeros((*shape, 64 * dim), **byte),
                         torch.zeros(shape, **byte), torch.zeros(shape, **byte),
                         torch.zeros((1, pages), dtype=torch.int32, device=device)], page


@pytest.mark.parametrize("make", [kv4, kv8])
def test_a_handle_lets_go_of_its_pools(make, monkeypatch):
    monkeypatch.setattr(_binding, "_ptr", lambda t: t.data_ptr())
    kind, pools, page = make("cpu")
    pools = [t.as_subclass(_OnGpu) for t in pools]
    cache = kind.of(*pools, page)
    alive = [weakref.ref(t) for t in pools]
    del pools
    gc.collect()
    assert all(r() is not None for r in alive)  # the handle's own
    del cache
    gc.collect()
    assert not any(r() is not None for r in alive)


@pytest.mark.gpu
@pytest.mark.parametrize("make", [kv4, kv8])
def test_pools_are_freed_on_the_gpu(make):
    """After calls through it, too; tables that are made anew for the same pools go one by one."""
    gc.collect()
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    kind, pools, page = make("cuda")
    held = torch.cuda.memory_allocated()
    rows = torch.zeros((4, 2, 64), dtype=torch.bfloat16, device="cuda")
    append = sd.sd_kv4_append if make is kv4 else sd.sd_kv8_append
    dims = sd.Dims(1, 0, 2, 2, 64, 32, 1, 1, 0)
    for n in range(4, 12):
        append(dims, kind.of(*pools[:4], pools[4].clone(), page), rows, rows, [0], [4], [n])
    torch.cuda.synchronize()
    del rows
    gc.collect()
    assert torch.cuda.memory_allocated() == held
    del pools
    gc.collect()
    assert torch.cuda.memory_allocated() == before
