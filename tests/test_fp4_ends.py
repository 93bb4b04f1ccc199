"""Rows near float32's end in the 4-bit cache: what is finite stays finite, on the oracle and on the GPU."""

import numpy as np
import pytest
import torch

import paper_2601_21622_amd as sd
from oracle import fp4

from test_gpu_kv4 import Cache, dims_of

MOST = {torch.float32: float(np.finfo(np.float32).max), torch.bfloat16: 255 * 2.0 ** 120}  # the types' largest numbers
# 6 * 2^125, the largest finite that a key's codes stand for, and values on either side of every border above it.
TOPS = [6 * 2.0 ** 125, np.nextafter(np.float32(6 * 2.0 ** 125), np.float32(0)), np.nextafter(np.float32(6 * 2.0 ** 125), np.float32(np.inf)),
        1.625 * 2.0 ** 127, np.nextafter(np.float32(1.75 * 2.0 ** 127), np.float32(0)), 1.75 * 2.0 ** 127, 1.875 * 2.0 ** 127,
        254 * 2.0 ** 120, 255 * 2.0 ** 120, np.nextafter(np.float32(255 * 2.0 ** 120), np.float32(np.inf)),
        MOST[torch.float32], 5.67e37 * 2, 1e38]


def near_the_end(dim, dtype):
    """[rows][2 heads][dim]: a largest element of every kind, others of any size below it."""
    rng = np.random.default_rng(dim)
    x = rng.uniform(-1, 1, (2 * len(TOPS), 2, dim)) * 2.0 ** rng.integers(-8, 1, (2 * len(TOPS), 2, dim))
    for i, top in enumerate(TOPS):
        x[2 * i:2 * i + 2] *= min(float(top), MOST[dtype])
        x[2 * i, :, 5::32], x[2 * i + 1, :, 5::32] = min(float(top), MOST[dtype]), -min(float(top), MOST[dtype])
    t = torch.from_numpy(x.astype(np.float32)).to(dtype)
    assert torch.isfinite(t).all()
    return t


def check_finite(x, k, v):
    """x [rows][dim] against its key and value. A key's scale is 2^125 at most: the nearest code is off by 2^125 (half of
    the step from 4 to 6), or by what lies past 6 * 2^125.  A value's is s = 170 * 2^118 at most, 6 s the largest
    bfloat16: off by s, past which no finite float32 lies by more."""
    assert np.isfinite(k).all() and np.isfinite(v).all()
    assert (np.abs(k - x) <= np.maximum(2.0 ** 125, np.abs(x) - 6 * 2.0 ** 125)).all()
    assert (np.abs(v - x) <= 170 * 2.0 ** 118).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dim", [64, 128])
def test_finite_rows_stay_finite(dim, dtype):
    x = near_the_end(dim, dtype).double().numpy()
    n = len(x)
    pools = [np.zeros((1, 2, 1, 32 * dim), np.uint8), np.zeros((1, 2, 1, 32 * dim), np.uint8), np.zeros((1, 2, 1, 2 * dim), np.uint8),
             np.zeros((1, 2, 1, 64), np.uint16)]
    pools = fp4.append(*pools, [[0]], x, x, [0], [n], [n])
    for h in range(2):
        k, v = fp4.rows(*pools, [0], 0, n, h)
        check_finite(x[:, h], k, v)
        again = fp4.append(*pools, [[0]], np.stack([k, k], 1), np.stack([v, v], 1), [0], [n], [n])
        for a, b in zip((k, v), fp4.rows(*again, [0], 0, n, h)):
            assert np.array_equal(a, b)
    assert pools[2].max() == 252 and pools[3].max() <= 0x7e2a


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dim", [64, 128])
def test_finite_rows_stay_finite_on_the_gpu(dim, dtype):
    """Bytes are the oracle's; rows are read back finite in either type."""
    x = near_the_end(dim, dtype)
    n = len(x)
    c = Cache(np.random.default_rng(3), [n], 2, dim, 64)
    c.append(x.double().numpy(), x.double().numpy(), [0], [n], [n])
    dev = x.cuda()
    sd.sd_kv4_append(dims_of(1, 2, dim, dtype), c.handle, dev, dev, [0], [n], [n])
    torch.cuda.synchronize()
    c.check()
    for t in (torch.float32, torch.bfloat16):
        out = [torch.full((n, 2, dim), float("nan"), dtype=t, device="cuda") for _ in range(2)]
        sd.sd_kv4_read(dims_of(1, 2, dim, t), c.handle, [0], [n], [0], *out)
        torch.cuda.synchronize()
        for h in range(2):
            want = fp4.rows(*c.host, c.table[0], 0, n, h)
            check_finite(x[:, h].double().numpy(), *want)
            for got, w in zip(out, want):
                assert torch.equal(got[:, h].cpu(), torch.from_numpy(w).float().to(t))
