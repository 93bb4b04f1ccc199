"""Pins of oracle.fp8: the code table against torch's e4m3 type, rounding
against torch's cast, the layouts against their documented index order, the
append against hand-worked blocks, the norm and the projection against plain
formulas."""

import numpy as np
import pytest
import torch

from oracle import fp8


def test_codes_are_torchs():
    v = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(fp8.VALUES, v, equal_nan=True)


def test_encode_is_torchs_cast():
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.normal(0, 100, 20000), rng.normal(0, 0.01, 20000), fp8.VALUES, -fp8.VALUES,
                        (fp8.VALUES[:126] + fp8.VALUES[1:127]) / 2,  # ties
                        [0.0, -0.0, 464.0, 464.1, 1e30, np.inf, -np.inf, np.nan, 2.0 ** -10, 2.0 ** -11]]).astype(np.float32)
    t = torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(fp8.decode(fp8.encode(x)), t, equal_nan=True)


@pytest.mark.parametrize("most,e", [(0.0, -100), (448.0, 0), (449.0, 1), (224.0, -1), (1.0, -8), (2.0 ** -130, -100),
                                    (3.3e38, 120)])
def test_scale_exponent(most, e):
    assert fp8.scale_exponent(most) == e


@pytest.mark.parametrize("dim", [64, 128])
def test_layouts(dim):
    """A pool written through the documented dimensions reads back by index."""
    x = np.arange(64 * dim).reshape(64, dim)
    k = np.empty((dim // 64, 4, 4, 16, 16), dtype=int)
    v = np.empty((dim // 16, 4, 16, 4, 4), dtype=int)
    for i, t, g, r, b in np.ndindex(k.shape):
        k[i, t, g, r, b] = x[16 * t + r, 64 * i + 16 * g + b]
    for i, g, d, t, r in np.ndindex(v.shape):
        v[i, g, d, t, r] = x[16 * t + 4 * g + r, 16 * i + d]
    assert np.array_equal(k.reshape(-1)[fp8.k_index(dim)], x)
    assert np.array_equal(v.reshape(-1)[fp8.v_index(dim)], x)


def test_append_by_hand():
    """One head, pages of one block: a block begun, then grown by a larger row,
    then cut back and overwritten; later bytes and other pages stay."""
    dim, idx = 64, fp8.k_index(64)
    pool = np.full((3, 1, 1, 64 * dim), 0x11, dtype=np.uint8)
    scales = np.full((3, 1, 1), 130, dtype=np.uint8)
    table = np.array([[2]])
    rows = np.zeros((4, 1, dim))
    rows[0, 0, 0], rows[1, 0, 1] = 448.0, -3.0
    p, s = fp8.append(pool, scales, table, rows, [0], [2], [2], idx)
    assert s[2, 0, 0] == 127 and (s[:2] == 130).all() and (p[:2] == 0x11).all()
    got = fp8.decode(p[2, 0, 0][idx])
    assert got[0, 0] == 448 and got[1, 1] == -3 and (got[:2] != 0).sum() == 2
    assert (p[2, 0, 0][idx][2:] == 0x11).all()
    rows[2, 0, 0] = 1000.0  # needs 2^2: 3 / 4 stays exact, 1000 / 4 = 250 rounds to 256
    p, s = fp8.append(p, s, table, rows, [2], [1], [3], idx)
    assert s[2, 0, 0] == 129
    got = fp8.cache_rows(p, s, table[0], 3, 0, idx)
    assert got[0, 0] == 448 and got[1, 1] == -3 and got[2, 0] == 1024
    rows[3, 0, 5] = np.inf  # cut back to one key: the scale does not shrink, infinity is NaN
    p, s = fp8.append(p, s, table, rows, [3], [1], [2], idx)
    got = fp8.cache_rows(p, s, table[0], 3, 0, idx)
    assert s[2, 0, 0] == 129 and got[0, 0] == 448 and np.isnan(got[1, 5]) and got[2, 0] == 1024
    q, z = fp8.append(p, s, table, rows, [0], [0], [3], idx)
    assert np.array_equal(p, q) and np.array_equal(s, z)


def test_segments_give_back_what_was_appended():
    rng = np.random.default_rng(1)
    dim, heads, lens = 64, 2, [70, 1, 130]
    table = np.array([[4, 1], [0, 0], [5, 2]])
    pools = [rng.integers(0, 255, (6, heads, 2, 64 * dim), dtype=np.uint8) & 0x77 for _ in range(2)]
    scales = [np.full((6, heads, 2), 127, dtype=np.uint8) for _ in range(2)]
    x = [fp8.decode(rng.integers(0, 120, (sum(lens), heads, dim))) for _ in range(2)]
    off = np.cumsum([0] + lens[:-1])
    idx = fp8.k_index(dim), fp8.v_index(dim)
    done = [fp8.append(pools[i], scales[i], table, x[i], off, lens, lens, idx[i]) for i in range(2)]
    k, v, seg = fp8.kv8_segments(done[0][0], done[1][0], done[0][1], done[1][1], table, lens)
    for got, want in ((k, x[0]), (v, x[1])):
        for b, n in enumerate(lens):
            part = got[seg[b]:seg[b] + heads * n * dim].reshape(heads, n, dim)
            ref = want[off[b]:off[b] + n].transpose(1, 0, 2)
            # codes of another power of two: exact where the block's scale leaves them in range
            assert np.all(np.abs(part - ref) <= 2.0 ** -10 * np.abs(ref).max())


def test_norm_and_projection():
    rng = np.random.default_rng(2)
    x, r, w = rng.normal(size=(3, 160)), rng.normal(size=(3, 160)), rng.normal(size=160)
    h, y, s = fp8.residual_norm(x, r, w, 1e-5)
    ref = torch.nn.functional.rms_norm(torch.from_numpy(x + r), (160,), torch.from_numpy(w), 1e-5).numpy()
    assert np.allclose(y, ref, rtol=1e-12) and np.array_equal(h, x + r) and s.shape == (2, 3)
    assert np.allclose(s[0], np.abs(y[:, :128]).max(1) / 448) and np.allclose(s[1], np.abs(y[:, 128:]).max(1) / 448)
    a, b = rng.integers(0, 126, (2, 160), dtype=np.uint8), rng.integers(128, 254, (130, 160), dtype=np.uint8)
    sa, sb = rng.random((2, 2)), rng.random((2, 2))
    got, mag = fp8.logits_fp8(a, sa, b, sb)
    for m, v in ((0, 0), (1, 127), (1, 128), (0, 129)):
        ref = sum(fp8.VALUES[a[m, k]] * sa[k // 128, m] * fp8.VALUES[b[v, k]] * sb[v // 128, k // 128] for k in range(160))
        assert np.isclose(got[m, v], ref, rtol=1e-12) and np.isclose(mag[m, v], -ref, rtol=1e-12)
