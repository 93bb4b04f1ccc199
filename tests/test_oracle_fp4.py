"""Pins of the 4-bit oracle that do not come from it."""

import itertools
from fractions import Fraction

import numpy as np
import pytest
import torch

from oracle import fp4, verify_attention


def test_codes_by_hand():
    """Every value, every border between neighbours (to the even code) and its surroundings."""
    assert fp4.VALUES.tolist() == [0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6]
    borders = {0.25: 0, 0.75: 2, 1.25: 2, 1.75: 4, 2.5: 4, 3.5: 6, 5.0: 6}
    for i, (x, code) in enumerate(borders.items()):
        assert fp4.encode(x) == code and fp4.encode(-x) == code + 8
        assert fp4.encode(np.nextafter(x, 0)) == i and fp4.encode(np.nextafter(x, 9)) == i + 1
    assert [int(fp4.encode(v)) for v in fp4.VALUES] == list(range(16))
    assert fp4.encode(-0.0) == 8 and fp4.encode(7.0) == 7 and fp4.encode(-100.0) == 15


def test_encode_is_nearest():
    x = np.random.default_rng(0).normal(size=5000) * 3
    got = np.abs(fp4.VALUES[fp4.encode(x)] - x)
    assert np.array_equal(got, np.abs(fp4.VALUES[None, :] - x[:, None]).min(1))


@pytest.mark.parametrize("x", [0.0, 1e-45, 2.0 ** -101, 6 * 2.0 ** -100, 1.0, 5.999, 6.0, 6.0000005, 12.0, 3.4e38, 8.8e37])
def test_scales_are_the_smallest(x):
    x = float(np.float32(x))
    e = fp4.scale_exponent(x)
    assert x <= 6 * 2.0 ** e and (e == -100 or x > 6 * 2.0 ** (e - 1))
    s = fp4.value_scale(x)
    assert Fraction(x) <= 6 * Fraction(float(fp4.bf16_value(s)))
    assert s == 27 << 7 or Fraction(x) > 6 * Fraction(float(fp4.bf16_value(s - 1)))
    assert float(fp4.bf16_value(s)) == float(torch.tensor([s], dtype=torch.int16).view(torch.bfloat16).double())


@pytest.mark.parametrize("dim", [64, 128])
def test_layouts_match_the_header(dim):
    """Index by index against the header's loops; every half byte is used once."""
    ki, vi, si = fp4.k_index(dim), fp4.v_index(dim), fp4.k_scale_index(dim)
    for index, size in ((ki, 64 * dim), (vi, 64 * dim), (si, 2 * dim)):
        assert sorted(index.reshape(-1).tolist()) == list(range(size))
    at = itertools.count()
    for t, g, r, b in itertools.product(range(4), range(4), range(16), range(dim // 8)):  # K's bytes in order
        byte = next(at)
        assert ki[16 * t + r, g * dim // 4 + 2 * b] == 2 * byte and ki[16 * t + r, g * dim // 4 + 2 * b + 1] == 2 * byte + 1
    at = itertools.count()
    for i, n, b in itertools.product(range(dim // 16), range(64), range(8)):
        byte = next(at)
        assert vi[n, 16 * i + 2 * b] == 2 * byte and vi[n, 16 * i + 2 * b + 1] == 2 * byte + 1
    at = itertools.count()
    for g, r, t in itertools.product(range(dim // 32), range(16), range(4)):
        assert si[16 * t + r, g] == next(at)
    b = np.random.default_rng(0).integers(0, 256, (3, 32 * dim), dtype=np.uint8)
    assert np.array_equal(fp4.pack(fp4.unpack(b)), b) and fp4.unpack(np.uint8([0x21])).tolist() == [1, 2]


def pools(rng, pages, heads, dim, blocks):
    return (rng.integers(0, 256, (pages, heads, blocks, 32 * dim), dtype=np.uint8),
            rng.integers(0, 256, (pages, heads, blocks, 32 * dim), dtype=np.uint8),
            rng.integers(110, 140, (pages, heads, blocks, 2 * dim), dtype=np.uint8),
            rng.integers(0x3e00, 0x4100, (pages, heads, blocks, 64), dtype=np.uint16))


@pytest.mark.parametrize("dim", [64, 128])
def test_append_by_hand(dim):
    """Rows land where the table says, within half a code step of what they were, all else as it was."""
    rng = np.random.default_rng(dim)
    p = pools(rng, 5, 2, dim, 2)
    table = np.array([[3, 1], [4, 0]])
    new, lens, off = [3, 0], [130, 70], [1, 0]
    k_new, v_new = (rng.normal(size=(5, 2, dim)).astype(np.float32) for _ in range(2))
    k_new[2, 1, 40] = np.inf
    v_new[3, 0, 5] = np.nan
    got = fp4.append(*p, table, k_new, v_new, off, new, lens)
    for h in range(2):
        k, v = fp4.rows(*got, table[0], 127, 3, h)
        for j in range(3):
            x = k_new[1 + j, h].astype(np.float64).reshape(-1, 32)
            for g, part in enumerate(x):
                y = k[j, 32 * g:32 * g + 32]
                if not np.isfinite(part).all():
                    assert np.isnan(y).all()
                    continue
                step = 2.0 ** np.ceil(np.log2(np.abs(part).max() / 6))
                assert (np.abs(y - part) <= step * (1 if np.abs(part).max() > 4 * step else 0.5) + 1e-12).all()
            if np.isfinite(v_new[1 + j, h]).all():
                assert (np.abs(v[j] - v_new[1 + j, h]) <= np.abs(v_new[1 + j, h]).max() / 6 * 1.01).all()
                assert np.abs(v[j]).max() >= np.abs(v_new[1 + j, h]).max()
            else:
                assert np.isnan(v[j]).all()
    # key 127 is the last of page 3's second block; 128 and 129 the first of page 1's first
    changed = [np.argwhere((a != b).reshape(5, 2, 2, -1).any((1, 3))).tolist() for a, b in zip(got, p)]
    assert all(c == [[1, 0], [3, 1]] for c in changed)
    ki = fp4.k_index(dim)
    same = np.ones(64 * dim, dtype=bool)
    same[ki[:2].reshape(-1)] = False
    assert np.array_equal(fp4.unpack(got[0][1, :, 0])[:, same], fp4.unpack(p[0][1, :, 0])[:, same])


def test_reading_and_appending_again_changes_nothing():
    """Rows that are read have the same scales' multiples, so appending them gives the same values."""
    rng = np.random.default_rng(3)
    p = pools(rng, 2, 1, 64, 1)
    table = np.array([[1]])
    x = rng.normal(size=(40, 1, 64)) * 2.0 ** rng.integers(-20, 20, (40, 1, 1))
    once = fp4.append(*p, table, x, x, [0], [40], [40])
    k, v = fp4.rows(*once, table[0], 0, 40, 0)
    twice = fp4.append(*once, table, k[:, None], v[:, None], [0], [40], [40])
    for a, b in zip((k, v), fp4.rows(*twice, table[0], 0, 40, 0)):
        assert np.array_equal(a, b)


def test_segments_are_the_rows():
    rng = np.random.default_rng(4)
    p = pools(rng, 6, 2, 64, 2)
    table = np.array([[5, 2], [0, 3]])
    lens = [130, 65]
    ks, vs, off = fp4.kv4_segments(*p, table, lens)
    for b, n in enumerate(lens):
        for h in range(2):
            k, v = fp4.rows(*p, table[b], 0, n, h)
            at = off[b] + h * n * 64
            assert np.array_equal(ks[at:at + n * 64].reshape(n, 64), k) and np.array_equal(vs[at:at + n * 64].reshape(n, 64), v)
    assert verify_attention(rng.normal(size=(2, 1, 2, 64)), ks, vs, off, lens, 2).shape == (2, 1, 2, 64)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_against_complex_numbers(interleaved):
    """Pairs are complex numbers turned by the angle; products of turned queries and keys
    depend on the positions' difference alone; other columns stay."""
    rng = np.random.default_rng(1)
    x, y = rng.normal(size=(2, 4, 3, 64))
    f = 1e4 ** (-np.arange(16) / 16)
    pos = np.array([0, 5, 100000, -3])
    got, mag = fp4.norm_rope(x, None, pos, f, 1e-6, interleaved)
    a, b = (slice(0, 32, 2), slice(1, 32, 2)) if interleaved else (slice(0, 16), slice(16, 32))
    z = (x[..., a] + 1j * x[..., b]) * np.exp(1j * pos[:, None, None] * f)
    assert np.allclose(got[..., a], z.real, atol=1e-9) and np.allclose(got[..., b], z.imag, atol=1e-9)
    assert np.array_equal(got[..., 32:], x[..., 32:]) and np.array_equal(got[0], x[0])
    assert (np.abs(got) <= mag + 1e-12).all()
    other, _ = fp4.norm_rope(y, None, pos + 7, f, 1e-6, interleaved)
    base, _ = fp4.norm_rope(x, None, pos * 0, f, 1e-6, interleaved)
    seven, _ = fp4.norm_rope(y, None, pos * 0 + 7, f, 1e-6, interleaved)
    assert np.allclose((got * other).sum(-1), (base * seven).sum(-1), atol=1e-8)


def test_norm_against_torch():
    rng = np.random.default_rng(2)
    x, w = rng.normal(size=(5, 2, 128)), rng.normal(size=128)
    got, _ = fp4.norm_rope(x, w, np.zeros(5), np.ones(8), 1e-3, False)
    ref = torch.nn.functional.rms_norm(torch.from_numpy(x), (128,), torch.from_numpy(w), 1e-3)
    assert np.allclose(got, ref.numpy(), rtol=1e-12)
