"""Weights of the 4-bit attention where a wave holds one block of 16 rows: they keep twice bfloat16's bits, so that an
output is off by little more than its own rounding."""

import numpy as np
import pytest
import torch

from oracle import fp4, verify_attention

from test_gpu_kv4 import filled
from test_gpu_kv4_chunks import FULL, attend

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G,group,heads,lens,joined", [(1, 4, 8, [1000], True), (1, 4, 8, [3, 64, 777, 1500], False), (9, 8, 2, [700], True),
                                                       (4, 4, 2, [FULL, 90], False), (16, 3, 2, [FULL], False)])
def test_outputs_are_off_by_their_rounding(G, group, heads, D, lens, joined):
    """Scores are sums of four products spread over tens, so that a few keys take the weight, with weights that are
    no bfloat16 numbers; values of a head are of one sign.

    Bound: half a step of bfloat16 at the output's size, and of A = sum p |v|, relatively: a score's sum, five roundings of
    at most 240 (four products of at most 30, and the reference), 5 * 2^-24 * 240 = 7.2e-5; its weight's exponent and
    exponential 2 * 60 * 2^-24 + 2^-23 = 7.3e-6 where the weight counts; both of these in numerator and denominator, 1.6e-4;
    the weight as two bfloat16 numbers, 2^-16 = 1.5e-5; sums of a lane's 16 keys of at most 64 blocks, and of partials,
    (1024 + 64) * 2^-24 = 6.5e-5 each of numerator and denominator, 1.3e-4: in all below 3.2e-4."""
    rng = np.random.default_rng(G + D + len(lens))
    c = filled(rng, lens, heads, D, 64)
    columns = [0, 1, D // 4, D // 2 + 1]
    codes, random = np.zeros((*c.host[0].shape[:3], 64 * D), dtype=np.uint8), rng.integers(0, 16, (*c.host[0].shape[:3], 64 * D), dtype=np.uint8)
    for col in columns:
        at = fp4.k_index(D)[:, col]
        codes[..., at] = random[..., at]
    c.host[0][...] = fp4.pack(codes)
    c.host[2][...] = 127
    c.host[1][...] &= 0x77  # values without signs
    c.upload()
    q = torch.zeros((len(lens), G, heads * group, D), dtype=torch.bfloat16)
    for col in columns:
        q[..., col] = torch.from_numpy(rng.uniform(0.5, 5, q.shape[:3]) * rng.choice([-1, 1], q.shape[:3])).bfloat16()
    got, chunks = attend(c, heads, G, group, D, lens, q, None, 1.0)
    assert (chunks == 0) == joined
    ref = verify_attention(q.double().numpy(), *c.segments(lens), lens, heads, 1.0)
    bound = 2.0 ** (np.frexp(ref)[1] - 9.0) + 3.2e-4 * np.abs(ref)
    bad = ~(np.abs(got - ref) <= bound)
    assert not bad.any(), f"{bad.sum()} of {bad.size} past the bound, by up to {(np.abs(got - ref) / bound).max():.2f}"
