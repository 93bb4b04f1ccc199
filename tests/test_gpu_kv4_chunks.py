"""Attention over 4-bit caches, each of its two ways and each number of row blocks to a wave by name: what a call
writes into its workspace shows whether it cut requests into chunks, and how many."""

import os
import re

import numpy as np
import pytest
import torch

import paper_2601_21622_amd as sd
from oracle import fp4, tree_attention, verify_attention
from oracle.tree import ancestor_masks
from paper_2601_21622_amd import build as sd_build

from gpu_util import announce
from test_gpu_kv4 import check_attention, filled, random_tree

pytestmark = pytest.mark.gpu

HKV = 8
FULL = 33000  # keys; 516 blocks, more than a workgroup takes whole
# Thresholds of the blocks of keys, times heads, per CU up to which a wave takes one and two row blocks at most.
ONE, TWO = 24, 40
# name: (requests, query heads of a KV head, positions, row blocks of a wave, uneven row groups)
KINDS = {
    "one": (3, 1, 16, 1, False),
    "one_token": (3, 4, 1, 1, False),
    "one_of_three_groups": (1, 3, 16, 1, False),
    "two": (3, 4, 8, 2, False),
    "two_and_one": (2, 3, 16, 2, True),
    "three": (3, 3, 16, 3, False),
    "four": (3, 4, 16, 4, False),
    "four_and_three": (3, 8, 14, 4, True),
    "five": (3, 8, 10, 5, False),
}


def check_kind(kind, lens):
    """The kernel that the rule in the source picks for these lengths is the one that the case is about."""
    with open(os.path.join(sd_build.CSRC, "kv4_attention.hip")) as f:
        rule = re.search(r"blocks <= (\d+) \* cu_count\(\) \? 1 : blocks <= (\d+) \* cu_count\(\) \? 2 : 5;", f.read())
    assert (int(rule[1]), int(rule[2])) == (ONE, TWO), "the rule has changed: choose the lengths of these tests anew"
    _, group, G, most, uneven = KINDS[kind]
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    blocks = sum(-(-n // 64) for n in lens) * HKV
    upto = 1 if blocks <= ONE * cus else 2 if blocks <= TWO * cus else 5
    of = -(-G * group // 16)  # row blocks
    groups = -(-of // upto)
    assert -(-of // groups) == most and (of % groups != 0) == uneven


def attend(c, heads, G, group, D, lens, q, parent, scale):
    """Outputs, and the chunks that the call's workspace shows (0: a workgroup took each request)."""
    B = len(lens)
    d = sd.Dims(B, G - 1, heads * group, heads, D, 32, 1, 1, 0)
    ws = torch.full((sd.sd_kv4_workspace_bytes(d, max(lens)) // 4,), -1, dtype=torch.int32, device="cuda")
    out = torch.full((B, G, heads * group, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    sd.sd_verify_attention_kv4(d, q.cuda(), c.handle, lens, None if parent is None else torch.from_numpy(parent).cuda(), scale, out, ws)
    torch.cuda.synchronize()
    # A partial is D + 2 numbers, none of them a NaN of all ones.
    written, per = int((ws != -1).sum()), heads * G * group * (D + 2)
    assert written % per == 0
    return out.double().cpu().numpy(), written // per


def chunk_blocks(lens, chunks):
    """64-key blocks of a chunk."""
    return next(n for n in range(1, 65) if sum(-(-(-(-x // 64)) // n) for x in lens) == chunks)


def lengths(requests, G, chunk):
    """Lengths whose last positions lie in one block, in two, and in two chunks."""
    return [FULL, 512 * 64 + (G + 1) // 2, 500 // chunk * chunk * 64 + max(1, G // 2)][:requests]


class Segments:
    """One request and KV head's cache for the oracle, with its values as they were before any became NaN."""

    def __init__(self, c):
        self.c, self.host, self.kept = c, [a.copy() for a in c.host], {}

    def of(self, b, head, n):
        if (b, head) not in self.kept:
            self.kept[b, head] = fp4.kv4_segments(*(a[:, head:head + 1] for a in self.host), self.c.table[b:b + 1], [FULL])
        k, v, off = self.kept[b, head]
        D = self.c.dim
        return k[:n * D], v[:n * D], off

    def check(self, got, q, b, head, group, n, parent, scale, what):
        rows = slice(head * group, head * group + group)
        return check_attention(got[b:b + 1, :, rows], q[b:b + 1, :, rows].double().numpy(), self.of(b, head, n), [n], 1,
                               None if parent is None else parent[b:b + 1], scale, f"{what}, request {b}, head {head}")


@pytest.fixture(scope="module")
def plain():
    made = {}

    def of(D):
        if D not in made:
            made.clear()
            made[D] = Segments(filled(np.random.default_rng(D), [FULL] * 3, HKV, D, 256))
        return made[D]
    return of


def planned(c, kind, D, rng, scale):
    """Lengths for this case, found by calls: chunks are as long as those that the last positions were placed for."""
    requests, group, G, _, _ = KINDS[kind]
    q, chunk = torch.from_numpy(rng.normal(size=(requests, G, HKV * group, D))).bfloat16(), 1
    for _ in range(4):
        lens = lengths(requests, G, chunk)
        now = chunk_blocks(lens, attend(c, HKV, G, group, D, lens, q, None, scale)[1])
        if now == chunk:
            break
        chunk = now
    check_kind(kind, lens)
    return lens, chunk


# The listing's order is by head dimension: one cache at a time.
CASES = [(D, kind) for D in (64, 128) for kind in KINDS]


@pytest.mark.parametrize("D,kind", CASES)
def test_trees_in_chunks(D, kind, plain):
    """Candidate trees (and single tokens) whose last positions lie in one block, across two, and across two chunks."""
    requests, group, G, _, _ = KINDS[kind]
    seg, rng, scale = plain(D), np.random.default_rng(G * group + D), D ** -0.5
    lens, chunk = planned(seg.c, kind, D, rng, scale)
    parent = random_tree(rng, requests, G - 1) if G > 1 else None
    q = torch.from_numpy(rng.normal(size=(requests, G, HKV * group, D))).bfloat16()
    got, chunks = attend(seg.c, HKV, G, group, D, lens, q, parent, scale)
    assert chunks > 16 * requests and chunk_blocks(lens, chunks) == chunk  # more than one thread joins
    worst = max(seg.check(got, q, b, head, group, lens[b], parent, scale, kind)
                for b, head in [(0, 0), (1, 3), (2, 7)][:requests])
    announce(f"kv4 tree in chunks of {chunk} blocks, {kind}, D {D}: {worst:.2f} of the bound")


@pytest.fixture(scope="module")
def odd():
    """Keys of one product (scores exact), magnitudes that jump from key to key and from region to region; head 4's values near
    the upper end of what sums hold, head 6's near the lower."""
    made = {}

    def of(D):
        if D not in made:
            made.clear()
            rng = np.random.default_rng(7 * D)
            c = filled(rng, [FULL] * 3, HKV, D, 256)
            codes = np.zeros((*c.host[0].shape[:3], 64 * D), dtype=np.uint8)
            codes[..., fp4.k_index(D)[:, 0]] = rng.integers(1, 8, (*codes.shape[:3], 64))
            c.host[0][...] = fp4.pack(codes)
            c.host[2][...] = 127
            c.host[2][..., :64] += rng.choice([0, 0, 4, 6], (*c.host[2].shape[:3], 64)).astype(np.uint8)
            for b in (0, 1):  # rising and falling by thirds of the cache, a few keys above their region
                for blk in range(-(-FULL // 64)):
                    at = int(c.table[b][blk * 64 // c.page]), slice(None), blk % (c.page // 64)
                    third = blk // 172 if b == 0 else 2 - blk // 172
                    up = np.full((HKV, 64), (0, 4, 6)[max(0, third)])
                    up[rng.random((HKV, 64)) < 0.004] = 6
                    c.host[2][at][:, :64] = 127 + up
            for head, e in ((4, 95), (6, -80)):
                c.host[3][:, head] = torch.from_numpy(rng.uniform(0.1, 0.6, c.host[3][:, head].shape) * 2.0 ** e).bfloat16().view(
                    torch.int16).numpy().view(np.uint16)
            seg = Segments(c)
            c.upload()
            made[D] = seg
        return made[D]
    return of


@pytest.mark.parametrize("D,kind", CASES)
def test_jumps_large_numbers_and_nan_in_chunks(D, kind, odd):
    """Scores that jump by hundreds within chunks and between them; head 5's queries 2^40 times as large, whose references
    are past 2^16; a NaN value of head 3 that some positions of request 0 see; a NaN key of head 2, mid-cache, that all of its last
    request see; a query of NaN.

    The bound of check_attention has a twentieth of 2^-8, 2e-4, for all but the weights' rounding.  Scores are one product,
    exact in float32; a weight's exponent is off by 3 * 2^-24 of at most 60 where the weight counts (1e-5), its exponential by
    2^-23, sums of up to 64 * 16 keys of a lane's chunk and of some 40 partials by (1024 + 40) * 2^-24 (6.4e-5) each, the
    numerator's and the denominator's: below 2e-4."""
    requests, group, G, _, _ = KINDS[kind]
    seg, rng = odd(D), np.random.default_rng(G * group + 3 * D)
    c, last = seg.c, requests - 1
    lens, chunk = planned(c, kind, D, rng, 1.0)
    parent = random_tree(rng, requests, G - 1) if G > 10 else None
    q = torch.zeros((requests, G, HKV * group, D), dtype=torch.bfloat16)
    q[..., 0] = torch.from_numpy(rng.choice([1.0, -1.0, 0.5], q.shape[:3])).bfloat16()
    q[:, :, 5 * group:6 * group] *= 2.0 ** 40
    q[last, G - 1, 7 * group, 1] = float("nan")
    put = [(3, 0, 3, lens[0] - max(1, G - 2)), (2, last, 2, 5000)]  # pool, request, head, key
    bits = []
    for pool, b, head, n in put:
        page, blk = int(c.table[b][n // c.page]), n % c.page // 64
        at = (page, head, blk, n % 64) if pool == 3 else (page, head, blk, int(fp4.k_scale_index(D)[n % 64, 1]))
        t = c.dev[pool].view(torch.int16) if pool == 3 else c.dev[pool]
        bits.append((t, at, t[at].clone()))
        t[at] = 0x7fc0 if pool == 3 else 255
    try:
        got, chunks = attend(c, HKV, G, group, D, lens, q, parent, 1.0)
    finally:
        for t, at, was in bits:
            t[at] = was
    assert chunks > 16 * requests and chunk_blocks(lens, chunks) == chunk
    want = np.zeros(got.shape[:3], dtype=bool)
    seen = min(2, G - 1)  # the position of the NaN value's key
    masks = np.array([(2 << g) - 1 for g in range(G)]) if parent is None else np.array([int(m) for m in ancestor_masks(parent[0])])
    want[0, (masks >> seen & 1).astype(bool), 3 * group:4 * group] = True
    want[last, :, 2 * group:3 * group] = True
    want[last, G - 1, 7 * group] = True
    assert np.array_equal(np.isnan(got).all(-1), want) and np.array_equal(np.isnan(got).any(-1), want)
    clean = q.nan_to_num(nan=0.0)
    for b, head in [(0, 3), (0, 4), (last, 5), (0, 6), (last, 7), (1 % requests, 1)]:
        rows = slice(head * group, head * group + group)
        if want[b, :, rows].any():  # the spoilt outputs: as the oracle's
            f = verify_attention if parent is None else lambda *a: tree_attention(*a[:-1], parent[b:b + 1], a[-1])
            ref = f(clean[b:b + 1, :, rows].double().numpy(), *seg.of(b, head, lens[b]), [lens[b]], 1, 1.0)
            got[b, :, rows] = np.where(want[b, :, rows, None], ref[0], got[b, :, rows])
        seg.check(got, clean, b, head, group, lens[b], parent, 1.0, kind)


@pytest.mark.parametrize("G,group,heads,D,lens,tree", [
    (16, 3, 8, 64, np.linspace(37, 3001, 13).astype(int).tolist(), True), (9, 8, 8, 128, [1500, 1437, 9, 1], False),
    (1, 4, 8, 128, [1, 2, 63, 64, 65, 1000], False), (2, 2, 2, 128, [2 + 5 * i for i in range(70)], False),
    (14, 8, 2, 64, list(range(14, 1200, 60)), True)])
def test_joined_requests(G, group, heads, D, lens, tree):
    """Short requests, which a workgroup takes whole: nothing is written into the workspace."""
    rng = np.random.default_rng(G + D)
    lens = [max(n, G) for n in lens]
    c = filled(rng, lens, heads, D, 128)
    q = torch.from_numpy(rng.normal(size=(len(lens), G, heads * group, D))).bfloat16()
    parent = random_tree(rng, len(lens), G - 1) if tree else None
    got, chunks = attend(c, heads, G, group, D, lens, q, parent, D ** -0.5)
    assert chunks == 0
    check_attention(got, q.double().numpy(), c.segments(lens), lens, heads, parent, D ** -0.5, "joined")


@pytest.mark.parametrize("lens,joined", [([150, 128], True), ([FULL, 130], False)])
def test_attention_clamps_bad_page_ids(lens, joined):
    """Ids outside the pool are clamped into it, by the attention too."""
    rng = np.random.default_rng(21)
    D, G, heads, page = 64, 3, 2, 128
    c = filled(rng, [page] * 12, heads, D, page)  # twelve pages of numbers
    good = c.table[:, 0]
    ids = good[rng.integers(0, 12, (2, -(-max(lens) // page)))]
    ids[0, ::3], ids[1, ::2] = 0, c.host[0].shape[0] - 1
    spare = np.setdiff1d([0, c.host[0].shape[0] - 1], good)  # pages of any bytes: give them a good one's
    for a in c.host:
        a[spare] = a[good[0]]
    c.upload()
    bad = ids.copy()
    bad[0, ::3], bad[1, ::2] = rng.choice([-1, -7, -2 ** 31], bad[0, ::3].shape), rng.choice([len(c.host[0]), 10 ** 6, 2 ** 31 - 1], bad[1, ::2].shape)
    c.table = ids
    c.handle = sd.KV4Cache.of(*c.dev[:3], c.dev[3].view(torch.bfloat16), torch.from_numpy(bad.astype(np.int32)).cuda(), page)
    q = torch.from_numpy(rng.normal(size=(2, G, 2 * heads, D))).bfloat16()
    got, chunks = attend(c, heads, G, 2, D, lens, q, None, D ** -0.5)
    assert (chunks == 0) == joined
    check_attention(got, q.double().numpy(), c.segments(lens), lens, heads, None, D ** -0.5, "bad ids")
