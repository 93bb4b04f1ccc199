"""The 8-bit KV cache on the GPU against the float64 oracle: appends code for
code, attention within a bound that is derived in check_attention."""

import numpy as np
import pytest
import torch

import paper_2601_21622_amd as sd
from oracle import fp8, tree_attention, verify_attention

from gpu_util import announce

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn


def make_table(rng, kv_len, page, spare=2):
    need = [-(-int(n) // page) for n in kv_len]
    n = sum(need) + spare
    ids = iter(rng.permutation(n).tolist())
    table = np.full((len(kv_len), max(1, max(need))), -1, dtype=np.int32)
    for j in range(table.shape[1]):
        for b in range(len(kv_len)):
            if j < need[b]:
                table[b, j] = next(ids)
    return table, n


class Cache:
    """A pool on both sides, its bytes seeded (codes of any kind, NaN among them)."""

    def __init__(self, rng, kv_len, heads, dim, page, batch=None):
        self.dim, self.page = dim, page
        self.table, n = make_table(rng, kv_len, page)
        shape = (n, heads, page // 64)
        self.k, self.v = (rng.integers(0, 256, (*shape, 64 * dim), dtype=np.uint8) for _ in range(2))
        self.ks, self.vs = (rng.integers(115, 125, shape, dtype=np.uint8) for _ in range(2))
        self.dev = [torch.from_numpy(a.copy()).cuda() for a in (self.k, self.v, self.ks, self.vs)]
        self.handle = sd.KV8Cache.of(self.dev[0].view(n, heads, page // 64, 64 * dim), *self.dev[1:],
                                     torch.from_numpy(self.table).cuda(), page)

    def upload(self):
        for d, a in zip(self.dev, (self.k, self.v, self.ks, self.vs)):
            d.copy_(torch.from_numpy(a))

    def append(self, k_new, v_new, off, new, lens):
        self.k, self.ks = fp8.append(self.k, self.ks, self.table, k_new, off, new, lens, fp8.k_index(self.dim))
        self.v, self.vs = fp8.append(self.v, self.vs, self.table, v_new, off, new, lens, fp8.v_index(self.dim))

    def check(self):
        for name, d, a in zip(("k", "v", "k_scale", "v_scale"), self.dev, (self.k, self.v, self.ks, self.vs)):
            got = d.cpu().numpy()
            if name in ("k", "v"):  # one NaN is as good as another
                got, a = (np.where(x & 127 == 127, 127, x) for x in (got, a))
            assert np.array_equal(got, a), f"{name}: {(got != a).sum()} of {a.size} differ"


def rows(rng, total, heads, dim, dtype, stride=None):
    """Token rows (magnitudes differ by head and row) on the GPU, and their exact values."""
    x = rng.normal(size=(total, heads, dim)) * 2.0 ** rng.integers(-12, 12, (1, heads, 1)) * 2.0 ** rng.integers(-2, 3, (total, 1, 1))
    full = torch.zeros((max(total, 1), stride or heads * dim), dtype=dtype)
    view = full[:, :heads * dim].unflatten(1, (heads, dim))
    view[:total] = torch.from_numpy(x).to(dtype)
    dev = full.cuda()[:, :heads * dim].unflatten(1, (heads, dim))
    return dev, view[:total].double().numpy()


APPENDS = {
    # name: heads, dim, page, dtype, stride, [(new, kv) per request]
    "one_row_each": (2, 128, 64, torch.bfloat16, None, [(1, 1), (1, 64), (1, 65), (1, 128), (1, 100)]),
    "step_over_pages": (4, 128, 64, torch.bfloat16, None, [(5, 5), (5, 66), (5, 130), (5, 64)]),
    "prompts": (2, 128, 256, torch.bfloat16, 3 * 256, [(300, 300), (64, 64), (1, 1), (0, 0), (513, 600)]),
    "d64": (3, 64, 128, torch.bfloat16, None, [(7, 60), (200, 200), (64, 128), (0, 50)]),
    "f32": (2, 128, 64, torch.float32, 264, [(70, 75), (3, 130)]),
    "f32_d64": (1, 64, 4096, torch.float32, None, [(130, 4000), (2, 64)]),
    "many": (1, 64, 64, torch.bfloat16, None, [(1 + i % 3, 4 + 5 * i) for i in range(70)]),
    "whole_blocks": (1, 128, 128, torch.bfloat16, None, [(128, 256), (64, 128)]),
}


@pytest.mark.parametrize("name", APPENDS)
def test_append(name):
    heads, dim, page, dtype, stride, req = APPENDS[name]
    rng = np.random.default_rng(len(name))
    new, lens = [a for a, _ in req], [b for _, b in req]
    c = Cache(rng, lens, heads, dim, page)
    off = np.cumsum([0] + new[:-1])
    (kd, kx), (vd, vx) = rows(rng, sum(new), heads, dim, dtype, stride), rows(rng, sum(new), heads, dim, dtype, stride)
    d = sd.Dims(len(req), 0, heads, heads, dim, 32, 1, 1 if dtype == torch.bfloat16 else 0, 0)
    for _ in range(2):  # a second time changes nothing but rows that the first rescaled once
        c.append(kx, vx, off, new, lens)
        sd.sd_kv8_append(d, c.handle, kd, vd, off, new, lens)
        torch.cuda.synchronize()
        c.check()


def test_append_steps_cut_back_and_odd_values():
    """A session's life: prompt, steps, a cut back to fewer keys, rows of
    zeros, infinities, NaN, the largest and smallest numbers; rows shared by requests."""
    rng = np.random.default_rng(5)
    heads, dim = 2, 64
    c = Cache(rng, [200, 200], heads, dim, 64)
    d = sd.Dims(2, 0, heads, heads, dim, 32, 1, 0, 0)
    for new, lens in (([90, 3], [90, 3]), ([5, 5], [95, 8]), ([5, 5], [97, 10]), ([1, 60], [98, 66]), ([30, 0], [120, 66]),
                      ([64, 1], [192, 1])):
        (kd, kx), (vd, vx) = rows(rng, 100, heads, dim, torch.float32), rows(rng, 100, heads, dim, torch.float32)
        for dev, x in ((kd, kx), (vd, vx)):
            odd = [0.0, -0.0, np.inf, -np.inf, np.nan, 3.4e38, -3.4e38, 1e-45, 1e-38]
            at = rng.integers(0, 100, len(odd)), rng.integers(0, heads, len(odd)), rng.integers(0, dim, len(odd))
            x[at] = np.float32(odd)
            x[7] = 0.0
            dev.copy_(torch.from_numpy(x.astype(np.float32)))
        off = [3, 3]  # both requests read the same rows
        c.append(kx, vx, off, new, lens)
        sd.sd_kv8_append(d, c.handle, kd, vd, off, new, lens)
        torch.cuda.synchronize()
        c.check()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new", [1, 4, 13, 14])
def test_append_steps_of_growing_rows(new, dim, dtype):
    """Steps at every place in a block, over its end too, of rows that outgrow the earlier scale and of rows that do not."""
    rng = np.random.default_rng(new)
    heads = 3
    lens = [new + i for i in range(0, 70, 3)]
    B = len(lens)
    c = Cache(rng, [n + 3 * new for n in lens], heads, dim, 64)
    d = sd.Dims(B, 0, heads, heads, dim, 32, 1, 1 if dtype == torch.bfloat16 else 0, 0)
    off = np.arange(B) * new
    for step, size in enumerate((1.0, 2.0 ** -5, 37.0, 2.0 ** 20)):
        x = [torch.from_numpy(rng.normal(size=(B * new, heads, dim)) * size).to(dtype) for _ in range(2)]
        at = [n + step * new for n in lens]
        c.append(*(a.double().numpy() for a in x), off, [new] * B, at)
        sd.sd_kv8_append(d, c.handle, *(a.cuda() for a in x), off, [new] * B, at)
        torch.cuda.synchronize()
        c.check()


# ---- attention -------------------------------------------------------------------

def check_attention(got, q, seg, kv_len, heads, parent, scale, what):
    """Bound: P is rounded to bf16 (half a step: 2^-8) where it is multiplied, and
    the sum that divides adds the rounded values, so |O - O*| <= 2^-8 (A + |O*|), A = sum p |v|;
    the output's own rounding adds 2^-8 |O|.  Scores are float32 sums of D exact products: a
    relative error of p of at most D 2^-24 |q| |k| scale and a few 2^-24 of |s|, which with the
    second-order terms is held within a twentieth of the bound for the scores used here (< 40)."""
    kseg, vseg, off = seg
    f = verify_attention if parent is None else lambda *a: tree_attention(*a[:-1], parent, a[-1])
    ref = f(q, kseg, vseg, off, kv_len, heads, scale)
    mag = f(q, kseg, np.abs(vseg), off, kv_len, heads, scale)
    bound = 1.05 * 2.0 ** -8 * (mag + 2 * np.abs(ref)) + 1e-30
    err = np.abs(got - ref)
    bad = ~(err <= bound)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} past the bound, first {np.argwhere(bad)[0]}"
    return float((err / bound).max())


ATTENDS = {
    # name: G, Hq, Hkv, D, page, lens, tree
    "single_token": (1, 8, 2, 128, 64, [1, 64, 65, 300], False),
    "single_token_mha": (1, 2, 2, 64, 64, [1, 2, 129], False),
    "mha": (5, 3, 3, 128, 64, [5, 64, 66, 68, 700], False),
    "gqa4": (7, 8, 2, 128, 128, [7, 63, 64, 65, 71, 1100], False),
    "gqa8_72": (9, 16, 2, 128, 256, [9, 130, 1500], False),
    "rows48_d64": (6, 16, 2, 64, 64, [6, 62, 128, 500], False),
    "rows64": (8, 8, 1, 128, 64, [8, 200], False),
    "rows88_two_groups": (11, 8, 1, 128, 64, [11, 300], False),
    "rows128": (16, 8, 1, 128, 4096, [16, 5000], False),
    "rows128_d64": (64, 4, 2, 64, 64, [64, 65, 127, 400], False),
    "g64": (64, 1, 1, 128, 64, [64, 191], False),
    "tree15": (16, 6, 2, 64, 128, [16, 37, 200, 801], True),
    "tree63": (64, 2, 1, 128, 64, [64, 100, 130], True),
    "many_requests": (2, 2, 2, 64, 64, [2 + 7 * i for i in range(70)], False),
}


def attend(G, Hq, Hkv, D, c, kv_len, q, parent, scale):
    B = len(kv_len)
    d = sd.Dims(B, G - 1, Hq, Hkv, D, 32, 1, 1, 0)
    ws = torch.full((sd.sd_fp8_workspace_bytes(d, max(kv_len)),), 0xff, dtype=torch.uint8, device="cuda")
    out = torch.full((B, G, Hq, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    sd.sd_verify_attention_kv8(d, q, c.handle, kv_len, parent, scale, out, ws)
    torch.cuda.synchronize()
    return out.double().cpu().numpy()


def filled(rng, kv_len, heads, dim, page):
    """A cache whose keys up to kv_len hold numbers, all other bytes anything (NaN too)."""
    c = Cache(rng, kv_len, heads, dim, page)
    total = int(sum(kv_len))
    x = [rng.normal(size=(total, heads, dim)) for _ in range(2)]
    off = np.cumsum([0] + list(kv_len[:-1]))
    c.append(*x, off, kv_len, kv_len)
    c.upload()
    return c


@pytest.mark.parametrize("name", ATTENDS)
def test_attention(name):
    G, Hq, Hkv, D, page, lens, tree = ATTENDS[name]
    rng = np.random.default_rng(100 + len(name))
    c = filled(rng, lens, Hkv, D, page)
    q = torch.from_numpy(rng.normal(size=(len(lens), G, Hq, D)) * 2).bfloat16()
    parent = pd = None
    if tree:
        parent = np.maximum(np.arange(G - 1)[None, :] - rng.integers(1, 5, (len(lens), G - 1)), -1).astype(np.int32)
        pd = torch.from_numpy(parent).cuda()
    scale = 1 / np.sqrt(D)
    got = attend(G, Hq, Hkv, D, c, lens, q.cuda(), pd, scale)
    seg = fp8.kv8_segments(c.k, c.v, c.ks, c.vs, c.table, lens)
    worst = check_attention(got, q.double().numpy(), seg, lens, Hkv, parent, scale, name)
    announce(f"kv8 attention {name}: {worst:.2f} of the bound")


def test_attention_of_large_and_growing_scores():
    """Keys that grow along the cache: the running maximum moves many times."""
    rng = np.random.default_rng(9)
    lens, G, H, D = [900, 333], 3, 2, 128
    c = Cache(rng, lens, H, D, 64)
    x = [rng.normal(size=(sum(lens), H, D)) for _ in range(2)]
    x[0] *= np.concatenate([np.linspace(0.01, 3, n) for n in lens])[:, None, None]
    c.append(*x, [0, 900], lens, lens)
    c.upload()
    q = torch.from_numpy(rng.normal(size=(2, G, H, D)) * 2).bfloat16()
    got = attend(G, H, H, D, c, lens, q.cuda(), None, 1 / np.sqrt(D))
    check_attention(got, q.double().numpy(), fp8.kv8_segments(c.k, c.v, c.ks, c.vs, c.table, lens), lens, H, None,
                    1 / np.sqrt(D), "growing scores")


@pytest.mark.parametrize("G,Hq,Hkv,D,page,tree", [
    (1, 16, 16, 128, 64, False), (5, 16, 16, 128, 64, False), (5, 8, 8, 64, 128, False), (9, 32, 4, 128, 256, False),
    (11, 32, 4, 128, 64, False), (16, 32, 4, 64, 64, True)])
def test_attention_of_long_chunks(G, Hq, Hkv, D, page, tree):
    """So many sequences that a wave folds many blocks of one: lengths from a few keys to 1,500."""
    rng = np.random.default_rng(G + D)
    lens = [1500 - 53 * i if i < 24 else G + 61 * (i - 24) for i in range(28)]
    c = filled(rng, lens, Hkv, D, page)
    q = torch.from_numpy(rng.normal(size=(len(lens), G, Hq, D)) * 2).bfloat16()
    parent = pd = None
    if tree:
        parent = np.maximum(np.arange(G - 1)[None, :] - rng.integers(1, 5, (len(lens), G - 1)), -1).astype(np.int32)
        pd = torch.from_numpy(parent).cuda()
    got = attend(G, Hq, Hkv, D, c, lens, q.cuda(), pd, 1 / np.sqrt(D))
    seg = fp8.kv8_segments(c.k, c.v, c.ks, c.vs, c.table, lens)
    worst = check_attention(got, q.double().numpy(), seg, lens, Hkv, parent, 1 / np.sqrt(D), "long chunks")
    announce(f"kv8 attention of long chunks G {G} D {D}: {worst:.2f} of the bound")


@pytest.mark.parametrize("G,D", [(5, 64), (8, 64), (9, 64), (16, 64), (5, 128), (8, 128), (9, 128), (16, 128)])
def test_attention_of_many_blocks(G, D):
    """Past 8,192 blocks of keys a wave holds all rows of a head that it can: 40, 64, 72 and 128 rows."""
    rng = np.random.default_rng(10 * G + D)
    Hkv, lens = 32, [3400, 3333, 3329, 3328, 3210]
    c = Cache(rng, lens, Hkv, D, 256)
    for a in (c.k, c.v):  # numbers up to 1 (code 0x38) and their negatives
        a[...] = rng.integers(0, 0x39, a.shape, dtype=np.uint8) | rng.integers(0, 2, a.shape, dtype=np.uint8) << 7
    c.ks[...] = 127 + rng.integers(-1, 2, c.ks.shape)
    c.vs[...] = 127 + rng.integers(-1, 2, c.vs.shape)
    c.upload()
    q = torch.from_numpy(rng.normal(size=(len(lens), G, 8 * Hkv, D)) * 2).bfloat16()
    got = attend(G, 8 * Hkv, Hkv, D, c, lens, q.cuda(), None, 1 / np.sqrt(D))
    for b in (0, 2, 4):  # each request against the oracle by itself
        seg = fp8.kv8_segments(c.k, c.v, c.ks, c.vs, c.table[b:b + 1], lens[b:b + 1])
        check_attention(got[b:b + 1], q[b:b + 1].double().numpy(), seg, lens[b:b + 1], Hkv, None, 1 / np.sqrt(D),
                        f"many blocks, request {b}")


@pytest.mark.parametrize("G,D", [(5, 64), (9, 64), (5, 128), (8, 128), (9, 128)])
def test_jumps_and_nan_among_many_blocks(G, D):
    """As test_attention_of_scores_that_jump (one product makes a score: exact but for the
    factors, 3 * 2^-24 * 256 of p), with three to five row blocks to a wave; and one NaN value that positions
    2 .. of one head see."""
    rng = np.random.default_rng(20 * G + D)
    Hkv, lens, page = 32, [3400, 3333, 3329, 3328, 3210], 256
    c = Cache(rng, lens, Hkv, D, page)
    c.k[...] = 0
    c.k[..., fp8.k_index(D)[:, 0]] = rng.integers(0x28, 0x39, (*c.k.shape[:3], 64))  # 1/4 .. 1
    c.v[...] = rng.integers(0, 0x39, c.v.shape, dtype=np.uint8) | rng.integers(0, 2, c.v.shape, dtype=np.uint8) << 7
    c.ks[...] = 127 + rng.choice([0, 0, 5, 7, 8], c.ks.shape)
    c.vs[...] = 127
    clean = c.v.copy()
    key, head, col = lens[0] - G + 2, 3, 7
    c.v[c.table[0, key // page], head, key % page // 64, fp8.v_index(D)[key % 64, col]] = 0x7f
    c.upload()
    q = torch.zeros((len(lens), G, 8 * Hkv, D), dtype=torch.bfloat16)
    q[..., 0] = torch.from_numpy(rng.choice([1.0, -1.0, 0.5], q.shape[:3])).bfloat16()
    got = attend(G, 8 * Hkv, Hkv, D, c, lens, q.cuda(), None, 1.0)
    hit = got[0, 2:, 8 * head:8 * head + 8, col]
    assert np.isnan(hit).all() and np.isnan(got).sum() == hit.size
    for b in (0, 3):
        seg = fp8.kv8_segments(c.k, clean, c.ks, c.vs, c.table[b:b + 1], lens[b:b + 1])
        if b == 0:  # the spoilt outputs: as the oracle's
            ref = verify_attention(q[:1].double().numpy(), *seg, lens[:1], Hkv, 1.0)
            got[0, 2:, 8 * head:8 * head + 8, col] = ref[0, 2:, 8 * head:8 * head + 8, col]
        check_attention(got[b:b + 1], q[b:b + 1].double().numpy(), seg, lens[b:b + 1], Hkv, None, 1.0,
                        f"jumps among many blocks, request {b}")


@pytest.mark.parametrize("G,Hq,Hkv,D", [(2, 16, 16, 128), (5, 16, 16, 64), (10, 32, 4, 128)])
def test_attention_of_scores_that_jump(G, Hq, Hkv, D):
    """Scores rise and fall by hundreds from one stretch of keys to the next, inside
    a wave's share too.  One column alone makes a score, so it is one product: exact in
    float32 but for the factors scale and log2 e, under 3 * 2^-24 * 300 = 5e-5 of p, within the bound's twentieth
    (2^-8 / 20 = 2e-4)."""
    rng = np.random.default_rng(G)
    B = 24
    lens = [1400 - 31 * i for i in range(B)]
    total = sum(lens)
    levels = np.array([0.0, 100.0, -200.0, 220.0, 220.0, 30.0, 290.0, 0.0])
    x = [rng.normal(size=(total, Hkv, D)) for _ in range(2)]
    x[0][...] = 0.0
    off = np.cumsum([0] + lens[:-1])
    for o, n in zip(off, lens):
        stretch = (np.arange(n) + rng.integers(0, 300)) // 150 % len(levels)
        x[0][o:o + n, :, 0] = levels[stretch][:, None] + rng.normal(size=(n, Hkv))
    c = Cache(rng, lens, Hkv, D, 64)
    c.append(*x, off, lens, lens)
    c.upload()
    q = torch.zeros((B, G, Hq, D), dtype=torch.bfloat16)
    q[..., 0] = torch.from_numpy(rng.choice([1.0, -1.0, 0.5], (B, G, Hq))).bfloat16()
    got = attend(G, Hq, Hkv, D, c, lens, q.cuda(), None, 1.0)
    seg = fp8.kv8_segments(c.k, c.v, c.ks, c.vs, c.table, lens)
    check_attention(got, q.double().numpy(), seg, lens, Hkv, None, 1.0, "scores that jump")


@pytest.mark.parametrize("D", [64, 128])
def test_nan_at_the_end_of_a_long_chunk(D):
    rng = np.random.default_rng(D)
    B, G, H = 24, 5, 16
    lens = [1300 - 29 * i for i in range(B)]
    off = np.cumsum([0] + lens[:-1])
    x = [rng.normal(size=(sum(lens), H, D)) for _ in range(2)]
    clean = [a.copy() for a in x]
    x[1][off[3] + lens[3] - G + 2, :, 7] = np.nan   # a value that positions 2 .. see
    x[0][off[9] + lens[9] - G + 4, :, 5] = np.nan   # a key that the last one sees
    x[1][off[11] + 700, 4, 9] = np.nan              # a value in the middle: its head and column alone
    c = Cache(rng, lens, H, D, 64)
    c.append(*x, off, lens, lens)
    c.upload()
    q = torch.from_numpy(rng.normal(size=(B, G, H, D))).bfloat16()
    got = attend(G, H, H, D, c, lens, q.cuda(), None, 1 / np.sqrt(D))
    assert np.isnan(got[3, 2:, :, 7]).all() and np.isnan(got[9, 4]).all() and np.isnan(got[11, :, 4, 9]).all()
    c.append(*clean, off, lens, lens)
    ref = verify_attention(q.double().numpy(), *fp8.kv8_segments(c.k, c.v, c.ks, c.vs, c.table, lens), lens, H)
    for b in range(B):
        if b in (3, 9, 11):
            first = {3: 2, 9: 4, 11: 0}[b]
            assert np.isfinite(got[b, :first]).all()
            assert np.abs(got[b, :first] - ref[b, :first]).max(initial=0) < 0.1 * np.abs(ref).max()
        else:
            assert np.isfinite(got[b]).all()
            assert np.abs(got[b] - ref[b]).max() < 0.02 * np.abs(ref).max()


@pytest.mark.parametrize("G,Hq,Hkv,D", [(4, 2, 1, 128), (4, 1, 1, 64), (9, 8, 1, 128)])
def test_nan_reaches_only_those_that_see_it(G, Hq, Hkv, D):
    """A draft whose rows are NaN spoils the positions from it on, not those before."""
    rng = np.random.default_rng(11)
    for L in (G, 62 + G // 2, 130):
        for which in (0, 1):
            c = Cache(rng, [L], Hkv, D, 64)
            x = [rng.normal(size=(L, Hkv, D)) for _ in range(2)]
            x[which][L - G + 2] = np.nan
            c.append(*x, [0], [L], [L])
            c.upload()
            q = torch.from_numpy(rng.normal(size=(1, G, Hq, D))).bfloat16()
            got = attend(G, Hq, Hkv, D, c, [L], q.cuda(), None, 1 / np.sqrt(D))
            assert np.isnan(got[0, 2:]).all()
            x[which][L - G + 2] = 0.0
            clean = Cache(rng, [L], Hkv, D, 64)
            clean.append(*x, [0], [L], [L])
            seg = fp8.kv8_segments(clean.k, clean.v, clean.ks, clean.vs, clean.table, [L])
            ref = verify_attention(q.double().numpy(), *seg, [L], Hkv)
            assert np.isfinite(got[0, :2]).all()
            assert np.abs(got[0, :2] - ref[0, :2]).max() < 0.1 * np.abs(ref).max()


def test_inactive_values_of_queries_and_extremes():
    """NaN and infinite queries spoil their own rows alone; a score far below the rest weighs nothing."""
    rng = np.random.default_rng(12)
    c = filled(rng, [200], 1, 128, 64)
    q = torch.from_numpy(rng.normal(size=(1, 4, 2, 128))).bfloat16()
    clean = attend(4, 2, 1, 128, c, [200], q.cuda(), None, 0.1)
    q[0, 1, 0, 5] = float("nan")
    q[0, 2, 1, 7] = float("inf")
    got = attend(4, 2, 1, 128, c, [200], q.cuda(), None, 0.1)
    assert np.isnan(got[0, 1, 0]).all() and np.isnan(got[0, 2, 1]).all()
    keep = np.ones((4, 2), dtype=bool)
    keep[1, 0] = keep[2, 1] = False
    assert np.array_equal(got[0][keep], clean[0][keep])
    big = torch.zeros((1, 4, 2, 128), dtype=torch.bfloat16)
    big[..., 0] = 2.0 ** 60
    got = attend(4, 2, 1, 128, c, [200], big.cuda(), None, 1.0)
    k, v, _ = fp8.kv8_segments(c.k, c.v, c.ks, c.vs, c.table, [200])
    best = k.reshape(200, 128)[:197, 0].argmax()
    if (k.reshape(200, 128)[:197, 0] == k.reshape(200, 128)[best, 0]).sum() == 1:
        assert np.abs(got[0, 0, 0] - v.reshape(200, 128)[best]).max() <= 2.0 ** -7 * np.abs(v).max()


def test_streams_graphs_and_workspaces():
    """Append and attention captured once, replayed with other data between
    eager calls; another stream than the current one."""
    rng = np.random.default_rng(13)
    lens, G, H, D = [70, 133], 3, 2, 128
    c = filled(rng, lens, H, D, 64)
    d, da = sd.Dims(2, G - 1, 2 * H, H, D, 32, 1, 1, 0), sd.Dims(2, 0, H, H, D, 32, 1, 1, 0)
    new = torch.randn((2 * G, H, D), device="cuda").bfloat16()
    q = torch.randn((2, G, 2 * H, D), device="cuda").bfloat16()
    out = torch.empty_like(q)
    n = sd.sd_fp8_workspace_bytes(d, max(lens))
    ws = torch.empty((n,), dtype=torch.uint8, device="cuda")

    def step(o, w, stream=None):
        sd.sd_kv8_append(da, c.handle, new, new, [0, G], [G, G], lens, stream=stream)
        sd.sd_verify_attention_kv8(d, q, c.handle, lens, None, 0.1, o, w, stream=stream)

    step(out, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out, ws)
    eager, ws2 = torch.empty_like(out), torch.empty_like(ws)
    side = torch.cuda.Stream()
    for i in range(4):
        new.normal_()
        q.normal_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        step(eager, ws2, stream=side if i % 2 else None)
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
        assert torch.isfinite(out).all()


def test_far_pages():
    """A pool past 4 GB: pages beyond 32-bit byte offsets."""
    rng = np.random.default_rng(14)
    heads, dim, page = 8, 128, 4096
    n = 1100  # 1100 * 8 * 4096 * 128 = 4.6 GB
    k, v = (torch.zeros((n, heads, page // 64, 64 * dim), dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.full((n, heads, page // 64), 127, dtype=torch.uint8, device="cuda") for _ in range(2))
    table = torch.tensor([[1099, 1030]], dtype=torch.int32, device="cuda")
    cache = sd.KV8Cache.of(k, v, ks, vs, table, page)
    L = 4096 + 70
    new = [torch.randn((L, heads, dim), device="cuda").bfloat16() for _ in range(2)]
    sd.sd_kv8_append(sd.Dims(1, 0, heads, heads, dim, 32, 1, 1, 0), cache, *new, [0], [L], [L])
    d = sd.Dims(1, 0, heads, heads, dim, 32, 1, 1, 0)
    q = torch.randn((1, 1, heads, dim), device="cuda").bfloat16()
    out = torch.empty_like(q)
    ws = torch.empty((sd.sd_fp8_workspace_bytes(d, L),), dtype=torch.uint8, device="cuda")
    sd.sd_verify_attention_kv8(d, q, cache, [L], None, dim ** -0.5, out, ws)
    host = [t[[1099, 1030]].cpu().numpy() for t in (k, v, ks, vs)]
    assert not k[1031:1099].any() and not k[:1030].any()
    seg = fp8.kv8_segments(*host, np.array([[0, 1]]), [L])
    check_attention(out.double().cpu().numpy(), q.double().cpu().numpy(), seg, [L], heads, None, dim ** -0.5, "far pages")
    x = new[0].double().cpu().numpy()
    got = seg[0].reshape(heads, L, dim).transpose(1, 0, 2)
    assert np.abs(got - x).max() <= 2.0 ** -4 * np.abs(x).max()


def test_binding_refuses_what_does_not_fit():
    rng = np.random.default_rng(15)
    c = filled(rng, [64], 2, 64, 64)
    d = sd.Dims(1, 0, 2, 2, 64, 32, 1, 1, 0)
    x = torch.zeros((1, 2, 64), dtype=torch.bfloat16, device="cuda")
    q = torch.zeros((1, 1, 2, 64), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty((1 << 20,), dtype=torch.uint8, device="cuda")
    for bad in (lambda: sd.sd_kv8_append(d, c.handle, x, x, [0], [2], [64]),              # past the rows
                lambda: sd.sd_kv8_append(d, c.handle, x.float(), x, [0], [1], [64]),
                lambda: sd.sd_kv8_append(d, c.handle, x[:, :1], x, [0], [1], [64]),
                lambda: sd.sd_kv8_append(d, c.handle, x, x, [0, 1], [1, 1], [64, 64]),
                lambda: sd.sd_kv8_append(sd.Dims(1, 0, 2, 2, 128, 32, 1, 1, 0), c.handle, x, x, [0], [1], [64]),
                lambda: sd.sd_verify_attention_kv8(d, q, c.handle, [64], None, 1.0, q.float(), ws),
                lambda: sd.sd_verify_attention_kv8(d, q[..., :32], c.handle, [64], None, 1.0, q, ws),
                lambda: sd.sd_verify_attention_kv8(d, q, c.handle, [64, 64], None, 1.0, q, ws),
                lambda: sd.KV8Cache.of(c.dev[0], c.dev[1], c.dev[2], c.dev[3], c.handle._tensors[4], 128),
                lambda: sd.KV8Cache.of(c.dev[0], c.dev[1], c.dev[2], c.dev[3], c.handle._tensors[4].long(), 64)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(sd.SdError):
        sd.sd_verify_attention_kv8(d, q, c.handle, [65], None, 1.0, torch.empty_like(q), ws)


# Chunks that end with the key of position 0: no block of them is masked, and its last key
# is the step's own.  (G, lengths, heads) with chunks of one block, and of several.
ENDS = {
    "one_token": (1, [64, 128, 1024], 2),
    "one_token_long_chunks": (1, [1408 - 64 * (i % 5) for i in range(24)], 16),
    "five_tokens": (5, [68, 132, 708], 2),
    "five_tokens_long_chunks": (5, [1412 - 64 * (i % 5) for i in range(24)], 16),
}


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("name", ENDS)
def test_attention_of_a_far_score_at_the_end_of_whole_blocks(name, D):
    """The key of position 0 scores 300 above all others and ends a block: the largest
    score of its chunk is found.  One column alone makes a score, as in test_attention_of_scores_that_jump."""
    G, lens, H = ENDS[name]
    rng = np.random.default_rng(G + D)
    off = np.cumsum([0] + lens[:-1])
    x = [rng.normal(size=(sum(lens), H, D)) for _ in range(2)]
    x[0][...] = 0.0
    x[0][..., 0] = rng.normal(size=(sum(lens), H))
    x[0][off + np.array(lens) - G, :, 0] = 300.0
    c = Cache(rng, lens, H, D, 64)
    c.append(*x, off, lens, lens)
    c.upload()
    q = torch.zeros((len(lens), G, H, D), dtype=torch.bfloat16)
    q[..., 0] = 1.0
    got = attend(G, H, H, D, c, lens, q.cuda(), None, 1.0)
    seg = fp8.kv8_segments(c.k, c.v, c.ks, c.vs, c.table, lens)
    check_attention(got, q.double().numpy(), seg, lens, H, None, 1.0, name)


def put_rows(c, pool, index, b, codes):
    """Codes [L][heads][D] of request b's keys into a pool of the cache's."""
    for n0 in range(0, len(codes), 64):
        part = codes[n0:n0 + 64].transpose(1, 0, 2)
        block = pool[c.table[b, n0 // c.page], :, n0 % c.page // 64]
        block[:, index[:part.shape[1]]] = part


@pytest.mark.parametrize("G,Hq,Hkv,D,lens", [
    (3, 8, 2, 128, [200, 333]), (3, 8, 2, 64, [200, 333]),
    (5, 16, 16, 128, [1400 - 31 * i for i in range(24)]), (5, 16, 16, 64, [1400 - 31 * i for i in range(24)]),
    (4, 32, 4, 128, [1400 - 31 * i for i in range(24)]),
    (9, 256, 32, 128, [3400, 3333, 3329, 3328, 3210]), (9, 256, 32, 64, [3400, 3333, 3329, 3328, 3210])])
def test_attention_of_huge_dense_queries(G, Hq, Hkv, D, lens):
    """Queries of all columns up to 2^101: a score summed from zero and one summed from the
    reference differ by their rounding, far more than the exponential takes.  Each row has one key of twice its signs, whose
    score exceeds all others by thousands in the exponential: the output is that key's value, to the bit
    (weights one and zero, a value of four bits)."""
    rng = np.random.default_rng(G + D)
    group = Hq // Hkv
    c = Cache(rng, lens, Hkv, D, 64)
    c.ks[...] = 127
    c.vs[...] = 127
    ki, vi = fp8.k_index(D), fp8.v_index(D)
    q = rng.uniform(1, 2, (len(lens), G, Hq, D)) * rng.choice([-1.0, 1.0], (len(lens), G, Hq, D))
    q = torch.from_numpy(q * 2.0 ** rng.choice([10, 20, 27, 28, 30, 40, 60, 100], (len(lens), G, Hq, 1))).bfloat16()
    want = np.empty(q.shape)
    for b, L in enumerate(lens):
        k = (rng.integers(0x38, 0x40, (L, Hkv, D)) | rng.integers(0, 2, (L, Hkv, D)) << 7).astype(np.uint8)  # 1 .. 1.875
        v = (rng.integers(0x20, 0x48, (L, Hkv, D)) | rng.integers(0, 2, (L, Hkv, D)) << 7).astype(np.uint8)
        rows_of_head = q[b].double().numpy().reshape(G, Hkv, group, D).transpose(1, 0, 2, 3).reshape(Hkv, G * group, D)
        for h in range(Hkv):
            at = rng.permutation(L - G)[:G * group]
            k[at, h] = 0x40 | np.where(rows_of_head[h] < 0, 0x80, 0)  # 2, the row's signs
            want[b, :, h * group:(h + 1) * group] = fp8.decode(v[at, h]).reshape(G, group, D)
            if h == 0:
                s = rows_of_head[h] @ fp8.decode(k[:, h]).T
                best = s[np.arange(len(at)), at].copy()
                s[np.arange(len(at)), at] = -np.inf
                assert ((best - s.max(axis=1)) / np.sqrt(D) > 2000).all()
        put_rows(c, c.k, ki, b, k)
        put_rows(c, c.v, vi, b, v)
    c.upload()
    got = attend(G, Hq, Hkv, D, c, lens, q.cuda(), None, 1 / np.sqrt(D))
    assert np.array_equal(got, want), f"{(got != want).any(axis=3).sum()} rows differ"


@pytest.mark.parametrize("D", [64, 128])
def test_nan_among_keys_that_are_taken_again(D):
    """A far score late in each chunk takes the item up again; a NaN value early in one makes its column
    NaN in its head, and nothing else."""
    G, H = 3, 16
    rng = np.random.default_rng(D)
    lens = [1400 - 31 * i for i in range(24)]
    off = np.cumsum([0] + lens[:-1])
    x = [rng.normal(size=(sum(lens), H, D)) for _ in range(2)]
    x[0][...] = 0.0
    x[0][..., 0] = rng.normal(size=(sum(lens), H))
    for o, n in zip(off, lens):
        x[0][o + 50:o + n:64, :, 0] = 300.0 + np.arange(len(range(50, n, 64)))[:, None]
    c = Cache(rng, lens, H, D, 64)
    c.append(*x, off, lens, lens)
    clean = c.v.copy()
    c.v[c.table[2, 1], 1, 0, fp8.v_index(D)[3, 5]] = 0xff
    c.upload()
    q = torch.zeros((len(lens), G, H, D), dtype=torch.bfloat16)
    q[..., 0] = 1.0
    got = attend(G, H, H, D, c, lens, q.cuda(), None, 1.0)
    seg = fp8.kv8_segments(c.k, clean, c.ks, c.vs, c.table, lens)
    hit = np.zeros(got.shape, dtype=bool)
    hit[2, :, 1, 5] = True
    assert np.array_equal(np.isnan(got), hit)
    got[hit] = verify_attention(q.double().numpy(), *seg, lens, H, 1.0)[hit]
    check_attention(got, q.double().numpy(), seg, lens, H, None, 1.0, "taken again")


@pytest.mark.parametrize("D", [64, 128])
def test_attention_of_scores_far_below_zero(D):
    """Rows whose every score lies between -2^119 and -2^112: the key of the least magnitude has all the weight."""
    rng = np.random.default_rng(D)
    G, H, lens = 3, 2, [3, 64, 500, 1411]
    c = Cache(rng, lens, H, D, 64)
    c.ks[...] = 127
    c.vs[...] = 127
    q = torch.from_numpy(rng.uniform(1, 2, (len(lens), G, H, D)) * 2.0 ** 110).bfloat16()
    want = np.empty(q.shape)
    for b, L in enumerate(lens):
        k = rng.integers(0xb8, 0xc0, (L, H, D)).astype(np.uint8)  # -1 .. -1.875
        v = (rng.integers(0x20, 0x48, (L, H, D)) | rng.integers(0, 2, (L, H, D)) << 7).astype(np.uint8)
        for h in range(H):
            at = rng.integers(0, L - G + 1)
            k[at, h] = 0xa8  # -1/4
            want[b, :, h] = fp8.decode(v[at, h])
        put_rows(c, c.k, fp8.k_index(D), b, k)
        put_rows(c, c.v, fp8.v_index(D), b, v)
    c.upload()
    got = attend(G, H, H, D, c, lens, q.cuda(), None, 1 / np.sqrt(D))
    assert np.array_equal(got, want)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("exponent", [0, 60, 75, 95])
def test_attention_of_large_values(exponent, D):
    """Values up to 2^(exponent + 1) and scores that grow by 40 (2^57.7 in the exponential) after a
    chunk's first keys: weights times values stay within float32.  One column alone makes a
    score, as in test_attention_of_scores_that_jump."""
    G, H, lens = 3, 16, [1400 - 31 * i for i in range(24)]
    rng = np.random.default_rng(D)
    c = Cache(rng, lens, H, D, 64)
    c.ks[...] = 127
    c.vs[...] = 127 + exponent
    for b, L in enumerate(lens):
        k = np.zeros((L, H, D), dtype=np.uint8)
        k[40::50, :, 0] = 0x62  # 40
        v = (rng.integers(0x30, 0x40, (L, H, D)) | rng.integers(0, 2, (L, H, D)) << 7).astype(np.uint8)
        put_rows(c, c.k, fp8.k_index(D), b, k)
        put_rows(c, c.v, fp8.v_index(D), b, v)
    c.upload()
    q = torch.zeros((len(lens), G, H, D), dtype=torch.bfloat16)
    q[..., 0] = 1.0
    got = attend(G, H, H, D, c, lens, q.cuda(), None, 1.0)
    seg = fp8.kv8_segments(c.k, c.v, c.ks, c.vs, c.table, lens)
    check_attention(got, q.double().numpy(), seg, lens, H, None, 1.0, f"values of 2^{exponent}")


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new", [3, 20])
def test_append_to_blocks_of_any_scale(new, dim):
    """Blocks that other programs filled hold any scale byte from 1 to 254."""
    rng = np.random.default_rng(new)
    bytes_ = [1, 2, 20, 26, 27, 100, 240, 247, 248, 252, 253, 254]
    lens = [40 + new] * len(bytes_)
    c = Cache(rng, lens, 2, dim, 64)
    for b, v in enumerate(bytes_):
        c.ks[c.table[b, 0]] = v
        c.vs[c.table[b, 0]] = v
    c.upload()
    x = [(rng.uniform(1, 2, (new, 2, dim)) * 2.0 ** rng.choice([-120, -3, 60, 127], (new, 2, dim))).astype(np.float32) for _ in range(2)]
    d = sd.Dims(len(lens), 0, 2, 2, dim, 32, 1, 0, 0)
    off, n = [0] * len(lens), [new] * len(lens)
    c.append(*(a.astype(np.float64) for a in x), off, n, lens)
    sd.sd_kv8_append(d, c.handle, *(torch.from_numpy(a).cuda() for a in x), off, n, lens)
    torch.cuda.synchronize()
    c.check()


def test_a_pool_of_another_size_is_refused():
    """Pages with bytes to spare would be read at the wrong places."""
    rng = np.random.default_rng(16)
    c = filled(rng, [64], 2, 64, 64)
    n = c.dev[0].shape[0]
    k, v = (torch.zeros((n, 2 * 64 * 64 + extra), dtype=torch.uint8, device="cuda") for extra in (64, 64))
    with pytest.raises(ValueError):
        sd.KV8Cache.of(k, v, c.dev[2], c.dev[3], c.handle._tensors[4], 64)
    k, v = (t[:, :2 * 64 * 64].contiguous() for t in (k, v))
    sd.KV8Cache.of(k, v, c.dev[2], c.dev[3], c.handle._tensors[4], 64)
