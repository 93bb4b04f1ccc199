"""The 4-bit KV cache on the GPU against the float64 oracle: appends code for
code, rows read back to a rounding, attention within a bound that is derived in
check_attention."""

import numpy as np
import pytest
import torch

import paper_2601_21622_amd as sd
from oracle import fp4, tree_attention, verify_attention

from gpu_util import announce

pytestmark = pytest.mark.gpu

TYPES = {torch.bfloat16: sd.SD_DTYPE_BF16, torch.float32: sd.SD_DTYPE_F32}


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
    """A pool on both sides, its bytes seeded (scales of any kind, NaN among them)."""

    def __init__(self, rng, kv_len, heads, dim, page):
        self.dim, self.page = dim, page
        self.table, n = make_table(rng, kv_len, page)
        shape = (n, heads, page // 64)
        self.host = [rng.integers(0, 256, (*shape, 32 * dim), dtype=np.uint8) for _ in range(2)]
        self.host.append(rng.integers(0, 256, (*shape, 2 * dim), dtype=np.uint8))
        self.host.append(rng.integers(0, 65536, (*shape, 64), dtype=np.uint16))
        self.dev = [torch.from_numpy(a.view(np.int16) if a.dtype == np.uint16 else a).cuda() for a in self.host]
        self.handle = sd.KV4Cache.of(*self.dev[:3], self.dev[3].view(torch.bfloat16), torch.from_numpy(self.table).cuda(), page)

    def upload(self):
        for d, a in zip(self.dev, self.host):
            d.copy_(torch.from_numpy(a.view(np.int16) if a.dtype == np.uint16 else a))

    def append(self, k_new, v_new, off, new, lens):
        self.host = list(fp4.append(*self.host, self.table, k_new, v_new, off, new, lens))

    def check(self):
        for name, d, a in zip(("k", "v", "k_scale", "v_scale"), self.dev, self.host):
            got = d.cpu().numpy().view(a.dtype)
            assert np.array_equal(got, a), f"{name}: {(got != a).sum()} of {a.size} differ, first {np.argwhere(got != a)[0]}"

    def segments(self, kv_len):
        return fp4.kv4_segments(*self.host, self.table, kv_len)


def dims_of(batch, heads, dim, dtype=torch.bfloat16, gamma=0, hq=None):
    return sd.Dims(batch, gamma, hq or heads, heads, dim, 32, 1, TYPES[dtype], 0)


def rows(rng, total, heads, dim, dtype, stride=None):
    """Token rows (magnitudes differ by head, row and column group) on the GPU, and their exact values."""
    x = rng.normal(size=(total, heads, dim)) * 2.0 ** rng.integers(-12, 12, (1, heads, 1)) * 2.0 ** rng.integers(-2, 3, (total, 1, 1))
    x *= np.repeat(2.0 ** rng.integers(-3, 4, (total, heads, dim // 32)), 32, axis=2)
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
    c.append(kx, vx, off, new, lens)
    for _ in range(2):  # a second time changes nothing
        sd.sd_kv4_append(dims_of(len(req), heads, dim, dtype), c.handle, kd, vd, off, new, lens)
        torch.cuda.synchronize()
        c.check()


@pytest.mark.parametrize("dim", [64, 128])
def test_append_steps_cut_back_and_odd_values(dim):
    """A session's life: prompt, steps, a cut back to fewer keys, rows of zeros, infinities,
    NaN, the largest and smallest numbers; rows shared by requests."""
    rng = np.random.default_rng(5)
    heads = 2
    c = Cache(rng, [200, 200], heads, dim, 64)
    for new, lens in (([90, 3], [90, 3]), ([5, 5], [95, 8]), ([5, 5], [97, 10]), ([1, 60], [98, 66]), ([30, 0], [120, 66]),
                      ([64, 1], [192, 1])):
        (kd, kx), (vd, vx) = rows(rng, 100, heads, dim, torch.float32), rows(rng, 100, heads, dim, torch.float32)
        for dev, x in ((kd, kx), (vd, vx)):
            odd = [0.0, -0.0, np.inf, -np.inf, np.nan, 3.4e38, -3.4e38, 1e-45, 1e-38, 2.0 ** -101, -6 * 2.0 ** -100]
            at = rng.integers(0, 100, len(odd)), rng.integers(0, heads, len(odd)), rng.integers(0, dim, len(odd))
            x[at] = np.float32(odd)
            x[7], x[8], x[9, :, 3:] = 0.0, 1e-45, -0.0
            dev.copy_(torch.from_numpy(x.astype(np.float32)))
        off = [3, 3]  # both requests read the same rows
        c.append(kx, vx, off, new, lens)
        sd.sd_kv4_append(dims_of(2, heads, dim, torch.float32), c.handle, kd, vd, off, new, lens)
        torch.cuda.synchronize()
        c.check()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_codes_at_the_borders(dtype):
    """Every border between codes, exactly and one float to either side, under scales that
    are and are not powers of two; the largest element fixes the scale."""
    rng = np.random.default_rng(6)
    dim, heads, keys = 128, 1, 192
    c = Cache(rng, [keys], heads, dim, 64)
    top = (torch.from_numpy(rng.uniform(1, 2, keys)) * 2.0 ** torch.from_numpy(rng.integers(-40, 40, keys))).to(dtype).double().numpy()
    top[:20] = 6 * 2.0 ** rng.integers(-20, 20, 20)
    step = 2.0 ** -7 if dtype == torch.bfloat16 else 2.0 ** -23
    x = np.empty((keys, 1, dim))
    for n in range(keys):
        s = float(fp4.bf16_value(fp4.value_scale(top[n]))) if n % 2 else 2.0 ** fp4.scale_exponent(top[n])
        border = rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], dim) * s
        border *= 1 + step * rng.integers(-1, 2, dim) * (border * (1 + step) < top[n])
        x[n, 0] = np.minimum(border, top[n]) * rng.choice([-1, 1], dim)
        x[n, 0, ::32] = top[n]
    dev = torch.from_numpy(x).to(dtype)
    c.append(dev.double().numpy(), dev.double().numpy(), [0], [keys], [keys])
    sd.sd_kv4_append(dims_of(1, 1, dim, dtype), c.handle, dev.cuda(), dev.cuda(), [0], [keys], [keys])
    torch.cuda.synchronize()
    c.check()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dim", [64, 128])
def test_read(dim, dtype):
    """Rows read back are the cached values rounded once (keys exactly), of NaN scales NaN; other rows stay."""
    rng = np.random.default_rng(7)
    heads, first, count = 3, [0, 5, 64, 130, 0, 63, 10], [1, 3, 64, 200, 0, 2, 55]
    lens = [f + n for f, n in zip(first, count)]
    c = Cache(rng, lens, heads, dim, 128)
    off = np.cumsum([2] + count[:-1])
    total = 2 + sum(count) + 3
    out = [torch.full((total, heads * dim + 8), 7.0, dtype=dtype, device="cuda") for _ in range(2)]
    view = [t[:, :heads * dim].unflatten(1, (heads, dim)) for t in out]
    d = dims_of(len(lens), heads, dim, dtype)
    sd.sd_kv4_read(d, c.handle, first, count, off, *view)
    torch.cuda.synchronize()
    got = [t.cpu() for t in out]
    for t in got:
        assert (t[:2] == 7).all() and (t[total - 3:] == 7).all() and (t[:, heads * dim:] == 7).all()
    for b in range(len(lens)):
        for h in range(heads):
            ref = fp4.rows(*c.host, c.table[b], first[b], count[b], h)
            for t, x in zip(got, ref):
                want = torch.from_numpy(x).to(torch.float32)
                y = t[off[b]:off[b] + count[b], h * dim:(h + 1) * dim].float()
                # A code times its scale has at most ten bits, exact in float32; bfloat16 rounds it once.
                assert torch.equal(y.nan_to_num(nan=123.0, posinf=3e38, neginf=-3e38),
                                   want.to(dtype).float().nan_to_num(nan=123.0, posinf=3e38, neginf=-3e38))
    for i in range(2):  # one of the two alone
        one = [None, None]
        one[i] = torch.full_like(out[i], 7.0)[:, :heads * dim].unflatten(1, (heads, dim))
        sd.sd_kv4_read(d, c.handle, first, count, off, *one)
        torch.cuda.synchronize()
        assert torch.equal(one[i].float().nan_to_num(nan=123.0), view[i].float().nan_to_num(nan=123.0))


# ---- attention -------------------------------------------------------------------

def check_attention(got, q, seg, kv_len, heads, parent, scale, what):
    """Bound: a weight times its value's scale is rounded to bf16 (half a step: 2^-8) where it multiplies
    the code, and the sum that divides adds the float32 weights, so |O - O*| <= 2^-8 A, A = sum p |v|; the output's
    own rounding adds 2^-8 |O|.  Scores are float32 sums of D exact products: a relative
    error of p of at most D 2^-24 |q| |k| scale and a few 2^-24 of |s|, which with the second-order
    terms is held within a twentieth of the bound for the scores used here (< 40)."""
    kseg, vseg, off = seg
    f = verify_attention if parent is None else lambda *a: tree_attention(*a[:-1], parent, a[-1])
    ref = f(q, kseg, vseg, off, kv_len, heads, scale)
    mag = f(q, kseg, np.abs(vseg), off, kv_len, heads, scale)
    bound = 1.05 * 2.0 ** -8 * (mag + np.abs(ref)) + 1e-30
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
    "rows48": (6, 16, 2, 128, 64, [6, 62, 128, 500], False),
    "rows64": (8, 8, 1, 128, 64, [8, 200], False),
    "rows88": (11, 8, 1, 128, 64, [11, 300], False),
    "rows128": (16, 8, 1, 128, 4096, [16, 5000], False),
    "rows128_d64": (64, 4, 2, 64, 64, [64, 65, 127, 400], False),
    "g64": (64, 1, 1, 128, 64, [64, 191], False),
    "tree15": (16, 6, 2, 64, 128, [16, 37, 200, 801], True),
    "tree63": (64, 2, 1, 128, 64, [64, 100, 130], True),
    "many_requests": (2, 2, 2, 64, 64, [2 + 7 * i for i in range(70)], False),
}


def attend(G, Hq, Hkv, D, c, kv_len, q, parent, scale, ws=None, stream=None):
    B = len(kv_len)
    d = sd.Dims(B, G - 1, Hq, Hkv, D, 32, 1, 1, 0)
    ws = torch.full((sd.sd_kv4_workspace_bytes(d, max(kv_len)),), 0xff, dtype=torch.uint8, device="cuda")
    out = torch.full((B, G, Hq, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    sd.sd_verify_attention_kv4(d, q, c.handle, kv_len, parent, scale, out, ws)
    torch.cuda.synchronize()
    return out.double().cpu().numpy()


def filled(rng, kv_len, heads, dim, page, key=1.0, value=1.0):
    """A cache whose keys up to kv_len hold numbers, all other bytes anything (NaN scales too).  Keys and
    values of magnitude about `key` and `value`."""
    c = Cache(rng, kv_len, heads, dim, page)
    ki, si = fp4.k_index(dim), fp4.k_scale_index(dim)
    blocks = page // 64
    for b, n in enumerate(kv_len):
        for n0 in range(0, int(n), 64):
            at = int(c.table[b][n0 // 64 // blocks]), slice(None), n0 // 64 % blocks
            m = min(64, int(n) - n0)
            e = 126 + int(np.log2(key)) + rng.integers(-1, 2, (heads, m, dim // 32))
            c.host[2][at][:, si[:m].reshape(-1)] = e.reshape(heads, -1)
            s = torch.from_numpy(rng.uniform(0.1, 0.6, (heads, m)) * value).bfloat16().view(torch.int16).numpy().view(np.uint16)
            c.host[3][at][:, :m] = s
    c.upload()
    return c


def random_tree(rng, B, N):
    return np.maximum(np.arange(N)[None, :] - rng.integers(1, 5, (B, N)), -1).astype(np.int32)


@pytest.mark.parametrize("name", ATTENDS)
def test_attention(name):
    G, Hq, Hkv, D, page, lens, tree = ATTENDS[name]
    rng = np.random.default_rng(100 + len(name))
    c = filled(rng, lens, Hkv, D, page)
    q = torch.from_numpy(rng.normal(size=(len(lens), G, Hq, D))).bfloat16()
    parent = random_tree(rng, len(lens), G - 1) if tree else None
    scale = 1 / np.sqrt(D)
    got = attend(G, Hq, Hkv, D, c, lens, q.cuda(), None if parent is None else torch.from_numpy(parent).cuda(), scale)
    worst = check_attention(got, q.double().numpy(), c.segments(lens), lens, Hkv, parent, scale, name)
    announce(f"kv4 attention {name}: {worst:.2f} of the bound")


@pytest.mark.parametrize("G,Hq,Hkv,D,lens", [(1, 4, 2, 128, [9000]), (5, 16, 8, 64, [2500, 70]), (9, 16, 2, 128, [6000, 3333])])
def test_attention_of_long_caches(G, Hq, Hkv, D, lens):
    """Chunks of many blocks, whose ring turns often, and a merge of many."""
    rng = np.random.default_rng(G)
    c = filled(rng, lens, Hkv, D, 512)
    q = torch.from_numpy(rng.normal(size=(len(lens), G, Hq, D))).bfloat16()
    got = attend(G, Hq, Hkv, D, c, lens, q.cuda(), None, 1 / np.sqrt(D))
    check_attention(got, q.double().numpy(), c.segments(lens), lens, Hkv, None, 1 / np.sqrt(D), "long")


MANY = [3600, 3593, 3585, 3584, 3521, 3500]  # of 32 heads, more than 40 blocks of keys per CU
SOME = MANY[:4]                              # more than 24


@pytest.mark.parametrize("lens", [MANY, SOME], ids=["many", "some"])
@pytest.mark.parametrize("G,D", [(3, 64), (5, 64), (8, 64), (9, 64), (14, 64), (3, 128), (5, 128), (8, 128), (9, 128), (11, 128),
                                 (14, 128), (16, 128)])
def test_attention_of_many_blocks(G, D, lens):
    """Caches so large that a wave holds more than one block of 16 rows of a head: of 24, 40, 64, 72, 88, 112 and
    128 rows, all in one wave, in several of one size and of two."""
    rng = np.random.default_rng(10 * G + D)
    Hkv = 32
    c = filled(rng, lens, Hkv, D, 256)
    q = torch.from_numpy(rng.normal(size=(len(lens), G, 8 * Hkv, D))).bfloat16()
    got = attend(G, 8 * Hkv, Hkv, D, c, lens, q.cuda(), None, 1 / np.sqrt(D))
    for b in (1, 3):  # each request against the oracle by itself
        seg = fp4.kv4_segments(*c.host, c.table[b:b + 1], lens[b:b + 1])
        check_attention(got[b:b + 1], q[b:b + 1].double().numpy(), seg, lens[b:b + 1], Hkv, None, 1 / np.sqrt(D),
                        f"many blocks, request {b}")


def place_of(c, b, at):
    """Page and block of request b's key."""
    return int(c.table[b][at // c.page]), at % c.page // 64


@pytest.mark.parametrize("G,D", [(3, 64), (5, 64), (9, 64), (3, 128), (5, 128), (8, 128), (9, 128)])
def test_jumps_and_nan_among_many_blocks(G, D):
    """Scores that jump by hundreds from key to key (one product makes a score: exact but for the factors, 4 * 2^-24 of
    512 log2 e, 2e-4 of a weight), with several row blocks to a wave; one NaN value that positions 2 .. of one head see; one
    head's queries 2^40 times as large, whose references are past 2^16."""
    rng = np.random.default_rng(20 * G + D)
    Hkv, lens, page = 32, MANY, 256
    c = filled(rng, lens, Hkv, D, page)
    column = fp4.k_index(D)[:, 0]
    codes = np.zeros((*c.host[0].shape[:3], 64 * D), dtype=np.uint8)
    codes[..., column] = rng.integers(1, 8, (*codes.shape[:3], 64))
    c.host[0][...] = fp4.pack(codes)
    del codes
    c.host[2][...] = 127
    c.host[2][..., :64] += rng.choice([0, 0, 4, 6], (*c.host[2].shape[:3], 64)).astype(np.uint8)
    at, (head, far) = lens[0] - G + 2, (3, 5)
    page_id, blk = place_of(c, 0, at)
    clean = [a.copy() for a in c.host]
    c.host[3][page_id, head, blk, at % 64] = 0x7fc0
    c.upload()
    q = torch.zeros((len(lens), G, 8 * Hkv, D), dtype=torch.bfloat16)
    q[..., 0] = torch.from_numpy(rng.choice([1.0, -1.0, 0.5], q.shape[:3])).bfloat16()
    q[:, :, 8 * far:8 * far + 8] *= 2.0 ** 40
    got = attend(G, 8 * Hkv, Hkv, D, c, lens, q.cuda(), None, 1.0)
    hit = got[0, 2:, 8 * head:8 * head + 8]
    assert np.isnan(hit).all() and np.isnan(got).sum() == hit.size
    for b in (0, 2):
        seg = fp4.kv4_segments(*clean, c.table[b:b + 1], lens[b:b + 1])
        if b == 0:  # the spoilt outputs: as the oracle's
            ref = verify_attention(q[:1].double().numpy(), *seg, lens[:1], Hkv, 1.0)
            got[0, 2:, 8 * head:8 * head + 8] = ref[0, 2:, 8 * head:8 * head + 8]
        check_attention(got[b:b + 1], q[b:b + 1].double().numpy(), seg, lens[b:b + 1], Hkv, None, 1.0,
                        f"jumps among many blocks, request {b}")


@pytest.mark.parametrize("B,G,Hq,Hkv,D,most", [(12, 1, 16, 16, 128, 2500), (20, 4, 16, 8, 64, 1900), (70, 2, 4, 2, 128, 400), (70, 3, 32, 32, 64, 130)])
def test_attention_of_requests_of_any_length(B, G, Hq, Hkv, D, most):
    """Lengths from the step's own positions to many blocks in one batch, of requests that a workgroup takes each (the first
    three) and that are cut into chunks; more requests than a launch holds."""
    rng = np.random.default_rng(B + D)
    lens = [G + int(x) for x in np.linspace(0, most - G, B)]
    rng.shuffle(lens)
    c = filled(rng, lens, Hkv, D, 64)
    q = torch.from_numpy(rng.normal(size=(B, G, Hq, D))).bfloat16()
    got = attend(G, Hq, Hkv, D, c, lens, q.cuda(), None, 1 / np.sqrt(D))
    check_attention(got, q.double().numpy(), c.segments(lens), lens, Hkv, None, 1 / np.sqrt(D), "lengths")



def key_rows(c, b, at):
    """The pool's place of request b's key."""
    blocks = c.page // 64
    return int(c.table[b][at // 64 // blocks]), slice(None), at // 64 % blocks


@pytest.mark.parametrize("G,Hq,Hkv,D", [(2, 16, 16, 128), (5, 16, 16, 64), (10, 32, 4, 128), (9, 8, 1, 64)])
def test_attention_of_scores_that_jump(G, Hq, Hkv, D):
    """Keys whose magnitude grows along the cache, and single ones far above the rest at a block's start
    and end, in whole blocks and in the last: references are set again, many times over."""
    rng = np.random.default_rng(11)
    lens = [700 + G, 64 + G, 64]
    c = filled(rng, lens, Hkv, D, 64)
    si = fp4.k_scale_index(D)
    for b, n in enumerate(lens):
        for at in range(n):
            up = at // 64 // 2 + (3 if at in (64, 127, 200, n - 1, n - G) else 0)
            p = key_rows(c, b, at)
            c.host[2][p][:, si[at % 64]] += np.uint8(up)
    c.upload()
    q = torch.from_numpy(rng.normal(size=(len(lens), G, Hq, D))).bfloat16()
    scale = 0.5 / np.sqrt(D)
    got = attend(G, Hq, Hkv, D, c, lens, q.cuda(), None, scale)
    # Scores reach 2^9: their float32 sums are off by up to D 2^-24 |q||k| scale, which stays below 2^-4 here, and
    # so does a weight's relative error; dominated rows are one value each.  Weights below 2^-126, float32's smallest
    # normal number, may be 0: of 701 keys with values below 4 they add up to less than 701 * 4 * 2^-126 < 1e-30.
    kseg, vseg, off = c.segments(lens)
    ref = verify_attention(q.double().numpy(), kseg, vseg, off, lens, Hkv, scale)
    mag = verify_attention(q.double().numpy(), kseg, np.abs(vseg), off, lens, Hkv, scale)
    smax = max(np.linalg.norm(q.double().numpy(), axis=-1).max() * np.linalg.norm(kseg.reshape(-1, D), axis=1).max() * scale, 1)
    tol = 1.05 * 2.0 ** -8 * (mag + np.abs(ref)) + 2 * D * 2.0 ** -24 * smax * (mag + np.abs(ref)) + 1e-30
    assert (np.abs(got - ref) <= tol).all(), np.abs(got - ref).max()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("size", [2.0 ** 14, 2.0 ** 30, 2.0 ** 100, -(2.0 ** 100)])
def test_attention_of_huge_scores(size, D):
    """Queries so large that scores pass 2^100: one key is far above the others and takes all the weight;
    twins of it, blocks apart, share it alike."""
    rng = np.random.default_rng(12)
    G, Hq, Hkv, lens = 3, 4, 2, [400, 67]
    c = filled(rng, lens, Hkv, D, 64)
    si, ki = fp4.k_scale_index(D), fp4.k_index(D)
    at = {0: [30, 130, 390], 1: [5, 62]}
    for b, keys in at.items():
        for n in range(lens[b]):
            p = key_rows(c, b, n)
            codes = fp4.unpack(c.host[0][p])
            # Products of equal sign: every key's score is size * (1 or 4) * D, the marked keys' the largest.
            big = n in keys
            codes[:, ki[n % 64]] = (6 if big else 2) if size > 0 else (2 if big else 6)
            c.host[0][p] = fp4.pack(codes)
            c.host[2][p][:, si[n % 64]] = 127
    c.upload()
    q = torch.full((2, G, Hq, D), float(size)).bfloat16()
    got = attend(G, Hq, Hkv, D, c, lens, q.cuda(), None, 1.0)
    _, vseg, off = c.segments(lens)
    for b, keys in at.items():
        V = vseg[off[b]:].reshape(-1)[:Hkv * lens[b] * D].reshape(Hkv, lens[b], D)
        for h in range(Hq):
            v = V[h // (Hq // Hkv)][keys]
            ref, mag = v.mean(0), np.abs(v).mean(0)
            assert (np.abs(got[b, :, h] - ref) <= 1.05 * 2.0 ** -8 * (mag + np.abs(ref))).all()


def test_nan_reaches_only_those_that_see_it():
    """A key of a NaN scale, and a value's: outputs of the positions that see it are NaN, the others'
    are the oracle's.  Bytes past the last key are anything already."""
    rng = np.random.default_rng(13)
    G, Hq, Hkv, D, lens = 4, 4, 2, 128, [70, 140, 200, 68]
    scale = 1 / np.sqrt(D)
    q = torch.from_numpy(rng.normal(size=(len(lens), G, Hq, D))).bfloat16()
    parent = np.array([[-1, 0, -1]] * 4, dtype=np.int32)  # positions 1 and 2 a chain, 3 another child of the root
    for pool in (2, 3):
        c = filled(rng, lens, Hkv, D, 64)
        clean = c.segments(lens)
        put = [(0, 68), (1, 3), (2, 199), (3, 65)]  # request, key; keys of positions 2, prefix, 3, 1
        for b, n in put:
            p = key_rows(c, b, n)
            if pool == 2:
                c.host[2][p][:, fp4.k_scale_index(D)[n % 64, 1]] = 255
            else:
                c.host[3][p][:, n % 64] = 0x7fc0
        c.upload()
        ref = tree_attention(q.double().numpy(), *clean, lens, Hkv, parent, scale)
        mag = tree_attention(q.double().numpy(), clean[0], np.abs(clean[1]), clean[2], lens, Hkv, parent, scale)
        got = attend(G, Hq, Hkv, D, c, lens, q.cuda(), torch.from_numpy(parent).cuda(), scale)
        sees = {0: [2], 1: [0, 1, 2, 3], 2: [3], 3: [1, 2]}
        for b in range(4):
            for g in range(G):
                if g in sees[b]:
                    assert np.isnan(got[b, g]).all(), (pool, b, g)
                else:
                    tol = 1.05 * 2.0 ** -8 * (mag[b, g] + np.abs(ref[b, g]))
                    assert (np.abs(got[b, g] - ref[b, g]) <= tol).all(), (pool, b, g)


@pytest.mark.parametrize("exponent", [-90, 0, 60, 105])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_of_large_and_small_values(exponent, D):
    """Values near both ends of what sums in float32 hold, among keys that grow."""
    rng = np.random.default_rng(14)
    G, Hq, Hkv, lens = 2, 4, 2, [300, 66]
    c = filled(rng, lens, Hkv, D, 64, value=2.0 ** exponent)
    si = fp4.k_scale_index(D)
    for n in range(300):
        c.host[2][key_rows(c, 0, n)][:, si[n % 64]] += np.uint8(n // 100)
    c.upload()
    q = torch.from_numpy(rng.normal(size=(2, G, Hq, D))).bfloat16()
    got = attend(G, Hq, Hkv, D, c, lens, q.cuda(), None, 1 / np.sqrt(D))
    check_attention(got, q.double().numpy(), c.segments(lens), lens, Hkv, None, 1 / np.sqrt(D), str(exponent))


@pytest.mark.parametrize("lens", [[133, 700, 64], [2500, 9000, 64]], ids=["joined", "chunks"])
def test_streams_graphs_and_workspaces(lens):
    """A captured step (append, attention) replayed over changing inputs, with eager work between the
    replays and calls on another stream with a workspace of their own; results do not depend on either."""
    rng = np.random.default_rng(15)
    G, Hq, Hkv, D = 5, 8, 4, 128
    c = filled(rng, lens, Hkv, D, 64)
    d = sd.Dims(3, G - 1, Hq, Hkv, D, 32, 1, 1, 0)
    n = sd.sd_kv4_workspace_bytes(d, max(lens))
    ws, ws2 = (torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(2))
    q = torch.zeros((3, G, Hq, D), dtype=torch.bfloat16, device="cuda")
    k_new, v_new = (torch.zeros((3 * G, Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    out, out2 = torch.zeros_like(q), torch.zeros_like(q)
    off = [0, G, 2 * G]

    def step(out, ws):
        sd.sd_kv4_append(d, c.handle, k_new, v_new, off, [G] * 3, lens)
        sd.sd_verify_attention_kv4(d, q, c.handle, lens, None, 0.1, out, ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(out, ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out, ws)
    for i in range(4):
        for t in (q, k_new, v_new):
            t.copy_(torch.from_numpy(rng.normal(size=t.shape)).bfloat16())
        graph.replay()
        torch.cuda.synchronize()
        first = out.clone()
        c.append(k_new.double().cpu().numpy(), v_new.double().cpu().numpy(), off, [G] * 3, lens)
        c.check()
        check_attention(first.double().cpu().numpy(), q.double().cpu().numpy(), c.segments(lens), lens, Hkv, None, 0.1, f"replay {i}")
        side.wait_stream(torch.cuda.current_stream())
        sd.sd_verify_attention_kv4(d, q, c.handle, lens, None, 0.1, out2, ws2, stream=side)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first) and torch.equal(out2, first)  # deterministic, whatever runs beside


def test_far_pages():
    """Pages past 4 GB of the pools: offsets pass 32 bits."""
    rng = np.random.default_rng(16)
    heads, dim, page = 2, 128, 4096
    pages = 17000  # 17000 * 2 * 4096 * 64 bytes = 8.9 GB each of K and V
    shape = (pages, heads, page // 64)
    k, v = (torch.zeros((*shape, 32 * dim), dtype=torch.uint8, device="cuda") for _ in range(2))
    ks = torch.zeros((*shape, 2 * dim), dtype=torch.uint8, device="cuda")
    vs = torch.zeros((*shape, 64), dtype=torch.bfloat16, device="cuda")
    ids = [16999, 8200, 4099]
    table = torch.tensor([ids], dtype=torch.int32, device="cuda")
    handle = sd.KV4Cache.of(k, v, ks, vs, table, page)
    n = 2 * page + 100
    (kd, kx), (vd, vx) = rows(rng, n, heads, dim, torch.bfloat16), rows(rng, n, heads, dim, torch.bfloat16)
    d = sd.Dims(1, 0, 2, heads, dim, 32, 1, 1, 0)
    sd.sd_kv4_append(d, handle, kd, vd, [0], [n], [n])
    out = [torch.empty((n, heads, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    sd.sd_kv4_read(d, handle, [0], [n], [0], *out)
    torch.cuda.synchronize()
    host = [a[ids].cpu() for a in (k, v, ks, vs)]
    host[3] = host[3].view(torch.int16)
    host = [a.numpy() for a in host]
    host[3] = host[3].view(np.uint16)
    local = np.array([[0, 1, 2]])
    for h in range(heads):
        for first in (0, page - 20, 2 * page + 50):
            for got, want in zip(out, fp4.rows(*host, local[0], first, 50, h)):
                assert torch.equal(got[first:first + 50, h].cpu(), torch.from_numpy(want).float().bfloat16())
        e = np.abs(kx[:, h].reshape(n, -1, 32)).max(2)
        assert (np.abs(out[0][:, h].double().cpu().numpy() - kx[:, h]).reshape(n, -1, 32) <= e[..., None] / 3).all()
    q = torch.from_numpy(rng.normal(size=(1, 1, 2, dim)) * 2.0 ** -8).bfloat16()
    ws = torch.empty(sd.sd_kv4_workspace_bytes(d, n), dtype=torch.uint8, device="cuda")
    got = torch.empty((1, 1, 2, dim), dtype=torch.bfloat16, device="cuda")
    sd.sd_verify_attention_kv4(d, q.cuda(), handle, [n], None, 2.0 ** -8, got, ws)
    torch.cuda.synchronize()
    check_attention(got.double().cpu().numpy(), q.double().numpy(), fp4.kv4_segments(*host, local, [n]), [n], heads, None,
                    2.0 ** -8, "far pages")


def test_bad_page_ids_are_clamped():
    """Ids outside the pool are clamped into it: nothing is read or written past its ends."""
    rng = np.random.default_rng(17)
    c = filled(rng, [64, 64], 1, 64, 64)
    pages = c.host[0].shape[0]
    handle = sd.KV4Cache.of(*c.dev[:3], c.dev[3].view(torch.bfloat16), torch.tensor([[-5], [10 ** 6]], dtype=torch.int32, device="cuda"), 64)
    c.table = np.array([[0], [pages - 1]])
    (kd, kx), (vd, vx) = rows(rng, 128, 1, 64, torch.bfloat16), rows(rng, 128, 1, 64, torch.bfloat16)
    c.append(kx, vx, [0, 64], [64, 64], [64, 64])
    d = dims_of(2, 1, 64)
    sd.sd_kv4_append(d, handle, kd, vd, [0, 64], [64, 64], [64, 64])
    out = torch.empty((128, 1, 64), dtype=torch.bfloat16, device="cuda")
    sd.sd_kv4_read(d, handle, [0, 0], [64, 64], [0, 64], out, None)
    torch.cuda.synchronize()
    c.check()
    for b in range(2):
        assert torch.equal(out[64 * b:64 * b + 64, 0].cpu(), torch.from_numpy(fp4.rows(*c.host, c.table[b], 0, 64, 0)[0]).bfloat16())


def test_a_step_of_all_calls():
    """As a step uses them: norms and rotation of a fused projection's rows, the append, the attention of a tree,
    acceptance's path read back and appended next to the root, then one token of plain decoding."""
    rng = np.random.default_rng(18)
    B, G, Hq, Hkv, D = 2, 6, 8, 2, 128
    old, page = [90, 60], 64
    lens = [n + G for n in old]
    c = filled(rng, lens, Hkv, D, page)
    parent = random_tree(rng, B, G - 1)
    depth = np.zeros((B, G), dtype=np.int32)
    for g in range(1, G):
        depth[:, g] = depth[np.arange(B), parent[:, g - 1] + 1] + 1
    fused = torch.from_numpy(rng.normal(size=(B * G, (Hq + 2 * Hkv) * D))).bfloat16()
    dev = fused.cuda()
    heads = dev.unflatten(1, (Hq + 2 * Hkv, D))
    pos = (np.array(old)[:, None] + depth).reshape(-1).astype(np.int32)
    f = (5e5 ** (-np.arange(D // 2) / (D // 2))).astype(np.float32)
    w = [torch.from_numpy(1 + 0.1 * rng.normal(size=D)).bfloat16() for _ in range(2)]
    q, k = heads[:, :Hq], heads[:, Hq:Hq + Hkv]
    sd.sd_qk_norm_rope(q, k, torch.from_numpy(pos).cuda(), torch.from_numpy(f).cuda(), w[0].cuda(), w[1].cuda(), 1e-6, q, k)
    d = sd.Dims(B, G - 1, Hq, Hkv, D, 32, 1, 1, 0)
    off = [0, G]
    v = heads[:, Hq + Hkv:]
    sd.sd_kv4_append(d, c.handle, k, v, off, [G] * B, lens)
    qc = q.contiguous()
    ws = torch.empty(sd.sd_kv4_workspace_bytes(d, 200), dtype=torch.uint8, device="cuda")
    out = torch.empty((B, G, Hq, D), dtype=torch.bfloat16, device="cuda")
    sd.sd_verify_attention_kv4(d, qc, c.handle, lens, torch.from_numpy(parent).cuda(), D ** -0.5, out, ws)
    torch.cuda.synchronize()
    host = heads.double().cpu().numpy()
    x = fused.double().numpy().reshape(B * G, -1, D)
    for part, weight in ((slice(0, Hq), w[0]), (slice(Hq, Hq + Hkv), w[1])):
        ref, mag = fp4.norm_rope(x[:, part], weight.double().numpy(), pos, f, 1e-6, False)
        assert (np.abs(host[:, part] - ref) <= 2.0 ** -8 * np.abs(ref) + 1e-5 * mag).all()
    assert np.array_equal(host[:, Hq + Hkv:], x[:, Hq + Hkv:])
    c.append(host[:, Hq:Hq + Hkv], host[:, Hq + Hkv:], off, [G] * B, lens)
    c.check()
    check_attention(out.double().cpu().numpy(), host[:, :Hq].reshape(B, G, Hq, D), c.segments(lens), lens, Hkv, parent, D ** -0.5, "tree")
    # A path of two nodes is accepted: their rows are read (keys old + 1 + node) and appended after the root.
    path = [[0, g] for g in [int(np.flatnonzero(parent[b] == 0)[0]) if (parent[b] == 0).any() else 1 for b in range(B)]]
    first, count = [], []
    for b in range(B):
        for node in path[b]:
            first.append(old[b] + 1 + node)
    d4 = sd.Dims(1, 0, Hkv, Hkv, D, 32, 1, 0, 0)  # one row at a time, in float32
    kr, vr = (torch.empty((4, Hkv, D), dtype=torch.float32, device="cuda") for _ in range(2))
    for i, at in enumerate(first):
        b = i // 2
        one = sd.KV4Cache.of(*c.dev[:3], c.dev[3].view(torch.bfloat16), torch.from_numpy(c.table[b:b + 1]).cuda(), page)
        sd.sd_kv4_read(d4, one, [at], [1], [i], kr, vr)
    now = [n + 3 for n in old]
    d2 = sd.Dims(B, 0, Hkv, Hkv, D, 32, 1, 0, 0)
    sd.sd_kv4_append(d2, c.handle, kr, vr, [0, 2], [2, 2], now)
    torch.cuda.synchronize()
    kept = [fp4.rows(*c.host, c.table[i // 2], at, 1, h) for i, at in enumerate(first) for h in range(Hkv)]
    c.append(kr.double().cpu().numpy(), vr.double().cpu().numpy(), [0, 2], [2, 2], now)
    for i, (kk, vv) in enumerate(kept):
        b, j, h = i // (2 * Hkv), i // Hkv % 2, i % Hkv
        k2, v2 = fp4.rows(*c.host, c.table[b], old[b] + 1 + j, 1, h)
        assert np.array_equal(k2, kk) and np.array_equal(v2, vv)
    c.check()
    d1 = sd.Dims(B, 0, Hq, Hkv, D, 32, 1, 1, 0)
    sd.sd_verify_attention_kv4(d1, qc[:B], c.handle, now, None, D ** -0.5, out, ws)
    torch.cuda.synchronize()
    check_attention(out.reshape(-1, Hq, D)[:B, None].double().cpu().numpy(), host[:B, None, :Hq], c.segments(now), now, Hkv, None, D ** -0.5, "token")


def test_binding_refuses_what_does_not_fit():
    rng = np.random.default_rng(19)
    c = filled(rng, [64], 2, 64, 64)
    d = dims_of(1, 2, 64)
    t = torch.zeros((4, 2, 64), dtype=torch.bfloat16, device="cuda")
    for bad in (dims_of(1, 1, 64), dims_of(1, 2, 128), dims_of(2, 2, 64)):
        with pytest.raises(ValueError):
            sd.sd_kv4_append(bad, c.handle, t, t, [0] * bad.batch, [1] * bad.batch, [1] * bad.batch)
    for args in ((t.float(), t, [0], [1], [1]), (t, t[:, :1], [0], [1], [1]), (t, t, [0], [5], [5]), (t, t, [0, 1], [1], [1]),
                 (t.transpose(0, 1), t, [0], [1], [1])):
        with pytest.raises(ValueError):
            sd.sd_kv4_append(d, c.handle, *args)
    with pytest.raises(ValueError):
        sd.sd_kv4_read(d, c.handle, [0], [5], [0], t, None)
    with pytest.raises(sd.SdError):
        sd.sd_kv4_read(d, c.handle, [62], [3], [0], t, None)
    with pytest.raises(ValueError):
        sd.sd_verify_attention_kv4(d, t[:1].float(), c.handle, [64], None, 0.1, t, t)
    with pytest.raises(sd.SdError):
        sd.sd_verify_attention_kv4(d, t, c.handle, [64], None, 0.1, t, torch.zeros(16, dtype=torch.uint8, device="cuda"))
    pools = [*c.dev[:3], c.dev[3].view(torch.bfloat16), torch.zeros((1, 1), dtype=torch.int32, device="cuda")]
    for i, bad in ((0, pools[0][:1]), (1, pools[1][..., :100].contiguous()), (2, pools[2][..., :64].contiguous()),
                   (3, pools[3].float()), (3, pools[3].half()), (4, pools[4].long())):
        with pytest.raises(ValueError):
            sd.KV4Cache.of(*pools[:i], bad, *pools[i + 1:], 64)
    with pytest.raises(ValueError):
        sd.KV4Cache.of(*pools, 128)
    sd.sd_kv4_append(d, c.handle, t[:0], t[:0], [0], [0], [0])  # nothing to append or read
    sd.sd_kv4_read(d, c.handle, [0], [0], [0], t[:0], None)
