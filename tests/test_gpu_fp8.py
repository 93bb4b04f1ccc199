"""The normed 8-bit rows and the 8-bit projection on the GPU against the
float64 oracle, and the 8-bit calls run together as a verification step."""

import numpy as np
import pytest
import torch

import paper_2601_21622_amd as sd
from oracle import accept_resample, fp8, near_threshold, verify_attention

from gpu_util import announce

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn
U = 2.0 ** -24


def run_norm(x, r, w, eps, store=True):
    rows, width = x.shape
    out = torch.full((rows, width), 0x55, dtype=torch.uint8, device="cuda").view(F8)
    scale = torch.full((-(-width // 128), rows), float("nan"), device="cuda")
    new = torch.empty_like(x) if store else None
    sd.sd_residual_norm_fp8(x, r, w, eps, new, out, scale)
    torch.cuda.synchronize()
    return new, out.view(torch.uint8).cpu().numpy(), scale.double().cpu().numpy()


@pytest.mark.parametrize("rows,width,dtype,residual", [
    (1, 32, torch.bfloat16, True), (3, 64, torch.float32, True), (5, 160, torch.bfloat16, False), (2, 512, torch.bfloat16, True),
    (7, 544, torch.float32, True), (4, 2048, torch.bfloat16, True), (9, 2080, torch.bfloat16, True), (33, 4096, torch.bfloat16, True),
    (6, 5120, torch.float32, True), (5, 8192, torch.bfloat16, False), (3, 8224, torch.bfloat16, True), (2, 16384, torch.float32, True),
    (2, 32768, torch.bfloat16, True), (300, 256, torch.bfloat16, True),
])
def test_norm(rows, width, dtype, residual):
    """Bounds: h is one float32 sum, 1/rms one rounding of a float64, y two products and
    the scale one division: y and the scale are within 6 2^-24 of the formula's, relative; a code
    stands for the value nearest to y / s, so |code s - y| is half a step of e4m3 there and
    16 2^-24 of |y| more (the factor 1/s and its product, and the above)."""
    rng = np.random.default_rng(rows + width)
    t = [torch.from_numpy(rng.normal(size=s) * m).to(dtype) for s, m in (((rows, width), 1), ((rows, width), 3), ((width,), 1))]
    t[0][0, 0] = 500.0
    x, r, w = (a.cuda() for a in t)
    new, code, scale = run_norm(x, r if residual else None, w, 1e-5)
    xs = [a.double().numpy() for a in t]
    h, y, s = fp8.residual_norm(xs[0], xs[1] if residual else None, xs[2], 1e-5)
    assert np.array_equal(new.double().cpu().numpy(), torch.from_numpy(h).float().to(dtype).double().numpy())
    assert np.all(np.abs(scale - s) <= 8 * U * s)
    per = np.repeat(scale.T, 128, axis=1)[:, :width]
    z = y / per
    step = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(np.abs(z), 1e-30))), -6) - 3)
    assert np.all(np.abs(fp8.decode(code) - z) <= step / 2 + 16 * U * np.abs(z))


def test_norm_of_odd_rows():
    """Zeros, NaN, infinities, numbers whose squares overflow; in place; no output of h."""
    x = torch.randn((8, 256), device="cuda")
    x[1] = 0
    x[2, 5] = float("nan")
    x[3, 200] = float("inf")
    x[4] *= 1e30
    x[5] *= 1e-30
    w = torch.ones((256,), device="cuda")
    _, code, scale = run_norm(x, None, w, 0.0 + 1e-12, store=False)
    v = fp8.decode(code)
    assert np.isfinite(scale).all()
    assert (v[1] == 0).all() and np.isnan(v[2]).all()
    assert np.isnan(v[3, 200]) and (np.delete(v[3], 200) == 0).all()
    for row in (0, 4):
        h = x[row].double().cpu().numpy()
        y = h / np.sqrt((h * h).mean() + 1e-12)
        assert np.all(np.abs(v[row] * np.repeat(scale[:, row], 128) - y) <= 2.0 ** -4 * np.abs(y) + 2.0 ** -9 * np.abs(y).max() / 448)
    h = torch.randn((4, 96), device="cuda").bfloat16()
    a, b = torch.randn_like(h), h.clone()
    wb = torch.ones((96,), device="cuda").bfloat16()
    new, code, scale = run_norm(a, b, wb, 1e-6)
    out, sc = torch.empty((4, 96), dtype=F8, device="cuda"), torch.empty((1, 4), device="cuda")
    sd.sd_residual_norm_fp8(a, b, wb, 1e-6, b, out, sc)  # new_residual is residual
    assert torch.equal(b, new) and np.array_equal(out.view(torch.uint8).cpu().numpy(), code)


def random_codes(rng, shape):
    c = rng.integers(0, 256, shape, dtype=np.uint8)
    return np.where(c & 127 == 127, 0x30, c).astype(np.uint8)


def run_logits(a, sa, w, sw, batch=None):
    M, K = a.shape
    V = w.shape[0]
    d = sd.Dims(batch or M, M // (batch or M) - 1, 1, 1, 128, K, V, 1, 0)
    dev = [torch.from_numpy(np.ascontiguousarray(t)).cuda() for t in (a, sa, w, sw)]
    logits = torch.full((M, V), float("nan"), device="cuda")
    lse = torch.empty((M,), device="cuda")
    ws = torch.full((sd.sd_fp8_workspace_bytes(d, 1 << 10),), 0xff, dtype=torch.uint8, device="cuda")
    sd.sd_verify_logits_fp8(d, dev[0], dev[1], dev[2], dev[3], logits, lse, ws)
    torch.cuda.synchronize()
    return logits.double().cpu().numpy(), lse.double().cpu().numpy()


def check_logits(got, lse, a, sa, w, sw, what):
    """Bound: products of codes are exact in float32 (4 by 4 bits), a block's sum adds 128 of
    them (127 roundings, as may be their alignment in the matrix instruction), two products with scales,
    one fused addition per block: (128 + 3 + blocks) 2^-24 of the sum of magnitudes.  The
    log-sum-exp: float32 sums over at most 512 entries of a tile, float64 beyond."""
    ref, mag = fp8.logits_fp8(a, sa, w, sw)
    bound = (131 + sa.shape[0]) * U * mag + 1e-37
    err = np.abs(got - ref)
    bad = ~(err <= bound)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} past the bound, first {np.argwhere(bad)[0]}"
    m = got.max(axis=1)
    want = m + np.log(np.exp(got - m[:, None]).sum(axis=1))
    assert np.all(np.abs(lse - want) <= (512 + 16) * U + 4 * U * np.abs(want))
    return float((err / bound).max())


@pytest.mark.parametrize("M,K,V", [
    (1, 32, 1), (1, 128, 128), (2, 160, 129), (5, 256, 1000), (17, 96, 70), (31, 1024, 333), (32, 4096, 515), (33, 224, 4001),
    (64, 544, 2000), (65, 128, 3000), (96, 2048, 777), (129, 320, 1500), (144, 8192, 700), (160, 8320, 300), (200, 512, 33000),
    (224, 1056, 40001), (225, 256, 2000), (320, 1024, 1700), (400, 64, 900), (7, 4096, 33001), (50, 128, 70003), (1, 16384, 40),
    (130, 256, 70000), (180, 128, 33001),
    # Odd numbers of lines in two parts, more lines than a wave holds scales of, and the same with undivided columns.
    (40, 20512, 700), (100, 17280, 900), (161, 384, 1200), (3, 64, 128), (97, 672, 33001), (192, 9120, 33000),
])
def test_logits(M, K, V):
    rng = np.random.default_rng(M + K + V)
    a, w = random_codes(rng, (M, K)), random_codes(rng, (V, K))
    sa, sw = (rng.random(s).astype(np.float32) * 0.01 + 1e-4 for s in ((-(-K // 128), M), (-(-V // 128), -(-K // 128))))
    sw /= np.float32(np.sqrt(K))
    got, lse = run_logits(a, sa, w, sw)
    worst = check_logits(got, lse, a, sa, w, sw, f"{M} x {K} x {V}")
    announce(f"fp8 logits {M} x {K} x {V}: {worst:.3f} of the bound")


def test_logits_codes_one_by_one():
    """Every code against every other: W rows that hold one code each."""
    a = np.zeros((256, 32), dtype=np.uint8)
    w = np.zeros((256, 32), dtype=np.uint8)
    a[:, 3] = w[:, 3] = np.arange(256)
    a[[127, 255]] = w[[127, 255]] = 0  # NaN apart
    got, _ = run_logits(a, np.ones((1, 256), np.float32), w, np.ones((2, 1), np.float32))
    v = np.nan_to_num(fp8.VALUES)
    assert np.array_equal(got, np.outer(v, v))


def test_logits_nan_stays_in_its_row_and_column():
    rng = np.random.default_rng(3)
    a, w = random_codes(rng, (40, 256)), random_codes(rng, (300, 256))
    a[7, 200], w[131, 3] = 0x7f, 0xff
    got, lse = run_logits(a, np.ones((2, 40), np.float32), w, np.ones((3, 2), np.float32))
    nan = np.isnan(got)
    want = np.zeros_like(nan)
    want[7], want[:, 131] = True, True
    assert np.array_equal(nan, want)


def test_logits_rows_do_not_depend_on_their_batch():
    """A request's logits are the same bits whichever rows share its tile shape; repeated calls agree."""
    rng = np.random.default_rng(4)
    a, w = random_codes(rng, (64, 512)), random_codes(rng, (900, 512))
    sa, sw = rng.random((4, 64)).astype(np.float32), rng.random((8, 4)).astype(np.float32)
    g1, l1 = run_logits(a, sa, w, sw)
    g2, l2 = run_logits(a, sa, w, sw, batch=16)
    assert np.array_equal(g1, g2) and np.array_equal(l1, l2)


def test_the_calls_as_one_step():
    """A pooled step on 8-bit data: append, attention, the residual and norm of
    its output, the projection, acceptance; each stage against the oracle on the
    stage's own inputs.  Then the accepted length cuts the cache back and the next step follows."""
    rng = np.random.default_rng(21)
    B, G, Hq, Hkv, D, V, page = 5, 4, 8, 2, 128, 3001, 64
    H = Hq * D
    pool = sd.KVPool(40, page)
    lens = np.array([30, 64, 100, 61, 7])
    n_blocks = page // 64
    k, v = (torch.zeros((40, Hkv, n_blocks, 64 * D), dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.zeros((40, Hkv, n_blocks), dtype=torch.uint8, device="cuda") for _ in range(2))
    w = torch.from_numpy(random_codes(rng, (V, H))).cuda().view(F8)
    sw = torch.from_numpy((rng.random((-(-V // 128), H // 128)) * 1e-3).astype(np.float32)).cuda()
    weight = torch.ones((H,), device="cuda").bfloat16()
    d = sd.Dims(B, G - 1, Hq, Hkv, D, H, V, 1, 0)
    ws = torch.empty((sd.sd_fp8_workspace_bytes(d, 400),), dtype=torch.uint8, device="cuda")
    wa = torch.empty((sd.sd_workspace_bytes(d, 400),), dtype=torch.uint8, device="cuda")
    start = np.zeros(B, dtype=int)
    for step in range(3):
        new = lens - start if step == 0 else np.full(B, G)
        end = start + new
        for b in range(B):
            pool.reserve(b, int(end[b]))
        table = torch.from_numpy(pool.block_table(range(B), 8)).cuda()
        cache = sd.KV8Cache.of(k, v, ks, vs, table, page)
        T = int(new.sum())
        qkv = torch.randn((T, (Hq + 2 * Hkv) * D), device="cuda").bfloat16()
        kn, vn = (qkv[:, a * D:(a + Hkv) * D].unflatten(1, (Hkv, D)) for a in (Hq, Hq + Hkv))
        off = np.cumsum(new) - new
        sd.sd_kv8_append(d, cache, kn, vn, off, new, end)
        q = torch.randn((B, G, Hq, D), device="cuda").bfloat16()
        attn = torch.empty_like(q)
        sd.sd_verify_attention_kv8(d, q, cache, end, None, D ** -0.5, attn, ws)
        stream = torch.randn((B * G, H), device="cuda").bfloat16()
        code, scale = torch.empty((B * G, H), dtype=F8, device="cuda"), torch.empty((H // 128, B * G), device="cuda")
        before = stream.clone()
        sd.sd_residual_norm_fp8(attn.view(B * G, H), stream, weight, 1e-5, stream, code, scale)
        logits, lse = torch.empty((B * G, V), device="cuda"), torch.empty((B * G,), device="cuda")
        sd.sd_verify_logits_fp8(d, code, scale, w, sw, logits, lse, ws)
        qd = torch.softmax(logits.view(B, G, V)[:, :-1] + torch.randn((B, G - 1, V), device="cuda"), -1).contiguous()
        draft = torch.multinomial(qd.view(-1, V), 1).view(B, G - 1).int().contiguous()
        u = torch.rand((B, G), device="cuda")
        acc, tok, left = (torch.empty(s, dtype=torch.int32, device="cuda") for s in ((B,), (B, G), (B,)))
        sd.sd_accept_resample(d, logits, lse, qd, draft, u, end.astype(np.int32), acc, tok, left, wa)
        torch.cuda.synchronize()
        host = [t.cpu().numpy() for t in (k, v, ks, vs)]
        seg = fp8.kv8_segments(*host, table.cpu().numpy(), end)
        ref = verify_attention(q.double().cpu().numpy(), *seg, end, Hkv)
        mag = verify_attention(q.double().cpu().numpy(), seg[0], np.abs(seg[1]), seg[2], end, Hkv)
        assert np.all(np.abs(attn.double().cpu().numpy() - ref) <= 1.05 * 2.0 ** -8 * (mag + 2 * np.abs(ref)))
        assert torch.equal(stream, (attn.view(B * G, H).float() + before.float()).bfloat16())
        y = fp8.residual_norm(attn.view(B * G, H).double().cpu().numpy(), before.double().cpu().numpy(), np.ones(H), 1e-5)[1]
        c8, s8 = code.view(torch.uint8).cpu().numpy(), scale.cpu().numpy()
        assert np.all(np.abs(fp8.dequantised(c8, s8.T.astype(np.float64)) - y) <= 2.0 ** -4 * np.abs(y) + 2.0 ** -9 * np.repeat(s8.T, 128, 1))
        check_logits(logits.double().cpu().numpy(), lse.double().cpu().numpy(), c8, s8, w.view(torch.uint8).cpu().numpy(),
                     sw.cpu().numpy(), f"step {step}")
        want = accept_resample(logits.cpu().numpy(), lse.cpu().numpy(), qd.cpu().numpy(), draft.cpu().numpy(), u.cpu().numpy(),
                               kv_len=end)
        keep = np.array([not near_threshold(t) for t in want["traces"]])
        assert np.array_equal(tok.cpu().numpy()[keep], want["out_tok"][keep])
        start = left.cpu().numpy().astype(int)
        for b in range(B):
            pool.truncate(b, int(start[b]))
    pool.close()


def test_norm_of_more_rows_than_a_launch_holds():
    """2^24 rows of 256 threads each: a launch holds fewer than 2^32 threads.  Every stretch of equal rows
    comes out as the first, which is the small call's."""
    width, part, times = 544, 1 << 14, 1 << 10
    rng = np.random.default_rng(5)
    few = torch.from_numpy(rng.normal(size=(part, width))).bfloat16().cuda()
    w = torch.from_numpy(rng.normal(size=(width,))).bfloat16().cuda()
    x = torch.empty((times, part, width), dtype=torch.bfloat16, device="cuda")
    x.copy_(few[None])
    out = torch.zeros((times * part, width), dtype=torch.uint8, device="cuda")
    scale = torch.zeros((-(-width // 128), times * part), device="cuda")
    flat = x.view(times * part, width)
    sd.sd_residual_norm_fp8(flat, None, w, 1e-5, flat, out.view(F8), scale)
    one, one_scale = torch.empty((part, width), dtype=torch.uint8, device="cuda"), torch.empty((scale.shape[0], part), device="cuda")
    sd.sd_residual_norm_fp8(few, None, w, 1e-5, None, one.view(F8), one_scale)
    for i in range(times):
        at = slice(i * part, (i + 1) * part)
        assert torch.equal(out[at], one) and torch.equal(scale[:, at], one_scale) and torch.equal(x[i], few), i


def test_norm_divides_by_the_scale():
    """Codes are those of y / s, ties to even: rows of ones (their mean square is one, y is the
    weight) and weights that lie halfway between two codes' values of their block's scale, to the bit."""
    width = 32768
    rng = np.random.default_rng(6)
    s = np.repeat(rng.integers(1 << 14, 1 << 15, width // 128) / 2.0 ** 15, 128)  # 15 bits: 448 s and tie s are exact
    halves = (fp8.VALUES[8:126] + fp8.VALUES[9:127]) / 2
    z = rng.choice(halves, width) * rng.choice([-1.0, 1.0], width)
    z[::128] = 448.0
    w = (z * s).astype(np.float32)
    assert np.array_equal(w.astype(np.float64), z * s)
    x = torch.ones((2, width), device="cuda")
    x[1, ::3] = -1
    _, code, scale = run_norm(x, None, torch.from_numpy(w).cuda(), 0.0)
    assert np.array_equal(scale, np.repeat(s[::128, None], 2, axis=1))
    assert np.array_equal(code, fp8.encode(z[None] * x.cpu().double().numpy()))


@pytest.mark.parametrize("exponent,dtype", [(-140, torch.float32), (-126, torch.float32), (-110, torch.float32), (110, torch.float32),
                                            (125, torch.float32), (-120, torch.bfloat16), (125, torch.bfloat16)])
def test_norm_of_rows_near_the_ends_of_float32(exponent, dtype):
    """Rows of magnitude 2^exponent and eps 0: the normed rows are of magnitude one.  The bounds of test_norm."""
    rng = np.random.default_rng(200 + exponent)
    x = torch.from_numpy(np.clip(rng.normal(size=(5, 544)), -3, 3) * 2.0 ** exponent).to(dtype)
    w = torch.from_numpy(rng.normal(size=(544,))).to(dtype)
    new, code, scale = run_norm(x.cuda(), None, w.cuda(), 0.0)
    assert torch.equal(new.cpu(), x)
    _, y, s = fp8.residual_norm(x.double().numpy(), None, w.double().numpy(), 0.0)
    assert np.all(np.abs(scale - s) <= 8 * U * s)
    z = y / np.repeat(scale.T, 128, axis=1)[:, :544]
    step = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(np.abs(z), 1e-30))), -6) - 3)
    assert np.all(np.abs(fp8.decode(code) - z) <= step / 2 + 16 * U * np.abs(z))


@pytest.mark.parametrize("V", [900, 33001])
def test_logits_of_a_row_among_other_rows(V):
    """A row's logits and log-sum-exp are the same bits at another place of a tile of the same shape, beside fewer rows."""
    rng = np.random.default_rng(V)
    a, w = random_codes(rng, (64, 544)), random_codes(rng, (V, 544))
    sa, sw = rng.random((5, 64)).astype(np.float32), rng.random((-(-V // 128), 5)).astype(np.float32)
    every, lse = run_logits(a, sa, w, sw)
    for n in (64, 40, 33):
        pick = rng.permutation(64)[:n]
        got, got_lse = run_logits(a[pick], sa[:, pick], w, sw)
        assert np.array_equal(got, every[pick]) and np.array_equal(got_lse, lse[pick]), n


def test_norm_codes_of_short_numbers():
    """bf16 rows and weights: h * weight is exact in float32, so codes are those of its quotient by the
    block's largest over 448, whatever 1 / rms is; a block of zeros has scale 2^-126 and codes 0."""
    rng = np.random.default_rng(7)
    x = torch.from_numpy(rng.normal(size=(300, 1024)) * 2.0 ** rng.choice([-140, -100, -3, 0, 60, 120], (300, 1))).bfloat16()
    w = torch.from_numpy(rng.normal(size=(1024,))).bfloat16()
    w[128:256] = 0
    for eps in (0.0, 1e-5):
        _, code, scale = run_norm(x.cuda(), None, w.cuda(), eps)
        v = x.double().numpy() * w.double().numpy()
        most = np.abs(v).reshape(300, 8, 128).max(axis=2)
        z = v / np.maximum(np.repeat(most, 128, axis=1) / 448, 1e-300)
        # Two roundings of the quotient, 2^-24 each: only values so near a halfway point may go either way.
        low, high = fp8.encode(z * (1 - 2.5 * U)), fp8.encode(z * (1 + 2.5 * U))
        none = (x.double().numpy() == 0).all(axis=1)  # bfloat16 ends at 2^-133: rows of zeros, 0 / 0 with eps 0
        assert 0 < none.sum() < 100
        if eps == 0.0:
            assert (code[none] & 127 == 127).all() and (scale[:, none] == 2.0 ** -126).all()
        ok = (code == low) | (code == high) | ((z == 0) & (code & 127 == 0))
        assert ok[~none | (eps > 0)].all()
        assert (scale[1] == 2.0 ** -126).all()
        assert (low != high).mean() < 1e-3


def test_norm_codes_do_not_depend_on_the_mean():
    """As test_norm_divides_by_the_scale, with rows of ones and twos: 1 / rms is no short number, but
    it divides out of y / s, and the codes are those of the exact halfway values, to the bit."""
    width = 32768
    rng = np.random.default_rng(8)
    s = np.repeat(rng.integers(1 << 14, 1 << 15, width // 128) / 2.0 ** 15, 128)
    halves = (fp8.VALUES[8:126] + fp8.VALUES[9:127]) / 2
    z = rng.choice(halves, width) * rng.choice([-1.0, 1.0], width)
    z[::128] = 448.0
    h = rng.choice([1.0, 2.0], width)
    w = (z * s / h).astype(np.float32)
    assert np.array_equal(w.astype(np.float64) * h, z * s)
    x = torch.from_numpy(np.stack([h, -h, h * 2.0 ** 30, h * 2.0 ** -130])).float().cuda()
    _, code, scale = run_norm(x, None, torch.from_numpy(w).cuda(), 0.0)
    assert np.array_equal(code, fp8.encode(z[None] * np.sign(x.cpu().double().numpy())))
    want = (s[::128] / np.sqrt((h * h).mean()))[:, None]
    assert np.all(np.abs(scale - want) <= 4 * U * want)
