"""Norms and rotation of queries and keys on the GPU against the float64 oracle."""

import numpy as np
import pytest
import torch

import paper_2601_21622_amd as sd
from oracle import fp4

pytestmark = pytest.mark.gpu

STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def make(rng, rows, heads, dim, dtype, wide, size=1.0):
    x = torch.from_numpy(rng.normal(size=(rows, wide)) * size).to(dtype)
    return x[:, :heads * dim].unflatten(1, (heads, dim)), x.cuda()[:, :heads * dim].unflatten(1, (heads, dim))


def check(got, x, w, pos, f, eps, interleaved, what):
    """Bound: half a step of the type for the output.  Before it float32: the sum of D squares and its root
    (D / 2 steps at most in a tree of sums, 8 + log2 D here), the factors 1/rms and weight, the cosine and sine
    (an absolute 2^-22, from an angle that is exact to 2^-25 revolutions), two products and a sum: under 40 half steps of
    the pair's magnitude."""
    ref, mag = fp4.norm_rope(x, w, pos, f, eps, interleaved)
    err = np.abs(got.double().cpu().numpy() - ref)
    bad = ~(err <= STEP[got.dtype] * np.abs(ref) + 40 * 2.0 ** -24 * mag)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size}, worst {np.nanmax(err / (mag + 1e-300))}"


CASES = {
    # name: rows, hq, hkv, dim, rotary, interleaved, norm (q, k), dtype, extra columns
    "one_row": (1, 1, 1, 128, 128, False, (True, True), torch.bfloat16, 0),
    "step": (30, 32, 32, 128, 128, False, (False, False), torch.bfloat16, 4096),
    "gqa": (7, 8, 2, 128, 128, False, (True, True), torch.bfloat16, 256),
    "d64": (13, 7, 3, 64, 64, False, (True, True), torch.float32, 8),
    "partial": (9, 5, 1, 128, 64, False, (True, False), torch.float32, 0),
    "partial16": (9, 24, 8, 64, 16, False, (False, True), torch.bfloat16, 0),
    "partial48": (5, 3, 2, 64, 48, False, (True, True), torch.float32, 0),
    "interleaved": (17, 8, 8, 128, 128, True, (True, True), torch.bfloat16, 0),
    "interleaved_partial": (17, 9, 2, 64, 32, True, (True, True), torch.float32, 16),
    "interleaved_d64": (3, 64, 8, 64, 64, True, (False, False), torch.float32, 0),
    "many_rows": (3001, 3, 1, 64, 64, False, (True, True), torch.bfloat16, 0),
    "many_heads": (2, 300, 100, 128, 112, False, (True, True), torch.bfloat16, 0),
}


@pytest.mark.parametrize("name", CASES)
@pytest.mark.parametrize("place", ["apart", "in place", "in the rows"])
def test_norm_rope(name, place):
    rows, hq, hkv, dim, rotary, inter, norm, dtype, extra = CASES[name]
    rng = np.random.default_rng(len(name))
    q, qd = make(rng, rows, hq, dim, dtype, hq * dim + extra)
    k, kd = make(rng, rows, hkv, dim, dtype, hkv * dim + extra)
    w = [torch.from_numpy(1 + 0.3 * rng.normal(size=dim)).to(dtype) if n else None for n in norm]
    pos = rng.integers(0, 5000, rows).astype(np.int32)
    pos[:1] = 0
    f = (1e4 ** (-np.arange(rotary // 2) / (rotary // 2))).astype(np.float32)
    if place == "apart":
        qo, ko = torch.full((rows, hq, dim), np.nan, dtype=dtype, device="cuda"), torch.full((rows, hkv, dim), np.nan, dtype=dtype, device="cuda")
    elif place == "in place":
        qo, ko = qd, kd
    else:
        full = torch.full((rows, (hq + hkv) * dim + 8), 7.0, dtype=dtype, device="cuda")
        qo, ko = full[:, :hq * dim].unflatten(1, (hq, dim)), full[:, hq * dim:-8].unflatten(1, (hkv, dim))
    dev = lambda t: None if t is None else t.cuda()
    sd.sd_qk_norm_rope(qd, kd, torch.from_numpy(pos).cuda(), torch.from_numpy(f).cuda(), dev(w[0]), dev(w[1]), 1e-6, qo, ko, inter)
    torch.cuda.synchronize()
    for got, x, weight in ((qo, q, w[0]), (ko, k, w[1])):
        check(got, x.double().numpy(), None if weight is None else weight.double().numpy(), pos, f, 1e-6, inter, name)
    if place == "in the rows":
        assert (full[:, -8:] == 7).all()


def test_far_and_negative_positions():
    """Angles of hundreds of millions of radians, the ends of int32, and positions below zero."""
    rng = np.random.default_rng(1)
    pos = np.array([0, 1, -1, 131072, 10 ** 6, 2 ** 24 + 1, 2 ** 31 - 1, -2 ** 31, 10 ** 9 + 7], dtype=np.int32)
    f = (5e5 ** (-np.arange(64) / 64)).astype(np.float32)
    q, qd = make(rng, len(pos), 2, 128, torch.float32, 256)
    out = [torch.empty_like(qd) for _ in range(2)]
    sd.sd_qk_norm_rope(qd, qd, torch.from_numpy(pos).cuda(), torch.from_numpy(f).cuda(), None, None, 0.0, *out)
    torch.cuda.synchronize()
    # The float64 product of angles below 2^31 is exact to 2^-22, on both sides: four half steps of float32 more.
    ref, mag = fp4.norm_rope(q.double().numpy(), None, pos, f, 0.0, False)
    for o in out:
        assert (np.abs(o.double().cpu().numpy() - ref) <= 2.0 ** -24 * np.abs(ref) + (40 * 2.0 ** -24 + 2.0 ** -21) * mag).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("size", [2.0 ** -70, 2.0 ** -40, 1e-12, 1e12, 2.0 ** 60, 2.0 ** 125])
def test_norm_of_large_and_small_rows(size, dtype):
    """Rows whose squares leave float32's range are normed alike, beside ordinary ones; zeros with
    eps give zeros, without NaN; a NaN or an infinity makes its head NaN (of an infinity, finite columns 0 or NaN)."""
    rng = np.random.default_rng(2)
    q, qd = make(rng, 12, 4, 128, dtype, 512, size)
    k, kd = make(rng, 12, 4, 128, dtype, 512)
    w = torch.from_numpy(1 + 0.1 * rng.normal(size=128)).to(dtype)
    pos, f = np.arange(12, dtype=np.int32), (1e4 ** (-np.arange(64) / 64)).astype(np.float32)
    out = [torch.empty_like(qd) for _ in range(2)]
    run = lambda eps: sd.sd_qk_norm_rope(qd, kd, torch.from_numpy(pos).cuda(), torch.from_numpy(f).cuda(), w.cuda(), w.cuda(), eps, *out)
    run(0.0)
    torch.cuda.synchronize()
    check(out[0], q.double().numpy(), w.double().numpy(), pos, f, 0.0, False, "q")
    check(out[1], k.double().numpy(), w.double().numpy(), pos, f, 0.0, False, "k")
    qd.zero_()
    qd[3, 1, 5], qd[4, 2, 7] = float("nan"), float("inf")
    run(1e-6)
    a = out[0].clone()
    run(0.0)
    torch.cuda.synchronize()
    plain = torch.ones(12, 4, dtype=torch.bool)
    plain[3, 1] = plain[4, 2] = False
    assert (a.cpu()[plain] == 0).all() and torch.isnan(out[0].cpu()[plain]).all()
    assert torch.isnan(a[3, 1]).all() and torch.isnan(a[4, 2, [7, 71]]).all()


def test_other_stream_and_graph():
    rng = np.random.default_rng(3)
    q, qd = make(rng, 20, 8, 128, torch.bfloat16, 1024)
    k, kd = make(rng, 20, 2, 128, torch.bfloat16, 256)
    pos = torch.arange(20, dtype=torch.int32, device="cuda")
    f = (1e4 ** (-np.arange(64) / 64)).astype(np.float32)
    fd = torch.from_numpy(f).cuda()
    out = [torch.empty_like(qd), torch.empty_like(kd)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    sd.sd_qk_norm_rope(qd, kd, pos, fd, None, None, 0.0, *out, stream=side)
    torch.cuda.synchronize()
    check(out[0], q.double().numpy(), None, np.arange(20), f, 0.0, False, "stream")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sd.sd_qk_norm_rope(qd, kd, pos, fd, None, None, 0.0, *out)
    for i in range(3):
        pos.fill_(100 * i)
        graph.replay()
        torch.cuda.synchronize()
        check(out[1], k.double().numpy(), None, np.full(20, 100 * i), f, 0.0, False, f"replay {i}")


def test_binding_refuses():
    t = torch.zeros((4, 2, 64), dtype=torch.bfloat16, device="cuda")
    pos, f = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.ones(32, device="cuda")
    ok = [t, t, pos, f, None, None, 1e-6, t.clone(), t.clone()]
    sd.sd_qk_norm_rope(*ok)
    for i, bad in ((0, t.half()), (0, t[:, :, :32]), (0, t.transpose(0, 1)), (1, t.float()), (1, t[:3]), (2, pos[:3]), (2, pos.long()),
                   (3, f.double()), (4, t[0, 0, :32]), (4, torch.zeros(64, device="cuda")), (7, t[:, :1]), (8, t[:3])):
        args = list(ok)
        args[i] = bad
        with pytest.raises(ValueError):
            sd.sd_qk_norm_rope(*args)
    for i, bad in ((3, f[:12].contiguous()), (3, torch.ones(64, device="cuda")), (6, -1.0)):
        args = list(ok)
        args[i] = bad
        with pytest.raises(sd.SdError):
            sd.sd_qk_norm_rope(*args)
    none = t[:0]
    sd.sd_qk_norm_rope(none, none, pos[:0], f, None, None, 1e-6, none, none)  # no rows
