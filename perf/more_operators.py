"""Measured cases of verification on a 4-bit KV cache, through the public entry points.

A case names an operator, a shape and its type:

  rope     sd_qk_norm_rope: norms of queries and keys for each head and the
           position rotation, on a fused projection's output
  append   sd_kv4_append: new key and value rows into paged caches of 4-bit codes
  read     sd_kv4_read: cached keys and values back as rows
  attend   sd_verify_attention_kv4: verification attention over such caches, of a
           draft chain, a candidate tree or single tokens

Layouts (codes are e2m1: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign bit, two to a byte, the
first column in the low half):

  K pool    [pages][Hkv][page/64][4 t][4 g][16 r][D/8]: key 16 t + r, columns g D/4 + 2 b and + 1
  K scales  [pages][Hkv][page/64][D/32][16 r][4 t] exponent bytes, 2^(byte - 127), one for
            each key and 32 columns
  V pool    [pages][Hkv][page/64][D/16][64 n][8]: key n, columns 16 i + 2 b and + 1
  V scales  [pages][Hkv][page/64][64 n] bfloat16, one for each key

A K scale is the smallest 2^e, a V scale the smallest bfloat16, with which no magnitude of its
columns passes 6 codes' units; neither is below 2^-100.

What an append leaves in the pools is returned as their bytes: equal codes are equal values,
and torch has no arithmetic on pairs of 4-bit values.

Lengths are spread between two ends (evenly, or geometrically with "spread": "log") and dealt
to the requests in an order that the seed draws, so a case's work does not depend on the seed.
"""

from __future__ import annotations

import math

import numpy as np
import torch

own = False

BLOCK = 64     # keys of a block
GROUP = 32     # columns of a K scale
LOWEST = -100  # exponent of the smallest scale


def listed():
    return [
        # One interactive session, one token at a time: the shortest call a decoding loop makes.
        dict(name="kv4_decode_single", op="attend", batch=1, gamma=0, hq=32, hkv=8, dim=128, page=64, len_min=1000,
             len_max=1000, spread="even", tree=False),
        # Plain decoding of an 8B-shaped target's pooled clients, a token each.
        dict(name="kv4_decode_pooled", op="attend", batch=32, gamma=0, hq=32, hkv=8, dim=128, page=64, len_min=700,
             len_max=8000, spread="even", tree=False),
        # The largest cache, one draft serving many clients: 64 pooled requests of widely mixed lengths, multi-head.
        dict(name="kv4_pooled", op="attend", batch=64, gamma=4, hq=32, hkv=32, dim=128, page=64, len_min=128,
             len_max=8192, spread="log", tree=False),
        # The most products: a 70B-shaped share with long contexts.
        dict(name="kv4_llama70b_share", op="attend", batch=16, gamma=8, hq=64, hkv=8, dim=128, page=256,
             len_min=16384, len_max=32768, spread="even", tree=False),
        # Candidate trees of 15 nodes, head dimension 64, odd lengths down to a short prompt.
        dict(name="kv4_tree_d64", op="attend", batch=13, gamma=15, hq=24, hkv=8, dim=64, page=128, len_min=37,
             len_max=3001, spread="even", tree=True),
        # What every verification step adds to the pooled caches: the step's five positions of 64 requests.
        dict(name="kv4_append_step", op="append", batch=64, hkv=32, dim=128, page=64, new_min=5, new_max=5, old_min=11,
             old_max=1019, dtype="bf16"),
        # Prompts of very different lengths entering at once.
        dict(name="kv4_append_prompts", op="append", batch=8, hkv=8, dim=128, page=256, new_min=1, new_max=6001,
             old_min=0, old_max=0, dtype="bf16"),
        # The rows of accepted paths, read to be appended again next to the root.
        dict(name="kv4_read_paths", op="read", batch=32, hkv=8, dim=128, page=64, len_min=1, len_max=7, first_min=500,
             first_max=4000, dtype="bf16"),
        # Whole sessions read for a pass that takes caches in bfloat16.
        dict(name="kv4_read_sessions", op="read", batch=8, hkv=8, dim=128, page=256, len_min=1, len_max=9001, first_min=0,
             first_max=0, dtype="bf16"),
        # The queries and keys of a pooled verification step, multi-head, rotated only.
        dict(name="rope_step", op="rope", rows=320, hq=32, hkv=32, dim=128, rotary=128, interleaved=False, norm=False,
             pos=8192, theta=1e4, dtype="bf16"),
        # A long prompt's, normed per head, at far positions.
        dict(name="rope_prompt", op="rope", rows=9001, hq=64, hkv=8, dim=128, rotary=128, interleaved=False, norm=True,
             pos=1000000, theta=5e5, dtype="bf16"),
        # Heads of 64 columns, half of each rotated, neighbours paired, in float32.
        dict(name="rope_partial_f32", op="rope", rows=77, hq=24, hkv=8, dim=64, rotary=32, interleaved=True, norm=True,
             pos=40000, theta=1e4, dtype="f32"),
    ]


# ---- drawn cases ------------------------------------------------------------

def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_once(rng):
    op = rng.choices(["attend", "append", "read", "rope"], [40, 20, 15, 25])[0]
    dim = rng.choice([64, 128, 128])
    if op == "rope":
        return dict(op=op, rows=_log(rng, 1, 9001), hq=rng.choice([1, 7, 8, 24, 32, 64]), hkv=rng.choice([1, 2, 8, 8, 32]),
                    dim=dim, rotary=rng.choice([dim, dim, dim // 2, 16]), interleaved=rng.random() < 0.3,
                    norm=rng.random() < 0.6, pos=_log(rng, 100, 4000000), theta=rng.choice([1e4, 5e5]),
                    dtype=rng.choice(["bf16", "bf16", "f32"]))
    c = dict(op=op, batch=_log(rng, 1, 64), hkv=rng.choice([1, 2, 4, 8, 8, 16, 32]), dim=dim,
             page=rng.choice([64, 64, 128, 256, 1024]))
    if op == "append":
        lo = _log(rng, 1, 300)
        c.update(new_min=lo, new_max=lo + rng.choice([0, _log(rng, 1, 4000)]), old_min=rng.randint(0, 200),
                 dtype=rng.choice(["bf16", "bf16", "f32"]))
        c["old_max"] = c["old_min"] + rng.randint(0, 1500)
        return c
    if op == "read":
        c.update(len_min=_log(rng, 1, 300), first_min=rng.randint(0, 200), dtype=rng.choice(["bf16", "bf16", "f32"]))
        c["len_max"] = c["len_min"] + rng.choice([0, _log(rng, 1, 9000)])
        c["first_max"] = c["first_min"] + rng.randint(0, 1500)
        return c
    c.update(gamma=rng.choice([0, 0, 1, 2, 3, 4, 5, 7, 8, 10, 14, 15]), spread=rng.choice(["even", "log"]))
    c["tree"] = c["gamma"] > 3 and rng.random() < 0.3
    c["hq"] = c["hkv"] * rng.choice([g for g in (1, 1, 2, 3, 4, 5, 8) if g * (c["gamma"] + 1) <= 128])
    c["len_min"] = c["gamma"] + 1 + rng.choice([0, _log(rng, 1, 4096)])
    c["len_max"] = c["len_min"] + _log(rng, 1, 20000)
    return c


def draw(rng):
    most = {"attend": 4.3e8, "append": 1.2e8, "read": 1.8e8, "rope": 3.3e8}
    while True:
        c = _draw_once(rng)
        # Padded to the longest request, the plain attention holds this many key values.
        padded = c["batch"] * c["len_max"] * c["hkv"] * c["dim"] if c["op"] == "attend" else 0
        if work(c)["bytes"] <= most[c["op"]] and padded <= 1.5e9:
            return c


# ---- inputs -----------------------------------------------------------------

def _spread(lo, hi, n, how="even"):
    if n == 1:
        v = np.array([hi])
    elif how == "log":
        v = np.rint(np.exp(np.linspace(math.log(max(lo, 1)), math.log(max(hi, 1)), n)))
    else:
        v = np.rint(np.linspace(lo, hi, n))
    return v.astype(np.int32)


def _ceil(a, b):
    return -(-a // b)


def _pages(rng, kv_len, page, spare=3):
    """A table that scatters every request's pages over a pool, whose size does not depend on
    how the lengths are dealt."""
    need = _ceil(kv_len.astype(np.int64), page)
    n = int(kv_len.astype(np.int64).sum()) // page + len(kv_len) + spare
    ids = rng.permutation(n)[:int(need.sum())].astype(np.int32)
    table = np.zeros((len(kv_len), max(1, int(need.max()))), dtype=np.int32)
    table[np.arange(table.shape[1])[None, :] < need[:, None]] = ids
    return table, n


def _codes(shape, gen):
    """Bytes of two codes of normal values, whose largest in 32 lies near the type's end."""
    n = int(np.prod(shape))
    out = torch.empty((n,), dtype=torch.uint8, device="cuda")
    edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device="cuda")
    for i in range(0, n, 1 << 26):
        m = min(1 << 26, n - i)
        x = torch.randn((m, 2), generator=gen, device="cuda").mul_(2.2)
        c = torch.bucketize(x.abs(), edges, out_int32=True) + (x < 0).int() * 8
        out[i:i + m] = (c[:, 0] + 16 * c[:, 1]).to(torch.uint8)
    return out.view(shape)


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _cache(c, n, gen):
    """A pool of n pages whose keys and values are of magnitude about one."""
    Hkv, D, nb = c["hkv"], c["dim"], c["page"] // BLOCK
    return dict(k=_codes((n, Hkv, nb, 4, 4, 16, D // 8), gen), v=_codes((n, Hkv, nb, D // 16, 64, 8), gen),
                k_scale=torch.randint(125, 128, (n, Hkv, nb, D // GROUP, 16, 4), generator=gen, device="cuda", dtype=torch.uint8),
                v_scale=(torch.rand((n, Hkv, nb, 64), generator=gen, device="cuda") * 0.6 + 0.2).bfloat16())


def _rows(c, total, width, gen):
    """Rows [total][Hkv][D], slices of rows of `width` elements (a fused projection's output);
    magnitudes differ from head to head and, as keys' do, from column to column."""
    x = torch.randn((total, width), generator=gen, device="cuda")
    x = x * torch.exp2(torch.randn((1, width), generator=gen, device="cuda"))
    return x.to(_dtype(c))[:, :c["hkv"] * c["dim"]].unflatten(1, (c["hkv"], c["dim"]))


def prepare(c, seed):
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s = {"case": c}
    if c["op"] == "rope":
        M, D, R, wide = c["rows"], c["dim"], c["rotary"], (c["hq"] + 2 * c["hkv"]) * c["dim"]
        x = torch.randn((M, wide), generator=gen, device="cuda").to(_dtype(c))
        s.update(q=x[:, :c["hq"] * D].unflatten(1, (c["hq"], D)),
                 k=x[:, c["hq"] * D:(c["hq"] + c["hkv"]) * D].unflatten(1, (c["hkv"], D)),
                 positions=torch.randint(0, c["pos"], (M,), generator=gen, device="cuda", dtype=torch.int32),
                 inv_freq=(c["theta"] ** (-torch.arange(0, R, 2, dtype=torch.float64) / R)).float().cuda(), eps=1e-6,
                 q_out=torch.empty((M, c["hq"], D), dtype=_dtype(c), device="cuda"),
                 k_out=torch.empty((M, c["hkv"], D), dtype=_dtype(c), device="cuda"))
        for w in ("q_weight", "k_weight"):
            s[w] = (1 + 0.2 * torch.randn((D,), generator=gen, device="cuda")).to(_dtype(c)) if c["norm"] else None
        return s
    B, Hkv, D, P = c["batch"], c["hkv"], c["dim"], c["page"]
    if c["op"] == "attend":
        G = c["gamma"] + 1
        kv_len = rng.permutation(_spread(c["len_min"], c["len_max"], B, c["spread"]))
        s.update(scale=1.0 / math.sqrt(D), q=torch.randn((B, G, c["hq"], D), generator=gen, device="cuda").bfloat16(),
                 out=torch.empty((B, G, c["hq"], D), dtype=torch.bfloat16, device="cuda"), parent=None)
        if c["tree"]:
            # Every node hangs on one of the few before it, as the layers of a proposal tree do.
            node = np.arange(c["gamma"])[None, :]
            s["parent"] = torch.from_numpy(np.maximum(node - rng.integers(1, 5, (B, c["gamma"])), -1).astype(np.int32)).cuda()
    else:
        ends = ("new_min", "new_max", "old_min", "old_max") if c["op"] == "append" else ("len_min", "len_max", "first_min", "first_max")
        count = rng.permutation(_spread(c[ends[0]], c[ends[1]], B)).astype(np.int32)
        first = rng.permutation(_spread(c[ends[2]], c[ends[3]], B)).astype(np.int32)
        kv_len, T = (first + count).astype(np.int32), int(count.sum())
        s.update(count=count, first=first, off=np.concatenate([[0], np.cumsum(count)[:-1]]).astype(np.int64))
        if c["op"] == "append":
            s.update(k_new=_rows(c, T, 3 * Hkv * D, gen), v_new=_rows(c, T, 3 * Hkv * D, gen))
        else:
            s.update({w: torch.empty((T, Hkv, D), dtype=_dtype(c), device="cuda") for w in ("k_out", "v_out")})
    table, n = _pages(rng, kv_len, P)
    s.update(kv_len=kv_len, table=torch.from_numpy(table).cuda(), **_cache(c, n, gen))
    if own:
        s["plan"] = _plan(s)
    return s


def _plan(s):
    """What a program keeps from step to step: the shape, the cache's handle, a workspace."""
    import paper_2601_21622_amd as sd

    c = s["case"]
    dtype = sd.SD_DTYPE_F32 if c.get("dtype") == "f32" else sd.SD_DTYPE_BF16
    dims = sd.Dims(c["batch"], c.get("gamma", 0), c.get("hq", c["hkv"]), c["hkv"], c["dim"], 128, 1, dtype, 0)
    plan = {"dims": dims, "cache": sd.KV4Cache.of(s["k"], s["v"], s["k_scale"], s["v_scale"], s["table"], c["page"])}
    if c["op"] == "attend":
        n = sd.sd_kv4_workspace_bytes(dims, int(s["kv_len"].max()))
        plan["ws"] = torch.empty((n,), dtype=torch.uint8, device="cuda")
    return plan


def work(c):
    if c["op"] == "rope":
        n, e = float(c["rows"] * (c["hq"] + c["hkv"]) * c["dim"]), 2 if c["dtype"] == "bf16" else 4
        return {"bytes": 2 * e * n + 4 * c["rows"] + 2 * c["rotary"], "flops": (6 if c["norm"] else 3) * n}
    key = c["hkv"] * (c["dim"] + c["dim"] / GROUP + 2)  # bytes of a cached key and its value
    if c["op"] == "attend":
        L = float(_spread(c["len_min"], c["len_max"], c["batch"], c["spread"]).astype(np.int64).sum())
        G, hq, D = c["gamma"] + 1, c["hq"], c["dim"]
        return {"bytes": L * key + 2 * 2 * c["batch"] * G * hq * D, "flops": 4 * L * G * hq * D}
    lo, hi = ("new_min", "new_max") if c["op"] == "append" else ("len_min", "len_max")
    T = float(_spread(c[lo], c[hi], c["batch"]).astype(np.int64).sum())
    e = 2 if c["dtype"] == "bf16" else 4
    return {"bytes": T * (key + 2 * e * c["hkv"] * c["dim"]), "flops": (6 if c["op"] == "append" else 2) * T * c["hkv"] * c["dim"]}


# ---- the operators' plain forms ------------------------------------------------

def _pow2(e):
    """2^e of an integer tensor, -126 <= e <= 127, exactly."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _values(b):
    """The two values of every byte [..., n] as [..., 2 n]."""
    c = torch.stack([b & 15, b >> 4], dim=-1).flatten(-2).int()
    m = c & 7
    x = torch.where(m < 5, m.float() * 0.5, torch.where(m < 7, m.float() - 2, 6.0))
    return torch.where(c > 7, -x, x)


def _keys_of(k, k_scale):
    """Blocks of K [..., 4 t, 4 g, 16 r, D/8] and their scales as float32 [..., 64, D]."""
    n = k.dim() - 4
    x = _values(k).transpose(n + 1, n + 2).flatten(n + 2).flatten(n, n + 1)
    scale = _pow2(k_scale.int() - 127).permute(*range(n), n + 2, n + 1, n).flatten(n, n + 1)
    return x * scale.repeat_interleave(GROUP, n + 1)


def _values_of(v, v_scale):
    """Blocks of V [..., D/16, 64, 8] and their scales as float32 [..., 64, D]."""
    n = v.dim() - 3
    return _values(v).transpose(n, n + 1).flatten(n + 1) * v_scale.float()[..., None]


def _plain_attend(s):
    c = s["case"]
    B, G, Hkv, D, group = c["batch"], c["gamma"] + 1, c["hkv"], c["dim"], c["hq"] // c["hkv"]
    table = s["table"].long()
    kv_len = torch.from_numpy(s["kv_len"]).cuda().long()
    # [B, pages, Hkv, blocks, 64, D] -> [B, Hkv, keys, D]
    k = torch.stack([_keys_of(s["k"][t], s["k_scale"][t]).transpose(0, 1).reshape(Hkv, -1, D) for t in table])
    v = torch.stack([_values_of(s["v"][t], s["v_scale"][t]).transpose(0, 1).reshape(Hkv, -1, D) for t in table])
    q = s["q"].float().view(B, G, Hkv, group, D).transpose(1, 2).reshape(B, Hkv, G * group, D)
    score = torch.matmul(q, k.transpose(2, 3).contiguous()) * s["scale"]
    del k
    key = torch.arange(v.shape[2], device="cuda")
    first = kv_len - G  # keys before the step's positions
    if s["parent"] is None:
        sees = torch.ones((G, G), device="cuda").tril().bool().expand(B, G, G)
    else:
        up = torch.nn.functional.one_hot(s["parent"].long() + 1, G).float()  # node i + 1 -> its parent's position
        up = torch.cat([torch.zeros((B, 1, G), device="cuda"), up], dim=1) + torch.eye(G, device="cuda")
        sees = torch.linalg.matrix_power(up, G) > 0
    tail = key[None, :] - first[:, None]
    seen = torch.gather(sees, 2, tail.clamp(0, G - 1)[:, None, :].expand(B, G, len(key)))
    seen = (tail < 0)[:, None, :] | (seen & (tail < G)[:, None, :])
    score = score.masked_fill(~seen[:, None, :, None, :].expand(B, 1, G, group, len(key)).reshape(B, 1, G * group, -1), -math.inf)
    p = torch.exp(score - score.amax(3, keepdim=True))
    v = v.masked_fill((tail >= G)[:, None, :, None], 0.0)
    o = torch.matmul(p, v) / p.sum(3, keepdim=True)
    return o.view(B, Hkv, G, group, D).transpose(1, 2).reshape(B, G, Hkv * group, D).bfloat16()


def _places(s):
    """Page, block of the page and key of the block for each of the rows, and its row number."""
    count, per = s["count"].astype(np.int64), s["case"]["page"]
    req = np.repeat(np.arange(len(count)), count)
    inside = np.arange(count.sum()) - (np.cumsum(count) - count)[req]
    key = inside + s["first"][req]
    page = s["table"][torch.from_numpy(req).cuda(), torch.from_numpy(key // per).cuda()].long()
    return (page, *(torch.from_numpy(a).cuda() for a in (key % per // BLOCK, key % BLOCK, s["off"][req] + inside)))


def _pack(y, x):
    """Bytes of the codes nearest to y, ties to the even code, with the signs of x."""
    a = y.abs()
    c = ((a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int() + (a > 2.5).int() + (a >= 3.5).int()
         + (a > 5).int() + torch.signbit(x).int() * 8)
    return (c[..., 0::2] + 16 * c[..., 1::2]).to(torch.uint8)


def _plain_append(s):
    page, blk, key, row = _places(s)
    D = s["case"]["dim"]
    x = s["k_new"][row].double().unflatten(2, (D // GROUP, GROUP))        # [T, Hkv, D/32, 32]
    m, e = torch.frexp(x.abs().amax(3))                                    # most = m 2^e, 1/2 <= m < 1
    e = torch.where(m > 0, e - 3 + (m > 0.75).int(), LOWEST).clamp(min=LOWEST)
    codes = _pack(x * torch.exp2(-e.double())[..., None], x).flatten(2).unflatten(2, (4, D // 8))
    s["k"].permute(0, 2, 3, 5, 1, 4, 6)[page, blk, key // 16, key % 16] = codes
    s["k_scale"].permute(0, 2, 5, 4, 1, 3)[page, blk, key // 16, key % 16] = (e + 127).to(torch.uint8)
    x = s["v_new"][row].double()
    most = x.abs().amax(2)
    bits = (most / 6).float().view(torch.int32) & -65536                   # bfloat16 at or next below
    for _ in range(2):
        bits = torch.where(bits.view(torch.float32).double() * 6 < most, bits + 65536, bits)
    scale = bits.view(torch.float32).clamp(min=2.0 ** LOWEST)
    codes = _pack(x / scale.double()[..., None], x).unflatten(2, (D // 16, 8))
    s["v"].permute(0, 2, 4, 1, 3, 5)[page, blk, key] = codes
    s["v_scale"].permute(0, 2, 3, 1)[page, blk, key] = scale.bfloat16()
    return _pools(s)


def _pools(s):
    return {"k": s["k"], "v": s["v"], "k_scale": s["k_scale"].view(torch.float8_e8m0fnu), "v_scale": s["v_scale"]}


def _plain_read(s):
    page, blk, key, row = _places(s)
    D = s["case"]["dim"]
    k = _values(s["k"].permute(0, 2, 3, 5, 1, 4, 6)[page, blk, key // 16, key % 16]).flatten(2)
    ks = _pow2(s["k_scale"].permute(0, 2, 5, 4, 1, 3)[page, blk, key // 16, key % 16].int() - 127)
    v = _values(s["v"].permute(0, 2, 4, 1, 3, 5)[page, blk, key]).flatten(2)
    vs = s["v_scale"].permute(0, 2, 3, 1)[page, blk, key].float()
    s["k_out"][row] = (k * ks.repeat_interleave(GROUP, 2)).to(s["k_out"].dtype)
    s["v_out"][row] = (v * vs[..., None]).to(s["v_out"].dtype)
    return {"k": s["k_out"], "v": s["v_out"]}


def _plain_rope(s):
    c = s["case"]
    R, out = c["rotary"], {}
    angle = s["positions"].double()[:, None] * s["inv_freq"].double()     # far positions pass float32's bits
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    for x, w, name in ((s["q"], s["q_weight"], "q"), (s["k"], s["k_weight"], "k")):
        y = x.float()
        if w is not None:
            y = y * torch.rsqrt(y.square().mean(2, keepdim=True) + s["eps"]) * w.float()
        a, b = (y[..., 0:R:2], y[..., 1:R:2]) if c["interleaved"] else (y[..., :R // 2], y[..., R // 2:R])
        pair = a * cos - b * sin, a * sin + b * cos
        turned = torch.stack(pair, -1).flatten(-2) if c["interleaved"] else torch.cat(pair, -1)
        out[name] = torch.cat([turned, y[..., R:]], -1).to(x.dtype)
    return out


# ---- one pass -------------------------------------------------------------------

def run(s):
    c = s["case"]
    if not own:
        return {"attend": _plain_attend, "append": _plain_append, "read": _plain_read, "rope": _plain_rope}[c["op"]](s)
    import paper_2601_21622_amd as sd

    if c["op"] == "rope":
        sd.sd_qk_norm_rope(s["q"], s["k"], s["positions"], s["inv_freq"], s["q_weight"], s["k_weight"], s["eps"], s["q_out"],
                           s["k_out"], interleaved=c["interleaved"])
        return {"q": s["q_out"], "k": s["k_out"]}
    plan = s["plan"]
    if c["op"] == "attend":
        sd.sd_verify_attention_kv4(plan["dims"], s["q"], plan["cache"], s["kv_len"], s["parent"], s["scale"], s["out"], plan["ws"])
        return s["out"]
    if c["op"] == "append":
        sd.sd_kv4_append(plan["dims"], plan["cache"], s["k_new"], s["v_new"], s["off"], s["count"], s["kv_len"])
        return _pools(s)
    sd.sd_kv4_read(plan["dims"], plan["cache"], s["first"], s["count"], s["off"], s["k_out"], s["v_out"])
    return {"k": s["k_out"], "v": s["v_out"]}


# ---- the operators in 64 bits ----------------------------------------------------

_E2M1 = [0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6]


def _index(D):
    """Byte of a block's K and of its V that holds key n, column d, [64][D] each, and of its K scale."""
    n, d = (torch.from_numpy(a).cuda() for a in np.meshgrid(np.arange(64), np.arange(D), indexing="ij"))
    k = ((n // 16 * 4 + d // (D // 4)) * 16 + n % 16) * (D // 8) + d % (D // 4) // 2
    v = (d // 16 * 64 + n) * 8 + d % 16 // 2
    return k, v, (d // GROUP * 16 + n % 16) * 4 + n // 16, d % 2 * 4


def _session(s, b, h, length):
    """Keys and values 0 .. length - 1 of request b, head h, in float64 [length][D]."""
    D = s["case"]["dim"]
    ki, vi, si, shift = _index(D)
    ids = s["table"][b, :_ceil(length, s["case"]["page"])].long()
    lut = torch.tensor(_E2M1, dtype=torch.float64, device="cuda")
    take = lambda pool, at: pool[ids, h].reshape(-1, 32 * D)[:, at]
    k = lut[((take(s["k"], ki) >> shift) & 15).long()]
    k = k * torch.exp2(s["k_scale"][ids, h].reshape(-1, 2 * D)[:, si].double() - 127)
    v = lut[((take(s["v"], vi) >> shift) & 15).long()] * s["v_scale"][ids, h].reshape(-1, 64, 1).double()
    return k.view(-1, D)[:length], v.view(-1, D)[:length]


def _exact_attend(s):
    c = s["case"]
    G, Hkv, D, group = c["gamma"] + 1, c["hkv"], c["dim"], c["hq"] // c["hkv"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    for b in range(c["batch"]):
        L = int(s["kv_len"][b])
        sees = np.zeros((G, L), dtype=bool)
        sees[:, :L - G] = True
        parent = None if s["parent"] is None else s["parent"][b].cpu().numpy()
        for g in range(G):
            a = g
            while True:
                sees[g, L - G + a] = True
                if a == 0:
                    break
                a = a - 1 if parent is None else int(parent[a - 1]) + 1
        sees = torch.from_numpy(sees).cuda().repeat_interleave(group, 0)
        for h in range(Hkv):
            k, v = _session(s, b, h, L)
            q = s["q"][b, :, h * group:(h + 1) * group].double().reshape(G * group, D)
            w = (q @ k.T * s["scale"]).masked_fill(~sees, -math.inf).softmax(1)
            out[b, :, h * group:(h + 1) * group] = (w @ v).view(G, group, D)
    return out


def _exact_append(s):
    """The scales after the append, key by key of the definition; the bytes have no value of their own."""
    c = s["case"]
    k_scale, v_scale = torch.exp2(s["k_scale"].double() - 127), s["v_scale"].double()
    fine = 2.0 ** -8  # a bfloat16 of [2^e, 2^(e + 1)) is a multiple of 2^(e + 1 - 8)
    for b in range(c["batch"]):
        first, n, off = int(s["first"][b]), int(s["count"][b]), int(s["off"][b])
        for lo in range(first // BLOCK * BLOCK, first + n, BLOCK):
            at = int(s["table"][b, lo // c["page"]]), slice(None), lo % c["page"] // BLOCK
            a, z = max(lo, first), min(lo + BLOCK, first + n)
            key = torch.arange(a - lo, z - lo, device="cuda")
            most = s["k_new"][off + a - first:off + z - first].double().abs().unflatten(2, (-1, GROUP)).amax(3)
            e = torch.ceil(torch.log2(most.clamp(min=1e-300) / 6))
            e = torch.where(torch.exp2(e - 1) * 6 >= most, e - 1, e)
            e = torch.where(torch.exp2(e) * 6 < most, e + 1, e).clamp(min=LOWEST)
            k_scale[at][:, :, key % 16, key // 16] = torch.exp2(e).permute(1, 2, 0)
            need = s["v_new"][off + a - first:off + z - first].double().abs().amax(2).clamp(min=6 * 2.0 ** LOWEST) / 6
            unit = torch.exp2(torch.floor(torch.log2(need)) + 1) * fine
            up = torch.ceil(need / unit) * unit
            up = torch.where((up - unit) * 6 >= need * 6, up - unit, up)
            v_scale[at][:, key] = up.T
    return {"k": None, "v": None, "k_scale": k_scale, "v_scale": v_scale}


def _exact_read(s):
    c = s["case"]
    out = {w: torch.empty(s["k_out"].shape, dtype=torch.float64, device="cuda") for w in ("k", "v")}
    for b in range(c["batch"]):
        first, n, off = int(s["first"][b]), int(s["count"][b]), int(s["off"][b])
        for h in range(c["hkv"]):
            k, v = _session(s, b, h, first + n)
            out["k"][off:off + n, h], out["v"][off:off + n, h] = k[first:], v[first:]
    return out


def _exact_rope(s):
    c, out = s["case"], {}
    half = c["rotary"] // 2
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                       s["positions"].double()[:, None] * s["inv_freq"].double())[:, None]
    for name in ("q", "k"):
        y = s[name].double()
        if s[name + "_weight"] is not None:
            y = s[name + "_weight"].double() * y / torch.sqrt((y * y).sum(2, keepdim=True) / c["dim"] + s["eps"])
        first = torch.arange(half, device="cuda") * (2 if c["interleaved"] else 1)
        second = first + (1 if c["interleaved"] else half)
        z = torch.complex(y[..., first], y[..., second]) * turn
        y = y.clone()
        y[..., first], y[..., second] = z.real, z.imag
        out[name] = y
    return out


def exact(c, seed):
    s = prepare(c, seed)
    return {"attend": _exact_attend, "append": _exact_append, "read": _exact_read, "rope": _exact_rope}[c["op"]](s)
