"""The operators of the 8-bit serving path as measurable cases: a plain torch form of each, and the library's call.

Four operators that one decoding or prefill step of a language model with 8-bit weights and an 8-bit KV cache runs
in turn (E4M3 values, FP32 scales):

* ``quantize``  BF16 rows to E4M3 with one power-of-two scale per 1 x 128 (activations) or 128 x 128 (weights) block;
* ``gemm``      C = (A * scale_a) (B * scale_b)^T for E4M3 A [M, K] and B [N, K] with those scales, BF16 result;
* ``append``    queries and keys rotated by their positions, keys and values written into a paged cache (BF16, or E4M3
                with one scale per cache block and KV head);
* ``decode``    one query token per sequence attends to an E4M3 paged cache.

``own`` false: elementary torch operations in FP32; true: the calls a user of the library makes.
"""
import math

import numpy as np
import torch

own = False

BLOCK = 128      # elements of K per scale
F8 = torch.float8_e4m3fn
F8_MAX = 448.0
MIN_EXP, MAX_EXP = -64, 127


def listed():
    return [
        # activations of a decoding batch of 16 tokens on their way into an 8-bit product (a launch's latency)
        {"name": "quantize_16x4096", "op": "quantize", "m": 16, "k": 4096, "block_rows": 1},
        # activations of an 8192-token prefill in front of the down projection of a 28672-wide MLP
        {"name": "quantize_8192x28672", "op": "quantize", "m": 8192, "k": 28672, "block_rows": 1},
        # next-token product with the up projection's weights: the weights stream once
        {"name": "gemm_16x28672x4096", "op": "gemm", "m": 16, "n": 28672, "k": 4096},
        # next-token product with a long K (down projection)
        {"name": "gemm_16x4096x28672", "op": "gemm", "m": 16, "n": 4096, "k": 28672},
        # a ragged chunk of prefill: no size is a multiple of a tile, K ends inside a scale block
        {"name": "gemm_777x5000x4200", "op": "gemm", "m": 777, "n": 5000, "k": 4200},
        # prefill through the up projection
        {"name": "gemm_8192x28672x4096", "op": "gemm", "m": 8192, "n": 28672, "k": 4096},
        # one new token for each of 32 running sequences, BF16 cache
        {"name": "append_bf16_s32_decode", "op": "append", "cache": "bf16", "seqs": 32, "new_lo": 1, "new_hi": 1, "ctx_lo": 2048, "ctx_hi": 4096,
         "heads": 32, "kv_heads": 4, "d": 128, "rot": 128, "interleaved": False, "block": 16},
        # a batch of prompts of 500 to 1500 tokens, BF16 cache
        {"name": "append_bf16_s8_prefill", "op": "append", "cache": "bf16", "seqs": 8, "new_lo": 500, "new_hi": 1500, "ctx_lo": 0, "ctx_hi": 0,
         "heads": 32, "kv_heads": 8, "d": 128, "rot": 128, "interleaved": False, "block": 16},
        # one new token for each of 32 running sequences, 8-bit cache: most fall into a block that holds tokens already
        {"name": "append_f8_s32_decode", "op": "append", "cache": "f8", "seqs": 32, "new_lo": 1, "new_hi": 1, "ctx_lo": 2048, "ctx_hi": 4096,
         "heads": 32, "kv_heads": 4, "d": 128, "rot": 128, "interleaved": False, "block": 16},
        # chunked prefill into an 8-bit cache: every chunk begins and ends inside a block; half of each head is rotated
        {"name": "append_f8_s8_chunks", "op": "append", "cache": "f8", "seqs": 8, "new_lo": 500, "new_hi": 1500, "ctx_lo": 100, "ctx_hi": 3000,
         "heads": 32, "kv_heads": 8, "d": 128, "rot": 64, "interleaved": True, "block": 16},
        # a decoding batch with grouped heads
        {"name": "decode_s32h32kv4d128_len2k-4k", "op": "decode", "seqs": 32, "lo": 2048, "hi": 4096, "heads": 32, "kv_heads": 4, "d": 128, "block": 16},
        # two long sequences, one query head per KV head
        {"name": "decode_s2h8d128_len32k", "op": "decode", "seqs": 2, "lo": 30000, "hi": 32768, "heads": 8, "kv_heads": 8, "d": 128, "block": 16},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["quantize", "gemm", "gemm", "append", "append", "decode", "decode"])
    if op == "quantize":
        return {"op": op, "m": _log(rng, 1, 8192), "k": _log(rng, 40, 28672), "block_rows": rng.choice([1, 1, BLOCK])}
    if op == "gemm":
        most = 8192 * 28672 * 4096
        m, n, k = _log(rng, 1, 8192), _log(rng, 40, 28672), _log(rng, 40, 28672)
        while m * n * k > most:
            m = max(1, m // 2)
        return {"op": op, "m": m, "n": n, "k": k}
    d = rng.choice([64, 128])
    kv = rng.choice([1, 2, 4, 8])
    heads = kv * rng.choice([1, 2, 4, 8])
    block = rng.choice([8, 16, 32])
    if op == "append":
        seqs = _log(rng, 1, 64)
        if rng.random() < 0.4:
            lo, hi = 1, 1
        else:
            hi = _log(rng, 2, max(2, 8192 // seqs))
            lo = rng.randint(0, hi)
        ctx_hi = _log(rng, 1, 4096) if rng.random() < 0.8 else 0
        return {"op": op, "cache": rng.choice(["bf16", "f8"]), "seqs": seqs, "new_lo": lo, "new_hi": hi, "ctx_lo": ctx_hi // 3, "ctx_hi": ctx_hi, "heads": heads,
                "kv_heads": kv, "d": d, "rot": rng.choice([d, d, d // 2, 16]), "interleaved": rng.random() < 0.5, "block": block}
    hi = _log(rng, 1, 32768)
    seqs = _log(rng, 1, max(1, min(200, 1048576 // (hi * kv))))
    return {"op": op, "seqs": seqs, "lo": rng.choice([0, hi // 2, hi]), "hi": hi, "heads": heads, "kv_heads": kv, "d": d, "block": block}


def _up(x, m):
    return (x + m - 1) // m * m


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _ints(seed, salt, lo, hi, n):
    return np.random.RandomState((int(seed) * 131 + salt) % (1 << 31)).randint(lo, hi + 1, n).astype(np.int64)


def _append_lengths(c):
    """New and earlier tokens of each sequence: they set the outputs' shapes, so they go by the case alone."""
    new, ctx = _ints(c["seqs"], 1, c["new_lo"], c["new_hi"], c["seqs"]), _ints(c["seqs"], 2, c["ctx_lo"], c["ctx_hi"], c["seqs"])
    new[0] = max(1, new[0])
    return new, ctx


def _dev32(a):
    return torch.from_numpy(np.ascontiguousarray(a).astype(np.int32)).cuda()


def _paged(c, seed, total_lens):
    """A block table whose sequences' blocks lie scattered over the pool (unused entries: -1), and the pool's size."""
    bs = c["block"]
    per = (total_lens + bs - 1) // bs
    blocks = int(per.sum()) + 3
    order = np.random.RandomState((int(seed) * 7919 + 13) % (1 << 31)).permutation(blocks)
    width = max(1, int(per.max()) if len(per) else 1)
    at = np.concatenate([[0], np.cumsum(per)])[:-1, None] + np.arange(width)[None, :]
    table = np.where(np.arange(width)[None, :] < per[:, None], order[np.minimum(at, blocks - 1)], -1)
    return table, blocks


def _filled_cache(c, blocks, g):
    """An E4M3 cache as earlier appends leave it: every block uses its scale's range, and the scales differ."""
    shape = (blocks, c["kv_heads"], c["block"], c["d"])
    scale = torch.exp2(torch.randint(-8, -5, shape[:2], generator=g, device="cuda").float())
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)
    q = (x.float() / scale[:, :, None, None]).clamp_(-F8_MAX, F8_MAX).to(F8)
    return q, scale


def prepare(case, seed):
    c, g = case, _gen(seed)
    if c["op"] == "quantize":
        x = torch.randn(c["m"], _up(c["k"], 8), generator=g, device="cuda", dtype=torch.bfloat16)
        x *= torch.exp2(torch.randint(-6, 3, (c["m"], 1), generator=g, device="cuda").to(torch.bfloat16))  # rows of different size
        x[:, c["k"] // 3] *= 50.0                                                                             # an outlier channel
        return {"case": c, "x": x[:, : c["k"]]}
    if c["op"] == "gemm":
        m, n, k, kb = c["m"], c["n"], c["k"], _up(c["k"], BLOCK) // BLOCK
        a = (torch.randn(m, _up(k, 16), generator=g, device="cuda", dtype=torch.bfloat16) * 100).to(F8)[:, :k]
        b = (torch.randn(n, _up(k, 16), generator=g, device="cuda", dtype=torch.bfloat16) * 100).to(F8)[:, :k]
        sa = torch.exp2(torch.randint(-9, -5, (kb, m), generator=g, device="cuda").float())                  # as the quantiser gives them
        sb = torch.rand(_up(n, BLOCK) // BLOCK, kb, generator=g, device="cuda") * 2e-4 + 1e-5                 # a checkpoint's, any value
        return {"case": c, "a": a, "b": b, "sa": sa, "sb": sb}
    if c["op"] == "append":
        S, H, Hk, D, R = c["seqs"], c["heads"], c["kv_heads"], c["d"], c["rot"]
        new, ctx = _append_lengths(c)
        table, blocks = _paged(c, seed, new + ctx)
        T = int(new.sum())
        qkv = torch.randn(T, (H + 2 * Hk) * D, generator=g, device="cuda", dtype=torch.bfloat16)
        top = int((new + ctx).max())
        ang = torch.arange(top, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, R, 2, device="cuda", dtype=torch.float64) / R)
        s = {"case": c, "q": qkv[:, : H * D].view(T, H, D), "k": qkv[:, H * D: (H + Hk) * D].view(T, Hk, D), "v": qkv[:, (H + Hk) * D:].view(T, Hk, D),
             "cos": torch.cos(ang).float(), "sin": torch.sin(ang).float(), "cu": _dev32(np.concatenate([[0], np.cumsum(new)])), "ctx": _dev32(ctx),
             "table": _dev32(table)}
        if c["cache"] == "f8":
            (s["kc"], s["ks"]), (s["vc"], s["vs"]) = _filled_cache(c, blocks, g), _filled_cache(c, blocks, g)
        else:
            shape = (blocks, Hk, c["block"], D)
            s["kc"], s["vc"] = (torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2))
        return s
    lens = _ints(seed, 3, c["lo"], c["hi"], c["seqs"])
    table, blocks = _paged(c, seed, lens)
    s = {"case": c, "table": _dev32(table), "lens": _dev32(lens), "scale": float(np.float32(1.0 / math.sqrt(c["d"])))}
    s["q"] = torch.randn(c["seqs"], c["heads"], c["d"], generator=g, device="cuda", dtype=torch.bfloat16)
    (s["kc"], s["ks"]), (s["vc"], s["vs"]) = _filled_cache(c, blocks, g), _filled_cache(c, blocks, g)
    s["ws"] = torch.empty(32 << 20, dtype=torch.uint8, device="cuda")  # scratch that a serving loop keeps
    return s


# ---------------------------------------------------------------- plain forms

def _pow2_scale(amax):
    """The smallest power of two 2^e with amax <= 448 * 2^e, -64 <= e (also for amax = 0)."""
    m, e = torch.frexp(amax)
    e = torch.where(amax > 0, e - 9 + (m > 0.875), torch.full_like(e, MIN_EXP)).clamp(MIN_EXP, MAX_EXP)
    return torch.ldexp(torch.ones_like(amax), e)


def _finite_abs(x):
    return torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x))


def _to_f8(x, scale):
    return (x * (1.0 / scale)).clamp(-F8_MAX, F8_MAX).to(F8)


def _plain_quantize(s):
    x, rows = s["x"].float(), s["case"]["block_rows"]
    m, k = x.shape
    mp, kp = _up(m, rows), _up(k, BLOCK)
    p = x.new_zeros(mp, kp)
    p[:m, :k] = x
    p = p.view(mp // rows, rows, kp // BLOCK, BLOCK)
    scale = _pow2_scale(_finite_abs(p).amax((1, 3)))
    q = _to_f8(p, scale[:, None, :, None]).view(mp, kp)[:m, :k]
    return q, (scale.t().contiguous() if rows == 1 else scale)


def _plain_gemm(s):
    k = s["case"]["k"]
    a = s["a"].float() * s["sa"].t().repeat_interleave(BLOCK, 1)[:, :k]
    b = s["b"].float() * s["sb"].repeat_interleave(BLOCK, 0)[: s["case"]["n"]].repeat_interleave(BLOCK, 1)[:, :k]
    return (a @ b.t()).to(torch.bfloat16)


def _rotated(x, cos, sin, interleaved):
    """x [T, heads, D] FP32 with the first 2 * cos.shape[1] elements of each head rotated in pairs."""
    h = cos.shape[1]
    c, s = cos[:, None, :], sin[:, None, :]
    r, rest = x[..., : 2 * h], x[..., 2 * h:]
    if interleaved:
        a, b = r[..., 0::2], r[..., 1::2]
        return torch.cat([torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2), rest], -1)
    a, b = r[..., :h], r[..., h:]
    return torch.cat([a * c - b * s, b * c + a * s, rest], -1)


def _plain_append(s):
    c, bs = s["case"], s["case"]["block"]
    T = s["q"].shape[0]
    t = torch.arange(T, device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(s["cu"], t, right=True) - 1
    pos = (t - s["cu"][seq] + s["ctx"][seq]).long()
    blk, off = s["table"][seq, pos // bs].long(), pos % bs
    cos, sin = s["cos"][pos], s["sin"][pos]
    q = _rotated(s["q"].float(), cos, sin, c["interleaved"]).to(torch.bfloat16)
    k, v = _rotated(s["k"].float(), cos, sin, c["interleaved"]), s["v"].float()
    if c["cache"] == "bf16":
        s["kc"][blk, :, off] = k.to(torch.bfloat16)
        s["vc"][blk, :, off] = v.to(torch.bfloat16)
        return q, s["kc"], s["vc"]
    ctx, new = s["ctx"].long(), (s["cu"][1:] - s["cu"][:-1]).long()
    part = ((ctx % bs > 0) & (new > 0)).nonzero()[:, 0]  # sequences whose first new token falls into a block that holds tokens
    pblk, held = s["table"][part, ctx[part] // bs].long(), ctx[part] % bs
    _append_f8(k, s["kc"], s["ks"], blk, off, pblk, held)
    _append_f8(v, s["vc"], s["vs"], blk, off, pblk, held)
    return q, s["kc"], s["ks"], s["vc"], s["vs"]


def _append_f8(x, cache, scale, blk, off, pblk, held):
    """x [T, heads, D] into cache[blk, :, off]; the blocks pblk hold `held` tokens that take over a larger scale."""
    top = torch.zeros_like(scale).index_reduce_(0, blk, _finite_abs(x).amax(-1), "amax")
    fresh = _pow2_scale(top)
    old = scale[pblk]
    larger = torch.maximum(old, fresh[pblk])
    rows = cache[pblk]
    moved = (rows.float() * (old / larger)[:, :, None, None]).clamp(-F8_MAX, F8_MAX).to(F8)
    keep = torch.arange(cache.shape[2], device="cuda")[None, None, :, None] < held[:, None, None, None]
    bits = cache.view(torch.uint8)
    bits[pblk] = torch.where(keep, moved.view(torch.uint8), rows.view(torch.uint8))
    scale[blk] = fresh[blk]
    scale[pblk] = larger
    bits[blk, :, off] = _to_f8(x, scale[blk][..., None]).view(torch.uint8)


def _plain_decode(s):
    c, bs = s["case"], s["case"]["block"]
    S, H, Hk, D = c["seqs"], c["heads"], c["kv_heads"], c["d"]
    phys = s["table"].long().clamp_min(0)
    n = phys.shape[1] * bs

    def gathered(cache, scale):  # [S, Hk, n, D]
        return (cache[phys].float() * scale[phys][..., None, None]).permute(0, 2, 1, 3, 4).reshape(S, Hk, n, D)

    seen = torch.arange(n, device="cuda")[None, :] < s["lens"][:, None]
    k, v = gathered(s["kc"], s["ks"]), gathered(s["vc"], s["vs"])
    sc = torch.matmul(s["q"].float().view(S, Hk, H // Hk, D) * s["scale"], k.transpose(2, 3))
    sc = torch.where(seen[:, None, None, :], sc, torch.full_like(sc, -math.inf))
    top = sc.amax(-1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, torch.zeros_like(top))
    p = torch.exp(sc - top)
    l = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(l > 0, l, torch.ones_like(l))
    return o.view(S, H, D).to(torch.bfloat16), (top + torch.log(l)).view(S, H)


def run(state):
    s, c = state, state["case"]
    if not own:
        return {"quantize": _plain_quantize, "gemm": _plain_gemm, "append": _plain_append, "decode": _plain_decode}[c["op"]](s)
    import paper_2503_14985_b200 as mlt
    if c["op"] == "quantize":
        return mlt.quantize_f8(s["x"], block_rows=c["block_rows"])
    if c["op"] == "gemm":
        return mlt.gemm_f8(s["a"], s["sa"], s["b"], s["sb"])
    if c["op"] == "append":
        if c["cache"] == "bf16":
            q = mlt.kv_append(s["q"], s["k"], s["v"], s["cos"], s["sin"], s["cu"], s["ctx"], s["table"], s["kc"], s["vc"], interleaved=c["interleaved"])
            return q, s["kc"], s["vc"]
        q = mlt.kv_append_f8(s["q"], s["k"], s["v"], s["cos"], s["sin"], s["cu"], s["ctx"], s["table"], s["kc"], s["vc"], s["ks"], s["vs"],
                             interleaved=c["interleaved"])
        return q, s["kc"], s["ks"], s["vc"], s["vs"]
    return mlt.paged_attn_decode_f8(s["q"], s["kc"], s["vc"], s["ks"], s["vs"], s["table"], s["lens"], scale=s["scale"], workspace=s["ws"])


def work(case):
    c = case
    if c["op"] == "quantize":
        blocks = -(-c["m"] // c["block_rows"]) * -(-c["k"] // BLOCK)
        return {"bytes": 3.0 * c["m"] * c["k"] + 4.0 * blocks, "flops": 2.0 * c["m"] * c["k"]}
    if c["op"] == "gemm":
        m, n, k, kb = c["m"], c["n"], c["k"], -(-c["k"] // BLOCK)
        return {"bytes": float(m * k + n * k + 2 * m * n + 4 * kb * (m + -(-n // BLOCK))), "flops": 2.0 * m * n * k}
    if c["op"] == "append":
        tokens = float(_append_lengths(c)[0].sum())
        H, Hk, D = c["heads"], c["kv_heads"], c["d"]
        wide = 1 if c["cache"] == "f8" else 2
        return {"bytes": tokens * (4.0 * H * D + 4.0 * Hk * D + 2.0 * wide * Hk * D + 4.0 * c["rot"]), "flops": tokens * 3.0 * c["rot"] * (H + Hk)}
    tokens = c["seqs"] * (c["lo"] + c["hi"]) / 2.0
    H, Hk, D = c["heads"], c["kv_heads"], c["d"]
    return {"bytes": tokens * Hk * (2.0 * D + 8.0 / c["block"]) + c["seqs"] * H * (4.0 * D + 4.0), "flops": 4.0 * tokens * H * D}


# ---------------------------------------------------------------- the definitions, in 64 bits

_E4M3 = None


def _nearest_f8(x):
    """64-bit values rounded to the nearest E4M3 value (ties to the even code), by a search in the table of values."""
    global _E4M3
    if _E4M3 is None:
        code = torch.arange(127, dtype=torch.float64)
        e, f = torch.div(code, 8, rounding_mode="floor"), code % 8
        _E4M3 = torch.where(e > 0, torch.exp2(e - 7) * (1 + f / 8), f * 2.0 ** -9).cuda()
    mag = x.abs().clamp(max=F8_MAX).contiguous()
    hi = torch.searchsorted(_E4M3, mag).clamp(max=126)
    lo = (hi - 1).clamp_min(0)
    up, down = _E4M3[hi] - mag, mag - _E4M3[lo]
    pick = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return torch.copysign(_E4M3[pick], x)


def _exact_scale(amax):
    """2^ceil(log2(amax / 448)), checked against its neighbours because a logarithm is rounded."""
    e = torch.ceil(torch.log2(amax.clamp_min(1e-300) / F8_MAX))
    e = torch.where(amax <= F8_MAX * torch.exp2(e - 1), e - 1, e)
    e = torch.where(amax > F8_MAX * torch.exp2(e), e + 1, e)
    return torch.exp2(e.clamp(MIN_EXP, MAX_EXP))


def _exact_append(s):
    c, bs = s["case"], s["case"]["block"]
    cu, ctx, table = (s[n].cpu().numpy() for n in ("cu", "ctx", "table"))
    h = s["cos"].shape[1]
    q, k, v = (s[n].double() for n in ("q", "k", "v"))
    cos, sin = s["cos"].double(), s["sin"].double()
    rot = []
    for i in range(c["seqs"]):
        rot += list(range(int(ctx[i]), int(ctx[i]) + int(cu[i + 1] - cu[i])))
    pos = torch.tensor(rot, device="cuda")
    turn = torch.complex(cos[pos], sin[pos])[:, None, :]
    for x in (q, k):
        first, second = (slice(0, 2 * h, 2), slice(1, 2 * h, 2)) if c["interleaved"] else (slice(0, h), slice(h, 2 * h))
        z = torch.complex(x[..., first], x[..., second]) * turn
        x[..., first], x[..., second] = z.real, z.imag
    if c["cache"] == "bf16":
        kc, vc = s["kc"].double(), s["vc"].double()
        for i in range(c["seqs"]):
            for b in range(int(ctx[i]) // bs, (int(ctx[i]) + int(cu[i + 1] - cu[i]) + bs - 1) // bs):
                p0, p1 = max(b * bs, int(ctx[i])), min((b + 1) * bs, int(ctx[i] + cu[i + 1] - cu[i]))
                t0 = int(cu[i]) + p0 - int(ctx[i])
                if p1 > p0:
                    for cache, x in ((kc, k), (vc, v)):
                        cache[int(table[i, b]), :, p0 - b * bs: p1 - b * bs] = x[t0: t0 + p1 - p0].transpose(0, 1)
        return q, kc, vc
    out = [q]
    for x, cache, scale in ((k, s["kc"].double(), s["ks"].double()), (v, s["vc"].double(), s["vs"].double())):
        for i in range(c["seqs"]):
            n = int(cu[i + 1] - cu[i])
            for b in range(int(ctx[i]) // bs, (int(ctx[i]) + n + bs - 1) // bs):
                p0, p1 = max(b * bs, int(ctx[i])), min((b + 1) * bs, int(ctx[i]) + n)
                if p1 <= p0:
                    continue
                t0, blk = int(cu[i]) + p0 - int(ctx[i]), int(table[i, b])
                rows = x[t0: t0 + p1 - p0].transpose(0, 1)  # [heads, tokens, D]
                want = _exact_scale(rows.abs().amax((1, 2)))
                if p0 > b * bs:
                    was = scale[blk].clone()
                    want = torch.maximum(was, want)
                    cache[blk, :, : p0 - b * bs] = _nearest_f8(cache[blk, :, : p0 - b * bs] * (was / want)[:, None, None])
                scale[blk] = want
                cache[blk, :, p0 - b * bs: p1 - b * bs] = _nearest_f8(rows / want[:, None, None])
        out += [cache, scale]
    return tuple(out)


def exact(case, seed):
    global own
    was, own = own, False
    s = prepare(case, seed)
    own = was
    c = case
    if c["op"] == "quantize":
        x = s["x"].double()
        rows, (m, k) = c["block_rows"], s["x"].shape
        kb = -(-k // BLOCK)
        q = torch.empty(m, k, dtype=torch.float64, device="cuda")
        scales = torch.empty(-(-m // rows), kb, dtype=torch.float64, device="cuda")
        step = 128
        for j in range(kb):
            part = x[:, j * BLOCK: (j + 1) * BLOCK]
            top = part.abs().amax(1)
            if rows > 1:
                top = torch.stack([t.max() for t in top.split(step)])
            scales[:, j] = _exact_scale(top)
            per_row = scales[:, j].repeat_interleave(rows)[:m]
            q[:, j * BLOCK: (j + 1) * BLOCK] = _nearest_f8(part / per_row[:, None])
        return q, (scales.t().contiguous() if rows == 1 else scales)
    if c["op"] == "gemm":
        acc = torch.zeros(c["m"], c["n"], dtype=torch.float64, device="cuda")
        for j in range(-(-c["k"] // BLOCK)):
            at = slice(j * BLOCK, (j + 1) * BLOCK)
            left = s["a"][:, at].double() * s["sa"][j].double()[:, None]
            right = s["b"][:, at].double() * s["sb"][:, j].double().repeat_interleave(BLOCK)[: c["n"], None]
            acc.addmm_(left, right.t())
        return acc
    if c["op"] == "append":
        return _exact_append(s)
    S, H, Hk, D, bs = c["seqs"], c["heads"], c["kv_heads"], c["d"], c["block"]
    o = torch.zeros(S, H, D, dtype=torch.float64, device="cuda")
    lse = torch.full((S, H), -math.inf, dtype=torch.float64, device="cuda")
    for i, n in enumerate(s["lens"].tolist()):
        if n == 0:
            continue
        blk = s["table"][i, : -(-n // bs)].long()
        for h in range(Hk):
            k = (s["kc"][blk, h].double() * s["ks"][blk, h].double()[:, None, None]).reshape(-1, D)[:n]
            v = (s["vc"][blk, h].double() * s["vs"][blk, h].double()[:, None, None]).reshape(-1, D)[:n]
            at = slice(h * (H // Hk), (h + 1) * (H // Hk))
            sc = (s["q"][i, at].double() @ k.t()) * s["scale"]
            lse[i, at] = torch.logsumexp(sc, -1)
            o[i, at] = torch.softmax(sc, -1) @ v
    return o, lse
