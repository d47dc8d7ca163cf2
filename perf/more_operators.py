"""The operators of the BF16 serving path as measurable cases: a plain torch form of each, and the library's call.

Four operators that a serving engine runs around the paged cache:

* ``packed``   attention over prompts of different lengths packed one behind another, grouped heads, causal or not;
* ``prefill``  new tokens of each sequence (a prompt, a chunk, a few speculated tokens) attend to the paged cache;
* ``shared``   one query token per sequence over the paged cache, where groups of sequences share a long prefix;
* ``w4``       few rows times 4-bit weights with group scales and optional zero points.

``own`` false: elementary torch operations in FP32; true: the calls a user of the library makes.
"""
import math

import numpy as np
import torch

own = False


def listed():
    return [
        # one short prompt (a chat turn): a call's latency
        {"name": "packed_1x37", "op": "packed", "seqs": 1, "lo": 37, "hi": 37, "ctx": 0, "causal": True, "heads": 32, "kv_heads": 8, "d": 128},
        # a batch of prompts of 500 to 1500 tokens, grouped heads
        {"name": "packed_8x500-1500", "op": "packed", "seqs": 8, "lo": 500, "hi": 1500, "ctx": 0, "causal": True, "heads": 32, "kv_heads": 8, "d": 128},
        # documents through an encoder: no mask, 64-wide heads, one key head per query head, ragged lengths
        {"name": "packed_full_24x100-1024_d64", "op": "packed", "seqs": 24, "lo": 100, "hi": 1024, "ctx": 0, "causal": False, "heads": 32, "kv_heads": 32,
         "d": 64},
        # long prompts
        {"name": "packed_4x4k-8k", "op": "packed", "seqs": 4, "lo": 4096, "hi": 8192, "ctx": 0, "causal": True, "heads": 32, "kv_heads": 8, "d": 128},
        # chunked prefill: chunks of 500 to 1500 tokens behind contexts of 100 to 3000
        {"name": "prefill_8x500-1500_behind_100-3000", "op": "prefill", "seqs": 8, "lo": 500, "hi": 1500, "ctx_lo": 100, "ctx_hi": 3000, "heads": 32,
         "kv_heads": 8, "d": 128, "block": 16},
        # five speculated tokens of each of 32 running sequences are checked at once
        {"name": "prefill_32x5_behind_2k-4k", "op": "prefill", "seqs": 32, "lo": 5, "hi": 5, "ctx_lo": 2048, "ctx_hi": 4096, "heads": 32, "kv_heads": 4,
         "d": 128, "block": 16},
        # one more question of 100 tokens behind a long document
        {"name": "prefill_1x100_behind_30k", "op": "prefill", "seqs": 1, "lo": 100, "hi": 100, "ctx_lo": 30000, "ctx_hi": 30000, "heads": 32,
         "kv_heads": 8, "d": 128, "block": 32},
        # 32 requests behind one system prompt of 4k tokens
        {"name": "shared_32_prefix4k", "op": "shared", "groups": 1, "seqs": 32, "prefix": 4096, "lo": 50, "hi": 500, "heads": 32, "kv_heads": 8, "d": 128,
         "block": 16},
        # 128 samples each behind one of two long documents
        {"name": "shared_128_prefix16k", "op": "shared", "groups": 2, "seqs": 128, "prefix": 16000, "lo": 0, "hi": 1000, "heads": 32, "kv_heads": 4,
         "d": 128, "block": 16},
        # next token of one sequence: the output projection
        {"name": "w4_1x4096x4096", "op": "w4", "m": 1, "n": 4096, "k": 4096, "group": 128, "zeros": False},
        # next token of one sequence: the up projection
        {"name": "w4_1x28672x4096", "op": "w4", "m": 1, "n": 28672, "k": 4096, "group": 128, "zeros": True},
        # next tokens of a batch: the down projection
        {"name": "w4_16x4096x28672", "op": "w4", "m": 16, "n": 4096, "k": 28672, "group": 64, "zeros": True},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


_MOST_PAIRS = 32 * 4 * 5000 * 5000  # score elements of a drawn case: below the largest listed one's


def draw(rng):
    op = rng.choice(["packed", "prefill", "prefill", "shared", "shared", "w4"])
    if op == "w4":
        group = rng.choice([32, 64, 128])
        m, n, k = _log(rng, 1, 64), _log(rng, 40, 28672), group * _log(rng, 1, 28672 // group)
        while m * n * k > 64 * 28672 * 4096:
            n = max(40, n // 2)
        return {"op": op, "m": m, "n": n, "k": k, "group": group, "zeros": rng.random() < 0.5}
    d, kv = rng.choice([64, 128]), rng.choice([1, 2, 4, 8])
    if op == "shared":
        heads = kv * rng.choice([1, 2, 4, 8])
        seqs, prefix = _log(rng, 2, 128), _log(rng, 1, 32000)
        hi = _log(rng, 1, 2000)
        return {"op": op, "groups": rng.randint(1, min(3, seqs)), "seqs": seqs, "prefix": prefix, "lo": rng.choice([0, hi // 2, hi]), "hi": hi,
                "heads": heads, "kv_heads": kv, "d": d, "block": rng.choice([8, 16, 32])}
    heads = kv * rng.choice([1, 2, 3, 4, 5, 7, 8])
    seqs = _log(rng, 1, 64)
    hi = _log(rng, 1, max(1, min(8192, 32768 // seqs)))
    lo = rng.choice([0, hi // 3, hi])
    ctx = 0 if rng.random() < 0.4 else _log(rng, 1, 32000)
    while seqs * hi * (hi + ctx) * heads > _MOST_PAIRS:
        hi, ctx = max(1, hi // 2), ctx // 2
        lo = min(lo, hi)
    if op == "packed":
        return {"op": op, "seqs": seqs, "lo": lo, "hi": hi, "ctx": min(ctx, 100000 // seqs), "causal": rng.random() < 0.7, "heads": heads,
                "kv_heads": kv, "d": d}
    ctx = min(ctx, 400000 // seqs)
    return {"op": op, "seqs": seqs, "lo": lo, "hi": hi, "ctx_lo": ctx // 3, "ctx_hi": ctx, "heads": heads, "kv_heads": kv, "d": d,
            "block": rng.choice([8, 16, 32])}


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _ints(seed, salt, lo, hi, n):
    return np.random.RandomState((int(seed) * 131 + salt) % (1 << 31)).randint(lo, hi + 1, n).astype(np.int64)


def _dev32(a):
    return torch.from_numpy(np.ascontiguousarray(a).astype(np.int32)).cuda()


def _cu(lens):
    return np.concatenate([[0], np.cumsum(lens)])


def _lengths(c):
    """New tokens of each sequence and the keys in front of them: they set the outputs' shapes, so they go by the case alone."""
    if c["op"] == "shared":
        return np.ones(c["seqs"], dtype=np.int64), _group_prefix(c) + _ints(c["seqs"], 2, c["lo"], c["hi"], c["seqs"]) - 1
    new = _ints(c["seqs"], 1, c["lo"], c["hi"], c["seqs"])
    new[0] = max(1, new[0])
    if c["op"] == "packed":
        return new, _ints(c["seqs"], 2, c["ctx"] // 2, c["ctx"], c["seqs"])
    return new, _ints(c["seqs"], 2, c["ctx_lo"], c["ctx_hi"], c["seqs"])


def _group_of(c):
    return np.arange(c["seqs"]) * c["groups"] // c["seqs"]


def _group_lens(c):
    """Prefix tokens of each group: whole blocks, as engines share them."""
    want = np.array([c["prefix"] // (1 + g) for g in range(c["groups"])])
    return np.maximum(1, want // c["block"]) * c["block"]


def _group_prefix(c):
    return _group_lens(c)[_group_of(c)]


def _table(c, seed, lens):
    """A block table whose blocks lie scattered over the pool (unused entries: -1), and the pool's size.  The sequences of a
    group have its prefix's blocks in common."""
    bs = c["block"]
    per = (lens + bs - 1) // bs
    width = max(1, int(per.max()))
    order = np.random.RandomState((int(seed) * 7919 + 13) % (1 << 31)).permutation(int(per.sum()) + 3)
    at = _cu(per)[:-1, None] + np.arange(width)[None, :]
    table = np.where(np.arange(width)[None, :] < per[:, None], order[np.minimum(at, len(order) - 1)], -1)
    if c["op"] == "shared":
        group, held = _group_of(c), _group_lens(c) // bs
        for g in range(c["groups"]):
            rows = np.nonzero(group == g)[0]
            table[rows, : held[g]] = order[at[rows[0], 0] + np.arange(held[g])]
    return table, len(order)


def prepare(case, seed):
    c, g = case, _gen(seed)
    if c["op"] == "w4":
        m, n, k, groups = c["m"], c["n"], c["k"], c["k"] // c["group"]
        s = {"case": c, "x": torch.randn(m, k, generator=g, device="cuda", dtype=torch.bfloat16)}
        s["x"][:, k // 3] *= 30.0                                                                        # an outlier channel
        s["w"] = torch.randint(0, 256, (n, k // 2), generator=g, device="cuda", dtype=torch.uint8)       # two weights per byte, the even one low
        s["scales"] = (torch.rand(n, groups, generator=g, device="cuda") * 0.01 + 0.002).to(torch.bfloat16)
        s["zeros"] = torch.randint(4, 12, (n, groups), generator=g, device="cuda", dtype=torch.uint8) if c["zeros"] else None
        return s
    H, Hk, D = c["heads"], c["kv_heads"], c["d"]
    new, ctx = _lengths(c)
    T = int(new.sum())
    s = {"case": c, "new": new.tolist(), "ctx": ctx.tolist(), "scale": float(np.float32(1.0 / math.sqrt(D))), "cu": _dev32(_cu(new))}
    if c["op"] == "packed":
        if c["ctx"] == 0:  # views of one fused projection
            qkv = torch.randn(T, (H + 2 * Hk) * D, generator=g, device="cuda", dtype=torch.bfloat16)
            s["q"], s["k"], s["v"] = qkv[:, : H * D].view(T, H, D), qkv[:, H * D: (H + Hk) * D].view(T, Hk, D), qkv[:, (H + Hk) * D:].view(T, Hk, D)
        else:
            s["q"] = torch.randn(T, H, D, generator=g, device="cuda", dtype=torch.bfloat16)
            s["k"], s["v"] = (torch.randn(int((new + ctx).sum()), Hk, D, generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2))
        s["cu_k"] = _dev32(_cu(new + ctx))
    else:
        s["q"] = torch.randn(T, H, D, generator=g, device="cuda", dtype=torch.bfloat16)
        table, blocks = _table(c, seed, new + ctx)
        s["table"], s["ctx_dev"], s["lens_dev"] = _dev32(table), _dev32(ctx), _dev32(new + ctx)
        s["kc"], s["vc"] = (torch.randn(blocks, Hk, c["block"], D, generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2))
        if c["op"] == "shared":
            s["prefix"] = _dev32(_group_lens(c))
            s["groups"] = _dev32(np.concatenate([[0], np.cumsum(np.bincount(_group_of(c), minlength=c["groups"]))]))
    s["ws"] = torch.empty(256 << 20, dtype=torch.uint8, device="cuda")  # scratch that a serving loop keeps
    return s


# ---------------------------------------------------------------- plain forms

def _sequences(s):
    """Keys, values [tokens, Hk, D] and the rows of q of each sequence."""
    c = s["case"]
    t = at = 0
    for i, (new, ctx) in enumerate(zip(s["new"], s["ctx"])):
        n = new + ctx
        if c["op"] == "packed":
            k, v = s["k"][at: at + n], s["v"][at: at + n]
        else:
            blk = s["table"][i, : -(-n // c["block"])].long()
            k, v = (x[blk].transpose(1, 2).reshape(-1, c["kv_heads"], c["d"])[:n] for x in (s["kc"], s["vc"]))
        yield slice(t, t + new), k, v
        t, at = t + new, at + n


def _plain_attention(s):
    c = s["case"]
    H, Hk, D = c["heads"], c["kv_heads"], c["d"]
    q = s["q"]
    o = torch.zeros(q.shape, device="cuda", dtype=torch.bfloat16)
    lse = torch.full(q.shape[:2], -math.inf, device="cuda")
    for rows, k, v in _sequences(s):
        n, nk = rows.stop - rows.start, k.shape[0]
        if n == 0:
            continue
        qs = q[rows].float().view(n, Hk, H // Hk, D).permute(1, 2, 0, 3).reshape(Hk, -1, D) * s["scale"]
        sc = torch.matmul(qs, k.float().permute(1, 2, 0)).view(Hk, H // Hk, n, nk)
        if c.get("causal", True):
            seen = torch.arange(nk, device="cuda")[None, :] <= torch.arange(n, device="cuda")[:, None] + (nk - n)
            sc.masked_fill_(~seen, -math.inf)
        top = sc.amax(-1, keepdim=True)
        p = torch.exp(sc.sub_(top))
        l = p.sum(-1, keepdim=True)
        out = torch.matmul(p.view(Hk, -1, nk), v.float().transpose(0, 1)).view(Hk, H // Hk, n, D) / l
        o[rows] = out.permute(2, 0, 1, 3).reshape(n, H, D).to(torch.bfloat16)
        lse[rows] = (top + torch.log(l)).permute(2, 0, 1, 3).reshape(n, H)
    return o, lse


def _plain_w4(s):
    c = s["case"]
    w = torch.stack([s["w"] & 15, s["w"] >> 4], -1).view(c["n"], -1, c["group"]).float()
    w = (w - (8.0 if s["zeros"] is None else s["zeros"].float()[..., None])) * s["scales"].float()[..., None]
    return (s["x"].float() @ w.view(c["n"], c["k"]).t()).to(torch.bfloat16)


def run(state):
    s, c = state, state["case"]
    if not own:
        return _plain_w4(s) if c["op"] == "w4" else _plain_attention(s)
    import paper_2503_14985_b200 as mlt
    if c["op"] == "w4":
        return mlt.gemm_w4(s["x"], s["w"], s["scales"], s["zeros"])
    if c["op"] == "packed":
        return mlt.mha_packed_fwd(s["q"], s["k"], s["v"], s["cu"], s["cu_k"], causal=c["causal"], scale=s["scale"], workspace=s["ws"])
    if c["op"] == "prefill":
        return mlt.paged_attn_prefill(s["q"], s["kc"], s["vc"], s["cu"], s["ctx_dev"], s["table"], scale=s["scale"], workspace=s["ws"])
    return mlt.paged_attn_decode_shared(s["q"], s["kc"], s["vc"], s["table"], s["lens_dev"], s["prefix"], s["groups"], scale=s["scale"],
                                        workspace=s["ws"])


def work(case):
    c = case
    if c["op"] == "w4":
        m, n, k, groups = c["m"], c["n"], c["k"], c["k"] // c["group"]
        return {"bytes": n * k / 2.0 + n * groups * (3.0 if c["zeros"] else 2.0) + 2.0 * m * k + 2.0 * m * n, "flops": 2.0 * m * n * k}
    H, Hk, D = c["heads"], c["kv_heads"], c["d"]
    new, ctx = _lengths(c)
    tokens, keys = float(new.sum()), float((new + ctx)[new > 0].sum())
    if c["op"] == "shared":
        keys -= float(_group_prefix(c).sum() - _group_lens(c).sum())
    if c.get("causal", True):
        pairs = float((new * ctx + new * (new + 1) // 2).sum())
    else:
        pairs = float((new * (new + ctx)).sum())
    return {"bytes": 4.0 * tokens * H * D + 4.0 * tokens * H + 4.0 * keys * Hk * D, "flops": 4.0 * pairs * H * D}


# ---------------------------------------------------------------- the definitions, in 64 bits

def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["op"] == "w4":
        out = torch.zeros(c["m"], c["n"], dtype=torch.float64, device="cuda")
        low, high = (s["w"] % 16).double(), torch.div(s["w"], 16, rounding_mode="floor").double()
        for j in range(c["k"] // c["group"]):
            half = slice(j * c["group"] // 2, (j + 1) * c["group"] // 2)
            x = s["x"][:, j * c["group"]: (j + 1) * c["group"]].double()
            part = x[:, 0::2] @ low[:, half].t() + x[:, 1::2] @ high[:, half].t()
            zero = 8.0 if s["zeros"] is None else s["zeros"][:, j].double()[None, :]
            out += (part - x.sum(1, keepdim=True) * zero) * s["scales"][:, j].double()[None, :]
        return out
    H, Hk, D = c["heads"], c["kv_heads"], c["d"]
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    cu, first_key = s["cu"].tolist(), 0
    for i in range(c["seqs"]):
        n = cu[i + 1] - cu[i]
        total = n + s["ctx"][i]
        if n > 0:
            for h in range(Hk):
                if c["op"] == "packed":
                    k, v = (s[x][first_key: first_key + total, h].double() for x in ("k", "v"))
                else:
                    where = torch.arange(total, device="cuda")
                    blk = s["table"][i].long()[where // c["block"]]
                    k, v = (s[x][blk, h, where % c["block"]].double() for x in ("kc", "vc"))
                for head in range(h * (H // Hk), (h + 1) * (H // Hk)):
                    for r in range(0, n, 2048):
                        q = s["q"][cu[i] + r: min(cu[i] + r + 2048, cu[i + 1]), head].double()
                        sc = s["scale"] * (q @ k.t())
                        if c.get("causal", True):
                            sc += torch.full_like(sc, -math.inf).triu(total - n + r + 1)
                        at = slice(cu[i] + r, cu[i] + r + q.shape[0])
                        lse[at, head] = torch.logsumexp(sc, -1)
                        o[at, head] = torch.softmax(sc, -1) @ v
        first_key += total
    return o, lse
