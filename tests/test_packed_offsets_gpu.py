"""Packed, paged and shared-prefix attention with offsets that do not ascend and key ranges that are cut: what is kept, and that nothing behind the
scratch is written.  Every case's plan is first run and checked on the CPU (packed_plan_util); the kernels go where the plan says."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2503_14985_b200 as mlt  # noqa: E402

from packed_plan_util import plan  # noqa: E402
from packed_util import check_rows, gathered, paged, rows_reference  # noqa: E402
from test_packed_gpu import visible  # noqa: E402
from test_packed_plan import alternating, cu as cu_host  # noqa: E402


def i32(x):
    return torch.tensor(np.asarray(x, np.int64), dtype=torch.int32, device="cuda")


def randn(*shape, seed=0):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda", dtype=torch.bfloat16)


def scratch(need):
    ws = torch.full((need + 65536,), 0xAB, dtype=torch.uint8, device="cuda")

    def untouched():
        torch.cuda.synchronize()
        assert (ws[need:] == 0xAB).all(), "written behind the scratch"
    return ws[:need], untouched


# queries, sequences (0, T, 0, T, ...), keys of each, heads per KV head, KV heads, D
REPEATED = [(1000, 15, 30000, 2, 8, 128), (5, 40, 30000, 4, 1, 64), (17, 40, 20000, 8, 1, 64), (300, 9, 9000, 4, 2, 128), (130, 30, 20000, 1, 3, 64)]


@pytest.mark.parametrize("T,S,keys,G,Hk,D", REPEATED)
def test_repeated_queries_write_nothing_behind_the_scratch(T, S, keys, G, Hk, D):
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    at, at_k = alternating(T, S), alternating(keys, S)
    assert plan("packed", T, at, G, Hk, D, cu_k=at_k, num_k=keys, sms=sms)["status"] == 9
    q, k, v = randn(T, G * Hk, D, seed=1), randn(keys, Hk, D, seed=2), randn(keys, Hk, D, seed=3)
    ws, untouched = scratch(mlt.mha_packed_workspace_bytes(T, S, G * Hk, Hk, D))
    mlt.mha_packed_fwd(q, k, v, i32(at), i32(at_k), causal=True, scale=0.1, workspace=ws)
    untouched()
    assert mlt.last_device_error()[0] == 9
    bs, blocks = 16, keys // 16
    ctx = keys // 16 * 16 - T
    assert plan("prefill", T, at, G, Hk, D, context=[ctx] * S, max_blocks=blocks, sms=sms)["status"] == 9
    kc, vc = randn(blocks, Hk, bs, D, seed=4), randn(blocks, Hk, bs, D, seed=5)
    table = i32(np.tile(np.arange(blocks), (S, 1)))
    mlt.paged_attn_prefill(q, kc, vc, i32(at), i32([ctx] * S), table, scale=0.1, workspace=ws)
    untouched()
    assert mlt.last_device_error()[0] == 9
    T = min(T, 150)
    at = alternating(T, S)
    lens, prefix = [ctx + T] * T, [ctx // 16 * 16] * S
    assert plan("shared", T, at, G, Hk, D, prefix=prefix, lens=lens, max_blocks=blocks, sms=sms)["status"] == 9
    ws, untouched = scratch(mlt.paged_attn_shared_workspace_bytes(T, S, G * Hk, Hk, D))
    mlt.paged_attn_decode_shared(q[:T].contiguous(), kc, vc, table[:1].repeat(T, 1).contiguous(), i32(lens), i32(prefix), i32(at), scale=0.1, workspace=ws)
    untouched()
    assert mlt.last_device_error()[0] == 9


def rows_of(kept):
    """kept: {sequence: (first token, tokens)} -> mask of rows that some kept sequence has"""
    return np.concatenate([np.arange(a, a + n) for a, n in kept.values()] + [np.zeros(0, int)]).astype(int)


# offsets of the queries; sequences that are kept and have tokens in common have the same ones (the result is then one of theirs)
@pytest.mark.parametrize("at,G,Hk,D", [([5, 9, 0, 4], 4, 2, 128), ([20, 23, 10, 17, 3, 9], 2, 1, 64), ([30, 60, 0, 29, 29, 30, 60], 8, 1, 64),
                                       ([9, 9, 2, 8, -1, 9, 10], 1, 3, 128), ([0, 40, 0, 40, 0, 40], 4, 1, 64)])
@pytest.mark.parametrize("kind", ["packed", "prefill"])
def test_kept_sequences_behind_descending_offsets(kind, at, G, Hk, D):
    """Key ranges are cut, so that the join has to find each row's sequence."""
    T, S, H, bs = max(at) + 3, len(at) - 1, G * Hk, 16
    m = [3000 + 700 * s for s in range(S)] if at[:2] != [0, 40] else [3000] * S
    at = np.asarray(at)
    n = at[1:] - at[:-1]
    kept = {s: (int(at[s]), int(n[s])) for s in range(S) if n[s] > 0 and at[s] >= 0}
    q = randn(T, H, D, seed=1)
    o = torch.full((T, H, D), 776.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((T, H), 776.0, device="cuda")
    if kind == "packed":
        at_k = cu_host(m)
        k, v = randn(at_k[-1], Hk, D, seed=2), randn(at_k[-1], Hk, D, seed=3)
        keys = {s: (k[at_k[s]: at_k[s + 1]].double(), v[at_k[s]: at_k[s + 1]].double()) for s in kept}
        if at[1] == 40:
            at_k, keys = alternating(3000, S), {s: (k[:3000].double(), v[:3000].double()) for s in kept}
        r = plan(kind, T, at, G, Hk, D, cu_k=at_k, num_k=len(k))
        mlt.mha_packed_fwd(q, k, v, i32(at), i32(at_k), causal=True, scale=0.125, O=o, LSE=lse)
    else:
        kc, vc, table = paged(m, Hk, D, bs, seed=4)
        if at[1] == 40:
            table = table[:1].repeat(S, 1).contiguous()
        ctx = np.asarray(m) - np.maximum(n, 0)
        keys = {s: (gathered(kc, table[s], m[s]), gathered(vc, table[s], m[s])) for s in kept}
        r = plan(kind, T, at, G, Hk, D, context=ctx, max_blocks=table.shape[1])
        mlt.paged_attn_prefill(q, kc, vc, i32(at), i32(ctx), table, scale=0.125, O=o, LSE=lse)
    assert r["chunk"] > 0 and (r["seqs"][list(kept), 1] > 0).all()
    assert mlt.last_device_error()[0] == 9
    right = {}
    for s, (a, count) in kept.items():
        ref = rows_reference(q[a: a + count].double(), *keys[s], visible(count, m[s], True), 0.125)
        try:
            check_rows(o[a: a + count], lse[a: a + count], ref, f"sequence {s}")
            right[a, count] = None
        except AssertionError as e:
            right.setdefault((a, count), e)
    for e in right.values():
        if e:
            raise e
    rest = np.setdiff1d(np.arange(T), rows_of(kept))
    assert (o[rest] == 776).all() and (lse[rest] == 776).all()


@pytest.mark.parametrize("G,Hk,D", [(4, 1, 64), (8, 2, 128)])
def test_sequences_of_groups_that_do_not_ascend(G, Hk, D):
    """Whatever the groups, a sequence's result is that of its own table: the prefix (the same for all here) and the tail meet once."""
    rng = np.random.RandomState(G)
    T, bs = 40, 16
    lens = (700 + rng.randint(0, 400, T)).tolist()
    kc, vc, table = paged(lens, Hk, D, bs, seed=6, share=[(list(range(T)), 40)])
    q = randn(T, G * Hk, D, seed=7)
    refs = [rows_reference(q[t: t + 1].double(), gathered(kc, table[t], lens[t]), gathered(vc, table[t], lens[t]), visible(1, lens[t], True), 0.125)
            for t in range(T)]
    answered = 0
    for case in range(30):
        S = int(rng.randint(2, 60))
        at = rng.randint(0, T + 1, S + 1) if case % 2 else np.where(rng.rand(S + 1) < 0.5, np.sort(rng.randint(0, T + 1, S + 1)), T + 9)
        prefix = [640 - 16 * int(x) for x in rng.randint(0, 30, S)]
        r = plan("shared", T, at, G, Hk, D, prefix=prefix, lens=lens, max_blocks=table.shape[1])
        o = torch.full((T, G * Hk, D), 776.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((T, G * Hk), 776.0, device="cuda")
        mlt.paged_attn_decode_shared(q, kc, vc, table, i32(lens), i32(prefix), i32(at), scale=0.125, O=o, LSE=lse)
        assert mlt.last_device_error()[0] == r["status"]
        if r["num"] == 0:
            assert (o == 776).all() and (lse == 776).all()
            continue
        answered += 1
        for t in range(T):
            check_rows(o[t: t + 1], lse[t: t + 1], refs[t], f"case {case}, sequence {t}")
    assert answered > 10
