"""mlt_mha_packed_fwd, mlt_paged_attn_prefill and mlt_paged_attn_decode_shared where they can go wrong: neighbours full of NaN, bad offsets and
tables, captured graphs, streams, scratch of any size, caches beyond 2^32 bytes, jumps of the running maximum (bounds: packed_util)."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2503_14985_b200 as mlt  # noqa: E402

from gpu_util import assert_device_healthy  # noqa: E402
from packed_util import check_rows, cu, gathered, paged, rows_reference  # noqa: E402
from test_packed_gpu import packed_inputs, run_packed, visible  # noqa: E402

NAN = math.nan


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def randn(*shape, seed=0):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda", dtype=torch.bfloat16)


@pytest.mark.parametrize("D,causal,lens", [(64, True, [100, 50, 77, 300]), (128, False, [100, 50, 77, 300]), (128, True, [3, 700, 1])])
def test_a_neighbour_of_nan_changes_nothing(D, causal, lens):
    q, k, v = (randn(sum(lens), h, D, seed=h) for h in (8, 2, 2))
    want, want_lse = run_packed(q, k, v, lens, lens, causal, 0.1)
    a, b = lens[0], lens[0] + lens[1]
    for x in (q, k, v):
        x[a:b] = NAN
    got, got_lse = run_packed(q, k, v, lens, lens, causal, 0.1)
    for rows in (slice(0, a), slice(b, None)):
        assert torch.equal(got[rows], want[rows]) and torch.equal(got_lse[rows], want_lse[rows])
    assert torch.isnan(got[a:b]).all()


@pytest.mark.parametrize("D", [64, 128])
def test_jumps_of_the_running_maximum(D):
    """One late key beats a row's earlier ones by up to e^100, in whole ranges and in cut ones; and rows that all lie far out."""
    for lens_q, lens_k in (([260], [1000]), ([3], [6000])):
        q, k, v = (randn(n, h, D, seed=n) for n, h in ((lens_q[0], 4), (lens_k[0], 2), (lens_k[0], 2)))
        k[lens_k[0] - 300] = q[min(1, lens_q[0] - 1), 0] * (60 / D)
        q[lens_q[0] // 2:] *= 8.0
        o, lse = run_packed(q, k, v, lens_q, lens_k, True, 1.0)
        check_rows(o, lse, rows_reference(q.double(), k.double(), v.double(), visible(lens_q[0], lens_k[0], True), 1.0))


def test_many_sequences_and_no_scratch_for_parts():
    g = np.random.RandomState(1)
    lens = g.randint(0, 4, 3000).tolist()
    q, k, v = packed_inputs(lens, lens, 4, 2, 64, seed=2)
    o, lse = run_packed(q, k, v, lens, lens, True, 0.125)
    a = 0
    for s, n in enumerate(lens):
        if s % 97 == 0 and n:
            ref = rows_reference(q[a: a + n].double(), k[a: a + n].double(), v[a: a + n].double(), visible(n, n, True), 0.125)
            check_rows(o[a: a + n], lse[a: a + n], ref, f"sequence {s}")
        a += n
    # scratch for the lists alone, for a few parts, for all: the same within the bounds
    q, k, v = randn(5, 8, 64, seed=1), randn(3000, 2, 64, seed=2), randn(3000, 2, 64, seed=3)
    ref = rows_reference(q.double(), k.double(), v.double(), visible(5, 3000, True), 0.125)
    full = mlt.mha_packed_workspace_bytes(5, 1, 8, 2, 64)
    row = 64 * 4 + 8
    lists = full - 320 * 2 * 5 * 4 * row
    for size in (lists, lists + 100 * row, lists + 1000 * row, full):
        ws = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")
        o, lse = mlt.mha_packed_fwd(q, k, v, cu([5]), cu([3000]), causal=True, scale=0.125, workspace=ws)
        check_rows(o, lse, ref, f"{size} bytes")
    with pytest.raises(mlt.MltError) as e:
        mlt.mha_packed_fwd(q, k, v, cu([5]), cu([3000]), causal=True, scale=0.125, workspace=ws[: lists - 256])
    assert e.value.status == 1
    o, lse = mlt.mha_packed_fwd(q, k, v, cu([5]), cu([3000]), causal=True, scale=0.125)  # its own scratch
    check_rows(o, lse, ref)
    assert mlt.mha_packed_fwd(q, k, v, cu([5]), cu([3000]), causal=True, scale=0.125, return_lse=False)[1] is None
    assert_device_healthy()


@pytest.mark.parametrize("bad_q,bad_k,left_out", [([0, 10, 5, 25], None, [1]), ([0, 10, 99, 25], None, [1, 2]), ([-3, 10, 20, 25], None, [0]),
                                                   (None, [0, 10, 7, 25], [1]), (None, [0, 10, 20, 99], [2])])
def test_offsets_that_do_not_fit_are_left_out_and_reported(bad_q, bad_k, left_out):
    lens = [10, 10, 5]
    q, k, v = (randn(25, h, 64, seed=h) for h in (4, 2, 2))
    o = torch.full((25, 4, 64), 776.0, dtype=torch.bfloat16, device="cuda")
    at_q, at_k = bad_q or [0, 10, 20, 25], bad_k or bad_q or [0, 10, 20, 25]
    _, lse = mlt.mha_packed_fwd(q, k, v, i32(at_q), i32(at_k), causal=True, scale=0.125, O=o)
    rc, _ = mlt.last_device_error()
    assert rc == 9
    assert mlt.last_device_error()[0] == 0
    for s in range(3):
        if s in left_out or (bad_q and s == 2 and 1 in left_out and bad_q[2] == 5):
            continue
        rows = slice(at_q[s], at_q[s + 1])
        keys = slice(at_k[s], at_k[s + 1])
        n, m = rows.stop - rows.start, keys.stop - keys.start
        ref = rows_reference(q[rows].double(), k[keys].double(), v[keys].double(), visible(n, m, True), 0.125)
        own = n if at_q != [0, 10, 5, 25] else 5                         # (rows 5 to 9 are the last sequence's too there)
        check_rows(o[rows][:own], lse[rows][:own], [x[:own] for x in ref], f"sequence {s}")
    if 0 in left_out:
        assert (o[:10] == 776).all()


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("at_q,at_k,T,M", [([3, 20], [5, 90], 30, 100), ([0, 37], [0, 0], 37, 0), ([4, 4], [0, 9], 9, 9), ([0, 200], [0, 180], 200, 256),
                                           ([2, 40], [0, 9], 39, 9), ([-1, 9], [0, 9], 9, 9), ([0, 9], [7, 3], 9, 9), ([0, 9], [0, 10], 9, 9)])
def test_one_short_sequence(at_q, at_k, T, M, causal):
    """One sequence that may leave rows in front and behind, without keys, without tokens, and with offsets that do not fit."""
    q, k, v = randn(T, 8, 64, seed=1), randn(M, 2, 64, seed=2), randn(M, 2, 64, seed=3)
    o = torch.full((T, 8, 64), 776.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((T, 8), 776.0, device="cuda")
    mlt.mha_packed_fwd(q, k, v, i32(at_q), i32(at_k), causal=causal, scale=0.125, O=o, LSE=lse)
    fits = 0 <= at_q[0] <= at_q[1] <= T and 0 <= at_k[0] <= at_k[1] <= M
    rc, detail = mlt.last_device_error()
    assert rc == (0 if fits else 9)
    a, b = at_q if fits else (0, 0)
    rows = slice(a, b)
    kk, vv = (x[at_k[0]: at_k[1]].double() for x in (k, v)) if fits else (k[:0].double(), v[:0].double())
    check_rows(o[rows], lse[rows], rows_reference(q[rows].double(), kk, vv, visible(b - a, kk.shape[0], causal), 0.125))
    for x in (o, lse):
        assert (x[:a] == 776).all() and (x[b:] == 776).all()


def test_offsets_whose_tiles_sum_up_beyond_32_bits():
    """0, T, 0, T, ...: every second sequence fits by itself, together they have 2.3e9 tile pairs."""
    T, S = 1 << 16, 140000
    q, k = torch.zeros(T, 128, 64, dtype=torch.bfloat16, device="cuda"), randn(8, 1, 64)
    at_q = torch.zeros(S + 1, dtype=torch.int32, device="cuda")
    at_q[1::2] = T
    o, lse = mlt.mha_packed_fwd(q, k, k, at_q, torch.zeros_like(at_q), causal=False, scale=0.125)
    assert mlt.last_device_error()[0] == 9
    assert (o == 0).all() and (lse == -math.inf).all()                  # (the first ones are within the call's tokens; no keys)
    assert_device_healthy()


@pytest.mark.parametrize("G,Hk,D", [(128, 1, 64), (128, 2, 128), (100, 1, 128), (64, 2, 64), (33, 3, 64)])
def test_many_heads_per_kv_head(G, Hk, D):
    H, bs = G * Hk, 16
    new, ctx = [1, 5, 0, 40], [700, 0, 9, 33]
    total = [a + b for a, b in zip(new, ctx)]
    kc, vc, table = paged(total, Hk, D, bs, seed=G)
    q = randn(sum(new), H, D, seed=1)
    o, lse = mlt.paged_attn_prefill(q, kc, vc, cu(new), i32(ctx), table, scale=0.11)
    a = 0
    for s, n in enumerate(new):
        kk, vv = gathered(kc, table[s], total[s]), gathered(vc, table[s], total[s])
        ref = rows_reference(q[a: a + n].double(), kk, vv, visible(n, total[s], True), float(np.float32(0.11)))
        check_rows(o[a: a + n], lse[a: a + n], ref, f"sequence {s}")
        a += n
    lens = [total[0], total[0] - 30, 0, 5]
    shared = table[:1].repeat(4, 1).contiguous()
    q = randn(4, H, D, seed=2)
    o, lse = mlt.paged_attn_decode_shared(q, kc, vc, shared, i32(lens), i32([640]), i32([0, 3]), scale=0.11)
    kk, vv = gathered(kc, table[0], total[0]), gathered(vc, table[0], total[0])
    for s, n in enumerate(lens):
        check_rows(o[s: s + 1], lse[s: s + 1], rows_reference(q[s: s + 1].double(), kk[:n], vv[:n], visible(1, n, True), float(np.float32(0.11))), f"shared {s}")
    assert_device_healthy()


def test_bad_blocks_and_positions():
    H, Hk, D, bs = 4, 2, 64, 16
    kc, vc, table = paged([100, 60, 40], Hk, D, bs, seed=5)
    q = randn(9, H, D, seed=6)
    new, ctx = [3, 4, 2], [97, 56, 38]
    good, _ = mlt.paged_attn_prefill(q, kc, vc, cu(new), i32(ctx), table, scale=0.2)
    assert_device_healthy()
    for entry in (-1, kc.shape[0], 2 ** 31 - 1, -2 ** 31):
        bad = table.clone()
        bad[1, 2] = entry
        got, lse = mlt.paged_attn_prefill(q, kc, vc, cu(new), i32(ctx), bad, scale=0.2)
        rc, detail = mlt.last_device_error()
        assert rc == 7 and detail[1] == 2
        assert torch.equal(got[:3], good[:3]) and torch.equal(got[7:], good[7:])
        k, v = gathered(kc, table[1], 60), gathered(vc, table[1], 60)  # a block of zeros
        k[32:48], v[32:48] = 0, 0
        check_rows(got[3:7], lse[3:7], rows_reference(q[3:7].double(), k, v, visible(4, 60, True), float(np.float32(0.2))))
    # contexts that are negative, or whose positions lie behind the table
    for c in (-1, 109, 2 ** 31 - 1):
        o = torch.full((9, H, D), 776.0, dtype=torch.bfloat16, device="cuda")
        mlt.paged_attn_prefill(q, kc, vc, cu(new), i32([97, c, 38]), table, scale=0.2, O=o)
        assert mlt.last_device_error()[0] == 9
        assert (o[3:7] == 776).all() and torch.equal(o[:3], good[:3]) and torch.equal(o[7:], good[7:])
    # shared prefixes: a group that descends is decoded sequence by sequence
    lens, one = i32([100, 60, 40]), q[:3].contiguous()
    got, lse = mlt.paged_attn_decode_shared(one, kc, vc, table, lens, i32([16, 16]), i32([3, 1, 2]), scale=0.2)
    assert mlt.last_device_error()[0] == 9
    for s, n in enumerate([100, 60, 40]):
        ref = rows_reference(one[s: s + 1].double(), gathered(kc, table[s], n), gathered(vc, table[s], n), visible(1, n, True), float(np.float32(0.2)))
        check_rows(got[s: s + 1], lse[s: s + 1], ref, f"sequence {s}")
    bad = table.clone()
    bad[0, 0] = -7
    mlt.paged_attn_decode_shared(one, kc, vc, bad, lens, i32([]), i32([0]), scale=0.2)
    assert mlt.last_device_error()[0] == 7


def test_overlapping_groups_write_nothing_out_of_bounds():
    S, H, Hk, D, bs = 300, 8, 8, 64, 16
    kc, vc, table = paged([40] * S, Hk, D, bs, seed=8, share=[(list(range(S)), 2)])
    q = randn(S, H, D, seed=9)
    groups = 400
    at = [0, S] * 200 + [0]                                             # every other group is all sequences
    need = mlt.paged_attn_shared_workspace_bytes(S, groups, H, Hk, D)
    ws = torch.full((need + 4096,), 0xAB, dtype=torch.uint8, device="cuda")
    mlt.paged_attn_decode_shared(q, kc, vc, table, i32([40] * S), i32([32] * groups), i32(at), scale=0.1, workspace=ws[:need])
    assert mlt.last_device_error()[0] == 9
    assert (ws[need:] == 0xAB).all()


def test_captured_and_replayed_with_other_lengths():
    H, Hk, D, bs, S = 8, 2, 128, 16, 4
    kc, vc, table = paged([500, 300, 700, 64], Hk, D, bs, seed=3)
    q = randn(40, H, D, seed=4)
    at, ctx, lens = cu([10, 10, 10, 10]), i32([490, 200, 0, 54]), i32([500, 300, 700, 64])
    prefix, groups = i32([0]), i32([0, 4])
    ws = [torch.empty(mlt.mha_packed_workspace_bytes(40, S, H, Hk, D), dtype=torch.uint8, device="cuda"),
          torch.empty(mlt.paged_attn_shared_workspace_bytes(S, 1, H, Hk, D), dtype=torch.uint8, device="cuda")]
    one = q[:S].contiguous()

    def step():
        return mlt.paged_attn_prefill(q, kc, vc, at, ctx, table, scale=0.1, workspace=ws[0]) + \
            mlt.paged_attn_decode_shared(one, kc, vc, table, lens, prefix, groups, scale=0.1, workspace=ws[1])

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for new, c, n in (([10, 10, 10, 10], [490, 200, 0, 54], [500, 300, 700, 64]), ([1, 30, 0, 9], [0, 270, 5, 55], [0, 17, 650, 64]),
                      ([40, 0, 0, 0], [460, 0, 0, 0], [1, 300, 1, 1])):
        at.copy_(cu(new)); ctx.copy_(i32(c)); lens.copy_(i32(n))
        for w in ws:
            w.fill_(0xFF)
        for t in captured:
            t.fill_(5.0)
        graph.replay()
        now = step()
        torch.cuda.synchronize()
        for a, b in zip(captured, now):
            assert torch.equal(a, b)
        t = 0
        for s, k in enumerate(new):
            if k:
                m = c[s] + k
                ref = rows_reference(q[t: t + k].double(), gathered(kc, table[s], m), gathered(vc, table[s], m), visible(k, m, True), float(np.float32(0.1)))
                check_rows(now[0][t: t + k], now[1][t: t + k], ref, f"sequence {s}")
            t += k
    assert_device_healthy()


def test_two_streams_with_scratch_of_their_own_and_inputs_from_the_call_in_front():
    """Calls on two streams at once, and lengths that a kernel just in front on the stream still has to write."""
    H, Hk, D, bs = 8, 2, 128, 16
    kc, vc, table = paged([3000, 2000], Hk, D, bs, seed=3)
    q = randn(6, H, D, seed=4)
    want = mlt.paged_attn_prefill(q, kc, vc, cu([2, 4]), i32([2998, 1996]), table, scale=0.1)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for rep in range(5):
        for st in streams:
            with torch.cuda.stream(st):
                ctx = torch.zeros(2, dtype=torch.int32, device="cuda")
                torch.cuda._sleep(200_000)
                ctx += torch.tensor([2998, 1996], dtype=torch.int32).cuda()
                got.append(mlt.paged_attn_prefill(q, kc, vc, cu([2, 4]), ctx, table, scale=0.1))
    got.append(mlt.paged_attn_prefill(q, kc, vc, cu([2, 4]), i32([2998, 1996]), table, scale=0.1, stream=streams[0]))
    torch.cuda.synchronize()
    for o, lse in got:
        assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
    assert_device_healthy()


def test_caches_and_rows_beyond_32_bits():
    H, Hk, D, bs = 8, 8, 128, 32
    blocks = 2 ** 32 // (Hk * bs * D) + 5                              # the last blocks begin behind 2^32 elements
    kc, vc = (torch.empty(blocks, Hk, bs, D, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    used = [blocks - 1, 0, blocks - 3, 2, blocks - 2]
    for x, c in enumerate((kc, vc)):
        for i, b in enumerate(used):
            c[b] = randn(Hk, bs, D, seed=10 * x + i)
    table = i32([used])
    q = randn(3, H, D, seed=1)
    o, lse = mlt.paged_attn_prefill(q, kc, vc, cu([3]), i32([150]), table, scale=0.1)
    k, v = gathered(kc, table[0], 153), gathered(vc, table[0], 153)
    check_rows(o, lse, rows_reference(q.double(), k, v, visible(3, 153, True), float(np.float32(0.1))))
    one = q[:1].contiguous()
    o, lse = mlt.paged_attn_decode_shared(one, kc, vc, table, i32([153]), i32([64]), i32([0, 1]), scale=0.1)
    check_rows(o, lse, rows_reference(one.double(), k, v, visible(1, 153, True), float(np.float32(0.1))))
    del kc, vc
    T, wide = 600000, 4096 + 8                                          # rows of a pitch with which the last ones begin behind 2^31 elements
    x = torch.empty(T, wide, device="cuda", dtype=torch.bfloat16)
    x[-700:] = randn(700, wide, seed=3)
    k, v = x[:, :256].unflatten(1, (2, 128)), x[:, 256:512].unflatten(1, (2, 128))
    q = x[:, 512:1536].unflatten(1, (8, 128))
    at = i32([T - 700, T - 690, T])
    o, lse = mlt.mha_packed_fwd(q, k, v, at, at, causal=True, scale=0.1, O=x[:, 2064:3088].unflatten(1, (8, 128)))
    ref = rows_reference(q[-690:].double(), k[-690:].double(), v[-690:].double(), visible(690, 690, True), float(np.float32(0.1)))
    check_rows(o[-690:], lse[-690:], ref)
    assert_device_healthy()


def test_two_heads_counts_and_random_shapes():
    g = np.random.RandomState(11)
    for case in range(14):
        D, Hk, G = int(g.choice([64, 128])), int(g.choice([1, 2, 3, 8])), int(g.choice([1, 2, 3, 4, 5, 6, 8, 9, 16, 20]))
        S = int(g.randint(1, 9))
        lens_q = np.exp(g.uniform(0, math.log(600), S)).astype(int) - 1
        lens_k = lens_q + (np.exp(g.uniform(0, math.log(4000), S)).astype(int) - 1) * (g.rand(S) < 0.6)
        causal = bool(g.rand() < 0.6)
        if lens_q.sum() == 0:
            lens_q[0], lens_k[0] = 3, 9
        q, k, v = packed_inputs(lens_q.tolist(), lens_k.tolist(), Hk * G, Hk, D, seed=case)
        o, lse = run_packed(q, k, v, lens_q.tolist(), lens_k.tolist(), causal, 0.11)
        a = b = 0
        for n, m in zip(lens_q, lens_k):
            ref = rows_reference(q[a: a + n].double(), k[b: b + m].double(), v[b: b + m].double(), visible(int(n), int(m), causal), float(np.float32(0.11)))
            check_rows(o[a: a + n], lse[a: a + n], ref, f"case {case}: {n} queries, {m} keys, {Hk} x {G}, D {D}")
            a, b = a + n, b + m
