"""Packed and paged prompt attention with so many work items that no key range is cut (more than three rounds of the SMs) and sequences of many key
blocks: the kernel that batches of prompts run (bounds: packed_util)."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2503_14985_b200 as mlt  # noqa: E402

from gpu_util import assert_device_healthy  # noqa: E402
from packed_plan_util import plan  # noqa: E402
from packed_util import check_rows, cu, gathered, guarded, paged, rows_reference  # noqa: E402
from test_packed_gpu import packed_inputs, run_packed, visible  # noqa: E402
from test_packed_plan import cu as cu_host  # noqa: E402


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def assert_many(r, Hk, lens_k):
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert r["part_rows"] == 0 and r["num"] * Hk > 3 * sms and np.max(lens_k) > 6 * 128


# new tokens and contexts of each sequence, heads per KV head, KV heads, D
SHAPES = [([1500, 700, 0, 129, 1, 1800, 900], [0] * 7, 4, 8, 128), ([1500, 700, 0, 129, 1, 1800, 900], [0] * 7, 4, 8, 64),
          ([640, 1100, 277, 1500, 1300], [900, 0, 3000, 129, 1], 3, 8, 64), ([640, 1100, 277, 1500, 1300], [900, 0, 3000, 129, 1], 3, 8, 128),
          ([900, 1024, 1023, 1025, 850, 3, 1200], [128, 0, 1, 5, 300, 2000, 0], 1, 32, 64), ([900, 1024, 1023, 1025, 850, 3, 1200], [128, 0, 1, 5, 300, 2000, 0], 1, 32, 128),
          ([500, 600, 700, 812], [2000, 1000, 0, 768], 16, 3, 128), ([500, 600, 700, 812], [2000, 1000, 0, 768], 16, 3, 64), ([1000, 930], [50, 700], 8, 8, 64)]


@pytest.mark.parametrize("new,ctx,G,Hk,D", SHAPES)
@pytest.mark.parametrize("causal", [True, False])
def test_packed(new, ctx, G, Hk, D, causal):
    total = [a + b for a, b in zip(new, ctx)]
    q, k, v = packed_inputs(new, total, G * Hk, Hk, D, seed=len(new) + D)
    assert_many(plan("packed", len(q), cu_host(new), G, Hk, D, cu_k=cu_host(total), num_k=len(k), causal=causal), Hk, total)
    o, lse = run_packed(q, k, v, new, total, causal, 0.11, pitch=G * Hk * D + 8)
    a = b = 0
    for s, (n, m) in enumerate(zip(new, total)):
        ref = rows_reference(q[a: a + n].double(), k[b: b + m].double(), v[b: b + m].double(), visible(n, m, causal), float(np.float32(0.11)))
        check_rows(o[a: a + n], lse[a: a + n], ref, f"sequence {s}")
        a, b = a + n, b + m
    again, again_lse = run_packed(q, k, v, new, total, causal, 0.11)
    assert torch.equal(again, o) and torch.equal(again_lse, lse), "two calls differ"


@pytest.mark.parametrize("new,ctx,G,Hk,D", SHAPES)
@pytest.mark.parametrize("bs", [8, 16, 32])
def test_prefill(new, ctx, G, Hk, D, bs):
    total = [a + b for a, b in zip(new, ctx)]
    kc, vc, table = paged(total, Hk, D, bs, seed=D + bs)
    T = sum(new)
    q = torch.randn(T + 2, G * Hk, D, generator=torch.Generator(device="cuda").manual_seed(bs), device="cuda", dtype=torch.bfloat16)
    q[T:] = math.nan
    assert_many(plan("prefill", T + 2, cu_host(new), G, Hk, D, context=ctx, bs=bs, max_blocks=table.shape[1]), Hk, total)
    o, o_ok = guarded((T + 2, G * Hk, D), torch.bfloat16)
    lse, lse_ok = guarded((T + 2, G * Hk), torch.float32)
    mlt.paged_attn_prefill(q, kc, vc, cu(new), i32(ctx), table, scale=0.11, O=o, LSE=lse)
    o_ok()
    lse_ok()
    assert (o[T:] == 776).all() and (lse[T:] == 776).all()
    a = 0
    for s, (n, m) in enumerate(zip(new, total)):
        ref = rows_reference(q[a: a + n].double(), gathered(kc, table[s], m), gathered(vc, table[s], m), visible(n, m, True), float(np.float32(0.11)))
        check_rows(o[a: a + n], lse[a: a + n], ref, f"sequence {s}")
        a += n
    assert_device_healthy()


@pytest.mark.parametrize("D", [64, 128])
def test_neighbours_of_nan_and_jumps_of_the_maximum(D):
    new, G, Hk = [1000, 300, 1400, 900, 1100], 4, 8
    q, k, v = packed_inputs(new, new, G * Hk, Hk, D, seed=D)
    at = cu_host(new)
    for s in (0, 3):                                                    # late keys far above a row's earlier ones
        k[at[s] + 700] = q[at[s] + 800, :Hk] * (60 / D)
        q[at[s] + 600: at[s] + 900] *= 8.0
    want, want_lse = run_packed(q, k, v, new, new, True, 1.0)
    for s in (0, 2, 3, 4):
        x = slice(at[s], at[s + 1])
        check_rows(want[x], want_lse[x], rows_reference(q[x].double(), k[x].double(), v[x].double(), visible(new[s], new[s], True), 1.0), f"sequence {s}")
    for t in (q, k, v):
        t[at[1]: at[2]] = math.nan
    got, got_lse = run_packed(q, k, v, new, new, True, 1.0)
    for x in (slice(0, at[1]), slice(at[2], at[-1])):
        assert torch.equal(got[x], want[x]) and torch.equal(got_lse[x], want_lse[x])
    assert torch.isnan(got[at[1]: at[2]]).all()


@pytest.mark.parametrize("D", [64, 128])
def test_bad_blocks_and_replays(D):
    new, ctx, G, Hk, bs = [1000, 1200, 1500], [100, 900, 0], 4, 8, 16
    total = [a + b for a, b in zip(new, ctx)]
    kc, vc, table = paged(total, Hk, D, bs, seed=D)
    q = torch.randn(sum(new), G * Hk, D, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda", dtype=torch.bfloat16)
    assert_many(plan("prefill", len(q), cu_host(new), G, Hk, D, context=ctx, bs=bs, max_blocks=table.shape[1]), Hk, total)
    at, context = cu(new), i32(ctx)
    ws = torch.empty(mlt.mha_packed_workspace_bytes(len(q), 3, G * Hk, Hk, D), dtype=torch.uint8, device="cuda")
    good = mlt.paged_attn_prefill(q, kc, vc, at, context, table, scale=0.1, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, lse = mlt.paged_attn_prefill(q, kc, vc, at, context, table, scale=0.1, workspace=ws)
    for _ in range(2):
        o.fill_(5.0)
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, good[0]) and torch.equal(lse, good[1])
    assert_device_healthy()
    saved = table[1, 77].item()
    table[1, 77] = kc.shape[0] + 5
    graph.replay()
    rc, detail = mlt.last_device_error()
    assert rc == 7 and detail[1] == 77
    a, b = new[0], new[0] + new[1]
    assert torch.equal(o[:a], good[0][:a]) and torch.equal(o[b:], good[0][b:])
    table[1, 77] = saved
    k, v = gathered(kc, table[1], total[1]), gathered(vc, table[1], total[1])
    k[77 * bs: 78 * bs], v[77 * bs: 78 * bs] = 0, 0                      # (a block of zeros)
    check_rows(o[a:b], lse[a:b], rows_reference(q[a:b].double(), k, v, visible(new[1], total[1], True), float(np.float32(0.1))))
