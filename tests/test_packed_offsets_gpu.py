"""Packed, paged and shared-prefix attention with offsets that do not ascend and key ranges that are cut: what is kept, and that nothing behind the
scratch is written.  Every case's plan is first run and checked on the CPU (packed_plan_util); the kernels go where the plan says."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2503_14985_b200 as mlt  # noqa: E402

from packed_plan_util import plan  # noqa: E402
from test_packed_plan import alternating  # noqa: E402


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
