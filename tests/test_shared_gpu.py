"""mlt_paged_attn_decode_shared against plain attention in 64 bits (bounds: packed_util)."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2503_14985_b200 as mlt  # noqa: E402

from gpu_util import assert_device_healthy  # noqa: E402
from packed_util import check_rows, gathered, guarded, paged, rows_reference  # noqa: E402


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def run_shared(q, kc, vc, table, lens, prefix, groups, scale):
    S, H, D = q.shape
    o, o_ok = guarded((S, H, D), torch.bfloat16)
    lse, lse_ok = guarded((S, H), torch.float32)
    need = mlt.paged_attn_shared_workspace_bytes(S, len(prefix), H, kc.shape[1], D)
    ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    mlt.paged_attn_decode_shared(q, kc, vc, table, i32(lens), i32(prefix), i32(groups), scale=scale, O=o, LSE=lse, workspace=ws[: need])
    torch.cuda.synchronize()
    o_ok()
    lse_ok()
    assert (ws[need:] == 0xFF).all(), "workspace overrun"
    return o, lse


# lengths in all; prefix of each group; the groups' offsets
SHARED = [
    ([20, 21, 300], [16], [0, 3], 8, 1, 64, 8), ([0, 16, 17, 0, 33, 5], [16], [0, 6], 8, 2, 128, 16), ([700, 600, 512, 513], [512], [0, 4], 32, 8, 128, 16),
    ([700, 600, 100, 513, 40, 900], [300, 33], [0, 2, 4], 4, 4, 128, 32), ([2000] * 3 + [1999] * 30, [1990, 100], [1, 20, 30], 16, 2, 64, 8),
    ([5000 + 3 * i for i in range(40)], [5000], [0, 40], 32, 8, 128, 16), ([9000 + i for i in range(70)], [9001, 9000], [0, 30, 70], 8, 4, 128, 16),
    ([30, 40, 50], [0, 7], [0, 1, 3], 8, 8, 64, 8), ([1], [1], [0, 1], 1, 1, 64, 8), ([130] * 200, [128], [0, 200], 8, 1, 64, 32),
    ([40] * 1100, [32], [0, 1100], 8, 2, 64, 16), ([40 + i % 5 for i in range(1100)], [32, 32], [0, 500, 1000], 4, 2, 128, 8),
]


@pytest.mark.parametrize("lens,prefix,groups,H,Hk,D,bs", SHARED)
def test_shared(lens, prefix, groups, H, Hk, D, bs):
    S = len(lens)
    share = [(list(range(groups[g], groups[g + 1])), prefix[g] // bs) for g in range(len(prefix))]
    kc, vc, table = paged(lens, Hk, D, bs, seed=S + D, share=share)
    gen = torch.Generator(device="cuda").manual_seed(S)
    q = torch.randn(S, H, D, generator=gen, device="cuda", dtype=torch.bfloat16)
    scale = float(np.float32(1 / math.sqrt(D)))
    o, lse = run_shared(q, kc, vc, table, lens, prefix, groups, scale)
    assert_device_healthy()
    for s in list(range(S)) if S < 100 else list(range(0, S, 37)) + [S - 1]:
        n = lens[s]
        ref = rows_reference(q[s: s + 1].double(), gathered(kc, table[s], n), gathered(vc, table[s], n), torch.ones(1, n, dtype=torch.bool, device="cuda"), scale)
        check_rows(o[s: s + 1], lse[s: s + 1], ref, f"sequence {s}")


@pytest.mark.parametrize("prefix,groups", [([], [0]), ([15], [0, 4]), ([64, 0], [1, 2, 4])])
def test_without_whole_blocks_in_common(prefix, groups):
    """No group, groups without a whole block in common, a group of one: plain decode (and mlt_paged_attn_decode within both paths' bounds)."""
    lens, H, Hk, D, bs = [100, 7, 0, 2000], 16, 4, 128, 16
    kc, vc, table = paged(lens, Hk, D, bs, seed=3)
    if groups[0] == 1:
        table[1, :4] = table[3, :4]  # (the second sequence is shorter than its prefix: its row goes on all the same)
    q = torch.randn(4, H, D, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda", dtype=torch.bfloat16)
    o, lse = run_shared(q, kc, vc, table, lens, prefix, groups, 0.1)
    ws = torch.empty(mlt.paged_attn_workspace_bytes(4, H, D), dtype=torch.uint8, device="cuda")
    plain, plain_lse = mlt.paged_attn_decode(q, kc, vc, table, i32(lens), scale=0.1, workspace=ws)
    for s, n in enumerate(lens):
        ref = rows_reference(q[s: s + 1].double(), gathered(kc, table[s], n), gathered(vc, table[s], n), torch.ones(1, n, dtype=torch.bool, device="cuda"), 0.1)
        check_rows(o[s: s + 1], lse[s: s + 1], ref, f"sequence {s}")
        check_rows(plain[s: s + 1], plain_lse[s: s + 1], ref, f"sequence {s}, plain")
    assert_device_healthy()
