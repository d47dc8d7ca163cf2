"""mlt_mha_packed_fwd and mlt_paged_attn_prefill against plain attention in 64 bits (bounds: packed_util)."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2503_14985_b200 as mlt  # noqa: E402

from gpu_util import assert_device_healthy  # noqa: E402
from packed_util import check_rows, cu, gathered, guarded, paged, rows_reference  # noqa: E402


def visible(n, m, causal, device="cuda"):
    j, i = torch.arange(m, device=device)[None, :], torch.arange(n, device=device)[:, None]
    return j <= i + (m - n) if causal else torch.ones(n, m, dtype=torch.bool, device=device)


def packed_inputs(lens_q, lens_k, H, Hk, D, seed, scale_rows=1.0, pad=3):
    """Fused rows (one projection's output) for self-attention, separate tensors else; `pad` rows of NaN behind the last sequence."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    T, Tk = int(np.sum(lens_q)), int(np.sum(lens_k))
    if list(lens_q) == list(lens_k):
        x = torch.randn(T + pad, (H + 2 * Hk) * D + 8, generator=g, device="cuda", dtype=torch.bfloat16)
        x[T:] = math.nan
        q, k, v = (x[:, a: b].unflatten(1, (-1, D)) for a, b in ((0, H * D), (H * D, (H + Hk) * D), ((H + Hk) * D, (H + 2 * Hk) * D)))
    else:
        q = torch.randn(T + pad, H, D, generator=g, device="cuda", dtype=torch.bfloat16)
        k, v = (torch.randn(Tk + pad, Hk, D, generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2))
        q[T:], k[Tk:], v[Tk:] = math.nan, math.nan, math.nan
    return q, k, v


def run_packed(q, k, v, lens_q, lens_k, causal, scale, workspace="full", pitch=None):
    T, H, D = q.shape
    o, o_ok = guarded((T, H, D), torch.bfloat16, pitch)
    lse, lse_ok = guarded((T, H), torch.float32)
    need = mlt.mha_packed_workspace_bytes(T, len(lens_q), H, k.shape[1], D)
    ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    mlt.mha_packed_fwd(q, k, v, cu(lens_q), cu(lens_k), causal=causal, scale=scale, O=o, LSE=lse, workspace=ws[: need])
    torch.cuda.synchronize()
    o_ok()
    lse_ok()
    assert (ws[need:] == 0xFF).all(), "workspace overrun"
    n = int(np.sum(lens_q))
    assert (o[n:] == 776).all() and (lse[n:] == 776).all(), "rows of no sequence written"
    assert_device_healthy()
    return o, lse


PACKED = [
    ([1], None, 1, 1, 64, True), ([1], None, 8, 1, 128, True), ([37], None, 32, 8, 128, True), ([128], None, 4, 4, 128, True),
    ([129], None, 4, 4, 64, True), ([255, 256, 257], None, 2, 2, 128, True), ([1, 1, 1, 1, 1], None, 8, 2, 64, False),
    ([0, 5, 0, 300, 1, 0], None, 6, 2, 128, True), ([0, 5, 0, 300, 1, 0], None, 6, 2, 64, False), ([700, 64, 333], None, 14, 2, 128, True),
    ([700, 64, 333], None, 10, 2, 64, True), ([90, 1000], None, 16, 1, 128, True), ([40, 17], None, 128, 1, 64, True), ([50], None, 120, 4, 128, False),
    ([3], [5000], 32, 8, 128, True), ([3, 1], [5000, 70], 7, 1, 64, True), ([200], [9000], 8, 2, 128, True), ([40], [9000], 4, 4, 64, False),
    ([10, 200, 30], [4, 130, 0], 8, 2, 128, True), ([10, 200, 30], [4, 130, 0], 8, 2, 64, True), ([300], [100], 4, 2, 128, True),
    ([10, 200, 30], [4, 130, 0], 3, 1, 64, False), ([2000, 1500, 30, 1, 800], None, 8, 8, 64, True), ([2000, 1500, 30, 1, 800], None, 8, 8, 128, False),
]


@pytest.mark.parametrize("lens_q,lens_k,H,Hk,D,causal", PACKED)
def test_packed(lens_q, lens_k, H, Hk, D, causal):
    lens_k = lens_q if lens_k is None else lens_k
    q, k, v = packed_inputs(lens_q, lens_k, H, Hk, D, seed=H * 1000 + D + len(lens_q))
    scale = 1 / math.sqrt(D)
    o, lse = run_packed(q, k, v, lens_q, lens_k, causal, float(np.float32(scale)), pitch=H * D + 16)
    a = b = 0
    for n, m in zip(lens_q, lens_k):
        ref = rows_reference(q[a: a + n].double(), k[b: b + m].double(), v[b: b + m].double(), visible(n, m, causal), float(np.float32(scale)))
        check_rows(o[a: a + n], lse[a: a + n], ref, f"sequence of {n} queries, {m} keys")
        a, b = a + n, b + m


PREFILL = [
    ([1], [0], 8, 8, 64, 8), ([1], [0], 32, 8, 128, 16), ([5, 5, 5], [100, 0, 4000], 8, 1, 128, 16), ([100], [3000], 32, 8, 128, 32),
    ([1, 0, 300, 77], [7, 50, 129, 0], 12, 4, 128, 8), ([1, 0, 300, 77], [7, 50, 129, 0], 14, 2, 64, 32), ([700, 513], [1000, 0], 4, 2, 64, 16),
    ([1200, 130], [37, 2000], 8, 8, 128, 8), ([64] * 40, list(range(0, 400, 10)), 8, 2, 128, 16), ([2], [20000], 4, 1, 64, 8),
]


@pytest.mark.parametrize("new,ctx,H,Hk,D,bs", PREFILL)
def test_prefill(new, ctx, H, Hk, D, bs):
    T = sum(new)
    lens = np.add(new, ctx)
    kc, vc, table = paged(lens * (np.asarray(new) > 0), Hk, D, bs, seed=H + D + bs)
    g = torch.Generator(device="cuda").manual_seed(7)
    q = torch.randn(T + 2, H, D, generator=g, device="cuda", dtype=torch.bfloat16)
    q[T:] = math.nan
    scale = float(np.float32(1 / math.sqrt(D)))
    o, o_ok = guarded((T + 2, H, D), torch.bfloat16)
    lse, lse_ok = guarded((T + 2, H), torch.float32)
    need = mlt.mha_packed_workspace_bytes(T + 2, len(new), H, Hk, D)
    ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    mlt.paged_attn_prefill(q, kc, vc, cu(new), torch.tensor(ctx, dtype=torch.int32, device="cuda"), table, scale=scale, O=o, LSE=lse, workspace=ws[: need])
    torch.cuda.synchronize()
    o_ok()
    lse_ok()
    assert (ws[need:] == 0xFF).all() and (o[T:] == 776).all() and (lse[T:] == 776).all()
    assert_device_healthy()
    a = 0
    for s, n in enumerate(new):
        if n:
            m = int(lens[s])
            k, v = gathered(kc, table[s], m), gathered(vc, table[s], m)
            check_rows(o[a: a + n], lse[a: a + n], rows_reference(q[a: a + n].double(), k, v, visible(n, m, True), scale), f"sequence {s}")
        a += n
