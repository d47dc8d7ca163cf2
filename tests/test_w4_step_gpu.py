"""The BF16 serving operators together, as a serving loop uses them: a prompt that several sequences share (project with 4-bit weights, rotate
and append, attend over the cache), a second chunk per sequence, then decoding behind the shared prefix; every stage against 64 bits on its actual
inputs, and the decoding step captured and replayed."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2503_14985_b200 as mlt  # noqa: E402

from gpu_util import assert_device_healthy  # noqa: E402
from packed_util import check_rows, cu, gathered, rows_reference  # noqa: E402
from test_gemm_w4_gpu import check as check_w4  # noqa: E402
from test_packed_gpu import visible  # noqa: E402

H, HKV, D, BS, WIDTH, GROUP, S = 8, 2, 64, 16, 384, 64, 3
QKV = (H + 2 * HKV) * D
SCALE = float(np.float32(D ** -0.5))


def weights(n, k, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = torch.randint(0, 256, (n, k // 2), generator=g, device="cuda", dtype=torch.uint8)
    s = (torch.rand(n, k // GROUP, generator=g, device="cuda") * 0.01 + 0.005).to(torch.bfloat16)
    z = torch.randint(6, 10, (n, k // GROUP), generator=g, device="cuda", dtype=torch.uint8)
    return w, s, z


class Layer:
    def __init__(self):
        self.w_in, self.w_out = weights(QKV, WIDTH, 1), weights(WIDTH, H * D, 2)
        ang = np.arange(256)[:, None] * 10000.0 ** (-np.arange(0, D, 2) / D)
        self.cos, self.sin = (torch.from_numpy(f(ang).astype(np.float32)).cuda() for f in (np.cos, np.sin))
        self.kc, self.vc = (torch.full((40, HKV, BS, D), math.nan, device="cuda", dtype=torch.bfloat16) for _ in range(2))

    def project(self, x, at, ctx, table):
        qkv = mlt.gemm_w4(x, *self.w_in)
        check_w4(qkv, x, *self.w_in, GROUP) if not torch.cuda.is_current_stream_capturing() else None
        q, k, v = (qkv[:, a * D: b * D].unflatten(1, (-1, D)) for a, b in ((0, H), (H, H + HKV), (H + HKV, H + 2 * HKV)))
        return mlt.kv_append(q, k, v, self.cos, self.sin, at, ctx, table, self.kc, self.vc)

    def back(self, o):
        y = mlt.gemm_w4(o.view(-1, H * D), *self.w_out)
        check_w4(y, o.view(-1, H * D), *self.w_out, GROUP) if not torch.cuda.is_current_stream_capturing() else None
        return y


def test_shared_prompt_chunks_and_decoding():
    layer = Layer()
    g = torch.Generator(device="cuda").manual_seed(0)

    def x(n):
        return torch.randn(n, WIDTH, generator=g, device="cuda", dtype=torch.bfloat16)

    def check(o, lse, q, row, first, n):
        k, v = gathered(layer.kc, table[row], first + n), gathered(layer.vc, table[row], first + n)
        check_rows(o, lse, rows_reference(q.double(), k, v, visible(n, first + n, True), SCALE))

    prefix = 80                                                          # five blocks that all sequences have in common
    table = torch.arange(36, dtype=torch.int32, device="cuda").view(S, 12) + 1
    table[:, :5] = table[0, :5]
    ctx0 = torch.zeros(1, dtype=torch.int32, device="cuda")
    q = layer.project(x(prefix), cu([prefix]), ctx0, table[:1].contiguous())
    o, lse = mlt.paged_attn_prefill(q, layer.kc, layer.vc, cu([prefix]), ctx0, table[:1].contiguous(), scale=SCALE)
    check(o, lse, q, 0, 0, prefix)
    # packed rows give the same as the cache that was made of them
    k, v = (gathered(c, table[0], prefix).to(torch.bfloat16) for c in (layer.kc, layer.vc))
    po, plse = mlt.mha_packed_fwd(q, k, v, cu([prefix]), causal=True, scale=SCALE)
    assert torch.equal(po, o) and torch.equal(plse, lse)
    # a chunk of its own for each sequence
    new = [7, 0, 30]
    ctx = torch.full((S,), prefix, dtype=torch.int32, device="cuda")
    q = layer.project(x(37), cu(new), ctx, table)
    o, lse = mlt.paged_attn_prefill(q, layer.kc, layer.vc, cu(new), ctx, table, scale=SCALE)
    check(o[:7], lse[:7], q[:7], 0, prefix, 7)
    check(o[7:], lse[7:], q[7:], 2, prefix, 30)
    layer.back(o)
    # decoding
    ctx += torch.tensor(new, dtype=torch.int32, device="cuda")
    lens, one = ctx + 1, cu([1] * S)
    prefixes, groups = torch.tensor([prefix], dtype=torch.int32, device="cuda"), torch.tensor([0, S], dtype=torch.int32, device="cuda")
    ws = torch.empty(mlt.paged_attn_shared_workspace_bytes(S, 1, H, HKV, D), dtype=torch.uint8, device="cuda")
    inp = x(S)

    def step():
        q = layer.project(inp, one, ctx, table)
        o, lse = mlt.paged_attn_decode_shared(q, layer.kc, layer.vc, table, lens, prefixes, groups, scale=SCALE, workspace=ws)
        return q, o, lse, layer.back(o)

    step()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        captured = step()
    for _ in range(18):
        now = step()
        for s in range(S):
            check(now[1][s: s + 1], now[2][s: s + 1], now[0][s: s + 1], s, int(ctx[s]), 1)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(now, captured):
            assert torch.equal(a, b)
        inp.copy_(x(S))
        ctx += 1
        lens += 1
    assert_device_healthy()


def test_w4_on_streams_captured_and_behind_its_input():
    g = torch.Generator(device="cuda").manual_seed(4)
    w = weights(1000, 512, 3)
    x = torch.randn(5, 512, generator=g, device="cuda", dtype=torch.bfloat16)
    want = mlt.gemm_w4(x, *w)
    check_w4(want, x, *w, GROUP)
    torch.cuda.synchronize()
    got, streams = [], [torch.cuda.Stream() for _ in range(2)]
    for _ in range(4):
        for st in streams:
            with torch.cuda.stream(st):
                late = torch.zeros_like(x)
                torch.cuda._sleep(200_000)
                late += x
                got.append(mlt.gemm_w4(late, *w))
    got.append(mlt.gemm_w4(x, *w, stream=streams[1]))
    got.append(mlt.gemm_w4(x, *w, stream=streams[0].cuda_stream))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        c = mlt.gemm_w4(x, *w)
        got.append(mlt.gemm_w4(c[:, :512].contiguous(), *w))
    chained = mlt.gemm_w4(want[:, :512].contiguous(), *w)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(c, want) and torch.equal(got.pop(), chained)
    for y in got:
        assert torch.equal(y, want)
    assert_device_healthy()
