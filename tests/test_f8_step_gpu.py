"""The 8-bit operators together, as a serving loop uses them: a prompt and decoding steps of one attention block (quantise,
project, rotate and append, attend, quantise, project back), every stage against the FP64 oracle on its actual inputs,
and the decoding step captured once and replayed."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2503_14985_b200 as mlt  # noqa: E402
from oracle import f8  # noqa: E402

from gpu_util import assert_device_healthy, to_f64  # noqa: E402

S, H, HKV, D, BS, WIDTH = 3, 8, 2, 64, 16, 384
QKV = (H + 2 * HKV) * D
MAX_BLOCKS, TOP = 8, 128


class Block:
    def __init__(self):
        g = torch.Generator().manual_seed(0)
        w = [torch.randn(r, k, generator=g).mul(k ** -0.5).to(torch.bfloat16).cuda() for r, k in ((QKV, WIDTH), (WIDTH, H * D))]
        self.w = [mlt.quantize_f8(x, block_rows=128) for x in w]
        ang = np.arange(TOP)[:, None] * 10000.0 ** (-np.arange(0, D, 2) / D)
        self.cos, self.sin = (torch.from_numpy(f(ang).astype(np.float32)).cuda() for f in (np.cos, np.sin))
        self.kc, self.vc = (torch.zeros(S * MAX_BLOCKS, HKV, BS, D, device="cuda").to(torch.float8_e4m3fn) for _ in range(2))
        self.ks, self.vs = (torch.zeros(S * MAX_BLOCKS, HKV, device="cuda") for _ in range(2))
        perm = torch.randperm(S * MAX_BLOCKS, generator=g).to(torch.int32)
        self.table = perm.view(S, MAX_BLOCKS).cuda()
        self.ws = torch.empty(mlt.paged_attn_f8_workspace_bytes(S, H, HKV, D), dtype=torch.uint8, device="cuda")

    def project_and_append(self, x, cu, ctx):
        q8, sq = mlt.quantize_f8(x)
        qkv = mlt.gemm_f8(q8, sq, *self.w[0])
        T = x.shape[0]
        parts = qkv[:, :H * D].view(T, H, D), qkv[:, H * D:(H + HKV) * D].view(T, HKV, D), qkv[:, (H + HKV) * D:].view(T, HKV, D)
        q = mlt.kv_append_f8(*parts, self.cos, self.sin, cu, ctx, self.table, self.kc, self.vc, self.ks, self.vs)
        return q8, sq, qkv, q

    def decode_step(self, x, cu, ctx, lens):
        q8, sq, qkv, q = self.project_and_append(x, cu, ctx)
        o, lse = mlt.paged_attn_decode_f8(q, self.kc, self.vc, self.ks, self.vs, self.table, lens, scale=D ** -0.5, workspace=self.ws)
        o8, so = mlt.quantize_f8(o.view(S, H * D))
        return q8, sq, qkv, q, o, lse, o8, so, mlt.gemm_f8(o8, so, *self.w[1])


def close(got, ref, mag, K):
    assert (np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + (K / 8 + 16) * 2.0 ** -23 * mag).all()  # as in the product's own test


def codes(t):
    return t.view(torch.uint8).cpu().numpy()


def check_step(b, x, ctx, lens, out):
    q8, sq, qkv, q, o, lse, o8, so, y = out
    want, scale = f8.quantize(to_f64(x), 1)
    assert np.array_equal(codes(q8), want) and np.array_equal(sq.cpu().numpy(), scale.T)
    close(to_f64(qkv), *f8.gemm(codes(q8), sq.cpu().numpy(), codes(b.w[0][0]), b.w[0][1].cpu().numpy()), WIDTH)
    raw = to_f64(qkv)
    ref = f8.rotate(raw[:, :H * D].reshape(S, H, D), ctx, b.cos.cpu().numpy(), b.sin.cpu().numpy(), False)
    assert (np.abs(to_f64(q) - ref) <= 2.0 ** -8 * np.abs(ref) + 12 * 2.0 ** -24 * np.abs(raw).max()).all()
    kc, vc = (f8.decode(codes(c)) * s.cpu().numpy().astype(np.float64)[..., None, None] for c, s in ((b.kc, b.ks), (b.vc, b.vs)))
    table = b.table.cpu().numpy()
    key = f8.rotate(raw[:, H * D:(H + HKV) * D].reshape(S, HKV, D), ctx, b.cos.cpu().numpy(), b.sin.cpu().numpy(), False)
    val = raw[:, (H + HKV) * D:].reshape(S, HKV, D)
    for s in range(S):
        blk, off = table[s, ctx[s] // BS], ctx[s] % BS
        for cache, x64, sc in ((kc, key[s], b.ks), (vc, val[s], b.vs)):
            step = sc[blk].double().cpu().numpy()[:, None]
            assert (np.abs(cache[blk, :, off] - x64) <= f8.half_step(x64 / step) * step + 12 * 2.0 ** -24 * np.abs(raw).max()).all()
    ro, rl, mag, dots = f8.paged_decode(to_f64(q), kc, vc, table, lens, float(np.float32(D ** -0.5)))
    d = (D * 2.0 ** -23 * dots)[..., None]
    assert (np.abs(to_f64(o) - ro) <= 2.0 ** -8 * np.abs(ro) + (2.0 ** -11 + 2.0 ** -16 + 2 * d) * mag).all()
    assert (np.abs(lse.cpu().numpy() - rl) <= d[..., 0] + 2.0 ** -19 * (1 + np.abs(rl))).all()
    want, scale = f8.quantize(to_f64(o).reshape(S, H * D), 1)
    assert np.array_equal(codes(o8), want) and np.array_equal(so.cpu().numpy(), scale.T)
    close(to_f64(y), *f8.gemm(codes(o8), so.cpu().numpy(), codes(b.w[1][0]), b.w[1][1].cpu().numpy()), H * D)


def test_prompt_then_decoding_steps_and_the_captured_step():
    b = Block()
    g = torch.Generator().manual_seed(1)
    new = np.array([40, 17, 1])
    cu = torch.tensor([0, 40, 57, 58], dtype=torch.int32, device="cuda")
    b.project_and_append(torch.randn(58, WIDTH, generator=g).to(torch.bfloat16).cuda(), cu, torch.zeros(S, dtype=torch.int32, device="cuda"))
    one = torch.arange(S + 1, dtype=torch.int32, device="cuda")
    x = torch.randn(S, WIDTH, generator=g).to(torch.bfloat16).cuda()
    ctx = torch.from_numpy(new.astype(np.int32)).cuda()
    lens = ctx + 1
    held = [t.clone() for t in (b.kc, b.vc, b.ks, b.vs)]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        captured = b.decode_step(x, one, ctx, lens)
    for step in range(18):  # every sequence passes from one cache block to the next at least once
        now = b.decode_step(x, one, ctx, lens)
        check_step(b, x, ctx.cpu().numpy(), lens.cpu().numpy(), now)
        after = [t.clone() for t in (b.kc, b.vc, b.ks, b.vs)]
        for t, was in zip((b.kc, b.vc, b.ks, b.vs), held):  # the same step again, replayed on the same state
            t.copy_(was)
        graph.replay()
        torch.cuda.synchronize()
        for a, c in zip(now + tuple(after), captured + (b.kc, b.vc, b.ks, b.vs)):
            assert torch.equal(a.contiguous().view(torch.uint8), c.contiguous().view(torch.uint8))
        held = after
        x.copy_(torch.randn(S, WIDTH, generator=g).to(torch.bfloat16))
        ctx += 1
        lens += 1
    assert_device_healthy()


def test_dependent_calls_back_to_back_and_one_by_one_give_the_same_bits():
    # the launches overlap the drain of the kernel before them: a call that read its inputs too early, or wrote before an earlier
    # call had read, would differ from the same chain with a synchronisation after every call
    g = torch.Generator().manual_seed(3)
    w = [mlt.quantize_f8((torch.randn(512, 512, generator=g) * 512 ** -0.5).to(torch.bfloat16).cuda(), block_rows=128) for _ in range(2)]
    x0 = torch.randn(48, 512, generator=g).to(torch.bfloat16).cuda()
    cu = torch.arange(49, dtype=torch.int32, device="cuda")
    cos, sin = (torch.randn(64, 32, generator=g).cuda() for _ in range(2))
    table = torch.randperm(48 * 4, generator=g).to(torch.int32).view(48, 4).cuda()
    ws = torch.empty(mlt.paged_attn_f8_workspace_bytes(48, 8, 2, 64), dtype=torch.uint8, device="cuda")
    q8, sq = torch.empty(48, 512, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn), torch.empty(4, 48, device="cuda")
    h = torch.empty(48, 512, dtype=torch.bfloat16, device="cuda")

    def chain(after):
        kc, vc = (torch.zeros(192, 2, 16, 64, device="cuda").to(torch.float8_e4m3fn) for _ in range(2))
        ks, vs = (torch.ones(192, 2, device="cuda") for _ in range(2))
        x, ctx = x0.clone(), torch.zeros(48, dtype=torch.int32, device="cuda")
        seen = []
        for step in range(40):
            mlt.quantize_f8(x, Q=q8, scales=sq); after()                      # buffers are written again while the call before
            mlt.gemm_f8(q8, sq, *w[step % 2], h); after()                     # may still be draining
            kv = h.view(48, 8, 64)
            mlt.kv_append_f8(kv, kv[:, 2:4], kv[:, 4:6], cos, sin, cu, ctx, table, kc, vc, ks, vs, Q_out=x.view(48, 8, 64)); after()
            ctx += 1; after()
            o, lse = mlt.paged_attn_decode_f8(x.view(48, 8, 64), kc, vc, ks, vs, table, ctx, scale=0.125, workspace=ws); after()
            x = o.view(48, 512)
            seen += [x, lse]
        torch.cuda.synchronize()
        return seen + [t.float() for t in (kc, vc, ks, vs)]

    one_by_one = chain(torch.cuda.synchronize)
    for _ in range(3):
        for a, b in zip(chain(lambda: None), one_by_one):
            assert torch.equal(a, b)
    assert_device_healthy()


@pytest.mark.parametrize("address", [False, True])
@pytest.mark.parametrize("op", ["quantize", "product", "append", "attend"])
def test_new_outputs_on_a_given_stream_are_not_memory_that_another_stream_still_writes(op, address):
    # blocks of the outputs' sizes go back to the allocator while the current stream is still going to write them: outputs of a
    # call on another stream must not lie there
    b = Block()
    g = torch.Generator().manual_seed(5)
    x = torch.randn(64, WIDTH, generator=g).to(torch.bfloat16).cuda()
    x8, sx = mlt.quantize_f8(x)
    cu = torch.tensor([0, 40, 57, 58], dtype=torch.int32, device="cuda")
    ctx = torch.zeros(S, dtype=torch.int32, device="cuda")
    lens = torch.tensor([40, 17, 1], dtype=torch.int32, device="cuda")
    q, k, v = (torch.randn(58, h, D, generator=g).to(torch.bfloat16).cuda() for h in (H, HKV, HKV))
    caches = b.kc, b.vc, b.ks, b.vs
    mlt.kv_append_f8(q, k, v, b.cos, b.sin, cu, ctx, b.table, *caches)
    run = {"quantize": lambda **kw: mlt.quantize_f8(x, **kw),
           "product": lambda **kw: (mlt.gemm_f8(x8, sx, *b.w[0], **kw),),
           "append": lambda **kw: (mlt.kv_append_f8(q, k, v, b.cos, b.sin, cu, ctx, b.table, *caches, **kw),),
           "attend": lambda **kw: mlt.paged_attn_decode_f8(q[:S].contiguous(), *caches, b.table, lens, scale=0.125, workspace=b.ws, **kw)}[op]
    want = [t.view(torch.uint8).clone() for t in run()]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    junk = [torch.empty_like(t) for t in want]
    torch.cuda._sleep(20_000_000)
    for t in junk:
        t.fill_(1)
    del junk, t
    got = run(stream=side.cuda_stream if address else side)
    torch.cuda.synchronize()
    assert [torch.equal(a.view(torch.uint8), w) for a, w in zip(got, want)] == [True] * len(want)
    assert_device_healthy()
