"""mlt_kv_append and mlt_kv_append_f8 against the FP64 oracle.

Tolerances.  A rotated value is two products and a sum in FP32: off by at most 3 * 2^-24 (|a| + |b|) (cos and sin are at
most 1 and taken as the FP32 numbers they are).  BF16 adds half a step, 2^-8 of the value.  E4M3 under a scale s: half a
step at x / s, and the FP32 error may move a value over a border between steps, which costs no more than that error
on top.  A scale must be the power of two that the FP64 maximum asks for, up to the FP32 error of that maximum."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2503_14985_b200 as mlt  # noqa: E402
from oracle import f8  # noqa: E402

from gpu_util import assert_device_healthy, to_f64  # noqa: E402

SENTINEL = 776.0  # exact in BF16


def case(new, ctx, H, Hkv, D, R, bs, interleaved, seed, pad_tokens=0, spare=3):
    rng = np.random.RandomState(seed)
    new, ctx = np.asarray(new), np.asarray(ctx)
    S, T = len(new), int(new.sum()) + pad_tokens
    per = -(-(new + ctx) // bs)
    blocks = int(per.sum()) + spare
    order = rng.permutation(blocks)
    table = np.full((S, max(1, int(per.max()))), -1, np.int32)
    at = 0
    for s in range(S):
        table[s, :per[s]] = order[at:at + per[s]]
        at += per[s]
    g = torch.Generator().manual_seed(seed)
    width = (H + 2 * Hkv) * D
    qkv = (torch.randn(T, width, generator=g) * torch.exp2(torch.randint(-3, 4, (T, 1), generator=g).float())).to(torch.bfloat16).cuda()
    top = max(1, int((new + ctx).max()))
    ang = np.arange(top)[:, None] * 10000.0 ** (-np.arange(0, R, 2) / max(R, 1))
    return dict(S=S, T=T, H=H, Hkv=Hkv, D=D, R=R, bs=bs, inter=interleaved, new=new, ctx=ctx, cu=np.concatenate([[0], np.cumsum(new)]).astype(np.int32),
                table=table, blocks=blocks, q=qkv[:, :H * D].view(T, H, D), k=qkv[:, H * D:(H + Hkv) * D].view(T, Hkv, D),
                v=qkv[:, (H + Hkv) * D:].view(T, Hkv, D), cos=np.cos(ang).astype(np.float32), sin=np.sin(ang).astype(np.float32), rng=rng)


def dev_args(c):
    cs = [torch.from_numpy(c[n]).cuda() if c["R"] else None for n in ("cos", "sin")]
    return [*cs, *(torch.from_numpy(np.ascontiguousarray(c[n]).astype(np.int32)).cuda() for n in ("cu", "ctx", "table"))]


def err_bound(c, x):
    """3 * 2^-24 (|a| + |b|) for every element of a rotated pair."""
    h, mag = c["R"] // 2, np.zeros_like(x)
    for i in range(h):
        a, b = (2 * i, 2 * i + 1) if c["inter"] else (i, i + h)
        mag[:, :, a] = mag[:, :, b] = np.abs(x[:, :, a]) + np.abs(x[:, :, b])
    return 3 * 2.0 ** -24 * mag


def check_q(c, Qo, n):
    seq, pos = f8.positions(c["cu"], c["ctx"])
    raw = to_f64(c["q"])[:n]
    ref = f8.rotate(raw, pos, c["cos"], c["sin"], c["inter"])
    assert (np.abs(to_f64(Qo)[:n] - ref) <= 2.0 ** -8 * np.abs(ref) + 2 * err_bound(c, raw)).all()


CASES = [  # new, ctx, H, H_kv, D, rotary, block, interleaved
    ([1], [0], 1, 1, 64, 64, 16, False),
    ([1, 1, 1], [0, 15, 16], 4, 2, 128, 128, 16, False),
    ([1, 1, 1, 1], [7, 8, 100, 0], 8, 1, 64, 64, 8, True),
    ([40], [0], 2, 2, 128, 128, 32, True),
    ([33, 0, 1, 70, 0, 5], [0, 9, 31, 5, 0, 64], 4, 4, 64, 32, 32, False),
    ([16, 17, 15, 31], [16, 8, 1, 3], 4, 2, 128, 64, 16, True),
    ([100, 3], [11, 250], 8, 8, 64, 16, 16, False),
    ([20, 9], [0, 5], 3, 1, 128, 0, 8, False),
    ([9, 64, 2], [7, 1, 62], 6, 2, 128, 112, 16, False),
    ([129], [1000], 16, 2, 128, 128, 8, False),
    ([200, 1], [31, 33], 2, 1, 64, 48, 32, True),
]


@pytest.mark.parametrize("new,ctx,H,Hkv,D,R,bs,inter", CASES)
def test_bf16_cache(new, ctx, H, Hkv, D, R, bs, inter):
    c = case(new, ctx, H, Hkv, D, R, bs, inter, seed=sum(new) + D + bs, pad_tokens=3)
    n = int(c["cu"][-1])
    Kc, Vc = (torch.full((c["blocks"], Hkv, bs, D), SENTINEL, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    Qo = torch.full((c["T"], H, D), SENTINEL, dtype=torch.bfloat16, device="cuda")
    out = mlt.kv_append(c["q"], c["k"], c["v"], *dev_args(c), Kc, Vc, interleaved=inter, Q_out=Qo)
    assert_device_healthy()
    assert out is Qo and (Qo[n:] == SENTINEL).all()
    check_q(c, Qo, n)
    seq, pos = f8.positions(c["cu"], c["ctx"])
    blk, off = c["table"][seq, pos // bs], pos % bs
    touched = np.zeros((c["blocks"], bs), bool); touched[blk, off] = True
    assert touched.sum() == n
    for cache, x, rot in ((Kc, to_f64(c["k"])[:n], True), (Vc, to_f64(c["v"])[:n], False)):
        got = to_f64(cache)
        ref = f8.rotate(x, pos, c["cos"], c["sin"], inter) if rot else x
        tol = 2.0 ** -8 * np.abs(ref) + 2 * err_bound(c, x) if rot else 0.0
        assert (np.abs(got[blk, :, off] - ref) <= tol).all()
        assert (got.transpose(0, 2, 1, 3)[~touched] == SENTINEL).all(), "a position without a new token was written"


def filled(c, rng):
    """A cache whose blocks use their scales' ranges, the scales powers of two of different size."""
    shape = (c["blocks"], c["Hkv"], c["bs"], c["D"])
    scale = np.exp2(rng.randint(-12, 3, shape[:2])).astype(np.float32)
    codes = f8.encode(rng.randn(*shape) * 100)
    return torch.from_numpy(codes).cuda().view(torch.float8_e4m3fn), torch.from_numpy(scale).cuda(), codes, scale.astype(np.float64)


def check_f8(c, x, err, cache, scale, codes, old):
    """Codes and scales of one cache after an append of x [T, heads, D] (FP64, each off by at most err)."""
    got, s = cache.view(torch.uint8).cpu().numpy(), scale.cpu().numpy().astype(np.float64)
    bs, want_codes, seen = c["bs"], codes.copy(), np.zeros(old.shape, bool)
    for i in range(c["S"]):
        n, ctx = int(c["new"][i]), int(c["ctx"][i])
        for b in range(ctx // bs, -(-(ctx + n) // bs) if n else ctx // bs):
            p0, p1 = max(b * bs, ctx), min((b + 1) * bs, ctx + n)
            t0, blk = int(c["cu"][i]) + p0 - ctx, int(c["table"][i, b])
            held = p0 - b * bs
            for h in range(c["Hkv"]):
                seen[blk, h] = True
                rows, e = x[t0:t0 + p1 - p0, h], err[t0:t0 + p1 - p0, h]
                fin = np.where(np.isfinite(rows), np.abs(rows), 0.0)
                low, high = f8.block_scale((fin - e).max(initial=0.0)), f8.block_scale((fin + e).max())
                if held:
                    low, high = max(low, old[blk, h]), max(high, old[blk, h])
                assert low <= s[blk, h] <= high, (low, s[blk, h], high)
                moved = f8.encode(f8.decode(codes[blk, h, :held]) * (old[blk, h] / s[blk, h]))
                assert np.array_equal(got[blk, h, :held], moved), "tokens that the block held already"
                val = f8.decode(got[blk, h, held:held + p1 - p0]) * s[blk, h]
                live = np.isfinite(rows)
                tol = f8.half_step(rows[live] / s[blk, h]) * s[blk, h] + 2 * e[live]
                assert (np.abs(val[live] - rows[live]) <= tol).all()
                want_codes[blk, h, :held + p1 - p0] = got[blk, h, :held + p1 - p0]
    assert np.array_equal(got, want_codes), "a position without a token was written"
    assert np.array_equal(s[~seen], old[~seen]), "the scale of an untouched block was written"


@pytest.mark.parametrize("new,ctx,H,Hkv,D,R,bs,inter", CASES)
def test_f8_cache(new, ctx, H, Hkv, D, R, bs, inter):
    c = case(new, ctx, H, Hkv, D, R, bs, inter, seed=sum(new) + D + bs + 1, pad_tokens=2)
    n = int(c["cu"][-1])
    (Kc, ks, kcodes, kold), (Vc, vs, vcodes, vold) = filled(c, c["rng"]), filled(c, c["rng"])
    Qo = torch.full((c["T"], H, D), SENTINEL, dtype=torch.bfloat16, device="cuda")
    mlt.kv_append_f8(c["q"], c["k"], c["v"], *dev_args(c), Kc, Vc, ks, vs, interleaved=inter, Q_out=Qo)
    assert_device_healthy()
    assert (Qo[n:] == SENTINEL).all()
    check_q(c, Qo, n)
    _, pos = f8.positions(c["cu"], c["ctx"])
    k, v = to_f64(c["k"])[:n], to_f64(c["v"])[:n]
    check_f8(c, f8.rotate(k, pos, c["cos"], c["sin"], inter), err_bound(c, k), Kc, ks, kcodes, kold)
    check_f8(c, v, np.zeros_like(v), Vc, vs, vcodes, vold)


def test_f8_special_values():
    # V is not rotated: infinities saturate and do not set the scale, NaN stays in its element, a block of zeros gets the
    # smallest scale, and a block that held tokens keeps a larger scale
    c = case([6, 4], [0, 20], 1, 1, 64, 0, 16, False, seed=3)
    c["v"][0, 0, 3], c["v"][1, 0, 4], c["v"][2, 0, 5] = float("inf"), float("-inf"), float("nan")
    c["v"][6:] = 0
    c["k"][:] = 0
    (Kc, ks, kcodes, kold), (Vc, vs, vcodes, vold) = filled(c, c["rng"]), filled(c, c["rng"])
    mlt.kv_append_f8(None, c["k"], c["v"], None, None, *dev_args(c)[2:], Kc, Vc, ks, vs)
    assert_device_healthy()
    v = to_f64(c["v"])
    check_f8(c, v, np.zeros_like(v), Vc, vs, vcodes, vold)
    blk = c["table"][0, 0]
    got, s = f8.decode(Vc.view(torch.uint8).cpu().numpy()[blk, 0]), float(vs[blk, 0])
    assert got[0, 3] == 448 and got[1, 4] == -448 and np.isnan(got[2, 5]) and np.isnan(got[:6]).sum() == 1
    assert s == f8.block_scale(np.abs(v[:6][np.isfinite(v[:6])]).max())
    assert float(ks[blk, 0]) == 2.0 ** -64 and (f8.decode(Kc.view(torch.uint8).cpu().numpy()[blk, 0, :6]) == 0).all()
    assert float(vs[c["table"][1, 1], 0]) == vold[c["table"][1, 1], 0]


@pytest.mark.parametrize("cache8", [False, True])
def test_token_by_token_is_the_whole_prompt(cache8):
    # BF16: the same bits.  E4M3 under powers of two: the same scales, and the same values up to the underflow of values that
    # were stored under a smaller scale first (at most half a subnormal step of the last scale more)
    T, H, Hkv, D, bs = 45, 2, 2, 64, 16
    c = case([T], [0], H, Hkv, D, 64, bs, False, seed=21)
    cs = dev_args(c)
    dtype = torch.float8_e4m3fn if cache8 else torch.bfloat16

    def empty():
        caches = [torch.zeros(c["blocks"], Hkv, bs, D, device="cuda").to(dtype) for _ in range(2)]
        return caches + ([torch.zeros(c["blocks"], Hkv, device="cuda") for _ in range(2)] if cache8 else [])

    call = mlt.kv_append_f8 if cache8 else mlt.kv_append
    whole, steps = empty(), empty()
    q_all = call(c["q"], c["k"], c["v"], *cs, *whole)
    one = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    for t in range(T):
        q = call(c["q"][t:t + 1], c["k"][t:t + 1], c["v"][t:t + 1], cs[0], cs[1], one, torch.tensor([t], dtype=torch.int32, device="cuda"), cs[4], *steps)
        assert torch.equal(q[0].view(torch.int16), q_all[t].view(torch.int16))
    assert_device_healthy()
    if not cache8:
        assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(whole, steps))
        return
    for i in range(2):
        assert torch.equal(whole[2 + i], steps[2 + i])
        a, b = (f8.decode(x[i].view(torch.uint8).cpu().numpy()) for x in (whole, steps))
        assert (np.abs(a - b) <= 2.0 ** -9).all() and (a == b).mean() > 0.95
        assert np.array_equal(a[np.abs(a) >= 2.0 ** -5], b[np.abs(a) >= 2.0 ** -5])


@pytest.mark.parametrize("S", [31, 32, 33, 300, 1100])
def test_many_sequences(S):
    # the search for a warp's sequence takes several rounds; some sequences have nothing new
    rng = np.random.RandomState(S)
    new, ctx = rng.randint(0, 4, S), rng.randint(0, 40, S)
    c = case(new, ctx, 1, 1, 64, 64, 8, False, seed=S)
    n = int(c["cu"][-1])
    Kc, Vc = (torch.full((c["blocks"], 1, 8, 64), SENTINEL, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    Qo = mlt.kv_append(c["q"], c["k"], c["v"], *dev_args(c), Kc, Vc)
    assert_device_healthy()
    check_q(c, Qo, n)
    seq, pos = f8.positions(c["cu"], c["ctx"])
    got = to_f64(Vc)
    assert np.array_equal(got[c["table"][seq, pos // 8], :, pos % 8], to_f64(c["v"])[:n])
    touched = np.zeros((c["blocks"], 8), bool); touched[c["table"][seq, pos // 8], pos % 8] = True
    assert (got.transpose(0, 2, 1, 3)[~touched] == SENTINEL).all()


@pytest.mark.parametrize("cache8", [False, True])
def test_no_tokens_and_no_sequences(cache8):
    call = mlt.kv_append_f8 if cache8 else mlt.kv_append
    kinds = dict(device="cuda", dtype=torch.int32)
    caches = [torch.ones(3, 2, 16, 64, device="cuda").to(torch.float8_e4m3fn if cache8 else torch.bfloat16) for _ in range(2)]
    scales = [torch.ones(3, 2, device="cuda") for _ in range(2)] if cache8 else []
    q, k = torch.zeros(0, 4, 64, device="cuda", dtype=torch.bfloat16), torch.zeros(0, 2, 64, device="cuda", dtype=torch.bfloat16)
    assert call(q, k, k, None, None, torch.zeros(3, **kinds), torch.zeros(2, **kinds), torch.zeros(2, 2, **kinds), *caches, *scales).shape == (0, 4, 64)
    q, k = (torch.ones(5, h, 64, device="cuda", dtype=torch.bfloat16) for h in (4, 2))  # a batch of padding alone
    out = torch.full_like(q, 3.0)
    call(q, k, k, None, None, torch.zeros(3, **kinds), torch.zeros(2, **kinds), torch.zeros(2, 2, **kinds), *caches, *scales, Q_out=out)
    call(q, k, k, None, None, torch.zeros(1, **kinds), torch.zeros(0, **kinds), torch.zeros(0, 2, **kinds), *caches, *scales, Q_out=out)
    assert_device_healthy()
    assert (out == 3).all() and all((c.float() == 1).all() for c in caches + scales)


def test_many_query_heads_and_few():
    # 71 heads do not fill the steps of a warp; the angles are shared by all of them
    for H, Hkv, D in ((71, 1, 64), (40, 5, 128), (1, 1, 128)):
        c = case([37, 2], [5, 40], H, Hkv, D, D, 16, False, seed=H)
        Kc, Vc = (torch.zeros(c["blocks"], Hkv, 16, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        check_q(c, mlt.kv_append(c["q"], c["k"], c["v"], *dev_args(c), Kc, Vc), 39)
    assert_device_healthy()


def test_queries_in_place_and_without_queries():
    c = case([19, 30], [3, 0], 4, 2, 128, 128, 16, False, seed=30)
    args = dev_args(c)
    ref = [torch.zeros(c["blocks"], 2, 16, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    q_ref = mlt.kv_append(c["q"], c["k"], c["v"], *args, *ref)
    alone = [torch.zeros_like(ref[0]) for _ in range(2)]
    assert mlt.kv_append(None, c["k"], c["v"], *args, *alone) is None
    assert torch.equal(alone[0].view(torch.int16), ref[0].view(torch.int16)) and torch.equal(alone[1].view(torch.int16), ref[1].view(torch.int16))
    q = c["q"].contiguous()
    assert mlt.kv_append(q, c["k"], c["v"], *args, *alone, Q_out=q) is q
    assert torch.equal(q.view(torch.int16), q_ref.view(torch.int16))
    fused = c["q"]  # a view of the fused projection, rotated where it lies
    mlt.kv_append(fused, c["k"], c["v"], *args, *alone, Q_out=fused)
    assert torch.equal(fused.contiguous().view(torch.int16), q_ref.view(torch.int16))
    assert torch.equal(alone[0].view(torch.int16), ref[0].view(torch.int16))


@pytest.mark.parametrize("cache8", [False, True])
def test_bad_tables_and_positions_are_reported_and_not_written(cache8):
    c = case([20, 20, 20, 20, 20], [0, 8, 5, 40, 30], 2, 1, 64, 64, 16, False, seed=40)
    dtype = torch.float8_e4m3fn if cache8 else torch.bfloat16
    call = mlt.kv_append_f8 if cache8 else mlt.kv_append

    def caches():
        x = [torch.full((c["blocks"], 1, 16, 64), 1.5, device="cuda").to(dtype) for _ in range(2)]
        return x + ([torch.ones(c["blocks"], 1, device="cuda") for _ in range(2)] if cache8 else [])

    cos, sin, cu, ctx, table = dev_args(c)
    good = caches()
    q_good = call(c["q"], c["k"], c["v"], cos, sin, cu, ctx, table, *good)
    assert mlt.last_device_error()[0] == 0

    bad = table.clone()
    bad[0, 1], bad[2, 0] = c["blocks"] + 5, -1
    got = caches()
    q = call(c["q"], c["k"], c["v"], cos, sin, cu, ctx, bad, *got)
    status, detail = mlt.last_device_error()
    assert status == 7 and (detail[1], detail[2]) in ((1, 0), (0, 2))
    assert torch.equal(q.view(torch.int16), q_good.view(torch.int16))  # the queries do not need the table
    left = [int(c["table"][0, 1]), int(c["table"][2, 0])]
    same = [b for b in range(c["blocks"]) if b not in left]
    assert (got[0][left].float() == 1.5).all() and (got[1][left].float() == 1.5).all()
    assert torch.equal(got[0][same].float(), good[0][same].float()) and torch.equal(got[1][same].float(), good[1][same].float())

    narrow = table[:, :2].contiguous()  # sequences 3 and 4 need a third and fourth block that the table does not have
    got = caches()
    call(c["q"], c["k"], c["v"], cos, sin, cu, ctx, narrow, *got)
    assert mlt.last_device_error()[0] == 7
    out = [int(b) for s in (3, 4) for b in c["table"][s, 2:] if b >= 0]
    assert (got[0][out].float() == 1.5).all()

    for cu2, ctx2, cos2, skipped in ((cu, torch.tensor([0, -1, 5, 40, 30], dtype=torch.int32, device="cuda"), cos, 1),
                                     (cu, ctx, cos[:59], 3),                       # position 59 has no row
                                     (torch.tensor([0, 20, 40, 60, 80, 101], dtype=torch.int32, device="cuda"), ctx, cos, 4)):
        got = caches()
        Qo = torch.full_like(q_good, SENTINEL)
        call(c["q"], c["k"], c["v"], cos2, sin[:cos2.shape[0]], cu2, ctx2, table, *got, Q_out=Qo)
        status, detail = mlt.last_device_error()
        assert status == 9 and detail[1] == skipped
        live = [t for t in range(100) if t // 20 != skipped]
        assert (Qo[skipped * 20:skipped * 20 + 20] == SENTINEL).all()
        assert torch.equal(Qo[live].view(torch.int16), q_good[live].view(torch.int16))
        mine = [int(b) for b in c["table"][skipped] if b >= 0]
        assert (got[0][mine].float() == 1.5).all() and (got[1][mine].float() == 1.5).all()
        assert mlt.last_device_error()[0] == 0  # cleared


def test_blocks_beyond_32_bit_element_offsets():
    # a BF16 cache of 2.4 G elements: the last blocks lie beyond 2^31 elements
    D, Hkv, bs, blocks = 128, 8, 16, 147000
    Kc = torch.empty(blocks, Hkv, bs, D, dtype=torch.bfloat16, device="cuda")
    Vc = torch.empty_like(Kc)
    table = torch.tensor([[blocks - 1], [blocks - 2]], dtype=torch.int32, device="cuda")
    k = torch.randn(2, Hkv, D, device="cuda").to(torch.bfloat16)
    cu, ctx = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda"), torch.tensor([3, 15], dtype=torch.int32, device="cuda")
    mlt.kv_append(None, k, k, None, None, cu, ctx, table, Kc, Vc)
    assert_device_healthy()
    assert torch.equal(Kc[-1, :, 3], k[0]) and torch.equal(Vc[-2, :, 15], k[1])


@pytest.mark.parametrize("cache8", [False, True])
def test_other_stream_and_captured_graph(cache8):
    # a captured step whose lengths are advanced on the device between replays, as a decoding loop does it
    c = case([1, 1, 1], [14, 3, 31], 4, 2, 64, 64, 16, False, seed=50, spare=8)
    table = np.full((3, 4), -1, np.int32); table[:, :] = np.arange(12).reshape(3, 4)
    c["table"], c["blocks"] = table, 12
    ang = np.arange(64)[:, None] * 10000.0 ** (-np.arange(0, 64, 2) / 64)
    c["cos"], c["sin"] = np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)
    dtype = torch.float8_e4m3fn if cache8 else torch.bfloat16
    call = mlt.kv_append_f8 if cache8 else mlt.kv_append

    def caches():
        x = [torch.zeros(12, 2, 16, 64, device="cuda").to(dtype) for _ in range(2)]
        return x + ([torch.ones(12, 2, device="cuda") for _ in range(2)] if cache8 else [])

    cos, sin, cu, ctx, tab = dev_args(c)
    ref, got, own = caches(), caches(), caches()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ctx_g = ctx.clone()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        q_g = call(c["q"], c["k"], c["v"], cos, sin, cu, ctx_g, tab, *got)
    for step in range(5):
        q_r = call(c["q"], c["k"], c["v"], cos, sin, cu, ctx + step, tab, *ref)
        with torch.cuda.stream(side):
            q_s = call(c["q"], c["k"], c["v"], cos, sin, cu, ctx + step, tab, *own)
        graph.replay()
        ctx_g += 1
        torch.cuda.synchronize()
        assert torch.equal(q_r.view(torch.int16), q_g.view(torch.int16)) and torch.equal(q_r.view(torch.int16), q_s.view(torch.int16))
    for a, b, d in zip(ref, got, own):
        assert torch.equal(a.float(), b.float()) and torch.equal(a.float(), d.float())
    assert_device_healthy()
