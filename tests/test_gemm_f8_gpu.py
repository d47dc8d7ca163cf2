"""mlt_gemm_f8 against the FP64 oracle.

Tolerance of an element: half a BF16 step of the result, 2^-8 |C|, and the FP32 sums.  With u = 2^-23 (the tensor core may
truncate) and at most K / 8 + 16 dependent additions and multiplications (its adders, the weighting and the sum over the
blocks, the slices), the sums are off by at most (K / 8 + 16) * 2^-23 times the sum of the terms' magnitudes."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2503_14985_b200 as mlt  # noqa: E402
from oracle import f8  # noqa: E402

from gpu_util import assert_device_healthy, to_f64  # noqa: E402


def operands(M, N, K, seed, pad=0):
    rng = np.random.RandomState(seed)
    up = (K + 15) // 16 * 16 + pad

    def codes(rows):
        c = np.full((rows, up), 0x7F, np.uint8)  # NaN in the padding
        c[:, :K] = f8.encode(rng.randn(rows, K) * 60)
        return c
    kb, nb = -(-K // 128), -(-N // 128)
    sa = np.exp2(rng.randint(-12, 4, (kb, M))).astype(np.float32)
    sb = (rng.rand(nb, kb) * 3e-3 + 1e-4).astype(np.float32)
    return codes(M), sa, codes(N), sb


def dev8(c, K):
    return torch.from_numpy(c).cuda().view(torch.float8_e4m3fn)[:, :K]


def run(M, N, K, a, sa, b, sb, guard=True):
    ldc = (N + 7) // 8 * 8 + 8
    buf = torch.full((M + 2, ldc), 776.0, dtype=torch.bfloat16, device="cuda")
    C = buf[1:M + 1, :N]
    mlt.gemm_f8(dev8(a, K), torch.from_numpy(sa).cuda(), dev8(b, K), torch.from_numpy(sb).cuda(), C)
    assert_device_healthy()
    assert (buf[0] == 776).all() and (buf[-1] == 776).all() and (buf[:, N:] == 776).all(), "written outside C"
    return to_f64(C)


def check(got, ref, mag, K):
    tol = 2.0 ** -8 * np.abs(ref) + (K / 8 + 16) * 2.0 ** -23 * mag
    worst = float((np.abs(got - ref) / np.maximum(tol, 1e-300)).max())
    assert worst <= 1.0, worst


SHAPES = [(1, 1, 1), (1, 8, 16), (1, 64, 128), (5, 40, 129), (16, 200, 700), (16, 256, 4096), (31, 130, 1000), (33, 65, 383), (64, 512, 512),
          (100, 77, 300), (128, 128, 128), (127, 640, 900), (129, 129, 129), (200, 1000, 260), (256, 256, 1024), (300, 520, 4200),
          (511, 390, 777), (777, 500, 130), (1024, 1024, 512), (1500, 770, 256), (2100, 300, 384), (4, 9000, 300), (16, 64, 20000)]


@pytest.mark.parametrize("M,N,K", SHAPES)
def test_parity(M, N, K):
    a, sa, b, sb = operands(M, N, K, seed=M + N + K, pad=16)
    ref, mag = f8.gemm(a[:, :K], sa, b[:, :K], sb)
    check(run(M, N, K, a, sa, b, sb), ref, mag, K)


# (M, N, K): which kernel; ragged in every direction, a pair whose second CTA has no rows (M mod 256 <= 128), right edges that
# are no multiple of 8 columns, more tiles than SMs
BY_KERNEL = {(4930, 261, 3931): 2, (5249, 333, 3500): 2, (3176, 546, 3552): 2, (4100, 4100, 2050): 2, (128, 20000, 300): 1, (64, 40000, 300): 1,
             (300, 39999, 200): 1, (2600, 5101, 1000): 1, (100, 20003, 600): 0, (16, 28671, 1030): 0}


@pytest.mark.parametrize("M,N,K", BY_KERNEL)
def test_every_kernel(M, N, K):
    assert mlt.gemm_f8_plan(M, N, K, sm_count=0)["kernel"] == BY_KERNEL[M, N, K]
    a, sa, b, sb = operands(M, N, K, seed=M + N + K)
    got = run(M, N, K, a, sa, b, sb)
    rows = np.unique(np.concatenate([np.arange(min(M, 40)), np.arange(max(0, M - 150), M), np.random.RandomState(0).randint(0, M, 200)]))
    ref, mag = f8.gemm(a[rows][:, :K], sa[:, rows], b[:, :K], sb)
    check(got[rows], ref, mag, K)


def test_padded_scale_pitches():
    M, N, K = 150, 300, 500
    a, sa, b, sb = operands(M, N, K, seed=2)
    ref, mag = f8.gemm(a[:, :K], sa, b[:, :K], sb)
    wide_a, wide_b = torch.full((4, M + 5), float("nan"), device="cuda"), torch.full((3, 4 + 3), float("nan"), device="cuda")
    wide_a[:, 1:M + 1], wide_b[:, 2:6] = torch.from_numpy(sa), torch.from_numpy(sb)
    got = to_f64(mlt.gemm_f8(dev8(a, K), wide_a[:, 1:M + 1], dev8(b, K), wide_b[:, 2:6]))
    check(got, ref, mag, K)


def test_output_beyond_32_bit_offsets():
    # 2.3 G results (4.6 GB): the last rows lie beyond 2^31 elements; every row of A is the same but the last three
    M, N, K = 80000, 28680, 128
    a, sa, b, sb = operands(4, N, K, seed=6)
    A = dev8(a, K)[:1].view(torch.uint8).expand(M, K).contiguous()
    A[-3:] = dev8(a, K)[1:].view(torch.uint8)
    s = torch.full((1, M), float(sa[0, 0]), device="cuda")
    s[0, -3:] = torch.from_numpy(sa[0, 1:]).cuda()
    C = mlt.gemm_f8(A.view(torch.float8_e4m3fn), s, dev8(b, K), torch.from_numpy(sb).cuda())
    ref, mag = f8.gemm(a[:, :K], sa, b[:, :K], sb)
    check(to_f64(C[-4:]), ref, mag, K)
    assert torch.equal(C[:-3].min(0).values, C[0]) and torch.equal(C[:-3].max(0).values, C[0])
    assert_device_healthy()


@pytest.mark.parametrize("seed", range(24))
def test_random_shapes(seed):
    rng = np.random.RandomState(900 + seed)
    M, N, K = (int(np.exp(rng.uniform(0, np.log(hi)))) for hi in (1200, 3000, 3000))
    a, sa, b, sb = operands(M, N, K, seed=seed, pad=int(rng.choice([0, 16, 48])))
    ref, mag = f8.gemm(a[:, :K], sa, b[:, :K], sb)
    check(run(M, N, K, a, sa, b, sb), ref, mag, K)


@pytest.mark.parametrize("M,N,K", [(7, 100, 300), (130, 300, 640), (600, 700, 1024)])
def test_small_integers_are_exact(M, N, K):
    # entries -1, 0, 1 and power-of-two scales that differ along K: every sum is an integer multiple of 1/4 below 2^14,
    # held exactly in FP32, so only the final rounding to BF16 is left
    rng = np.random.RandomState(K)
    a, b = f8.encode(rng.randint(-1, 2, (M, K))), f8.encode(rng.randint(-1, 2, (N, K)))
    a, b = (np.pad(x, ((0, 0), (0, -K % 16))) for x in (a, b))
    sa, sb = np.exp2(rng.randint(-1, 2, (-(-K // 128), M))).astype(np.float32), np.exp2(rng.randint(-1, 2, (-(-N // 128), -(-K // 128)))).astype(np.float32)
    ref, _ = f8.gemm(a[:, :K], sa, b[:, :K], sb)
    assert np.abs(ref).max() < 2 ** 14
    want = torch.from_numpy(ref).to(torch.bfloat16).double().numpy()
    assert np.array_equal(run(M, N, K, a, sa, b, sb), want)


def test_scales_reach_their_blocks():
    # all ones; every scale a different power of two, so that a swapped or shifted scale shows
    M, N, K = 150, 300, 500
    one = np.pad(np.full((1, K), 0x38, np.uint8), ((0, 0), (0, -K % 16)))
    sa = np.exp2((np.arange(4)[:, None] * 3 + np.arange(M)[None, :]) % 11).astype(np.float32)
    sb = np.exp2((np.arange(3)[:, None] * 5 + np.arange(4)[None, :] * 2) % 7).astype(np.float32)
    a, b = np.repeat(one, M, 0), np.repeat(one, N, 0)
    ref, mag = f8.gemm(a[:, :K], sa, b[:, :K], sb)
    check(run(M, N, K, a, sa, b, sb), ref, mag, K)


def test_nan_and_zero_stay_in_their_rows_and_columns():
    M, N, K = 140, 140, 260
    a, sa, b, sb = operands(M, N, K, seed=5)
    a[3, 17], b[135, 259] = 0x7F, 0xFF
    sa[:, 77] = 0.0
    ref, mag = f8.gemm(a[:, :K], sa, b[:, :K], sb)
    got = run(M, N, K, a, sa, b, sb)
    assert np.isnan(got[3]).all() and np.isnan(got[:, 135]).all()
    rest = np.ones((M, N), bool); rest[3] = False; rest[:, 135] = False
    assert (got[77][rest[77]] == 0).all() and np.isfinite(got[rest]).all()
    check(got[rest], ref[rest], mag[rest], K)


def test_empty_problems():
    f = lambda *s: torch.zeros(*s, device="cuda").to(torch.float8_e4m3fn)  # noqa: E731
    one = lambda *s: torch.ones(*s, device="cuda")  # noqa: E731
    assert mlt.gemm_f8(f(0, 64), one(1, 0), f(8, 64), one(1, 1)).shape == (0, 8)
    assert mlt.gemm_f8(f(4, 64), one(1, 4), f(0, 64), one(0, 1)).shape == (4, 0)
    C = torch.full((4, 8), 5.0, dtype=torch.bfloat16, device="cuda")
    mlt.gemm_f8(f(4, 0), one(0, 4), f(8, 0), one(1, 0), C)
    assert (C == 0).all()


@pytest.mark.parametrize("M,N,K", [(16, 300, 4096), (300, 500, 900), (1024, 1030, 640)])
def test_repeatable_bits_on_any_stream_and_in_a_graph(M, N, K):
    a, sa, b, sb = operands(M, N, K, seed=8)
    args = [dev8(a, K), torch.from_numpy(sa).cuda(), dev8(b, K), torch.from_numpy(sb).cuda()]
    c0 = mlt.gemm_f8(*args)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c1 = mlt.gemm_f8(*args)
    c2 = mlt.gemm_f8(*args)  # at the same time as the call on the other stream
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        c3 = mlt.gemm_f8(*args)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    for c in (c1, c2, c3):
        assert torch.equal(c.view(torch.int16), c0.view(torch.int16))
    args[1].mul_(2.0)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(c3.float(), c0.float() * 2)


def test_quantized_operands_reproduce_the_bf16_product():
    # quantiser and product together: against the exact product of the BF16 matrices the error is the quantisation's, at
    # most 2^-4 of every factor (half an E4M3 step), plus the product's own
    M, N, K = 70, 390, 1000
    g = torch.Generator().manual_seed(3)
    x, w = (torch.randn(r, K, generator=g).to(torch.bfloat16).cuda() for r in (M, N))
    q, sq = mlt.quantize_f8(x)
    p, sp = mlt.quantize_f8(w, block_rows=128)
    got = to_f64(mlt.gemm_f8(q, sq, p, sp))
    fx, fw = to_f64(x), to_f64(w)
    mag = np.abs(fx) @ np.abs(fw).T
    lost = 2.0 ** -10 * 2.0 ** -6  # E4M3 subnormals: half a step, times the largest scale that unit-variance blocks get
    tol = (2 * 2.0 ** -4 + 2.0 ** -8) * mag + 2.0 ** -8 * np.abs(fx @ fw.T) + lost * (np.abs(fx).sum(1)[:, None] + np.abs(fw).sum(1)[None, :])
    assert (np.abs(got - fx @ fw.T) <= tol).all()
    assert np.linalg.norm(got - fx @ fw.T) <= 0.052 * np.linalg.norm(fx @ fw.T)  # two uniform roundings of up to 2^-4: rms at most 2^-4 * sqrt(2 / 3) = 0.051
