"""mlt_gemm_w4 against the definition in 64 bits.

Bound of an output element, with T = sum over groups of |scale| sum |x| in them: half a BF16 step, 2^-8 |C|; a group's products are exact
and its partial sums at most 15 sum |x|, so each of its at most group / 8 additions costs at most 2^-23 of that: group / 8 * 15 * 2^-23 T;
an element of x below 2^-27 of its group's largest is off by at most 2^-38 of that one: 15 * group * 2^-38 T; scales, and the sums over
groups and warps, at most K / group + 24 roundings of 2^-23 in terms of 15 T: (K / group + 24) * 15 * 2^-23 T.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2503_14985_b200 as mlt  # noqa: E402

from gpu_util import assert_device_healthy  # noqa: E402


def inputs(M, N, K, group, zeros, seed, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(M, K + 8 * pad, generator=g, device="cuda", dtype=torch.bfloat16)
    w = torch.randint(0, 256, (N, (K // 2 + 15) // 16 * 16 + 16 * pad), generator=g, device="cuda", dtype=torch.uint8)
    s = (torch.rand(N, K // group + pad, generator=g, device="cuda") * 0.02 - 0.005).to(torch.bfloat16)
    z = torch.randint(0, 16, (N, K // group + pad), generator=g, device="cuda", dtype=torch.uint8) if zeros else None
    if pad:
        x[:, K:] = float("nan")
        s[:, K // group:] = float("nan")
    return x[:, :K], w[:, : K // 2], s[:, : K // group], None if z is None else z[:, : K // group]


def check(c, x, w, s, z, group):
    M, K = x.shape
    N = w.shape[0]
    q = torch.stack([w & 15, w >> 4], -1).reshape(N, K).double()
    zz = torch.full((N, K // group), 8.0, dtype=torch.float64, device="cuda") if z is None else z.double()
    wd = ((q.view(N, -1, group) - zz[..., None]) * s.double()[..., None]).reshape(N, K)
    ref = x.double() @ wd.t()
    T = x.double().abs().view(M, -1, group).sum(-1) @ s.double().abs().t()
    bound = 2.0 ** -8 * ref.abs() + 15 * (group / 8 + group * 2.0 ** -15 + K / group + 24) * 2.0 ** -23 * T + 1e-30
    err = (c.double() - ref).abs()
    assert torch.isfinite(c).all()
    assert (err <= bound).all(), f"off by {(err / bound).max().item():.3f} of the bound"


CASES = [(1, 1, 32, 32, False), (1, 33, 64, 64, True), (1, 40, 128, 128, True), (3, 100, 96, 32, True), (8, 64, 192, 64, False), (9, 65, 1152, 128, True),
         (16, 128, 4096, 128, False), (1, 4096, 4096, 128, True), (2, 5000, 2048, 64, True), (5, 1000, 4160, 32, False), (16, 4096, 28672, 64, True),
         (13, 96, 28672, 128, True), (17, 200, 512, 32, True), (33, 777, 4096, 128, False), (64, 300, 1024, 64, True), (100, 64, 256, 128, True),
         (7, 28672, 896, 128, True), (16, 50, 102400, 32, True), (1, 31, 200000 // 128 * 128, 128, False), (16, 2000, 100352, 128, True)]


@pytest.mark.parametrize("M,N,K,group,zeros", CASES)
def test_gemm_w4(M, N, K, group, zeros):
    for pad in (0, 3):
        x, w, s, z = inputs(M, N, K, group, zeros, seed=M * 7 + N + pad, pad=pad)
        buf = torch.full((M + 2, N + 5), 776.0, dtype=torch.bfloat16, device="cuda")
        c = buf[1: M + 1, 2: N + 2]
        mlt.gemm_w4(x, w, s, z, c)
        torch.cuda.synchronize()
        check(c, x, w, s, z, group)
        buf[1: M + 1, 2: N + 2] = 776.0
        assert (buf == 776).all(), "written outside C"
    again = mlt.gemm_w4(x, w, s, z)
    assert torch.equal(again, mlt.gemm_w4(x, w, s, z)), "two calls differ"
    assert_device_healthy()


@pytest.mark.parametrize("M,N,K,group", [(16, 80000, 4096, 128), (15, 10000, 28672, 32), (16, 10000, 4864, 128), (11, 5000, 9728, 64)])
def test_several_sets_of_row_tiles(M, N, K, group):
    """A CTA's row tiles are more than the memory beside x holds sums of (the first two, with and without clusters), or would be."""
    x, w, s, z = inputs(M, N, K, group, True, seed=N)
    c = mlt.gemm_w4(x, w, s, z)
    check(c, x, w, s, z, group)
    assert torch.equal(c, mlt.gemm_w4(x, w, s, z)), "two calls differ"
    assert_device_healthy()


def test_exact_on_small_integers():
    """Whole numbers that BF16 and FP32 hold: every output is exact."""
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randint(-1, 2, (4, 256), generator=g, device="cuda").to(torch.bfloat16) * (torch.rand(4, 256, generator=g, device="cuda") < 0.1)
    w = torch.randint(0, 256, (70, 128), generator=g, device="cuda", dtype=torch.uint8)
    s = torch.ones(70, 2, device="cuda", dtype=torch.bfloat16)
    z = torch.randint(0, 16, (70, 2), generator=g, device="cuda", dtype=torch.uint8)
    q = torch.stack([w & 15, w >> 4], -1).reshape(70, 2, 128).double() - z.double()[..., None]
    ref = x.double() @ q.reshape(70, 256).t()
    assert ref.abs().max() <= 256
    assert torch.equal(mlt.gemm_w4(x.to(torch.bfloat16), w, s, z).double(), ref)


def test_empty():
    x = torch.zeros(3, 0, device="cuda", dtype=torch.bfloat16)
    w, s = torch.zeros(5, 0, device="cuda", dtype=torch.uint8), torch.zeros(5, 0, device="cuda", dtype=torch.bfloat16)
    c = torch.full((3, 5), 7.0, device="cuda", dtype=torch.bfloat16)
    mlt.gemm_w4(x, w, s, None, c)
    assert (c == 0).all()
    assert mlt.gemm_w4(x[:0], w, s).shape == (0, 5) and mlt.gemm_w4(x, w[:0], s[:0]).shape == (3, 0)
    assert_device_healthy()
