"""mlt_gemm_w4 over the whole range of BF16 activations and scales, against the definition in 64 bits.

The bound of test_gemm_w4_gpu, and for small numbers 2^-138 |scale| per group (its sum is rounded there) and 2^-138 per group and warp (what
the sums over groups and warps are rounded at), and half of the smallest BF16 number, 2^-134.
"""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2503_14985_b200 as mlt  # noqa: E402

from gpu_util import assert_device_healthy  # noqa: E402


def reference(x, w, s, z, group):
    M, K = x.shape
    N = w.shape[0]
    q = torch.stack([w & 15, w >> 4], -1).reshape(N, K).double()
    zz = torch.full((N, K // group), 8.0, dtype=torch.float64, device="cuda") if z is None else z.double()
    wd = ((q.view(N, -1, group) - zz[..., None]) * s.double()[..., None]).reshape(N, K)
    T = x.double().abs().view(M, -1, group).sum(-1) @ s.double().abs().t()
    ref = x.double() @ wd.t()
    small = (s.double().abs().sum(-1) + K // group + 24) * 2.0 ** -138 + 2.0 ** -134
    return ref, 2.0 ** -8 * ref.abs() + 15 * (group / 8 + group * 2.0 ** -15 + K / group + 24) * 2.0 ** -23 * T + small


def inputs(M, N, K, group, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(M, K, generator=g, device="cuda").clamp(-3.9, 3.9) / 3.9      # (below 1)
    w = torch.randint(0, 256, (N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    s = (torch.rand(N, K // group, generator=g, device="cuda") - 0.3)
    z = torch.randint(0, 16, (N, K // group), generator=g, device="cuda", dtype=torch.uint8)
    return x, w, s, z


# exponents of x and of the scales, over which the groups go
@pytest.mark.parametrize("x_exp,s_exp", [((118, 128), (-40, -30)), ((128, 128), (-16, -14)), ((90, 100), (20, 20)), ((100, 100), (14, 16)), ((-20, 20), (80, 90)),
                                         ((-126, -112), (0, 8)), ((-133, -127), (20, 40)), ((-133, 128), (-120, -20)), ((-60, 60), (-60, 60)), ((0, 0), (110, 112)),
                                         ((-128, -124), (-3, 3))])
@pytest.mark.parametrize("M,N,K,group", [(1, 70, 1024, 128), (16, 50, 512, 32), (5, 40, 2048, 64)])
def test_range(x_exp, s_exp, M, N, K, group):
    x, w, s, z = inputs(M, N, K, group, seed=M)
    g = torch.Generator(device="cuda").manual_seed(K)
    ex = torch.randint(x_exp[0], x_exp[1] + 1, (M, K // group, 1), generator=g, device="cuda").double()
    es = torch.randint(s_exp[0], s_exp[1] + 1, (N, K // group), generator=g, device="cuda").double()
    x = (x.double().view(M, -1, group) * 2.0 ** ex).view(M, K).clamp(-3.38e38, 3.38e38).to(torch.bfloat16)
    s = (s.double() * 2.0 ** es).clamp(-3.38e38, 3.38e38).to(torch.bfloat16)
    assert torch.isfinite(x).all() and torch.isfinite(s).all()
    for zeros in (z, None):
        ref, bound = reference(x, w, s, zeros, group)
        c = mlt.gemm_w4(x, w, s, zeros)
        fits = ref.abs() + bound < 2.0 ** 127
        assert fits.any()
        err = (c.double() - ref).abs()
        assert torch.isfinite(c[fits]).all() and not torch.isnan(c).any()
        assert (err[fits] <= bound[fits]).all(), f"off by {(err[fits] / bound[fits]).max().item():.3f} of the bound"
    assert_device_healthy()


def test_largest_x_of_one_sign_and_weights_without_effect():
    """128 of the largest BF16 numbers in a group add up beyond FP32; weights at the zero point give 0 whatever x and scale are."""
    x = torch.full((3, 256), 3.3895313892515355e38, device="cuda", dtype=torch.bfloat16)
    x[1, 128:] = -x[1, 128:]
    x[2, ::2] = 0
    w = torch.full((40, 128), 0x55, device="cuda", dtype=torch.uint8)
    w[20:] = 0x66
    s = torch.full((40, 2), 2.0 ** -12, device="cuda", dtype=torch.bfloat16)
    s[10:20] = 3.3895313892515355e38
    z = torch.full((40, 2), 5, device="cuda", dtype=torch.uint8)
    c = mlt.gemm_w4(x, w, s, z)
    assert (c[:, :20] == 0).all()
    ref, bound = reference(x, w, s, z, 128)
    assert torch.isfinite(c).all() and ((c.double() - ref).abs() <= bound)[:, 20:].all()
    assert_device_healthy()
