"""mlt_gemm_f8 at full sizes, every element against FP64 sums on the GPU (tolerance: test_gemm_f8_gpu.py), with finite operands only:
one NaN code among the weights would hide a column."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2503_14985_b200 as mlt  # noqa: E402

from gpu_util import assert_device_healthy  # noqa: E402


@pytest.mark.parametrize("M,N,K", [(16, 28672, 4096), (16, 4096, 28672), (777, 5000, 4200), (8192, 28672, 4096)])
def test_every_element(M, N, K):
    g = torch.Generator(device="cuda").manual_seed(M + N)
    kb, nb, up = -(-K // 128), -(-N // 128), (K + 15) // 16 * 16

    def codes(rows):
        return (torch.randn(rows, up, generator=g, device="cuda") * 100).clamp_(-448, 448).to(torch.float8_e4m3fn)[:, :K]

    A, B = codes(M), codes(N)
    sa = torch.exp2(torch.randint(-9, -5, (kb, M), generator=g, device="cuda").float())
    sb = torch.rand(nb, kb, generator=g, device="cuda") * 2e-4 + 1e-5
    C = mlt.gemm_f8(A, sa, B, sb)
    assert_device_healthy()
    assert torch.isfinite(C).all()
    col = torch.arange(K, device="cuda") // 128
    for n0 in range(0, N, 4096):                                # columns, a part at a time
        n1 = min(N, n0 + 4096)
        a = A.double() * sa.double().t()[:, col]
        b = B[n0:n1].double() * sb.double()[torch.arange(n0, n1, device="cuda") // 128][:, col]
        ref, mag = a @ b.t(), a.abs() @ b.abs().t()
        worst = (C[:, n0:n1].double() - ref).abs() / (2.0 ** -8 * ref.abs() + (K / 8 + 16) * 2.0 ** -23 * mag)
        assert float(worst.max()) <= 1.0, float(worst.max())
