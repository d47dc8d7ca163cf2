"""mlt_gemm_w4 at the longest K of 16, 8, 4, 2 and 1 rows per pass (bounds: test_gemm_w4_gpu)."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2503_14985_b200 as mlt  # noqa: E402

from gpu_util import assert_device_healthy  # noqa: E402
from test_gemm_w4_gpu import check, inputs  # noqa: E402


@pytest.mark.parametrize("rows,K,group", [(16, 34816, 32), (16, 38912, 128), (8, 71680, 32), (8, 75776, 64), (4, 157696, 128), (2, 309248, 64), (1, 583680, 32),
                                          (1, 618496, 64), (1, 636928, 128)])
def test_longest_k(rows, K, group):
    for M in (rows, rows + 1):
        for k in (K, K + group) if rows > 1 else (K,):
            x, w, s, z = inputs(M, 65, k, group, True, seed=K)
            c = mlt.gemm_w4(x, w, s, z)
            check(c, x, w, s, z, group)
    assert_device_healthy()
