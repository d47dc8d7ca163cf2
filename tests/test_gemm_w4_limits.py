"""mlt_gemm_w4 refuses what it has no grid or memory for before any CUDA call (no GPU needed).

Every call has a misaligned x, which is refused next (status 3): nothing is ever launched."""
import pytest

import __graft_entry__ as entry
from paper_2503_14985_b200 import binding


@pytest.fixture(scope="module", autouse=True)
def lib():
    entry.build()


def call(M, K, group, **kw):
    a = dict(X=8, W=16, scales=16, zeros=0, C=16, M=M, N=100, K=K, group=group, ldx=K, ldw=(K // 2 + 15) // 16 * 16, lds=K // group, ldz=0, ldc=100)
    a.update(kw)
    return binding.gemm_w4_raw(**a)


# the longest K of 16, 8, 4, 2 and 1 rows per pass
@pytest.mark.parametrize("group,longest", [(32, (34816, 71680, 145408, 290816, 583680)), (64, (36864, 75776, 153600, 309248, 618496)),
                                           (128, (38912, 77824, 157696, 317440, 636928))])
def test_more_passes_than_a_grid_has(group, longest):
    for i, K in enumerate(longest):
        rows = 16 >> i
        most = min(65535 * rows, 1 << 19)
        assert call(most + 1, K, group) == 2 and call(most, K, group) == 3 and call(1, K, group) == 3
        if i < 4:                                                       # one group more: half as many rows per pass
            most = min(65535 * rows // 2, 1 << 19)
            assert call(most + 1, K + group, group) == 2 and call(most, K + group, group) == 3


def test_a_row_that_fits_no_cluster():
    for group, K in ((32, 583680), (64, 618496), (128, 636928)):
        assert call(1, K, group) == 3
        assert call(1, K + group, group) == 2
        assert call(1, (2 ** 31 - 2048) // 128 * 128, group) == 2
