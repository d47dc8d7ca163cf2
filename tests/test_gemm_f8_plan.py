"""The launch plan of mlt_gemm_f8 (host arithmetic, no GPU): every plan fits the kernel it names."""
import random

import pytest

import paper_2503_14985_b200 as mlt


def check(M, N, K, sm_count):
    p = mlt.gemm_f8_plan(M, N, K, sm_count)
    kb = -(-K // 128)
    assert p["kernel"] in (0, 1, 2)
    if p["kernel"]:
        assert p["tile_n"] == 256 and N >= 128 and p["cluster"] == 1  # the tensor map of C needs 8 columns at least
        return p
    assert p["tile_n"] % 16 == 0 and 16 <= p["tile_n"] <= 256
    assert p["cluster"] in (1, 2, 4, 8) and p["cluster"] <= kb, "an empty slice of K"
    rows = min(128, -(-M // 8) * 8)
    assert rows * (p["tile_n"] + 4) * 4 + 1024 <= p["smem"] <= 208 * 1024
    assert 2 * (rows + p["tile_n"]) * 128 + 1024 <= p["smem"], "two stages at least"
    return p


@pytest.mark.parametrize("sm_count", [2, 7, 132, 148])
def test_plans_are_valid_over_the_range(sm_count):
    rng = random.Random(sm_count)
    for _ in range(600):
        check(*(int(2 ** rng.uniform(0, 17)) for _ in range(3)), sm_count)
    for M, N, K in ((1, 1, 1), (128, 256, 128), (129, 127, 129), (1, 10 ** 6, 1), (10 ** 6, 1, 10 ** 5), (8192, 28672, 4096)):
        check(M, N, K, sm_count)


def test_kernels_by_shape():
    kinds = {s: check(*s, 148) for s in ((16, 28672, 4096), (16, 4096, 28672), (128, 28672, 4096), (200, 5000, 4200), (777, 5000, 4200),
                                         (4096, 4096, 4096), (8192, 28672, 4096), (1, 64, 64))}
    assert kinds[16, 28672, 4096]["kernel"] == 0 and kinds[16, 28672, 4096]["cluster"] == 1
    assert kinds[16, 4096, 28672]["kernel"] == 0 and kinds[16, 4096, 28672]["cluster"] > 1
    assert kinds[200, 5000, 4200]["kernel"] == 0 and kinds[128, 28672, 4096]["kernel"] == 1 and kinds[777, 5000, 4200]["kernel"] == 1
    assert kinds[4096, 4096, 4096]["kernel"] == 2 and kinds[8192, 28672, 4096]["kernel"] == 2


def test_refusals():
    for args in ((0, 1, 1, 148), (1, 0, 1, 148), (1, 1, 0, 148), (1, 1, 1, 1), (1, 1, 1, -2)):
        with pytest.raises(mlt.MltError):
            mlt.gemm_f8_plan(*args)
