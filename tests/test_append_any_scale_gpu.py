"""mlt_kv_append_f8 into blocks whose scale, set by someone else, is no power of two: a value still has one rounding, to the E4M3
value nearest to x / s, and a token that moves to a larger scale one more.  Scales are made such that the quotients lie next to the
middle between two E4M3 values, on either side, where any rounding in between goes wrong.  The codes must be equal: the quotient
of a 24-bit and an 8-bit number is at least 2^-33 of itself away from such a middle if it is not the middle, which FP64 resolves."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2503_14985_b200 as mlt  # noqa: E402
from oracle import f8  # noqa: E402

from gpu_util import assert_device_healthy, to_f64  # noqa: E402

S, HKV, BS, HELD, NEW = 200, 2, 16, 5, 6


def operands(D, moved, seed):
    """Held codes [S, HKV, BS, D], old scales [S, HKV], new tokens [S * NEW, HKV, D] (BF16 values)."""
    rng = np.random.RandomState(seed)
    middle = 1 + (2 * rng.randint(0, 8, (S, HKV)) + 1) / 16.0
    ulps = rng.randint(-1, 2, (S, HKV)).astype(np.int32)
    if moved:  # held * old next to a middle; the new tokens ask for a larger scale
        held = 1 + rng.randint(0, 8, (S, HKV)) / 8.0
        old = ((middle / held).astype(np.float32).view(np.int32) + ulps).view(np.float32)
        codes = f8.encode(rng.choice([-1.0, 1.0], (S, HKV, BS, D)) * held[..., None, None] * np.exp2(rng.randint(-6, 6, (S, HKV, BS, D))))
        x = np.zeros((S, NEW, HKV, D))
        x[:, 1, :, 3] = 448.0 * np.exp2(rng.randint(3, 9, (S, HKV)))
    else:      # x / old next to a middle
        lead = 1 + rng.randint(0, 128, (S, HKV)) / 128.0
        old = ((lead / middle).astype(np.float32).view(np.int32) + ulps).view(np.float32)
        codes = rng.randint(0, 120, (S, HKV, BS, D)).astype(np.uint8)
        x = rng.choice([-1.0, 1.0], (S, NEW, HKV, D)) * lead[:, None, :, None] * np.exp2(rng.randint(-10, 6, (S, NEW, HKV, D)))
    return codes, old, x.reshape(S * NEW, HKV, D)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("moved", [False, True])
def test_one_rounding(D, moved):
    kinds = dict(dtype=torch.int32, device="cuda")
    cu, ctx = torch.arange(0, S * NEW + 1, NEW, **kinds), torch.full((S,), HELD, **kinds)
    table = torch.arange(S, **kinds)[:, None]
    sides = [operands(D, moved, seed) for seed in (D, D + 1)]   # K (not rotated here) and V
    caches = [torch.from_numpy(c).cuda().view(torch.float8_e4m3fn) for c, _, _ in sides]
    scales = [torch.from_numpy(o).cuda() for _, o, _ in sides]
    new = [torch.from_numpy(x).to(torch.bfloat16).cuda() for _, _, x in sides]
    mlt.kv_append_f8(None, *new, None, None, cu, ctx, table, *caches, *scales)
    assert_device_healthy()
    for (codes, old, x), cache, scale, t in zip(sides, caches, scales, new):
        assert np.array_equal(to_f64(t), x)
        got, s = cache.view(torch.uint8).cpu().numpy(), scale.cpu().numpy().astype(np.float64)
        need = f8.block_scale(np.abs(x).reshape(S, NEW, HKV, D).max((1, 3)))
        assert np.array_equal(s, np.maximum(need, old)) and ((need > old) == moved).all()
        want = codes.copy()
        want[:, :, HELD:HELD + NEW] = f8.encode(x.reshape(S, NEW, HKV, D).transpose(0, 2, 1, 3) / s[..., None, None])
        if moved:
            want[:, :, :HELD] = f8.encode(f8.decode(codes[:, :, :HELD]) * old.astype(np.float64)[..., None, None] / s[..., None, None])
        assert np.array_equal(got, want), int((got != want).sum())


def test_infinities_and_nan_under_such_a_scale():
    kinds = dict(dtype=torch.int32, device="cuda")
    v = torch.zeros(3, 1, 64, dtype=torch.bfloat16, device="cuda")
    v[0, 0, 0], v[1, 0, 1], v[2, 0, 2], v[2, 0, 3], v[2, 0, 4] = float("inf"), float("-inf"), float("nan"), 3.0, 1e-38
    cache = [torch.ones(1, 1, 16, 64, device="cuda").to(torch.float8_e4m3fn) for _ in range(2)]
    scale = [torch.full((1, 1), 1.3, device="cuda") for _ in range(2)]
    mlt.kv_append_f8(None, v, v, None, None, torch.tensor([0, 3], **kinds), torch.tensor([4], **kinds), torch.zeros(1, 1, **kinds), *cache, *scale)
    assert_device_healthy()
    for c, s in zip(cache, scale):
        got = c.float().cpu()[0, 0]
        assert float(s) == np.float32(1.3) and got[4, 0] == 448 and got[5, 1] == -448 and got[6, 2].isnan() and got.isnan().sum() == 1
        assert got[6, 3] == 2.25 and got[6, 4] == 0 and (got[:4] == 1).all() and (got[7:] == 1).all()
