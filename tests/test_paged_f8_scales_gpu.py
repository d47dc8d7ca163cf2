"""mlt_paged_attn_decode_f8 where V's scales and the probabilities differ by far, in either direction.

The tolerance is that of test_paged_f8_gpu.py (weights p * |v_scale| in FP16, whose rounding is relative down to 2^-28 of the
row's largest) and what a weight below that loses: half of FP16's smallest step, 2^-25 where the largest weight is 2^14 at least, so
2^-39 max(p |v_scale|) / l |V code| per token; and half of BF16's smallest step, 2^-134."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2503_14985_b200 as mlt  # noqa: E402
from oracle import f8  # noqa: E402

from gpu_util import assert_device_healthy, to_f64  # noqa: E402
from test_paged_f8_gpu import Case  # noqa: E402

NATS = math.log(2.0)


class Scales(Case):
    """Blocks with given scores (in units of log2, the same for all their tokens) and V scales; V codes of magnitude 1 to 2."""

    def __init__(self, lens, H, Hkv, D, bs, levels, vs, seed):
        super().__init__(lens, H, Hkv, D, bs, seed, poison=False)
        rng = np.random.RandomState(seed + 1)
        self.q[:] = 0.5
        self.kc[:] = f8.encode(np.ones(self.kc.shape))
        step = NATS / (self.scale * 0.5 * D)                    # k_scale of a score of one unit
        self.vc = f8.encode(rng.choice([-1.0, 1.0, 1.0, 1.0], self.vc.shape) * rng.uniform(1.0, 2.0, self.vc.shape))
        for s in range(self.S):
            for i, b in enumerate(self.table[s, :-(-int(self.lens[s]) // bs)]):
                self.ks[b], self.vs[b] = levels(s, i) * step, vs(s, i)

    def check(self, o, lse, rows=None):
        ro, rl, mag, dots = self.reference()
        d = (self.D * 2.0 ** -23 * dots)[..., None]
        G = self.H // self.Hkv
        lost = np.zeros_like(ro)
        for s in range(self.S):
            n = int(self.lens[s])
            blk = self.table[s, :-(-n // self.bs)]
            for h in range(self.H):
                at = np.s_[blk, h // G]
                sc = np.repeat(0.5 * self.D * self.scale * self.ks[at].astype(np.float64), self.bs)[:n]
                w = np.exp(sc - rl[s, h]) * np.repeat(np.abs(self.vs[at]).astype(np.float64), self.bs)[:n]
                lost[s, h] = 2.0 ** -39 * w.max() * np.abs(f8.decode(self.vc[at])).reshape(-1, self.D)[:n].sum(0)
        tol = 2.0 ** -8 * np.abs(ro) + (2.0 ** -11 + 2.0 ** -16 + 2 * d) * mag + lost + 2.0 ** -134
        assert np.isfinite(o).all()
        assert (np.abs(o - ro) / tol).max() <= 1.0, float((np.abs(o - ro) / tol).max())
        assert (np.abs(lse - rl) <= d[..., 0] + 2.0 ** -19 * (1 + np.abs(rl))).all()

    def check_all(self):
        slot = mlt.paged_attn_f8_workspace_bytes(2, self.H, self.Hkv, self.D) - mlt.paged_attn_f8_workspace_bytes(1, self.H, self.Hkv, self.D)
        slot //= self.Hkv
        for ws in ("full", 0, slot * (self.S * self.Hkv + 3)):  # every share there is; none; three
            self.check(*self.run(ws))
        assert_device_healthy()


SHAPES = [([64], 1, 1, 64, 16), ([64, 200], 8, 1, 128, 32), ([4000, 33], 8, 2, 64, 8), ([2000], 4, 1, 128, 16)]


@pytest.mark.parametrize("lens,H,Hkv,D,bs", SHAPES)
@pytest.mark.parametrize("where", ["first", "middle", "last"])
@pytest.mark.parametrize("below,ratio", [(58, 40), (30, 28), (20, 45), (200, 40), (120, 100), (90, 120)])
def test_large_scale_of_unlikely_tokens(lens, H, Hkv, D, bs, where, below, ratio):
    # one block with a large V scale, its tokens far less likely than the others, whose scale is 1
    def special(s, i):
        blocks = -(-lens[s] // bs)
        return i == {"first": 0, "middle": blocks // 2, "last": blocks - 1}[where]

    c = Scales(lens, H, Hkv, D, bs, lambda s, i: 4.0 if special(s, i) else 4.0 + below, lambda s, i: 2.0 ** ratio if special(s, i) else 1.0,
               seed=below + ratio)
    c.check_all()


@pytest.mark.parametrize("lens,H,Hkv,D,bs", SHAPES)
@pytest.mark.parametrize("below,ratio", [(290, -45), (60, -45), (45, -45), (100, -100), (10, -64)])
def test_small_scale_of_likely_tokens(lens, H, Hkv, D, bs, below, ratio):
    # every third block is likely and has a small scale, the others have scale 1
    c = Scales(lens, H, Hkv, D, bs, lambda s, i: 4.0 + below if i % 3 == 1 else 4.0, lambda s, i: 2.0 ** ratio * 1.3 if i % 3 == 1 else 1.0,
               seed=below)
    c.check_all()


@pytest.mark.parametrize("lens,H,Hkv,D,bs", SHAPES)
@pytest.mark.parametrize("span", [3, 30, 100])
def test_scales_that_make_up_for_the_probabilities(lens, H, Hkv, D, bs, span):
    # every block contributes about as much as the others, with probabilities over 2^span; scales of either sign, no powers of two
    rng = np.random.RandomState(span)
    level = {(s, i): float(rng.randint(0, span + 1)) for s in range(len(lens)) for i in range(-(-lens[s] // bs))}
    c = Scales(lens, H, Hkv, D, bs, lambda s, i: 1.0 + level[s, i],
               lambda s, i: rng.choice([-1.0, 1.0, 1.0, 1.0]) * rng.uniform(1, 2) * 2.0 ** (20 - level[s, i]), seed=span + D)
    c.check_all()


@pytest.mark.parametrize("lens,H,Hkv,D,bs", SHAPES)
def test_zero_and_extreme_scales(lens, H, Hkv, D, bs):
    # the likely blocks hold zeros (scale 0): what is left comes from the others, 2^-58 times as likely
    c = Scales(lens, H, Hkv, D, bs, lambda s, i: 60.0 if i % 2 == 0 else 2.0, lambda s, i: 0.0 if i % 2 == 0 else 1.0, seed=1)
    if min(lens) > bs:
        assert np.abs(c.reference()[0]).max() > 2.0 ** -60
    c.check_all()
    for size in (2.0 ** 120, 2.0 ** -64, 2.0 ** -126, 2.0 ** -131):  # the largest and the smallest the library makes, and smaller still
        c = Scales(lens, H, Hkv, D, bs, lambda s, i: 1.0 + i % 5, lambda s, i: size * (1 + i % 2), seed=2)
        c.check_all()


def test_scale_grows_or_shrinks_all_along():
    # the reference moves with every block: likelier and smaller, less likely and larger, and both together
    blocks = 100
    for dl, de in ((1.0, -1.5), (-1.0, 1.5), (-2.0, 2.0), (1.0, 0.7), (-0.5, -0.9)):
        c = Scales([blocks * 8 - 3], 8, 1, 64, 8, lambda s, i: 1 + (i if dl > 0 else i - blocks) * dl, lambda s, i: 2.0 ** (de * (i - blocks / 2)),
                   seed=int(10 * (dl + 5)))
        c.check_all()


@pytest.mark.parametrize("lens,H,Hkv,D,bs", SHAPES)
@pytest.mark.parametrize("ratio", [40, -40, 120, -120])
def test_scores_far_beyond_a_scales_exponent(lens, H, Hkv, D, bs, ratio):
    # scores of 2^40 and more, powers of two and hence exact: the softmax is the mean over the last block, whose scale is far from the
    # others'.  Weights 1 and V's values: as in check(), without any error of the scores
    c = Scales(lens, H, Hkv, D, bs, lambda s, i: 1.0, lambda s, i: 1.0, seed=200 + ratio)
    last = [int(c.table[s, -(-n // bs) - 1]) for s, n in enumerate(lens)]
    c.scale, c.ks[:], c.ks[last], c.vs[last] = 0.125, 2.0 ** 40, 2.0 ** 41, 2.0 ** ratio
    slot = (mlt.paged_attn_f8_workspace_bytes(2, H, Hkv, D) - mlt.paged_attn_f8_workspace_bytes(1, H, Hkv, D)) // Hkv
    for ws in ("full", 0, slot * (c.S * Hkv + 3)):
        o, lse = c.run(ws)
        for s, n in enumerate(lens):
            v = f8.decode(c.vc[last[s]])[:, :n - (-(-n // bs) - 1) * bs] * 2.0 ** ratio
            ref, mag = (x.repeat(H // Hkv, 0) for x in (v.mean(1), np.abs(v).mean(1)))
            assert (np.abs(o[s] - ref) <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -11 + 2.0 ** -16) * mag).all()
            top = 0.125 * 0.5 * D * 2.0 ** 41
            assert (np.abs(lse[s] - top) <= 2.0 ** -20 * top).all()
    assert_device_healthy()
