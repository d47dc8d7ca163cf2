"""mlt_paged_attn_decode_f8 against the FP64 oracle.

Tolerance of an output element, with P = sum of p |v| / l: half a BF16 step, 2^-8 |O|; the probabilities' rounding to FP16,
2^-11 P; the scores' FP32 error d (D products, each sum or product off by at most 2^-23 of the terms' magnitudes, which
moves a probability and the sum by a relative d each), 2 d P; exponentials, scales and sums, 2^-16 P.  LSE: d, and
2^-19 (1 + |LSE|) for the logarithm, the exponentials and the sums."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2503_14985_b200 as mlt  # noqa: E402
from oracle import f8  # noqa: E402

from gpu_util import assert_device_healthy, to_f64  # noqa: E402


class Case:
    def __init__(self, lens, H, Hkv, D, bs, seed, exps=(-9, -5), spare=3, poison=True, width=None):
        rng = np.random.RandomState(seed)
        self.lens, self.H, self.Hkv, self.D, self.bs = np.asarray(lens, np.int32), H, Hkv, D, bs
        self.S = S = len(lens)
        per = -(-self.lens // bs)
        self.blocks = int(per.sum()) + spare
        order, at = rng.permutation(self.blocks), 0
        self.table = np.full((S, width or max(1, int(per.max()))), -1, np.int32)
        used = np.zeros((self.blocks, bs), bool)
        for s in range(S):
            blk = order[at:at + per[s]]
            self.table[s, :per[s]] = blk
            for i, b in enumerate(blk):
                used[b, :min(bs, self.lens[s] - i * bs)] = True
            at += per[s]
        shape = (self.blocks, Hkv, bs, D)
        self.q = torch.from_numpy(rng.randn(S, H, D)).to(torch.bfloat16)
        self.ks, self.vs = (np.exp2(rng.randint(*exps, shape[:2]) + rng.rand(*shape[:2])).astype(np.float32) for _ in range(2))
        self.kc, self.vc = (f8.encode(rng.randn(*shape) / s.astype(np.float64)[..., None, None]) for s in (self.ks, self.vs))
        if poison:  # NaN wherever no sequence may look
            for c in (self.kc, self.vc):
                c.transpose(0, 2, 1, 3)[~used] = 0x7F
            for s in (self.ks, self.vs):
                s[~used.any(1)] = np.nan
        self.scale = float(np.float32(1 / math.sqrt(D)))

    def dev(self):
        c = [torch.from_numpy(x).cuda().view(torch.float8_e4m3fn) for x in (self.kc, self.vc)]
        return [self.q.cuda(), *c, *(torch.from_numpy(x).cuda() for x in (self.ks, self.vs, self.table, self.lens))]

    def run(self, workspace="full", table=None, lens=None):
        guard = 256
        S, H, D = self.S, self.H, self.D
        ob = torch.full((S * H * D + 2 * guard,), 776.0, dtype=torch.bfloat16, device="cuda")
        lb = torch.full((S * H + 2 * guard,), 776.0, device="cuda")
        O, L = ob[guard:-guard].view(S, H, D), lb[guard:-guard].view(S, H)
        n = mlt.paged_attn_f8_workspace_bytes(S, H, self.Hkv, D) if workspace == "full" else workspace
        ws = torch.full((n + 64,), 0xFF, dtype=torch.uint8, device="cuda") if n else None  # NaN: an unwritten partial shows
        args = self.dev()
        if table is not None:
            args[5] = torch.from_numpy(table).cuda()
        if lens is not None:
            args[6] = torch.from_numpy(np.asarray(lens, np.int32)).cuda()
        mlt.paged_attn_decode_f8(*args, scale=self.scale, workspace=ws[:n] if n else None, O=O, LSE=L)
        torch.cuda.synchronize()
        for b in (ob, lb):
            assert (b[:guard] == 776).all() and (b[-guard:] == 776).all(), "guard band written"
        if ws is not None:
            assert (ws[n:] == 0xFF).all(), "workspace overrun"
        return to_f64(O), L.cpu().numpy().astype(np.float64)

    def reference(self):
        k, v = (f8.decode(c) * s.astype(np.float64)[..., None, None] for c, s in ((self.kc, self.ks), (self.vc, self.vs)))
        return f8.paged_decode(to_f64(self.q.cuda()), k, v, self.table, self.lens, self.scale)

    def check(self, o, lse, rows=None):
        ro, rl, mag, dots = self.reference()
        d = (self.D * 2.0 ** -23 * dots)[..., None]
        tol = 2.0 ** -8 * np.abs(ro) + (2.0 ** -11 + 2.0 ** -16 + 2 * d) * mag
        live = self.lens > 0
        if rows is not None:
            live &= rows
        bad = np.abs(o - ro)[live] / np.maximum(tol[live], 1e-300)
        assert bad.max(initial=0.0) <= 1.0, float(bad.max())
        assert (np.abs(lse[live] - rl[live]) <= d[..., 0][live] + 2.0 ** -19 * (1 + np.abs(rl[live]))).all()
        for s in np.flatnonzero(self.lens == 0):
            assert (o[s] == 0).all() and np.isneginf(lse[s]).all()


CASES = [  # lens, H, H_kv, D, block
    ([1], 1, 1, 64, 16), ([1, 2, 15, 16, 17], 2, 2, 128, 16), ([100, 0, 3], 4, 4, 64, 8), ([31, 32, 33, 127, 128, 129], 8, 2, 128, 32),
    ([300, 17, 255], 8, 1, 64, 16), ([700, 50, 257], 8, 2, 128, 8), ([1500, 200], 4, 2, 64, 32), ([5000], 2, 1, 128, 16), ([5000], 16, 2, 64, 8),
    ([2000, 1, 64, 65], 16, 2, 128, 32), ([0, 0, 1, 0], 8, 8, 128, 16), ([0, 0], 4, 2, 64, 8), ([9, 1000, 8], 4, 1, 128, 32), ([640, 641, 639], 32, 4, 128, 16),
]


@pytest.mark.parametrize("lens,H,Hkv,D,bs", CASES)
def test_parity_and_any_workspace(lens, H, Hkv, D, bs):
    c = Case(lens, H, Hkv, D, bs, seed=sum(lens) + H + D)
    slot = H // Hkv * (4 * D + 8)
    for ws in ("full", 0, slot * (len(lens) * Hkv + 3), slot * len(lens) * Hkv, 16):
        o, lse = c.run(ws)
        assert_device_healthy()
        c.check(o, lse)


@pytest.mark.parametrize("seed", range(24))
def test_random_shapes(seed):
    rng = np.random.RandomState(700 + seed)
    Hkv, G = int(rng.choice([1, 2, 3, 8])), int(rng.choice([1, 2, 4, 8]))
    top = int(np.exp(rng.uniform(0, np.log(3000))))
    lens = rng.randint(0, top + 1, int(rng.randint(1, 9)))
    c = Case(lens, Hkv * G, Hkv, int(rng.choice([64, 128])), int(rng.choice([8, 16, 32])), seed=seed)
    o, lse = c.run()
    assert_device_healthy()
    c.check(o, lse)


def test_one_long_row_split_over_every_cta():
    c = Case([70000], 4, 1, 128, 16, seed=1, poison=False)
    c.check(*c.run())
    assert_device_healthy()


def test_more_sequences_than_the_scan_table():
    lens = np.random.RandomState(2).randint(0, 60, 1100)
    c = Case(lens, 2, 1, 64, 16, seed=2)
    c.check(*c.run())
    c = Case(lens[:1024], 4, 1, 64, 8, seed=3)
    c.check(*c.run())
    assert_device_healthy()


def test_more_units_than_one_batch_of_table_entries():
    # a warp reads the entries and scales of 32 of its units (4096 tokens) at a time; without scratch one CTA walks the whole row
    for bs in (8, 16, 32):
        c = Case([20000, 8191, 4097], 2, 1, 64, bs, seed=20 + bs)
        for ws in ("full", 0):
            c.check(*c.run(ws))
    assert_device_healthy()


def test_block_scales_of_very_different_size():
    # powers of two from 2^-40 to 2^15 from block to block: V's scale is applied relative to the largest met so far
    c = Case([400, 333], 8, 2, 128, 8, seed=4)
    rng = np.random.RandomState(5)
    c.vs = np.exp2(rng.randint(-40, 16, c.vs.shape)).astype(np.float32)
    c.check(*c.run())
    c.vs[c.table[0, 3]] = 0.0                                   # a block whose values are all zero
    c.vs[c.table[1, :]] = 0.0                                   # ... and a whole sequence of them
    o, lse = c.run()
    assert (o[1] == 0).all()
    c.check(o, lse)
    assert_device_healthy()


def test_scales_that_favour_tiny_values():
    # the most likely tokens carry values 2^-20 times those of the least likely ones
    c = Case([256], 1, 1, 64, 16, seed=6)
    c.q[:] = 0.5
    c.kc[:] = f8.encode(np.full(c.kc.shape, 16.0))
    c.ks[:] = 2.0 ** -6
    late = c.table[0, 8:]
    c.ks[late] = 2.0 ** -3                                      # scores 1 and 8
    c.vs[:] = 1.0
    c.vs[late] = 2.0 ** -20
    c.check(*c.run())


def test_queries_far_from_unit_size():
    c = Case([100, 200], 4, 2, 64, 16, seed=7)
    c.q[0, 0] *= 2.0 ** -100
    c.q[0, 1] = 0
    c.q[1, 0, 5] = 1e-30                                        # one element far below its row
    c.check(*c.run())
    c.q[1, 1] *= 2.0 ** 60                                      # one score dominates: the softmax is a single token
    o, lse = c.run()
    ro = c.reference()[0]
    assert (np.abs(o[1, 1] - ro[1, 1]) <= 2.0 ** -8 * np.abs(ro[1, 1])).all()
    assert_device_healthy()


def test_nan_in_one_head_stays_there():
    c = Case([60, 60], 4, 2, 64, 16, seed=8)
    blk = c.table[0, 1]
    c.kc[blk, 0, 2, 7] = 0x7F
    o, lse = c.run()
    assert np.isnan(o[0, :2]).all() and np.isnan(lse[0, :2]).all()
    rest = np.ones((2, 4), bool); rest[0, :2] = False
    ro, rl, mag, dots = c.reference()
    assert np.isfinite(o[rest]).all() and np.abs(o[rest] - ro[rest]).max() < 0.02
    assert_device_healthy()


def test_length_beyond_the_table_is_cut_and_negative_is_empty():
    c = Case([1200, 1200, 40], 4, 4, 128, 16, seed=9)
    assert c.table.shape[1] == 75
    for ws in ("full", 0):
        o, lse = c.run(ws, lens=[1237, 2 ** 31 - 1, 40])
        c.check(o, lse)
        o, lse = c.run(ws, lens=[-5, 1200, 40])
        assert (o[0] == 0).all() and np.isneginf(lse[0]).all()
    assert_device_healthy()


@pytest.mark.parametrize("bs", [8, 16, 32])
def test_bad_entries_are_reported_and_only_their_tokens_left_out(bs):
    c = Case([700, 90], 8, 2, 64, bs, seed=10, poison=False)
    bad = c.table.copy()
    bad[0, 3], bad[0, 8], bad[1, 0] = -7, c.blocks, c.blocks + 10 ** 6
    for ws in ("full", 0):
        o, lse = c.run(ws, table=bad)
        status, detail = mlt.last_device_error()
        assert status == 7 and (detail[1], detail[2]) in ((3, 0), (8, 0), (0, 1))
        keep = Case.__new__(Case)  # the same sequences without those blocks
        keep.__dict__.update(c.__dict__)
        rows = [[b for i, b in enumerate(c.table[s]) if b >= 0 and (s, i) not in ((0, 3), (0, 8), (1, 0))] for s in range(2)]
        keep.table = np.array([r + [0] * (len(rows[0]) - len(r)) for r in rows], np.int32)
        keep.lens = np.array([700 - 2 * bs, 90 - bs], np.int32)
        keep.check(o, lse)
        c.check(*c.run(ws))                                     # the next call is clean
        assert_device_healthy()


def test_bits_repeat_on_any_stream_and_in_a_graph():
    c = Case([900, 1, 333, 0, 2100], 8, 2, 128, 16, seed=11)
    args = c.dev()
    ws = [torch.empty(mlt.paged_attn_f8_workspace_bytes(5, 8, 2, 128), dtype=torch.uint8, device="cuda") for _ in range(3)]
    o0, l0 = mlt.paged_attn_decode_f8(*args, scale=c.scale, workspace=ws[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        o1, l1 = mlt.paged_attn_decode_f8(*args, scale=c.scale, workspace=ws[1])
    o2, none = mlt.paged_attn_decode_f8(*args, scale=c.scale, workspace=ws[0], return_lse=False)
    assert none is None
    torch.cuda.synchronize()
    assert torch.equal(o0, o1) and torch.equal(l0, l1) and torch.equal(o0, o2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o3, l3 = mlt.paged_attn_decode_f8(*args, scale=c.scale, workspace=ws[2])
    for lens in ([900, 1, 333, 0, 2100], [5, 1, 0, 0, 100]):    # lengths change under the captured call
        args[6].copy_(torch.tensor(lens, dtype=torch.int32))
        graph.replay()
        o4, l4 = mlt.paged_attn_decode_f8(*args, scale=c.scale, workspace=ws[0])
        torch.cuda.synchronize()
        assert torch.equal(o3, o4) and torch.equal(l3, l4)
    assert_device_healthy()


def test_cache_beyond_32_bit_byte_offsets():
    # 4.8 GB of keys: the last blocks lie beyond 2^32 bytes
    D, Hkv, bs, blocks = 128, 8, 32, 147000
    kc = torch.full((blocks, Hkv, bs, D), 0x7F, dtype=torch.uint8, device="cuda")
    vc, scales = torch.full_like(kc, 0x7F), torch.full((blocks, Hkv), float("nan"), device="cuda")
    c = Case([70], 8, 8, D, bs, seed=12, spare=0)
    last = torch.arange(blocks - c.blocks, blocks)
    for big, small in ((kc, c.kc), (vc, c.vc)):
        big[last] = torch.from_numpy(small).cuda()
    ks, vs = scales.clone(), scales.clone()
    ks[last], vs[last] = torch.from_numpy(c.ks).cuda(), torch.from_numpy(c.vs).cuda()
    args = c.dev()
    table = torch.from_numpy(c.table + (blocks - c.blocks)).to(torch.int32).cuda()
    o, lse = mlt.paged_attn_decode_f8(args[0], kc.view(torch.float8_e4m3fn), vc.view(torch.float8_e4m3fn), ks, vs, table, args[6], scale=c.scale)
    c.check(to_f64(o), lse.cpu().numpy().astype(np.float64))
    assert_device_healthy()


@pytest.mark.parametrize("H,Hkv,D,bs", [(4, 4, 64, 16), (32, 4, 128, 8), (8, 2, 64, 32)])
def test_more_rows_than_shares(H, Hkv, D, bs):
    # most rows lie inside one share, some cross a border, some are empty; a few long ones lie in many shares
    rng = np.random.RandomState(H + D + bs)
    lens = rng.randint(0, 90, 2600 // Hkv)
    lens[rng.randint(0, len(lens), 40)] = 0
    lens[-3:] = 0
    lens[7] = 2500
    assert len(lens) * Hkv > 2048
    c = Case(lens, H, Hkv, D, bs, seed=9)
    c.check(*c.run())
    c.check(*c.run((len(lens) * Hkv + 9) * (H // Hkv * (4 * D + 8) + 8)))
    assert_device_healthy()
