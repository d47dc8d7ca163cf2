"""Pins of the 8-bit oracle: the format against its published landmarks and torch's conversion, the operations against
closed forms and brute force."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import f8  # noqa: E402


def test_format_landmarks_and_torch_values():
    t = f8.e4m3_table()
    assert t[0] == 0 and t[0x01] == 2.0 ** -9 and t[0x08] == 2.0 ** -6 and t[0x38] == 1.0 and t[0x7E] == 448.0 and np.isnan(t[0x7F])
    ref = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).to(torch.float64).numpy()
    assert np.array_equal(t, ref, equal_nan=True)
    assert np.signbit(t[0x80]) and t[0x80] == 0


def test_encode_round_trips_ties_and_saturates():
    codes = np.array([c for c in range(256) if c & 127 != 127], np.uint8)
    assert np.array_equal(f8.encode(f8.decode(codes)), codes)
    grid = f8.e4m3_table()[:127]
    mid = (grid[1:] + grid[:-1]) / 2
    even = np.where(np.arange(126) % 2 == 0, np.arange(126), np.arange(1, 127)).astype(np.uint8)
    assert np.array_equal(f8.encode(mid), even)
    assert np.array_equal(f8.encode(np.nextafter(mid, np.inf)), np.arange(1, 127))
    assert f8.encode(np.array([1e9, np.inf, -np.inf, np.nan])).tolist() == [0x7E, 0x7E, 0xFE, 0x7F]


def test_encode_agrees_with_torch():
    x = torch.randn(20000, generator=torch.Generator().manual_seed(1), dtype=torch.float32) * torch.logspace(-4, 2.4, 20000)
    x = x.clamp(-448, 448)
    assert np.array_equal(f8.encode(x.numpy().astype(np.float64)), x.to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_half_step_is_the_distance_to_the_rounding_border():
    grid = f8.e4m3_table()[1:127]
    nxt = np.append(grid[1:], 480.0)
    assert np.array_equal(f8.half_step(grid), (nxt - grid) / 2)
    assert f8.half_step(np.array([1e-5])) == 2.0 ** -10


def test_block_scale_is_the_smallest_power_of_two_that_holds_the_maximum():
    amax = np.array([0.0, 1e-30, 1.0, 448.0, np.nextafter(448.0, 500), 449.0, 896.0, 3.38e38, 1.75, 1.7501])
    s = f8.block_scale(amax)
    assert s[0] == s[1] == 2.0 ** -64 and s[3] == 1.0 and s[4] == s[5] == s[6] == 2.0
    live = amax > 1e-19
    assert (amax[live] <= 448 * s[live]).all() and (amax[live] > 224 * s[live]).all()


def test_quantize_reconstructs_within_half_a_step():
    rng = np.random.RandomState(0)
    x = rng.randn(37, 300) * np.exp2(rng.randint(-9, 9, (37, 1)))
    for rows in (1, 128):
        codes, scales = f8.quantize(x, rows)
        s = np.repeat(np.repeat(scales, rows, 0)[:37], 128, 1)[:, :300]
        assert (np.abs(f8.decode(codes) * s - x) <= f8.half_step(x / s) * s).all()


def test_gemm_against_a_loop_and_a_hand_worked_product():
    rng = np.random.RandomState(1)
    M, N, K = 3, 130, 200
    a, b = rng.randint(0, 127, (M, K)).astype(np.uint8), rng.randint(0, 127, (N, K)).astype(np.uint8)
    sa, sb = rng.rand(2, M).astype(np.float32), rng.rand(2, 2).astype(np.float32)
    c, mag = f8.gemm(a, sa, b, sb)
    for i, j in ((0, 0), (2, 129), (1, 127), (1, 128)):
        want = sum(f8.decode(a[i, k]) * f8.decode(b[j, k]) * float(sa[k // 128, i]) * float(sb[j // 128, k // 128]) for k in range(K))
        assert abs(c[i, j] - want) <= 1e-12 * mag[i, j]
    one = np.full((1, 256), 0x38, np.uint8)  # all ones: 128 * (2 * 5 + 3 * 7)
    assert f8.gemm(one, np.array([[2.0], [3.0]]), one, np.array([[5.0, 7.0]]))[0][0, 0] == 128 * 31


def test_rotation_keeps_lengths_composes_and_places_pairs():
    rng = np.random.RandomState(2)
    ang = np.arange(40)[:, None] * np.array([1.0, 0.1, 0.01, 0.001])
    x = rng.randn(3, 2, 12)
    for inter in (False, True):
        y = f8.rotate(x, np.array([0, 5, 39]), np.cos(ang), np.sin(ang), inter)
        assert np.array_equal(y[0], x[0]) and np.array_equal(y[:, :, 8:], x[:, :, 8:])
        assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))
        z = f8.rotate(f8.rotate(x, np.array([3, 3, 3]), np.cos(ang), np.sin(ang), inter), np.array([4, 4, 4]), np.cos(ang), np.sin(ang), inter)
        assert np.allclose(z, f8.rotate(x, np.array([7, 7, 7]), np.cos(ang), np.sin(ang), inter))
    unit = np.zeros((1, 1, 8)); unit[0, 0, 0] = 1.0
    quarter = np.full((1, 4), np.pi / 2)
    assert np.allclose(f8.rotate(unit, np.array([0]), np.cos(quarter), np.sin(quarter), True)[0, 0], np.eye(8)[1])
    assert np.allclose(f8.rotate(unit, np.array([0]), np.cos(quarter), np.sin(quarter), False)[0, 0], np.eye(8)[4])


def test_positions_of_new_tokens():
    seq, pos = f8.positions(np.array([0, 2, 2, 5]), np.array([7, 3, 0]))
    assert seq.tolist() == [0, 0, 2, 2, 2] and pos.tolist() == [7, 8, 0, 1, 2]


def test_paged_decode_equal_keys_give_the_mean_and_empty_rows_nothing():
    rng = np.random.RandomState(3)
    k = np.ones((4, 1, 8, 4)); v = rng.randn(4, 1, 8, 4); q = rng.randn(2, 2, 4)
    table = np.array([[2, 0], [1, 3]])
    o, lse, mag, dots = f8.paged_decode(q, k, v, table, np.array([11, 0]), 0.5)
    want = np.concatenate([v[2, 0], v[0, 0, :3]])
    assert np.allclose(o[0, 0], want.mean(0)) and np.allclose(lse[0, 1], 0.5 * q[0, 1].sum() + np.log(11))
    assert (o[1] == 0).all() and np.isneginf(lse[1]).all() and np.allclose(mag[0, 1], np.abs(want).mean(0))
