"""CPU oracle (FP64, NumPy) for the 8-bit serving path -- TEST INFRASTRUCTURE, as oracle/__init__.py.

Plain definitions over the exact stored values: E4M3 by its fields, block scales, the scaled product, the cache append
and attention over the cache.  Shares nothing with the product package.
"""
from __future__ import annotations

import numpy as np

F8_MAX = 448.0
MIN_EXP = -64


def e4m3_table() -> np.ndarray:
    """The 256 values of E4M3: sign, 4 exponent bits (bias 7), 3 fraction bits; no infinities, 0x7F and 0xFF are NaN."""
    code = np.arange(256)
    e, f = (code >> 3) & 15, code & 7
    mag = np.where(e > 0, np.ldexp(1.0 + f / 8.0, e - 7), np.ldexp(f / 8.0, -6))
    v = np.where(code & 128, -mag, mag)
    v[(code & 127) == 127] = np.nan
    return v


_TABLE = e4m3_table()


def decode(codes: np.ndarray) -> np.ndarray:
    return _TABLE[np.asarray(codes, dtype=np.uint8)]


def encode(x: np.ndarray) -> np.ndarray:
    """FP64 -> nearest E4M3 code, ties to the even code; magnitudes beyond 448 become 448, NaN becomes 0x7F."""
    x = np.asarray(x, dtype=np.float64)
    mag = np.minimum(np.where(np.isnan(x), 0.0, np.abs(x)), F8_MAX)
    grid = _TABLE[:127]
    hi = np.minimum(np.searchsorted(grid, mag), 126)
    lo = np.maximum(hi - 1, 0)
    up, down = grid[hi] - mag, mag - grid[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo).astype(np.uint8)
    code = code | np.where(np.signbit(x), 128, 0).astype(np.uint8)
    return np.where(np.isnan(x), np.uint8(0x7F), code).astype(np.uint8)


def half_step(x: np.ndarray) -> np.ndarray:
    """Half the distance between the E4M3 values around |x| (2^-4 of its power of two; 2^-10 below 2^-6)."""
    mag = np.maximum(np.abs(np.asarray(x, dtype=np.float64)), 2.0 ** -6)
    return np.ldexp(1.0, np.frexp(mag)[1] - 1 - 4)


def block_scale(amax) -> np.ndarray:
    """The smallest 2^e, e >= -64, with amax <= 448 * 2^e."""
    m, e = np.frexp(np.asarray(amax, dtype=np.float64))
    e = np.where(m <= 0.875, e - 9, e - 8)
    e = np.where(np.asarray(amax) > 0, np.maximum(e, MIN_EXP), MIN_EXP)
    return np.ldexp(1.0, e)


def quantize(x: np.ndarray, block_rows: int):
    """x [M, K] FP64 -> (codes [M, K], scales [row blocks, K blocks])."""
    M, K = x.shape
    rb, kb = -(-M // block_rows), -(-K // 128)
    codes = np.empty((M, K), np.uint8)
    scales = np.empty((rb, kb))
    fin = np.where(np.isfinite(x), np.abs(x), 0.0)
    for i in range(rb):
        for j in range(kb):
            at = np.s_[i * block_rows:(i + 1) * block_rows, j * 128:(j + 1) * 128]
            scales[i, j] = block_scale(fin[at].max())
            codes[at] = encode(x[at] / scales[i, j])
    return codes, scales


def gemm(a: np.ndarray, sa: np.ndarray, b: np.ndarray, sb: np.ndarray):
    """a [M, K], b [N, K] codes; sa [K blocks, M], sb [N blocks, K blocks].  Returns (C, sum of the terms' magnitudes)."""
    K = a.shape[1]
    at = np.arange(K) // 128
    fa = decode(a) * sa.astype(np.float64).T[:, at]
    fb = decode(b) * sb.astype(np.float64)[np.arange(b.shape[0]) // 128][:, at]
    return fa @ fb.T, np.abs(fa) @ np.abs(fb).T


def rotate(x: np.ndarray, pos: np.ndarray, cos: np.ndarray, sin: np.ndarray, interleaved: bool) -> np.ndarray:
    """x [T, heads, D] FP64 with the first 2 * cos.shape[1] elements of every head rotated by the angles of its position."""
    h = cos.shape[1]
    out = x.copy()
    for i in range(h):
        p, q = (2 * i, 2 * i + 1) if interleaved else (i, i + h)
        c, s = cos[pos, i].astype(np.float64)[:, None], sin[pos, i].astype(np.float64)[:, None]
        out[:, :, p] = x[:, :, p] * c - x[:, :, q] * s
        out[:, :, q] = x[:, :, q] * c + x[:, :, p] * s
    return out


def positions(cu: np.ndarray, ctx: np.ndarray):
    """(sequence, position) of every new token."""
    seq = np.concatenate([np.full(cu[s + 1] - cu[s], s) for s in range(len(ctx))] + [np.zeros(0)]).astype(int)
    t = np.arange(len(seq))
    return seq, t - cu[seq] + ctx[seq] if len(seq) else t


def paged_decode(q, k, v, table, lens, scale):
    """q [S, H, D], caches k, v [blocks, H_kv, block, D], all FP64 values.  Returns (O, LSE, sum of p |v|, max sum |q k|)."""
    S, H, D = q.shape
    _, Hkv, bs, _ = k.shape
    o, lse = np.zeros((S, H, D)), np.full((S, H), -np.inf)
    mag, dots = np.zeros((S, H, D)), np.zeros((S, H))
    for s in range(S):
        n = int(lens[s])
        if n == 0:
            continue
        blk = table[s, :-(-n // bs)]
        for h in range(H):
            kk = k[blk, h // (H // Hkv)].reshape(-1, D)[:n]
            vv = v[blk, h // (H // Hkv)].reshape(-1, D)[:n]
            sc = float(scale) * (kk @ q[s, h])
            m = sc.max()
            p = np.exp(sc - m)
            l = p.sum()
            o[s, h], mag[s, h], lse[s, h] = p @ vv / l, p @ np.abs(vv) / l, m + np.log(l)
            dots[s, h] = float(scale) * (np.abs(kk) @ np.abs(q[s, h])).max()
    return o, lse, mag, dots
