"""Plain attention in 64 bits over packed sequences and paged caches, with the magnitudes that error bounds need.

Bound of an output element, with P = sum of p |v| / l: half a BF16 step of the result, 2^-8 |O|; the weights' rounding to BF16,
2^-8 P; the scores' FP32 error d (D products, each sum or product off by at most 2^-23 of the terms' magnitudes), which moves a
weight and the sum by a relative d each, 2 d P; the exponentials, some of which are polynomials whose exponent has steps of 252 * 2^-24
(half a step is 5.3e-6 of the value) and which are off by 2.2e-7 themselves, in weights and sum, 2 * 6e-6 P; scales, sums and
joins, 2^-16 P.  LSE: d + 6e-6, and 2^-19 (1 + |LSE|) for the logarithm and the sums.
"""
import math

import numpy as np
import torch

GUARD = 512


def rows_reference(q, k, v, seen, scale):
    """q [n, H, D], k and v [m, Hk, D] (64 bits), seen [n, m] or [n, H, m] bool -> O, LSE, P, d."""
    n, H, D = q.shape
    m, Hk, _ = k.shape
    o, mag = torch.zeros(n, H, D, dtype=torch.float64, device=q.device), torch.zeros(n, H, D, dtype=torch.float64, device=q.device)
    lse, d = torch.full((n, H), -math.inf, dtype=torch.float64, device=q.device), torch.zeros(n, H, dtype=torch.float64, device=q.device)
    if n == 0 or m == 0:
        return o, lse, mag, d
    for h in range(H):
        kh, vh = k[:, h // (H // Hk)], v[:, h // (H // Hk)]
        any_seen = seen.any(0)
        kh = torch.where(any_seen[:, None], kh, torch.zeros_like(kh))
        vh = torch.where(any_seen[:, None], vh, torch.zeros_like(vh))
        s = (q[:, h] @ kh.t()) * scale
        s = torch.where(seen, s, torch.full_like(s, -math.inf))
        top = s.amax(-1, keepdim=True)
        top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
        p = torch.exp(s - top)
        l = p.sum(-1, keepdim=True)
        some = l[:, 0] > 0
        safe = torch.where(l > 0, l, torch.ones_like(l))
        o[:, h], mag[:, h] = p @ vh / safe, p @ vh.abs() / safe
        lse[some, h] = (top + torch.log(safe))[some, 0]
        d[:, h] = D * 2.0 ** -23 * scale * torch.where(seen, q[:, h].abs() @ kh.abs().t(), torch.zeros_like(s)).amax(-1)
    return o, lse, mag, d


def check_rows(o, lse, ref, what=""):
    ro, rl, mag, d = ref
    dd = d[..., None]
    bound = 2.0 ** -8 * ro.abs() + (2.0 ** -8 + 2 * dd + 2 * 6e-6 + 2.0 ** -16) * mag + 2.0 ** -126
    err = (o.double() - ro).abs()
    assert torch.isfinite(o).all(), f"{what}: not finite"
    assert (err <= bound).all(), f"{what}: O off by {(err / bound).max().item():.3f} of its bound"
    empty = torch.isinf(rl)
    assert torch.equal(torch.isinf(lse) & (lse < 0), empty), f"{what}: LSE of empty rows"
    assert (o[empty] == 0).all(), f"{what}: O of empty rows"
    err = torch.where(empty, torch.zeros_like(rl), (lse.double() - rl).abs())
    bound = d + 6e-6 + 2.0 ** -19 * (1 + torch.where(empty, torch.zeros_like(rl), rl).abs())
    assert (err <= bound).all(), f"{what}: LSE off by {(err / bound).max().item():.3f} of its bound"


def guarded(shape, dtype, pitch=None):
    """A tensor (rows of a larger pitch, if given) inside a buffer of a marker value, and the buffer's check."""
    rows, width = shape[0], int(np.prod(shape[1:]))
    pitch = pitch or width
    buf = torch.full((rows * pitch + 2 * GUARD,), 776.0, dtype=dtype, device="cuda")
    body = buf[GUARD: GUARD + rows * pitch].view(rows, pitch)
    view = body[:, :width].unflatten(1, shape[1:]) if rows else body[:, :width].reshape(shape)

    def untouched():
        assert (buf[:GUARD] == 776).all() and (buf[GUARD + rows * pitch:] == 776).all() and (body[:, width:] == 776).all(), "guard band written"
    return view, untouched


def cu(lens):
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")


def paged(lens, Hk, D, bs, seed, width=None, share=None):
    """A cache whose blocks lie scattered, NaN wherever no sequence looks; share: (rows, blocks) whose first blocks are the
    same (one of them must have that many)."""
    rng = np.random.RandomState(seed)
    lens = np.asarray(lens)
    per = -(-lens // bs)
    blocks = int(per.sum()) + 3
    order, at = rng.permutation(blocks), 0
    table = np.full((len(lens), width or max(1, int(per.max()))), -1, np.int32)
    for s in range(len(lens)):
        table[s, : per[s]] = order[at: at + per[s]]
        at += per[s]
    for rows, held in share or []:  # (also for rows that do not reach that far themselves)
        longest = max(rows, key=lambda s: lens[s])
        table[rows, :held] = table[longest, :held]
    used = np.zeros((blocks, bs), bool)
    for s in range(len(lens)):
        for i in range(per[s]):
            used[table[s, i], : min(bs, lens[s] - i * bs)] = True
    g = torch.Generator(device="cuda").manual_seed(seed)
    caches = []
    for _ in range(2):
        c = torch.randn(blocks, Hk, bs, D, generator=g, device="cuda", dtype=torch.bfloat16)
        c.transpose(1, 2)[~torch.from_numpy(used).cuda()] = math.nan
        caches.append(c)
    return caches[0], caches[1], torch.from_numpy(table).cuda()


def gathered(cache, table_row, n):
    """[n, Hk, D] in 64 bits of a sequence's cached tokens."""
    bs = cache.shape[2]
    blk = table_row[: -(-n // bs)].long()
    return cache[blk].transpose(1, 2).reshape(-1, cache.shape[1], cache.shape[3])[:n].double()
