"""The plan of the packed attention, run on the CPU (packed_plan_util checks each: every key block of every tile once, parts in rows of their own
within the scratch, the join's list in line with it), for lengths as they come and for offsets that do not ascend."""
import numpy as np
import pytest

from packed_plan_util import plan


def lengths(rng, n, most):
    return np.floor(np.exp(rng.uniform(0, np.log(most + 1), n))).astype(int) - (rng.rand(n) < 0.2)


def cu(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(int)


def heads(rng):
    return int(rng.choice([1, 2, 3, 4, 5, 8, 16, 100, 128])), int(rng.choice([1, 2, 3, 8])), int(rng.choice([64, 128]))


@pytest.mark.parametrize("kind", ["packed", "prefill", "shared"])
def test_lengths_as_they_come(kind):
    rng = np.random.RandomState(len(kind))
    cut = 0
    for i in range(60):
        G, Hk, D = heads(rng)
        S = int(np.exp(rng.uniform(0, np.log(200 if kind != "packed" else 3000))))
        bs = int(rng.choice([8, 16, 32]))
        if kind == "shared":
            lens = np.maximum(lengths(rng, S, 20000), 0)
            groups = int(rng.randint(0, min(S, 4) + 1))
            at = np.sort(rng.choice(S + 1, groups + 1, replace=False)) if groups else np.zeros(1, int)
            r = plan(kind, S, at, G, Hk, D, prefix=lengths(rng, groups, 20000), lens=lens, bs=bs, max_blocks=20000 // bs + 1)
        else:
            q = np.maximum(lengths(rng, S, max(1, 20000 // S)), 0)
            more = np.maximum(lengths(rng, S, 50000 // S + 1), 0)
            T = int(q.sum()) + int(rng.randint(0, 3))
            if T == 0:
                continue
            if kind == "packed":
                k = q + more * (rng.rand(S) < 0.7)
                r = plan(kind, T, cu(q), G, Hk, D, cu_k=cu(k), num_k=int(k.sum()), causal=bool(rng.rand() < 0.6), sms=int(rng.choice([148, 7])),
                         parts=None if rng.rand() < 0.7 else int(rng.randint(0, 3000)))
            else:
                r = plan(kind, T, cu(q), G, Hk, D, context=more, bs=bs, max_blocks=int((q + more).max()) // bs + 1)
            assert (r["seqs"][:, 1] == q).all()
        assert r["status"] == 0
        cut += r["chunk"] > 0
    assert cut > 10                                                     # (both ways of the plan were there)


def alternating(T, S):
    at = np.zeros(S + 1, int)
    at[1::2] = T
    return at


def test_repeated_queries_with_cut_key_ranges():
    """0, T, 0, T, ...: more tile pairs than the lists hold, behind keys long enough for parts; the first ones fit and are kept."""
    T, S = 1000, 15
    r = plan("packed", T, alternating(T, S), 2, 8, 128, cu_k=alternating(30000, S), num_k=30000)
    assert r["status"] == 9 and r["part_rows"] > 0
    W2, most = 128, r["max_tiles"]
    kept = most // -(-T // W2)
    assert (r["seqs"][: 2 * kept: 2, 1] == T).all() and r["seqs"][:, 1].sum() == kept * T
    r = plan("packed", 5, alternating(5, 40), 4, 1, 64, cu_k=alternating(30000, 40), num_k=30000)
    assert r["status"] == 9 and r["chunk"] > 0 and r["seqs"][:, 1].sum() == 5 * 20    # (one tile each: as many as sequences)
    # 20 sequences of 17 tokens, two tiles each, where lists of 21 tiles are enough for what does not repeat
    r = plan("packed", 17, alternating(17, 40), 8, 1, 64, cu_k=alternating(30000, 40), num_k=30000)
    assert r["status"] == 9 and r["chunk"] > 0


@pytest.mark.parametrize("kind", ["packed", "prefill", "shared"])
def test_offsets_that_do_not_ascend(kind):
    rng = np.random.RandomState(7 + len(kind))
    dropped = cut = 0
    for i in range(150):
        G, Hk, D = heads(rng)
        T, S = int(np.exp(rng.uniform(0, 7.5))), int(rng.randint(2, 60 if i % 10 else 1500))
        at = alternating(T, S)
        if i % 3 == 1:
            at = rng.randint(0, T + 1, S + 1)
        elif i % 3 == 2:
            at = np.where(rng.rand(S + 1) < 0.9, rng.randint(0, T + 1, S + 1), rng.choice([-1, -2 ** 31, T + 1, 2 ** 31 - 1], S + 1))
        keys = int(np.exp(rng.uniform(0, 10.5)))
        own = (at[:-1] >= 0) & (at[1:] >= at[:-1]) & (at[1:] <= T)
        if kind == "packed":
            ck = alternating(keys, S) if i % 2 else np.where(rng.rand(S + 1) < 0.95, rng.randint(0, keys + 1, S + 1), 2 ** 31 - 1)
            own &= (ck[:-1] >= 0) & (ck[1:] >= ck[:-1]) & (ck[1:] <= keys)
            r = plan(kind, T, at, G, Hk, D, cu_k=ck, num_k=keys, causal=bool(i & 1))
        elif kind == "prefill":
            ctx = np.where(rng.rand(S) < 0.9, keys, rng.choice([-1, -2 ** 31, 2 ** 31 - 1], S))
            blocks = (keys + T) // 16 + 1
            own &= (ctx >= 0) & ((at[1:] == at[:-1]) | (ctx.astype(np.int64) + at[1:] - at[:-1] <= blocks * 16))
            r = plan(kind, T, at, G, Hk, D, context=ctx, max_blocks=blocks)
        else:
            lens = np.where(rng.rand(T) < 0.8, keys + rng.randint(0, 300, T), rng.choice([0, -5, 2 ** 31 - 1], T))
            r = plan(kind, T, at, G, Hk, D, prefix=np.where(rng.rand(S) < 0.9, keys, rng.choice([-1, 2 ** 31 - 1], S)), lens=lens, max_blocks=keys // 16 + 30)
        n = np.where(own, at[1:] - at[:-1], 0)
        if kind != "shared":                                            # whole or left out, and in order as long as the lists have room
            got = r["seqs"][:, 1]
            assert ((got == n) | (got == 0)).all()
            room = np.cumsum(-(-n // (2 * r["W"]))) <= r["max_tiles"]
            assert (got[room] == n[room]).all()
            dropped += (~room).any()
        else:
            fits = r["status"] == 0 or r["num"] > 0
            dropped += not fits
        if not own.all():
            assert r["status"] == 9
        cut += r["chunk"] > 0
    assert dropped > 3 and cut > 3, (dropped, cut)
