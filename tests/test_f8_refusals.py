"""The 8-bit entry points validate before any CUDA call (there may be no GPU here): statuses of the C ABI and the
exceptions of the Python wrappers."""
import pytest

torch = pytest.importorskip("torch")

import paper_2503_14985_b200 as mlt  # noqa: E402

INVALID, UNSUPPORTED, ALIGNMENT = 1, 2, 3


def test_quantize_statuses():
    q = mlt.quantize_f8_raw  # X, Q, scales, M, K, ldx, ldq, lds, block_rows
    assert q(16, 16, 16, -1, 8, 8, 16, 8, 1) == INVALID
    assert q(0, 0, 0, 0, 8, 8, 16, 8, 1) == 0 and q(0, 0, 0, 8, 0, 8, 16, 8, 128) == 0
    assert q(16, 16, 16, 4, 8, 8, 16, 4, 64) == UNSUPPORTED
    assert q(0, 16, 16, 4, 8, 8, 16, 4, 1) == INVALID and q(16, 16, 0, 4, 8, 8, 16, 4, 1) == INVALID
    assert q(16, 16, 16, 4, 8, 0, 16, 4, 1) == INVALID and q(16, 16, 16, 4, 24, 24, 16, 4, 1) == INVALID
    assert q(16, 16, 16, 4, 8, 8, 16, 3, 1) == INVALID and q(16, 16, 16, 4, 300, 304, 304, 2, 128) == INVALID
    assert q(18, 16, 16, 4, 8, 8, 16, 4, 1) == ALIGNMENT and q(16, 24, 16, 4, 8, 8, 16, 4, 1) == ALIGNMENT
    assert q(16, 16, 18, 4, 8, 8, 16, 4, 1) == ALIGNMENT
    assert q(16, 16, 16, 4, 8, 12, 16, 4, 1) == ALIGNMENT and q(16, 16, 16, 4, 8, 8, 24, 4, 1) == ALIGNMENT
    assert q(16, 16, 16, 2 ** 31, 8, 8, 16, 2 ** 31, 1) == UNSUPPORTED


def test_gemm_statuses():
    g = mlt.gemm_f8_raw  # A, sa, B, sb, C, M, N, K, lda, ldb, ldc, ldsa, ldsb
    assert g(16, 16, 16, 16, 16, -1, 8, 8, 16, 16, 8, 4, 1) == INVALID
    assert g(0, 0, 0, 0, 0, 0, 8, 8, 16, 16, 8, 4, 1) == 0 and g(0, 0, 0, 0, 0, 8, 0, 8, 16, 16, 8, 8, 1) == 0
    assert g(16, 16, 16, 16, 0, 4, 8, 8, 16, 16, 8, 4, 1) == INVALID
    for i in range(4):
        ptr = [16] * 5
        ptr[i] = 0
        assert g(*ptr, 4, 8, 8, 16, 16, 8, 4, 1) == INVALID
    assert g(16, 16, 16, 16, 16, 4, 8, 40, 32, 48, 8, 4, 1) == INVALID and g(16, 16, 16, 16, 16, 4, 8, 40, 48, 32, 8, 4, 1) == INVALID
    assert g(16, 16, 16, 16, 16, 4, 16, 8, 16, 16, 8, 4, 1) == INVALID
    assert g(16, 16, 16, 16, 16, 4, 8, 8, 16, 16, 8, 3, 1) == INVALID and g(16, 16, 16, 16, 16, 4, 8, 129, 144, 144, 8, 4, 1) == INVALID
    assert g(16, 16, 16, 16, 16, 4, 8, 8, 24, 16, 8, 4, 1) == ALIGNMENT and g(16, 16, 16, 16, 16, 4, 8, 8, 16, 24, 8, 4, 1) == ALIGNMENT
    assert g(16, 16, 16, 16, 16, 4, 8, 8, 16, 16, 12, 4, 1) == ALIGNMENT
    assert g(24, 16, 16, 16, 16, 4, 8, 8, 16, 16, 8, 4, 1) == ALIGNMENT and g(16, 18, 16, 16, 16, 4, 8, 8, 16, 16, 8, 4, 1) == ALIGNMENT
    assert g(16, 16, 16, 16, 24, 4, 8, 8, 16, 16, 8, 4, 1) == ALIGNMENT
    assert g(16, 16, 16, 16, 16, 2 ** 31, 8, 8, 16, 16, 8, 2 ** 31, 1) == UNSUPPORTED


APPEND = dict(Q=16, K=16, V=16, cos=16, sin=16, cu_tokens=16, context_lens=16, block_table=16, Q_out=16, K_cache=16, V_cache=16, k_scale=16,
              v_scale=16, num_tokens=4, num_seqs=2, H=8, H_kv=2, D=64, rotary_dim=64, interleaved=0, block_size=16, max_blocks=4,
              num_blocks=9, max_position=100, ldq=512, ldk=128, ldv=128, ldqo=512)


def append(f8, **changes):
    a = {**APPEND, **changes}
    if not f8:
        a.pop("k_scale"), a.pop("v_scale")
    return (mlt.kv_append_f8_raw if f8 else mlt.kv_append_raw)(**a)


@pytest.mark.parametrize("f8", [False, True])
def test_append_statuses(f8):
    assert append(f8, num_tokens=0) == 0 and append(f8, num_seqs=0) == 0
    for name in ("num_tokens", "num_seqs", "H", "H_kv", "rotary_dim", "max_blocks", "num_blocks", "max_position"):
        assert append(f8, **{name: -1}) == INVALID
    for name in ("K", "V", "K_cache", "V_cache", "cu_tokens", "context_lens", "block_table", "Q_out", "cos", "sin"):
        assert append(f8, **{name: 0}) == INVALID
    assert append(f8, H_kv=0) == INVALID and append(f8, H=0) == INVALID and append(f8, rotary_dim=80) == INVALID
    assert append(f8, D=96) == UNSUPPORTED and append(f8, block_size=64) == UNSUPPORTED and append(f8, rotary_dim=24) == UNSUPPORTED
    assert append(f8, H=65536, ldq=65536 * 64, ldqo=65536 * 64) == UNSUPPORTED and append(f8, num_seqs=2 ** 30) == UNSUPPORTED
    assert append(f8, ldk=120) == INVALID and append(f8, ldv=120) == INVALID and append(f8, ldq=504) == INVALID and append(f8, ldqo=504) == INVALID
    assert append(f8, ldk=132) == ALIGNMENT and append(f8, ldv=132) == ALIGNMENT and append(f8, ldq=516) == ALIGNMENT and append(f8, ldqo=516) == ALIGNMENT
    for name in ("Q", "K", "V", "Q_out", "K_cache", "V_cache", "cos", "sin"):
        assert append(f8, **{name: 24}) == ALIGNMENT
    if f8:
        assert append(f8, k_scale=0) == INVALID and append(f8, v_scale=0) == INVALID


DECODE = dict(Q=16, K_cache=16, V_cache=16, k_scale=16, v_scale=16, block_table=16, seq_lens=16, O=16, LSE=16, num_seqs=2, H=8, H_kv=2, D=64,
              block_size=16, max_blocks=4, num_blocks=9, scale=0.1)


def decode(**changes):
    return mlt.paged_attn_decode_f8_raw(**{**DECODE, **changes})


def test_decode_statuses():
    assert decode(num_seqs=0) == 0 and decode(H=0) == 0
    for name in ("num_seqs", "H", "H_kv", "max_blocks", "num_blocks"):
        assert decode(**{name: -1}) == INVALID
    for name in ("Q", "K_cache", "V_cache", "k_scale", "v_scale", "block_table", "seq_lens", "O"):
        assert decode(**{name: 0}) == INVALID
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert decode(scale=scale) == INVALID
    assert decode(H_kv=0) == INVALID and decode(H_kv=3) == INVALID
    assert decode(D=80) == UNSUPPORTED and decode(H=6) == UNSUPPORTED and decode(H=32) == UNSUPPORTED and decode(block_size=64) == UNSUPPORTED
    assert decode(num_blocks=2 ** 30) == UNSUPPORTED
    for name in ("Q", "K_cache", "V_cache", "O"):
        assert decode(**{name: 24}) == ALIGNMENT
    assert decode(workspace=24, workspace_bytes=1000) == ALIGNMENT


def test_workspace_bytes():
    w = mlt.paged_attn_f8_workspace_bytes
    assert w(0, 8, 2, 64) == 0 and w(4, 8, 3, 64) == 0
    assert w(4, 8, 2, 64) >= (4 * 2 + 2) * 4 * (64 * 4 + 8) and w(5, 8, 2, 64) > w(4, 8, 2, 64)


def test_bad_position_status_has_a_name():
    assert mlt.binding.STATUS_NAMES[9] == "MLT_ERR_BAD_POSITION" and "position" in mlt.status_string(9)


def test_wrappers_refuse_wrong_types_shapes_and_devices():
    bf, f8, i32 = torch.bfloat16, torch.float8_e4m3fn, torch.int32
    x = torch.zeros(4, 64, dtype=bf)
    with pytest.raises(ValueError):
        mlt.quantize_f8(x)                                      # not on a GPU
    with pytest.raises(TypeError):
        mlt.quantize_f8(x.float())
    with pytest.raises(ValueError):
        mlt.quantize_f8(x, block_rows=32)
    with pytest.raises(ValueError):
        mlt.quantize_f8(x.t())                                  # inner stride
    with pytest.raises(ValueError):
        mlt.quantize_f8(x, scales=torch.zeros(4, 1))            # layout of the other block form
    a, b, sa, sb = torch.zeros(4, 64).to(f8), torch.zeros(8, 64).to(f8), torch.ones(1, 4), torch.ones(1, 1)
    with pytest.raises(ValueError):
        mlt.gemm_f8(a, sa, b, sb)
    with pytest.raises(TypeError):
        mlt.gemm_f8(x, sa, b, sb)
    with pytest.raises(ValueError):
        mlt.gemm_f8(a, sa.t(), b, sb)
    with pytest.raises(ValueError):
        mlt.gemm_f8(a, sa, b, torch.ones(2, 1))
    q, k = torch.zeros(3, 4, 64, dtype=bf), torch.zeros(3, 2, 64, dtype=bf)
    cs, cu, ctx, table = torch.zeros(10, 32), torch.zeros(2, dtype=i32), torch.zeros(1, dtype=i32), torch.zeros(1, 2, dtype=i32)
    cache, ones = torch.zeros(5, 2, 16, 64, dtype=bf), torch.ones(5, 2)
    c8 = cache.to(f8)
    good = [q, k, k, cs, cs, cu, ctx, table, cache, cache]
    for i, wrong, err in ((0, q.float(), TypeError), (1, q, ValueError), (3, None, ValueError), (3, cs.double(), TypeError), (5, ctx, ValueError),
                          (6, ctx.long(), TypeError), (7, table[0], ValueError), (8, c8, TypeError), (9, cache[:4].contiguous(), ValueError),
                          (0, q.transpose(0, 1), ValueError)):
        bad = list(good)
        bad[i] = wrong
        with pytest.raises(err):
            mlt.kv_append(*bad)
    with pytest.raises(ValueError):
        mlt.kv_append(*good)                                    # not on a GPU
    with pytest.raises(TypeError):
        mlt.kv_append_f8(*good[:8], c8, c8, ones, ones.t())
    with pytest.raises(TypeError):
        mlt.kv_append_f8(*good, ones, ones)                     # a BF16 cache
    d = [q[:1], c8, c8, ones, ones, table, ctx]
    for i, wrong, err in ((0, q[:1].float(), TypeError), (1, cache, TypeError), (3, ones[:4], TypeError), (5, table.long(), TypeError),
                          (6, cu, ValueError), (0, torch.zeros(1, 4, 128, dtype=bf), ValueError)):
        bad = list(d)
        bad[i] = wrong
        with pytest.raises(err):
            mlt.paged_attn_decode_f8(*bad, scale=0.1)
    with pytest.raises(ValueError):
        mlt.paged_attn_decode_f8(*d, scale=0.1)                 # not on a GPU
