"""The packed and paged attention entry points refuse what they cannot do before any CUDA call (no GPU needed)."""
import pytest

import __graft_entry__ as entry
from paper_2503_14985_b200 import binding

BIG = 1 << 40


@pytest.fixture(scope="module", autouse=True)
def lib():
    entry.build()


def packed(**kw):
    a = dict(Q=16, K=16, V=16, cu_q=16, cu_k=16, O=16, LSE=0, num_q=10, num_k=10, num_seqs=2, H=8, H_kv=2, D=128, causal=1, scale=1.0, ldq=1024,
             ldk=256, ldv=256, ldo=1024, workspace=256, workspace_bytes=BIG)
    a.update(kw)
    return binding.mha_packed_fwd_raw(**a)


def prefill(**kw):
    a = dict(Q=16, K_cache=16, V_cache=16, cu_tokens=16, context_lens=16, block_table=16, O=16, LSE=0, num_tokens=10, num_seqs=2, H=8, H_kv=2, D=128,
             block_size=16, max_blocks=4, num_blocks=9, scale=1.0, ldq=1024, ldo=1024, workspace=256, workspace_bytes=BIG)
    a.update(kw)
    return binding.paged_attn_prefill_raw(**a)


@pytest.mark.parametrize("call,tokens", [(packed, "num_q"), (prefill, "num_tokens")])
def test_shared_refusals(call, tokens):
    assert call(**{tokens: 0}) == 0 and call(num_seqs=0) == 0          # nothing to do
    assert call(**{tokens: -1}) == 1 and call(num_seqs=-1) == 1
    assert call(Q=0) == 1 and call(O=0) == 1 and call(workspace=0) == 1
    assert call(H=9) == 1 and call(H_kv=0) == 1
    assert call(scale=0.0) == 1 and call(scale=float("nan")) == 1 and call(scale=float("inf")) == 1
    assert call(D=96, ldq=4096, ldo=4096) == 2
    assert call(H=258, H_kv=2, ldq=258 * 128, ldo=258 * 128) == 2      # 129 query heads per KV head
    assert call(ldq=1016) == 1 and call(ldo=1016) == 1
    assert call(ldq=1028) == 3 and call(ldo=1028) == 3
    assert call(Q=18) == 3 and call(O=24) == 3 and call(workspace=8) == 3
    assert call(workspace_bytes=100) == 1                              # too little for the list of work items


def test_counts_that_do_not_fit():
    for call in (packed, prefill):
        assert call(num_seqs=1 << 20) == 2                             # tile pairs
        assert call(num_seqs=(1 << 18) + 1, H=4096, H_kv=4096, ldq=4096 * 128, ldo=4096 * 128) == 2  # times KV heads


def test_packed_refusals():
    assert packed(K=0) == 1 and packed(cu_q=0) == 1 and packed(cu_k=0) == 1 and packed(num_k=-1) == 1
    assert packed(ldk=248) == 1 and packed(ldv=248) == 1 and packed(ldk=260) == 3


def test_prefill_refusals():
    assert prefill(K_cache=0) == 1 and prefill(context_lens=0) == 1 and prefill(block_table=0) == 1
    assert prefill(block_size=12) == 2 and prefill(block_size=64) == 2
    assert prefill(num_blocks=-1) == 1 and prefill(max_blocks=-1) == 1
    assert prefill(num_blocks=2 ** 30, H_kv=2) == 2


def test_workspace_size():
    size = binding.mha_packed_workspace_bytes
    assert size(0, 1, 8, 2, 128) == 0 and size(10, 1, 9, 2, 128) == 0
    assert size(10, 1, 8, 2, 128) >= 2 * 10 * 8 * (128 * 4 + 8)
    assert size(100000, 100, 32, 8, 128) >= 320 * 256 * (128 * 4 + 8)


def test_shared_refusals():
    def call(**kw):
        a = dict(Q=16, K_cache=16, V_cache=16, block_table=16, seq_lens=16, prefix_lens=16, cu_groups=16, O=16, LSE=0, num_seqs=10, num_groups=2, H=8,
                 H_kv=2, D=128, block_size=16, max_blocks=4, num_blocks=9, scale=1.0, workspace=256, workspace_bytes=BIG)
        a.update(kw)
        return binding.paged_attn_decode_shared_raw(**a)

    assert call(num_seqs=0) == 0 and call(num_seqs=0, workspace=0) == 0
    assert call(num_seqs=0, num_groups=0) == 0
    assert call(num_groups=-1) == 1 and call(prefix_lens=0) == 1 and call(cu_groups=0) == 1 and call(workspace=0) == 1
    assert call(workspace=8) == 3 and call(workspace_bytes=10000) == 1
    assert call(Q=0) == 1 and call(seq_lens=0) == 1 and call(block_table=0) == 1 and call(H=7) == 1 and call(scale=-1.0) == 1
    assert call(H=258, H_kv=2) == 2 and call(D=96) == 2 and call(block_size=64) == 2
    assert call(num_seqs=4090) == 2 and call(num_groups=4090) == 2 and call(num_blocks=2 ** 30) == 2
    size = binding.paged_attn_shared_workspace_bytes
    assert size(0, 1, 8, 2, 128) == 0 and size(8, 0, 8, 2, 128) >= 2 * 8 * 8 * (128 * 4 + 8)
    assert size(8, 1, 8, 2, 128) >= (2 * 8 * 8 + 256 * 2) * (128 * 4 + 8)


def test_w4_refusals():
    def call(**kw):
        a = dict(X=16, W=16, scales=16, zeros=16, C=16, M=4, N=100, K=256, group=64, ldx=256, ldw=128, lds=4, ldz=4, ldc=100)
        a.update(kw)
        return binding.gemm_w4_raw(**a)

    assert call(M=0) == 0 and call(N=0) == 0 and call(M=0, X=0, C=0) == 0
    assert call(M=-1) == 1 and call(X=0) == 1 and call(W=0) == 1 and call(scales=0) == 1 and call(C=0) == 1
    assert call(group=16) == 2 and call(group=256) == 2 and call(K=224, group=64) == 1
    assert call(ldx=248) == 1 and call(ldw=112) == 1 and call(lds=3) == 1 and call(ldz=3) == 1 and call(ldc=99) == 1
    assert call(ldx=260) == 3 and call(ldw=136) == 3 and call(X=8) == 3 and call(W=24) == 3 and call(scales=17) == 3 and call(C=17) == 3
    assert call(M=1 << 20) == 2
