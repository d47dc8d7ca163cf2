"""Block tables so wide that a position no longer fits 32 bits are refused, and what just fits is planned right (no GPU needed)."""
import pytest

import __graft_entry__ as entry
from packed_plan_util import plan
from test_packed_refusals import BIG, prefill
from paper_2503_14985_b200 import binding


@pytest.fixture(scope="module", autouse=True)
def lib():
    entry.build()


@pytest.mark.parametrize("bs", [8, 16, 32])
def test_tables_beyond_32_bits(bs):
    def shared(**kw):
        a = dict(Q=16, K_cache=16, V_cache=16, block_table=16, seq_lens=16, prefix_lens=16, cu_groups=16, O=16, LSE=0, num_seqs=10, num_groups=2, H=8,
                 H_kv=2, D=128, block_size=bs, max_blocks=4, num_blocks=9, scale=1.0, workspace=256, workspace_bytes=BIG)
        a.update(kw)
        return binding.paged_attn_decode_shared_raw(**a)

    most = (2 ** 31 - 128) // bs
    for n in (most + 1, 2 ** 31 // bs, 2 ** 31 - 1):
        assert prefill(block_size=bs, max_blocks=n) == 2 and shared(max_blocks=n) == 2
    # (too little scratch is found later: what fits is not refused for its width)
    assert prefill(block_size=bs, max_blocks=most, workspace_bytes=100) == 1 and shared(max_blocks=most, workspace_bytes=100) == 1


@pytest.mark.parametrize("bs", [8, 32])
def test_the_longest_sequences(bs):
    most = 2 ** 31 - 128
    r = plan("prefill", 20, [0, 20], 4, 2, 128, context=[most - 20], bs=bs, max_blocks=most // bs)
    assert r["status"] == 0 and r["seqs"][0, 2] == most and r["entries"][:, 3].sum() == most // 128
    r = plan("prefill", 20, [0, 20], 4, 2, 128, context=[most - 19], bs=bs, max_blocks=most // bs)
    assert r["status"] == 9 and r["num"] == 0
    r = plan("shared", 3, [0, 3], 4, 2, 128, prefix=[most - 128], lens=[2 ** 31 - 1, 5, most - 127], bs=bs, max_blocks=most // bs)
    assert r["status"] == 0 and r["seqs"][:, 2].tolist() == [most - 128, 128, 0, 1]
