"""Calls of the 8-bit path whose inputs a long-running call just in front of them still has to write."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2503_14985_b200 as mlt  # noqa: E402

from gpu_util import assert_device_healthy  # noqa: E402

F8 = torch.float8_e4m3fn


def long_product(S, lens):
    """Operands of a product of 8 x 64 with a K of 2^20 (its few CTAs are busy for some hundred microseconds, store their result at
    the end, and release the launches behind them at the start) whose first row, read as 32-bit integers, is `lens`: lengths
    2048 + 16 f are the bit patterns of the BF16 numbers 2^-111 (1 + f / 8)."""
    K, KB = 1 << 20, 1 << 13
    A, B = torch.zeros(8, K, device="cuda").to(F8), torch.zeros(64, K, dtype=torch.uint8, device="cuda").view(F8)
    A[0, 0] = 1.0
    for s in range(S):
        B[2 * s, 0] = 1.0 + (int(lens[s]) - 2048) / 16 / 8
    sa, sb = torch.ones(KB, 8, device="cuda"), torch.ones(1, KB, device="cuda")
    sa[0, 0] = 2.0 ** -111
    return A, sa, B, sb


@pytest.mark.parametrize("S,H,Hkv", [(1, 8, 8), (2, 8, 1), (9, 4, 4), (32, 8, 2)])
def test_lengths_written_by_the_call_in_front(S, H, Hkv):
    D, bs, g = 64, 16, torch.Generator().manual_seed(S)
    lens = 2048 + 16 * torch.randint(0, 8, (S,), generator=g)
    width = 136                                                 # 2176 tokens
    table = torch.randperm(S * width, generator=g).view(S, width).to(torch.int32).cuda()
    kc, vc = (torch.randn(S * width, Hkv, bs, D, generator=g).to(F8).cuda() for _ in range(2))
    ks, vs = (torch.exp2(torch.randint(-3, 3, (S * width, Hkv), generator=g).float()).cuda() for _ in range(2))
    q = torch.randn(S, H, D, generator=g).to(torch.bfloat16).cuda()
    ws = torch.empty(mlt.paged_attn_f8_workspace_bytes(S, H, Hkv, D), dtype=torch.uint8, device="cuda")
    product = long_product(S, lens)
    C = torch.empty(8, 64, dtype=torch.bfloat16, device="cuda")
    seq_lens = C.view(torch.int32)[0, :S]

    def decode(O, LSE):
        mlt.paged_attn_decode_f8(q, kc, vc, ks, vs, table, seq_lens, scale=0.125, workspace=ws, O=O, LSE=LSE)

    def outputs():
        ws.fill_(0xFF)
        C.view(torch.int32).fill_(7)                            # the lengths of the step before
        return torch.full((S, H, D), 776.0, dtype=torch.bfloat16, device="cuda"), torch.full((S, H), 776.0, device="cuda")

    want = outputs()
    mlt.gemm_f8(*product, C)
    torch.cuda.synchronize()
    assert torch.equal(seq_lens.cpu(), lens.to(torch.int32))
    decode(*want)
    torch.cuda.synchronize()
    for _ in range(3):
        got = outputs()
        torch.cuda.synchronize()
        mlt.gemm_f8(*product, C)
        decode(*got)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph, got = torch.cuda.CUDAGraph(), outputs()
    with torch.cuda.graph(graph):
        mlt.gemm_f8(*product, C)
        decode(*got)
    outputs()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert_device_healthy()
