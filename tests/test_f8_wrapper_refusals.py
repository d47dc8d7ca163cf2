"""Arguments that the Python entry points of the 8-bit path must refuse before anything is launched (no GPU needed)."""
import pytest

torch = pytest.importorskip("torch")

import paper_2503_14985_b200 as mlt  # noqa: E402

BF, F8, I32 = torch.bfloat16, torch.float8_e4m3fn, torch.int32


def decode_args():
    q, cache, ones = torch.zeros(2, 4, 64, dtype=BF), torch.zeros(5, 2, 16, 64).to(F8), torch.ones(5, 2)
    return [q, cache, cache, ones, ones, torch.zeros(2, 3, dtype=I32), torch.zeros(2, dtype=I32)]


@pytest.mark.parametrize("ws", [torch.zeros(1 << 16, dtype=torch.uint8)[::2], torch.zeros(256, 256, dtype=torch.uint8).t(), torch.zeros(256, 256, dtype=torch.uint8)[:, :128],
                                torch.zeros(1, dtype=torch.uint8).expand(1 << 16)])
def test_workspace_that_is_not_contiguous(ws):
    # the call takes the address and as many bytes as the view has elements: it would write what lies between them, or behind them
    with pytest.raises(TypeError, match="workspace"):
        mlt.paged_attn_decode_f8(*decode_args(), scale=0.1, workspace=ws)


@pytest.mark.parametrize("shape", [(2, 3), (2, 1, 2), (2, 0)])
def test_lengths_that_are_not_a_vector(shape):
    # [sequences, 3], say, would be read as if its first row held the lengths
    args = decode_args()
    args[6] = torch.zeros(shape, dtype=I32)
    with pytest.raises(ValueError, match="seq_lens"):
        mlt.paged_attn_decode_f8(*args, scale=0.1)
    q, k, cache = torch.zeros(3, 4, 64, dtype=BF), torch.zeros(3, 2, 64, dtype=BF), torch.zeros(5, 2, 16, 64, dtype=BF)
    cu, ctx, table = torch.zeros(3, dtype=I32), torch.zeros(2, dtype=I32), torch.zeros(2, 2, dtype=I32)
    wide = torch.zeros((3,) + shape[1:], dtype=I32)
    for c, x in ((wide, ctx), (cu, torch.zeros(shape, dtype=I32))):
        with pytest.raises(ValueError, match="cu_tokens"):
            mlt.kv_append(q, k, k, None, None, c, x, table, cache, cache)
        with pytest.raises(ValueError, match="cu_tokens"):
            mlt.kv_append_f8(q, k, k, None, None, c, x, table, cache.to(F8), cache.to(F8), torch.ones(5, 2), torch.ones(5, 2))


def test_columns_of_one_element_serve_as_vectors():
    args = decode_args()
    args[6] = args[6][:, None]
    with pytest.raises(ValueError, match="CUDA"):               # the next check: the tensors are not on a GPU
        mlt.paged_attn_decode_f8(*args, scale=0.1)
    k, cache = torch.zeros(3, 2, 64, dtype=BF), torch.zeros(5, 2, 16, 64, dtype=BF)
    with pytest.raises(ValueError, match="CUDA"):
        mlt.kv_append(None, k, k, None, None, torch.zeros(2, 1, dtype=I32), torch.zeros(1, 1, dtype=I32), torch.zeros(1, 2, dtype=I32), cache, cache)
