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
