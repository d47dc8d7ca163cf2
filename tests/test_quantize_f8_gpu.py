"""mlt_quantize_f8 against the FP64 oracle: codes and scales bit for bit (the scales are powers of two, so x / s is exact
and the one rounding has one right answer)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2503_14985_b200 as mlt  # noqa: E402
from oracle import f8  # noqa: E402

from gpu_util import assert_device_healthy, to_f64  # noqa: E402


def source(M, K, ldx, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(M, ldx, generator=g) * torch.exp2(torch.randint(-20, 20, (M, 1), generator=g).float())
    x = x.to(torch.bfloat16).cuda()
    x[:, K:] = float("nan")  # padding that a read would turn into a wrong code or scale
    return x[:, :K]


def check(x, block_rows, Q=None, scales=None):
    Q, scales = mlt.quantize_f8(x, block_rows=block_rows, Q=Q, scales=scales)
    assert_device_healthy()
    codes, want = f8.quantize(to_f64(x), block_rows)
    got = Q.view(torch.uint8).cpu().numpy()
    ref = f8.decode(codes)
    assert np.array_equal(f8.decode(got), ref, equal_nan=True)
    live = ~np.isnan(ref)
    assert np.array_equal(got[live], codes[live])  # the sign of zero too
    assert np.array_equal(scales.cpu().numpy().astype(np.float64), want.T if block_rows == 1 else want)


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("M,K", [(1, 1), (1, 128), (3, 40), (5, 129), (17, 300), (130, 257), (128, 256), (7, 1031), (300, 8), (16, 4096)])
def test_codes_and_scales(M, K, block_rows):
    check(source(M, K, (K + 7) // 8 * 8 + 8, seed=M * 1000 + K), block_rows)


@pytest.mark.parametrize("block_rows", [1, 128])
def test_special_values(block_rows):
    x = torch.zeros(140, 512, dtype=torch.bfloat16)
    x[0, :128] = float("inf")                                   # nothing finite
    x[1, 5], x[1, 6], x[1, 7], x[1, 8] = float("inf"), float("-inf"), float("nan"), 3.0
    x[2, 128:256] = -0.0
    x[3, 300] = 3.3895e38                                       # largest BF16
    x[3, 301] = 1e-38
    x[4, 400] = 1e-40                                           # subnormal alone: the smallest scale
    x[5, 0], x[5, 1] = 448.0, 1.0
    x[6, 0], x[6, 1] = 450.0, -1.0                              # just over: the next power of two
    x[7, 10:40] = torch.linspace(-17, 17, 30).to(torch.bfloat16)
    x[139, 511] = float("nan")
    check(x.cuda(), block_rows)


@pytest.mark.parametrize("block_rows", [1, 128])
def test_views_and_outputs_of_the_caller_and_nothing_outside(block_rows):
    M, K = 37, 200
    x = source(M, K, 264, seed=9)[:, 16:]                       # 16-byte aligned start inside a row
    K = x.shape[1]
    shape = (2, M) if block_rows == 1 else (1, 2)
    buf, sbuf = torch.full((M + 2, 256), 0x55, dtype=torch.uint8, device="cuda"), torch.full((shape[0] + 1, shape[1] + 3), 7.0, device="cuda")
    check(x, block_rows, buf[1:M + 1].view(torch.float8_e4m3fn)[:, :K], sbuf[:shape[0], :shape[1]])
    rest = buf.cpu().numpy()
    assert (rest[0] == 0x55).all() and (rest[-1] == 0x55).all() and (rest[1:-1, K:] == 0x55).all()
    assert (sbuf[shape[0]:] == 7.0).all() and (sbuf[:, shape[1]:] == 7.0).all()


def test_empty_and_misaligned():
    q, s = mlt.quantize_f8(torch.zeros(0, 128, dtype=torch.bfloat16, device="cuda"))
    assert q.shape == (0, 128) and s.shape == (1, 0)
    q, s = mlt.quantize_f8(torch.zeros(4, 0, dtype=torch.bfloat16, device="cuda"))
    assert q.shape == (4, 0) and s.shape == (0, 4)
    with pytest.raises(mlt.MltError) as e:
        mlt.quantize_f8(torch.zeros(4, 136, dtype=torch.bfloat16, device="cuda")[:, 4:])
    assert e.value.status == 3
    with pytest.raises(mlt.MltError) as e:
        mlt.quantize_f8(torch.zeros(4, 132, dtype=torch.bfloat16, device="cuda"))
    assert e.value.status == 3


def test_offsets_beyond_32_bits():
    # a matrix of 2.2 G elements: the last rows lie beyond 2^31 elements and (as BF16) 2^32 bytes
    M, K = 70000, 31744
    x = torch.empty(M, K, dtype=torch.bfloat16, device="cuda").fill_(1.0)
    x[-3:] = torch.randn(3, K, generator=torch.Generator().manual_seed(4)).to(torch.bfloat16).cuda()
    q, s = mlt.quantize_f8(x)
    codes, want = f8.quantize(to_f64(x[-3:]), 1)
    assert np.array_equal(q[-3:].view(torch.uint8).cpu().numpy(), codes)
    assert np.array_equal(s[:, -3:].cpu().numpy().astype(np.float64), want.T)
    assert (q[:100].float() == 256.0).all() and (s[:, :100] == 2.0 ** -8).all()


def test_other_stream_and_captured_graph():
    x = source(33, 500, 504, seed=11)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    q0, s0 = mlt.quantize_f8(x)
    with torch.cuda.stream(side):
        q1, s1 = mlt.quantize_f8(x)
    q2, s2 = mlt.quantize_f8(x, stream=side)
    torch.cuda.synchronize()
    for q, s in ((q1, s1), (q2, s2)):
        assert torch.equal(q.view(torch.uint8), q0.view(torch.uint8)) and torch.equal(s, s0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q3, s3 = mlt.quantize_f8(x)
    x.copy_(source(33, 500, 504, seed=12))
    graph.replay()
    q4, s4 = mlt.quantize_f8(x)
    torch.cuda.synchronize()
    assert torch.equal(q3.view(torch.uint8), q4.view(torch.uint8)) and torch.equal(s3, s4) and not torch.equal(s3, s0)
