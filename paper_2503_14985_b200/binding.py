"""Thin ctypes binding over the C ABI of include/mlt.h.

Argument marshalling only: every step of the GEMM and of the attention forward
runs inside the CUDA kernels of libmlt.so.  There is no fallback: if the library
is missing or the device is not sm_100, calls raise.
"""
from __future__ import annotations

import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmlt.so")

MLT_OK = 0
STATUS_NAMES = {0: "MLT_OK", 1: "MLT_ERR_INVALID_ARG", 2: "MLT_ERR_UNSUPPORTED", 3: "MLT_ERR_ALIGNMENT",
                4: "MLT_ERR_CUDA", 5: "MLT_ERR_ARCH", 6: "MLT_ERR_TIMEOUT", 7: "MLT_ERR_BAD_BLOCK",
                8: "MLT_ERR_SCRATCH_LIMIT", 9: "MLT_ERR_BAD_POSITION"}
PAGED_STATIC_SCRATCH_BYTES = 16 * 1024 * 1024

EXPORTS = ("mlt_gemm", "mlt_gemm_f16", "mlt_gemm_ex", "mlt_gemm_workspace_bytes", "mlt_mha_fwd", "mlt_paged_attn_decode", "mlt_paged_attn_decode_static",
           "mlt_paged_attn_workspace_bytes",
           "mlt_quantize_f8", "mlt_gemm_f8", "mlt_kv_append", "mlt_kv_append_f8", "mlt_paged_attn_decode_f8", "mlt_paged_attn_f8_workspace_bytes",
           "mlt_mha_packed_fwd", "mlt_mha_packed_workspace_bytes", "mlt_paged_attn_prefill",
           "mlt_paged_attn_decode_shared", "mlt_paged_attn_shared_workspace_bytes", "mlt_gemm_w4",
           "mlt_last_device_error", "mlt_debug_wait_timeout_selftest", "mlt_debug_last_clock_mhz", "mlt_debug_gemm_plan", "mlt_debug_gemm_f8_plan", "mlt_status_string",
           "mlt_version")

_lib = None


class MltError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {STATUS_NAMES.get(status, status)} ({status_string(status)})")


def load() -> ctypes.CDLL:
    """Load libmlt.so (built in-tree by paper_2503_14985_b200.build); raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(f"{LIB_PATH} not found: build it with `python -m paper_2503_14985_b200.build`")
        lib = ctypes.CDLL(LIB_PATH)
        i64, p, i32 = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int
        lib.mlt_gemm.argtypes = [p, p, p, i64, i64, i64, i64, i64, i64, p]
        lib.mlt_gemm.restype = i32
        lib.mlt_debug_wait_timeout_selftest.argtypes = [ctypes.c_uint64, p]
        lib.mlt_debug_wait_timeout_selftest.restype = i32
        lib.mlt_debug_last_clock_mhz.argtypes = [i32, ctypes.POINTER(ctypes.c_double)]
        lib.mlt_debug_last_clock_mhz.restype = i32
        lib.mlt_debug_gemm_plan.argtypes = [i64, i64, i64, ctypes.c_size_t, i32, ctypes.POINTER(ctypes.c_int)]
        lib.mlt_debug_gemm_plan.restype = i32
        lib.mlt_debug_gemm_f8_plan.argtypes = [i64, i64, i64, i32, ctypes.POINTER(ctypes.c_int)]
        lib.mlt_debug_gemm_f8_plan.restype = i32
        lib.mlt_gemm_f16.argtypes = [p, p, p, i64, i64, i64, i64, i64, i64, i32, p]
        lib.mlt_gemm_f16.restype = i32
        lib.mlt_gemm_ex.argtypes = [p, p, p, i64, i64, i64, i64, i64, i64, p, ctypes.c_size_t, p]
        lib.mlt_gemm_ex.restype = i32
        lib.mlt_gemm_workspace_bytes.argtypes = [i64, i64, i64]
        lib.mlt_gemm_workspace_bytes.restype = ctypes.c_size_t
        lib.mlt_mha_fwd.argtypes = [p, p, p, p, p, i32, i32, i32, i32, i32, i32, ctypes.c_float, p]
        lib.mlt_mha_fwd.restype = i32
        lib.mlt_paged_attn_workspace_bytes.argtypes = [i32, i32, i32]
        lib.mlt_paged_attn_workspace_bytes.restype = ctypes.c_size_t
        lib.mlt_paged_attn_decode.argtypes = [p, p, p, p, p, p, p, i32, i32, i32, i32, i32, i32, i32, ctypes.c_float,
                                              p, ctypes.c_size_t, p]
        lib.mlt_paged_attn_decode.restype = i32
        lib.mlt_paged_attn_decode_static.argtypes = [p, p, p, p, p, p, p, i32, i32, i32, i32, i32, i32, i32,
                                                     ctypes.c_float, p]
        lib.mlt_paged_attn_decode_static.restype = i32
        lib.mlt_quantize_f8.argtypes = [p, p, p, i64, i64, i64, i64, i64, i32, p]
        lib.mlt_quantize_f8.restype = i32
        lib.mlt_gemm_f8.argtypes = [p, p, p, p, p, i64, i64, i64, i64, i64, i64, i64, i64, p]
        lib.mlt_gemm_f8.restype = i32
        lib.mlt_kv_append.argtypes = [p] * 11 + [i32] * 11 + [i64] * 4 + [p]
        lib.mlt_kv_append.restype = i32
        lib.mlt_kv_append_f8.argtypes = [p] * 13 + [i32] * 11 + [i64] * 4 + [p]
        lib.mlt_kv_append_f8.restype = i32
        lib.mlt_paged_attn_f8_workspace_bytes.argtypes = [i32, i32, i32, i32]
        lib.mlt_paged_attn_f8_workspace_bytes.restype = ctypes.c_size_t
        lib.mlt_paged_attn_decode_f8.argtypes = [p] * 9 + [i32] * 7 + [ctypes.c_float, p, ctypes.c_size_t, p]
        lib.mlt_paged_attn_decode_f8.restype = i32
        lib.mlt_mha_packed_workspace_bytes.argtypes = [i32] * 5
        lib.mlt_mha_packed_workspace_bytes.restype = ctypes.c_size_t
        lib.mlt_mha_packed_fwd.argtypes = [p] * 7 + [i32] * 7 + [ctypes.c_float] + [i64] * 4 + [p, ctypes.c_size_t, p]
        lib.mlt_mha_packed_fwd.restype = i32
        lib.mlt_paged_attn_prefill.argtypes = [p] * 8 + [i32] * 8 + [ctypes.c_float] + [i64] * 2 + [p, ctypes.c_size_t, p]
        lib.mlt_paged_attn_prefill.restype = i32
        lib.mlt_paged_attn_shared_workspace_bytes.argtypes = [i32] * 5
        lib.mlt_paged_attn_shared_workspace_bytes.restype = ctypes.c_size_t
        lib.mlt_paged_attn_decode_shared.argtypes = [p] * 9 + [i32] * 8 + [ctypes.c_float, p, ctypes.c_size_t, p]
        lib.mlt_paged_attn_decode_shared.restype = i32
        lib.mlt_gemm_w4.argtypes = [p] * 5 + [i64] * 3 + [i32] + [i64] * 5 + [p]
        lib.mlt_gemm_w4.restype = i32
        lib.mlt_last_device_error.argtypes = [p]
        lib.mlt_last_device_error.restype = i32
        lib.mlt_status_string.argtypes = [i32]
        lib.mlt_status_string.restype = ctypes.c_char_p
        lib.mlt_version.restype = i32
        _lib = lib
    return _lib


def status_string(status: int) -> str:
    return load().mlt_status_string(int(status)).decode()


def version() -> int:
    return int(load().mlt_version())


def gemm_raw(A: int, B: int, C: int, M: int, N: int, K: int, lda: int, ldb: int, ldc: int, stream: int = 0) -> int:
    """mlt_gemm with raw device addresses; returns the status code."""
    return int(load().mlt_gemm(A, B, C, M, N, K, lda, ldb, ldc, stream))


def debug_wait_timeout_selftest(budget_cycles: int, stream: int = 0) -> int:
    """Launches the bounded-wait self-test (a wait that runs out after `budget_cycles` SM clocks); returns the status."""
    return int(load().mlt_debug_wait_timeout_selftest(budget_cycles, stream))


def gemm_f16_raw(A: int, B: int, C: int, M: int, N: int, K: int, lda: int, ldb: int, ldc: int, accumulate: int,
                 stream: int = 0) -> int:
    """mlt_gemm_f16 (FP16 operands, FP32 result, optional C += A*B) with raw device addresses."""
    return int(load().mlt_gemm_f16(A, B, C, M, N, K, lda, ldb, ldc, accumulate, stream))


def gemm_workspace_bytes(M: int, N: int, K: int) -> int:
    return int(load().mlt_gemm_workspace_bytes(M, N, K))


def gemm_ex_raw(A: int, B: int, C: int, M: int, N: int, K: int, lda: int, ldb: int, ldc: int, workspace: int = 0,
                workspace_bytes: int = 0, stream: int = 0) -> int:
    """mlt_gemm_ex (split-K with caller scratch for skinny problems) with raw device addresses."""
    return int(load().mlt_gemm_ex(A, B, C, M, N, K, lda, ldb, ldc, workspace, workspace_bytes, stream))


def mha_fwd_raw(Q: int, K: int, V: int, O: int, LSE: int, B: int, H: int, Nq: int, Nk: int, D: int, causal: int,
                scale: float, stream: int = 0) -> int:
    """mlt_mha_fwd with raw device addresses; returns the status code."""
    return int(load().mlt_mha_fwd(Q, K, V, O, LSE, B, H, Nq, Nk, D, causal, scale, stream))


def paged_attn_workspace_bytes(num_seqs: int, H: int, D: int) -> int:
    return int(load().mlt_paged_attn_workspace_bytes(num_seqs, H, D))


def paged_attn_decode_raw(Q: int, K_cache: int, V_cache: int, block_table: int, seq_lens: int, O: int, LSE: int,
                          num_seqs: int, H: int, H_kv: int, D: int, block_size: int, max_blocks: int, num_blocks: int,
                          scale: float, workspace: int = 0, workspace_bytes: int = 0, stream: int = 0) -> int:
    """mlt_paged_attn_decode with raw device addresses; returns the status code."""
    return int(load().mlt_paged_attn_decode(Q, K_cache, V_cache, block_table, seq_lens, O, LSE, num_seqs, H, H_kv, D,
                                            block_size, max_blocks, num_blocks, scale, workspace, workspace_bytes,
                                            stream))


def paged_attn_decode_static_raw(Q: int, K_cache: int, V_cache: int, block_table: int, seq_lens: int, O: int, LSE: int,
                                 num_seqs: int, H: int, H_kv: int, D: int, block_size: int, max_blocks: int,
                                 num_blocks: int, scale: float, stream: int = 0) -> int:
    """mlt_paged_attn_decode_static (scratch inside the library, nothing allocated) with raw device addresses."""
    return int(load().mlt_paged_attn_decode_static(Q, K_cache, V_cache, block_table, seq_lens, O, LSE, num_seqs, H,
                                                   H_kv, D, block_size, max_blocks, num_blocks, scale, stream))


def quantize_f8_raw(X: int, Q: int, scales: int, M: int, K: int, ldx: int, ldq: int, lds: int, block_rows: int,
                    stream: int = 0) -> int:
    """mlt_quantize_f8 with raw device addresses; returns the status code."""
    return load().mlt_quantize_f8(X, Q, scales, M, K, ldx, ldq, lds, block_rows, stream)


def gemm_f8_raw(A: int, scale_a: int, B: int, scale_b: int, C: int, M: int, N: int, K: int, lda: int, ldb: int, ldc: int,
                ldsa: int, ldsb: int, stream: int = 0) -> int:
    """mlt_gemm_f8 with raw device addresses; returns the status code."""
    return load().mlt_gemm_f8(A, scale_a, B, scale_b, C, M, N, K, lda, ldb, ldc, ldsa, ldsb, stream)


def kv_append_raw(Q: int, K: int, V: int, cos: int, sin: int, cu_tokens: int, context_lens: int, block_table: int,
                  Q_out: int, K_cache: int, V_cache: int, num_tokens: int, num_seqs: int, H: int, H_kv: int, D: int,
                  rotary_dim: int, interleaved: int, block_size: int, max_blocks: int, num_blocks: int, max_position: int,
                  ldq: int, ldk: int, ldv: int, ldqo: int, stream: int = 0) -> int:
    """mlt_kv_append (BF16 cache) with raw device addresses; returns the status code."""
    return load().mlt_kv_append(Q, K, V, cos, sin, cu_tokens, context_lens, block_table, Q_out, K_cache, V_cache, num_tokens,
                                num_seqs, H, H_kv, D, rotary_dim, interleaved, block_size, max_blocks, num_blocks,
                                max_position, ldq, ldk, ldv, ldqo, stream)


def kv_append_f8_raw(Q: int, K: int, V: int, cos: int, sin: int, cu_tokens: int, context_lens: int, block_table: int,
                     Q_out: int, K_cache: int, V_cache: int, k_scale: int, v_scale: int, num_tokens: int, num_seqs: int,
                     H: int, H_kv: int, D: int, rotary_dim: int, interleaved: int, block_size: int, max_blocks: int,
                     num_blocks: int, max_position: int, ldq: int, ldk: int, ldv: int, ldqo: int, stream: int = 0) -> int:
    """mlt_kv_append_f8 (E4M3 cache) with raw device addresses; returns the status code."""
    return load().mlt_kv_append_f8(Q, K, V, cos, sin, cu_tokens, context_lens, block_table, Q_out, K_cache, V_cache, k_scale,
                                   v_scale, num_tokens, num_seqs, H, H_kv, D, rotary_dim, interleaved, block_size,
                                   max_blocks, num_blocks, max_position, ldq, ldk, ldv, ldqo, stream)


def paged_attn_f8_workspace_bytes(num_seqs: int, H: int, H_kv: int, D: int) -> int:
    return int(load().mlt_paged_attn_f8_workspace_bytes(num_seqs, H, H_kv, D))


def paged_attn_decode_f8_raw(Q: int, K_cache: int, V_cache: int, k_scale: int, v_scale: int, block_table: int,
                             seq_lens: int, O: int, LSE: int, num_seqs: int, H: int, H_kv: int, D: int, block_size: int,
                             max_blocks: int, num_blocks: int, scale: float, workspace: int = 0, workspace_bytes: int = 0,
                             stream: int = 0) -> int:
    """mlt_paged_attn_decode_f8 with raw device addresses; returns the status code."""
    return load().mlt_paged_attn_decode_f8(Q, K_cache, V_cache, k_scale, v_scale, block_table, seq_lens, O, LSE, num_seqs, H,
                                           H_kv, D, block_size, max_blocks, num_blocks, scale, workspace, workspace_bytes,
                                           stream)


def mha_packed_workspace_bytes(num_q: int, num_seqs: int, H: int, H_kv: int, D: int) -> int:
    return int(load().mlt_mha_packed_workspace_bytes(num_q, num_seqs, H, H_kv, D))


def mha_packed_fwd_raw(Q: int, K: int, V: int, cu_q: int, cu_k: int, O: int, LSE: int, num_q: int, num_k: int, num_seqs: int, H: int,
                       H_kv: int, D: int, causal: int, scale: float, ldq: int, ldk: int, ldv: int, ldo: int, workspace: int,
                       workspace_bytes: int, stream: int = 0) -> int:
    """mlt_mha_packed_fwd with raw device addresses; returns the status code."""
    return load().mlt_mha_packed_fwd(Q, K, V, cu_q, cu_k, O, LSE, num_q, num_k, num_seqs, H, H_kv, D, causal, scale, ldq, ldk, ldv, ldo,
                                     workspace, workspace_bytes, stream)


def paged_attn_prefill_raw(Q: int, K_cache: int, V_cache: int, cu_tokens: int, context_lens: int, block_table: int, O: int, LSE: int,
                           num_tokens: int, num_seqs: int, H: int, H_kv: int, D: int, block_size: int, max_blocks: int, num_blocks: int,
                           scale: float, ldq: int, ldo: int, workspace: int, workspace_bytes: int, stream: int = 0) -> int:
    """mlt_paged_attn_prefill with raw device addresses; returns the status code."""
    return load().mlt_paged_attn_prefill(Q, K_cache, V_cache, cu_tokens, context_lens, block_table, O, LSE, num_tokens, num_seqs, H, H_kv, D,
                                         block_size, max_blocks, num_blocks, scale, ldq, ldo, workspace, workspace_bytes, stream)


def paged_attn_shared_workspace_bytes(num_seqs: int, num_groups: int, H: int, H_kv: int, D: int) -> int:
    return int(load().mlt_paged_attn_shared_workspace_bytes(num_seqs, num_groups, H, H_kv, D))


def paged_attn_decode_shared_raw(Q: int, K_cache: int, V_cache: int, block_table: int, seq_lens: int, prefix_lens: int, cu_groups: int, O: int,
                                 LSE: int, num_seqs: int, num_groups: int, H: int, H_kv: int, D: int, block_size: int, max_blocks: int,
                                 num_blocks: int, scale: float, workspace: int, workspace_bytes: int, stream: int = 0) -> int:
    """mlt_paged_attn_decode_shared with raw device addresses; returns the status code."""
    return load().mlt_paged_attn_decode_shared(Q, K_cache, V_cache, block_table, seq_lens, prefix_lens, cu_groups, O, LSE, num_seqs, num_groups,
                                               H, H_kv, D, block_size, max_blocks, num_blocks, scale, workspace, workspace_bytes, stream)


def gemm_w4_raw(X: int, W: int, scales: int, zeros: int, C: int, M: int, N: int, K: int, group: int, ldx: int, ldw: int, lds: int, ldz: int,
                ldc: int, stream: int = 0) -> int:
    """mlt_gemm_w4 with raw device addresses; returns the status code."""
    return load().mlt_gemm_w4(X, W, scales, zeros, C, M, N, K, group, ldx, ldw, lds, ldz, ldc, stream)


def last_device_error():
    """Synchronise, read and clear the device status word: (status, [code, barrier, block, aux])."""
    detail = (ctypes.c_uint32 * 4)()
    rc = int(load().mlt_last_device_error(ctypes.cast(detail, ctypes.c_void_p)))
    return rc, list(detail)


def last_clock_mhz(which: int) -> float:
    """SM clock in MHz that the last GEMM (which = 0) or attention (which = 1) launch ran at; 0.0 if none has run."""
    mhz = ctypes.c_double(0.0)
    rc = int(load().mlt_debug_last_clock_mhz(which, ctypes.byref(mhz)))
    if rc != MLT_OK:
        raise MltError(rc, "mlt_debug_last_clock_mhz")
    return float(mhz.value)


def gemm_plan(M: int, N: int, K: int, workspace_bytes: int = 0, sm_count: int = 148) -> dict:
    """Launch plan of gemm / gemm_ex for a shape: tile variant, K slices through the workspace, CTAs per K-cutting
    cluster, K blocks of 64 per slice.  sm_count >= 2: host arithmetic for such a device, no GPU; 0: the current device."""
    out = (ctypes.c_int * 4)()
    rc = int(load().mlt_debug_gemm_plan(M, N, K, workspace_bytes, sm_count, out))
    if rc != MLT_OK:
        raise MltError(rc, "mlt_debug_gemm_plan")
    return {"variant": out[0], "split_k": out[1], "cluster": out[2], "kb_per_split": out[3]}


def gemm_f8_plan(M: int, N: int, K: int, sm_count: int = 148) -> dict:
    """Launch plan of gemm_f8 for a shape: kernel (0: one tile per cluster, 1: 128 x 256 tiles, 2: CTA pairs), tile width, CTAs
    per K-cutting cluster, shared memory of kernel 0.  sm_count as in gemm_plan."""
    out = (ctypes.c_int * 4)()
    rc = int(load().mlt_debug_gemm_f8_plan(M, N, K, sm_count, out))
    if rc != MLT_OK:
        raise MltError(rc, "mlt_debug_gemm_f8_plan")
    return {"kernel": out[0], "tile_n": out[1], "cluster": out[2], "smem": out[3]}


def _stream(stream) -> int:
    import torch
    if stream is None:
        return int(torch.cuda.current_stream().cuda_stream)
    return int(getattr(stream, "cuda_stream", stream))


def gemm(A, B, C=None, *, M=None, N=None, K=None, stream=None):
    """C = A @ B for torch.bfloat16 CUDA tensors: A (M, K), B (K, N), row-major with unit inner stride.

    Row pitches are taken from the tensors' strides, so padded views work.  Returns C.
    """
    import torch
    if A.dtype != torch.bfloat16 or B.dtype != torch.bfloat16 or not A.is_cuda or not B.is_cuda:
        raise TypeError("A and B must be CUDA bfloat16 tensors")
    M = A.shape[0] if M is None else M
    K = A.shape[1] if K is None else K
    N = B.shape[1] if N is None else N
    if C is None:
        C = torch.empty((M, N), dtype=torch.bfloat16, device=A.device)
    for t in (A, B, C):
        if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
            raise ValueError("operands must be 2-D with unit inner stride")
    lda = A.stride(0) if A.shape[0] > 1 else max(A.stride(0), K)
    ldb = B.stride(0) if B.shape[0] > 1 else max(B.stride(0), N)
    ldc = C.stride(0) if C.shape[0] > 1 else max(C.stride(0), N)
    rc = gemm_raw(A.data_ptr(), B.data_ptr(), C.data_ptr(), M, N, K, lda, ldb, ldc, _stream(stream))
    if rc != MLT_OK:
        raise MltError(rc, "mlt_gemm")
    return C


def mha_fwd(Q, K, V, *, causal: bool, scale: float, O=None, LSE=None, return_lse: bool = True, stream=None):
    """Attention forward for contiguous torch.bfloat16 CUDA tensors Q [B,H,Nq,D], K,V [B,H,Nk,D].

    Returns (O [B,H,Nq,D] bfloat16, LSE [B,H,Nq] float32 or None).
    """
    import torch
    for t in (Q, K, V):
        if t.dtype != torch.bfloat16 or not t.is_cuda or not t.is_contiguous() or t.dim() != 4:
            raise TypeError("Q, K, V must be contiguous 4-D CUDA bfloat16 tensors")
    Bn, H, Nq, D = Q.shape
    Nk = K.shape[2]
    if tuple(K.shape) != (Bn, H, Nk, D) or K.shape != V.shape:
        raise ValueError("shape mismatch")
    if O is None:
        O = torch.empty_like(Q)
    if LSE is None and return_lse:
        LSE = torch.empty((Bn, H, Nq), dtype=torch.float32, device=Q.device)
    rc = mha_fwd_raw(Q.data_ptr(), K.data_ptr(), V.data_ptr(), O.data_ptr(), LSE.data_ptr() if LSE is not None else 0,
                     Bn, H, Nq, Nk, D, int(bool(causal)), float(scale), _stream(stream))
    if rc != MLT_OK:
        raise MltError(rc, "mlt_mha_fwd")
    return O, LSE


def paged_attn_decode(Q, K_cache, V_cache, block_table, seq_lens, *, scale: float, workspace=None, O=None, LSE=None,
                      return_lse: bool = True, stream=None):
    """Paged-attention decode for CUDA tensors: Q [S,H,D] bfloat16, caches [num_blocks,H_kv,block_size,D] bfloat16,
    block_table [S,max_blocks] int32, seq_lens [S] int32.  `workspace` is an optional uint8 CUDA tensor (see
    paged_attn_workspace_bytes).  Returns (O [S,H,D] bfloat16, LSE [S,H] float32 or None).
    """
    import torch
    for t in (Q, K_cache, V_cache):
        if t.dtype != torch.bfloat16 or not t.is_cuda or not t.is_contiguous():
            raise TypeError("Q and the caches must be contiguous CUDA bfloat16 tensors")
    for t in (block_table, seq_lens):
        if t.dtype != torch.int32 or not t.is_cuda or not t.is_contiguous():
            raise TypeError("block_table and seq_lens must be contiguous CUDA int32 tensors")
    S, H, D = Q.shape
    NB, H_kv, bs, _ = K_cache.shape
    if O is None:
        O = torch.empty_like(Q)
    if LSE is None and return_lse:
        LSE = torch.empty((S, H), dtype=torch.float32, device=Q.device)
    rc = paged_attn_decode_raw(Q.data_ptr(), K_cache.data_ptr(), V_cache.data_ptr(), block_table.data_ptr(),
                               seq_lens.data_ptr(), O.data_ptr(), LSE.data_ptr() if LSE is not None else 0, S, H, H_kv, D,
                               bs, block_table.shape[1], NB, float(scale),
                               workspace.data_ptr() if workspace is not None else 0,
                               workspace.numel() * workspace.element_size() if workspace is not None else 0,
                               _stream(stream))
    if rc != MLT_OK:
        raise MltError(rc, "mlt_paged_attn_decode")
    return O, LSE


_f8_dtype = None


def _f8():
    global _f8_dtype
    if _f8_dtype is None:
        import torch
        _f8_dtype = torch.float8_e4m3fn
    return _f8_dtype


def _call(name, fn, tensors, args, stream):
    """fn(*args, stream address) with the tensors' device current; they must all be CUDA tensors of one device.

    The stream is torch's current one of that device (asked for by its raw handle: building a torch.cuda.Stream object
    takes 3 us), or the caller's.
    """
    import torch
    index = tensors[0].get_device()
    for t in tensors:
        if t.get_device() != index:
            index = -1
    if index < 0:
        raise ValueError("all tensors must be on one CUDA device")
    st = torch._C._cuda_getCurrentRawStream(index) if stream is None else _stream(stream)
    if torch._C._cuda_getDevice() == index:
        rc = fn(*args, st)
    else:
        with torch.cuda.device(index):
            rc = fn(*args, st)
    if rc != MLT_OK:
        raise MltError(rc, name)


def _new(t, shape, dtype, stream):
    """An output on t's device.  Its memory belongs to the stream that the call runs on: the allocator's blocks of another
    stream may still be in use by what that stream has under way."""
    if stream is None or not t.is_cuda:
        return t.new_empty(shape, dtype=dtype)
    import torch
    if not isinstance(stream, torch.cuda.Stream):
        address = _stream(stream)
        stream = torch.cuda.ExternalStream(address, device=t.device) if address else torch.cuda.default_stream(t.device)
    with torch.cuda.stream(stream):
        return t.new_empty(shape, dtype=dtype)


def _pitch(t, width):
    """Row pitch of a 2-D tensor with unit inner stride (of a single row: any pitch serves)."""
    st = t.stride()
    if len(st) != 2 or (st[1] != 1 and t.shape[1] > 1):
        raise ValueError("matrices must be 2-D with unit inner stride")
    return st[0] if t.shape[0] > 1 else width


def quantize_f8(X, *, block_rows: int = 1, Q=None, scales=None, stream=None):
    """X [M, K] bfloat16 -> (Q [M, K] float8_e4m3fn, scales float32), one power-of-two scale per block.

    block_rows 1 (activations): 1 x 128 blocks, scales [ceil(K / 128), M].  block_rows 128 (weights): 128 x 128 blocks,
    scales [ceil(M / 128), ceil(K / 128)].  Both are what gemm_f8 takes.  Row pitches come from the tensors' strides; the
    pitch of a new Q is K rounded up to 16.
    """
    import torch
    if X.dtype != torch.bfloat16:
        raise TypeError("X must be bfloat16")
    if block_rows not in (1, 128):
        raise ValueError("block_rows must be 1 or 128")
    M, K = X.shape
    up16 = (K + 15) // 16 * 16
    kb = (K + 127) // 128
    shape = (kb, M) if block_rows == 1 else ((M + 127) // 128, kb)
    ldx = _pitch(X, (K + 7) // 8 * 8)
    if Q is None:
        Q = _new(X, (M, up16), _f8(), stream)
        if up16 != K:
            Q = Q[:, :K]
        ldq = up16
    elif Q.dtype != _f8():
        raise TypeError("Q must be float8_e4m3fn")
    elif Q.shape != X.shape:
        raise ValueError("Q must have the shape of X")
    else:
        ldq = _pitch(Q, up16)
    if scales is None:
        scales = _new(X, shape, torch.float32, stream)
        lds = shape[1]
    elif scales.dtype != torch.float32:
        raise TypeError("scales must be float32")
    elif tuple(scales.shape) != shape:
        raise ValueError(f"scales must be {shape}")
    else:
        lds = _pitch(scales, shape[1])
    _call("mlt_quantize_f8", load().mlt_quantize_f8, (X, Q, scales),
          (X.data_ptr(), Q.data_ptr(), scales.data_ptr(), M, K, ldx, ldq, lds, block_rows), stream)
    return Q, scales


def gemm_f8(A, scale_a, B, scale_b, C=None, *, stream=None):
    """C = (A scaled) @ (B scaled).T in bfloat16 for float8_e4m3fn A [M, K] and B [N, K] with K contiguous.

    scale_a [ceil(K / 128), M] and scale_b [ceil(N / 128), ceil(K / 128)], float32 (see quantize_f8).  Row pitches come
    from the tensors' strides (A, B: multiples of 16 bytes; C: of 8 elements; a new C has N rounded up to 8).
    """
    import torch
    f8, f32 = _f8(), torch.float32
    if A.dtype != f8 or B.dtype != f8 or scale_a.dtype != f32 or scale_b.dtype != f32:
        raise TypeError("A and B must be float8_e4m3fn, the scales float32")
    (M, K), (N, Kb) = A.shape, B.shape
    kb = (K + 127) // 128
    if Kb != K or tuple(scale_a.shape) != (kb, M) or tuple(scale_b.shape) != ((N + 127) // 128, kb):
        raise ValueError("shape mismatch")
    up8, up16 = (N + 7) // 8 * 8, (K + 15) // 16 * 16
    if C is None:
        C = _new(A, (M, up8), torch.bfloat16, stream)
        if up8 != N:
            C = C[:, :N]
        ldc = up8
    elif C.dtype != torch.bfloat16 or tuple(C.shape) != (M, N):
        raise ValueError("C must be bfloat16 [M, N]")
    else:
        ldc = _pitch(C, up8)
    _call("mlt_gemm_f8", load().mlt_gemm_f8, (A, scale_a, B, scale_b, C),
          (A.data_ptr(), scale_a.data_ptr(), B.data_ptr(), scale_b.data_ptr(), C.data_ptr(), M, N, K, _pitch(A, up16), _pitch(B, up16),
           ldc, _pitch(scale_a, M), _pitch(scale_b, kb)), stream)
    return C


def _rows(t, heads, D):
    """Token pitch of [T, heads, D] whose heads lie side by side."""
    st, sh = t.stride(), t.shape
    if len(sh) != 3 or sh[1] != heads or sh[2] != D or st[2] != 1 or (heads > 1 and st[1] != D):
        raise ValueError("queries, keys and values must be [tokens, heads, D] with a token's heads side by side")
    return st[0] if sh[0] > 1 else heads * D


def _kv_append(name, Q, K, V, cos, sin, cu_tokens, context_lens, block_table, K_cache, V_cache, scales, interleaved, Q_out, stream):
    import torch
    bf16, f32, i32 = torch.bfloat16, torch.float32, torch.int32
    cache_type = _f8() if scales else bf16
    if K.dtype != bf16 or V.dtype != bf16 or (Q is not None and Q.dtype != bf16):
        raise TypeError("Q, K and V must be bfloat16")
    if K_cache.dtype != cache_type or V_cache.dtype != cache_type or not K_cache.is_contiguous() or not V_cache.is_contiguous():
        raise TypeError(f"the caches must be contiguous {cache_type} tensors")
    num_blocks, H_kv, block_size, D = K_cache.shape
    T = K.shape[0]
    if V_cache.shape != K_cache.shape or V.shape != K.shape or (Q is not None and Q.shape[0] != T):
        raise ValueError("shape mismatch")
    for t in (cu_tokens, context_lens, block_table):
        if t.dtype != i32 or not t.is_contiguous():
            raise TypeError("cu_tokens, context_lens and block_table must be contiguous int32 tensors")
    S, table = context_lens.numel(), block_table.shape  # (columns of one element serve as vectors)
    if cu_tokens.numel() != S + 1 or len(table) != 2 or table[0] != S:
        raise ValueError("cu_tokens must be [sequences + 1], context_lens [sequences], block_table [sequences, blocks]")
    held = [K, V, K_cache, V_cache, cu_tokens, context_lens, block_table]
    ks = vs = ()
    if scales:
        for t in scales:
            if t.dtype != f32 or not t.is_contiguous() or tuple(t.shape) != (num_blocks, H_kv):
                raise TypeError("k_scale and v_scale must be contiguous float32 [num_blocks, H_kv] tensors")
        held += scales
        ks, vs = (scales[0].data_ptr(),), (scales[1].data_ptr(),)
    ldk, ldv = _rows(K, H_kv, D), _rows(V, H_kv, D)
    H = ldq = ldqo = rotary = top = q = qo = c = s = 0
    if Q is not None:
        H = Q.shape[1]
        ldq = _rows(Q, H, D)
        if Q_out is None:
            Q_out = _new(Q, (T, H, D), bf16, stream)
            ldqo = H * D
        elif Q_out.dtype != bf16 or Q_out.shape != Q.shape:
            raise ValueError("Q_out must be bfloat16 of Q's shape")
        else:
            ldqo = _rows(Q_out, H, D)
        held += (Q, Q_out)
        q, qo = Q.data_ptr(), Q_out.data_ptr()
    if (cos is None) != (sin is None):
        raise ValueError("cos and sin come together")
    if cos is not None:
        if cos.dtype != f32 or sin.dtype != f32 or not cos.is_contiguous() or not sin.is_contiguous():
            raise TypeError("cos and sin must be contiguous float32 tensors")
        if cos.shape != sin.shape or cos.dim() != 2:
            raise ValueError("cos and sin must be [positions, rotary_dim / 2]")
        top, rotary = cos.shape
        rotary *= 2
        held += (cos, sin)
        c, s = cos.data_ptr(), sin.data_ptr()
    _call(name, load().mlt_kv_append_f8 if scales else load().mlt_kv_append, held,
          (q, K.data_ptr(), V.data_ptr(), c, s, cu_tokens.data_ptr(), context_lens.data_ptr(), block_table.data_ptr(), qo, K_cache.data_ptr(),
           V_cache.data_ptr(), *ks, *vs, T, S, H, H_kv, D, rotary, 1 if interleaved else 0, block_size, table[1], num_blocks, top, ldq, ldk, ldv,
           ldqo), stream)
    return Q_out if Q is not None else None


def kv_append(Q, K, V, cos, sin, cu_tokens, context_lens, block_table, K_cache, V_cache, *, interleaved: bool = False,
              Q_out=None, stream=None):
    """Rotates Q and K by their positions and appends K and V to a bfloat16 paged cache; returns the rotated Q.

    Q [T, H, D] (or None: only the cache is written), K and V [T, H_kv, D] bfloat16, a token's heads side by side (views
    of one fused projection work); cos, sin [positions, rotary_dim / 2] float32 (both None: no rotation); cu_tokens
    [S + 1], context_lens [S], block_table [S, max_blocks] int32; caches [num_blocks, H_kv, block_size, D].  Tokens from
    cu_tokens[S] on (a padded batch) are left out: their rows of Q_out are not written, so those of a new Q_out hold
    whatever its memory held.  Q_out may be Q.
    """
    return _kv_append("mlt_kv_append", Q, K, V, cos, sin, cu_tokens, context_lens, block_table, K_cache, V_cache, (),
                      interleaved, Q_out, stream)


def kv_append_f8(Q, K, V, cos, sin, cu_tokens, context_lens, block_table, K_cache, V_cache, k_scale, v_scale, *,
                 interleaved: bool = False, Q_out=None, stream=None):
    """kv_append into a float8_e4m3fn cache with one float32 scale per block and head: k_scale, v_scale [num_blocks, H_kv]."""
    return _kv_append("mlt_kv_append_f8", Q, K, V, cos, sin, cu_tokens, context_lens, block_table, K_cache, V_cache,
                      (k_scale, v_scale), interleaved, Q_out, stream)


def paged_attn_decode_f8(Q, K_cache, V_cache, k_scale, v_scale, block_table, seq_lens, *, scale: float, workspace=None, O=None,
                         LSE=None, return_lse: bool = True, stream=None):
    """paged_attn_decode over float8_e4m3fn caches with float32 scales k_scale, v_scale [num_blocks, H_kv].

    `workspace` is an optional contiguous uint8 CUDA tensor (see paged_attn_f8_workspace_bytes); without one a single CTA
    works on each (sequence, KV head), which is slow for few or long sequences.  Returns (O [S,H,D] bfloat16, LSE [S,H]
    float32 or None).
    """
    import torch
    if Q.dtype != torch.bfloat16 or not Q.is_contiguous() or Q.dim() != 3:
        raise TypeError("Q must be a contiguous [S, H, D] bfloat16 tensor")
    for t in (K_cache, V_cache):
        if t.dtype != _f8() or not t.is_contiguous() or t.dim() != 4:
            raise TypeError("the caches must be contiguous 4-D float8_e4m3fn tensors")
    for t in (block_table, seq_lens):
        if t.dtype != torch.int32 or not t.is_contiguous():
            raise TypeError("block_table and seq_lens must be contiguous int32 tensors")
    S, H, D = Q.shape
    NB, H_kv, bs, _ = K_cache.shape
    for t in (k_scale, v_scale):
        if t.dtype != torch.float32 or not t.is_contiguous() or tuple(t.shape) != (NB, H_kv):
            raise TypeError("k_scale and v_scale must be contiguous float32 [num_blocks, H_kv] tensors")
    if seq_lens.numel() != S or block_table.dim() != 2 or block_table.shape[0] != S:
        raise ValueError("seq_lens must be [sequences], block_table [sequences, blocks]")
    if V_cache.shape != K_cache.shape or K_cache.shape[3] != D:
        raise ValueError("shape mismatch")
    if O is None:
        O = _new(Q, Q.shape, torch.bfloat16, stream)
    elif O.dtype != torch.bfloat16 or O.shape != Q.shape or not O.is_contiguous():
        raise ValueError("O must be contiguous bfloat16 of Q's shape")
    if LSE is None and return_lse:
        LSE = _new(Q, (S, H), torch.float32, stream)
    elif LSE is not None and (LSE.dtype != torch.float32 or tuple(LSE.shape) != (S, H) or not LSE.is_contiguous()):
        raise ValueError("LSE must be contiguous float32 [S, H]")
    held = [Q, K_cache, V_cache, k_scale, v_scale, block_table, seq_lens, O]
    lse = ws = ws_bytes = 0
    if LSE is not None:
        held.append(LSE)
        lse = LSE.data_ptr()
    if workspace is not None:
        if not workspace.is_contiguous():
            raise TypeError("workspace must be contiguous")
        held.append(workspace)
        ws, ws_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    _call("mlt_paged_attn_decode_f8", load().mlt_paged_attn_decode_f8, held,
          (Q.data_ptr(), K_cache.data_ptr(), V_cache.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), block_table.data_ptr(),
           seq_lens.data_ptr(), O.data_ptr(), lse, S, H, H_kv, D, bs, block_table.shape[1], NB, float(scale), ws, ws_bytes), stream)
    return O, LSE


def _out_rows(Q, O, LSE, return_lse, stream):
    """O [T, H, D] with its token pitch, and LSE [T, H] or None: the caller's, checked, or new ones."""
    import torch
    T, H, D = Q.shape
    ldo = H * D
    if O is None:
        O = _new(Q, (T, H, D), torch.bfloat16, stream)
    elif O.dtype != torch.bfloat16 or O.shape != Q.shape:
        raise ValueError("O must be bfloat16 of Q's shape")
    else:
        ldo = _rows(O, H, D)
    if LSE is None and return_lse:
        LSE = _new(Q, (T, H), torch.float32, stream)
    elif LSE is not None and (LSE.dtype != torch.float32 or tuple(LSE.shape) != (T, H) or not LSE.is_contiguous()):
        raise ValueError("LSE must be contiguous float32 [T, H]")
    return O, ldo, LSE


def _scratch(Q, workspace, need, stream):
    """The caller's workspace, or a new one of the size that is always enough."""
    import torch
    if workspace is None:
        return _new(Q, (need(),), torch.uint8, stream)
    if not workspace.is_contiguous():
        raise TypeError("workspace must be contiguous")
    return workspace


def _vectors(*tensors):
    import torch
    for t in tensors:
        if t.dtype != torch.int32 or not t.is_contiguous():
            raise TypeError("token offsets, lengths and block tables must be contiguous int32 tensors")


def mha_packed_fwd(Q, K, V, cu_q, cu_k=None, *, causal: bool, scale: float, O=None, LSE=None, return_lse: bool = True, workspace=None,
                   stream=None):
    """Attention forward over sequences packed one behind another, with grouped heads.

    Q [T, H, D], K and V [T_k, H_kv, D] bfloat16, a token's heads side by side (views of one fused projection work); cu_q, cu_k
    [S + 1] int32: sequence s has the queries cu_q[s] .. cu_q[s + 1] - 1 and the keys cu_k[s] .. cu_k[s + 1] - 1 (cu_k None: cu_q).
    Causal masks are aligned bottom-right, as in mha_fwd; a query without a visible key gives O = 0 and LSE = -inf.  Rows of no
    sequence are not written.  `workspace`: a contiguous uint8 CUDA tensor of mha_packed_workspace_bytes (a new one without).
    Returns (O [T, H, D] bfloat16, LSE [T, H] float32 or None).
    """
    import torch
    for t in (Q, K, V):
        if t.dtype != torch.bfloat16 or t.dim() != 3:
            raise TypeError("Q, K and V must be [tokens, heads, D] bfloat16 tensors")
    if cu_k is None:
        cu_k = cu_q
    _vectors(cu_q, cu_k)
    T, H, D = Q.shape
    Tk, H_kv, _ = K.shape
    if V.shape != K.shape or K.shape[2] != D:
        raise ValueError("shape mismatch")
    S = cu_q.numel() - 1
    if S < 0 or cu_k.numel() != S + 1:
        raise ValueError("cu_q and cu_k must be [sequences + 1]")
    O, ldo, LSE = _out_rows(Q, O, LSE, return_lse, stream)
    workspace = _scratch(Q, workspace, lambda: mha_packed_workspace_bytes(T, S, H, H_kv, D), stream)
    held = [Q, K, V, cu_q, cu_k, O, workspace]
    lse = 0
    if LSE is not None:
        held.append(LSE)
        lse = LSE.data_ptr()
    _call("mlt_mha_packed_fwd", load().mlt_mha_packed_fwd, held,
          (Q.data_ptr(), K.data_ptr(), V.data_ptr(), cu_q.data_ptr(), cu_k.data_ptr(), O.data_ptr(), lse, T, Tk, S, H, H_kv, D,
           1 if causal else 0, float(scale), _rows(Q, H, D), _rows(K, H_kv, D), _rows(V, H_kv, D), ldo, workspace.data_ptr(),
           workspace.numel() * workspace.element_size()), stream)
    return O, LSE


def paged_attn_prefill(Q, K_cache, V_cache, cu_tokens, context_lens, block_table, *, scale: float, O=None, LSE=None,
                       return_lse: bool = True, workspace=None, stream=None):
    """Causal attention of new tokens over the paged cache, which holds their own keys and values already (see kv_append, whose
    cu_tokens, context_lens and block_table these are).

    Q [T, H, D] bfloat16 (rotated, a token's heads side by side); caches [num_blocks, H_kv, block_size, D] bfloat16.  Token t of
    sequence s sees the cache positions 0 .. context_lens[s] + t - cu_tokens[s].  Rows of no sequence are not written.  `workspace`
    as for mha_packed_fwd.  Returns (O [T, H, D] bfloat16, LSE [T, H] float32 or None).
    """
    import torch
    if Q.dtype != torch.bfloat16 or Q.dim() != 3:
        raise TypeError("Q must be a [tokens, heads, D] bfloat16 tensor")
    for t in (K_cache, V_cache):
        if t.dtype != torch.bfloat16 or not t.is_contiguous() or t.dim() != 4:
            raise TypeError("the caches must be contiguous 4-D bfloat16 tensors")
    _vectors(cu_tokens, context_lens, block_table)
    T, H, D = Q.shape
    num_blocks, H_kv, block_size, _ = K_cache.shape
    if V_cache.shape != K_cache.shape or K_cache.shape[3] != D:
        raise ValueError("shape mismatch")
    S = context_lens.numel()
    if cu_tokens.numel() != S + 1 or block_table.dim() != 2 or block_table.shape[0] != S:
        raise ValueError("cu_tokens must be [sequences + 1], context_lens [sequences], block_table [sequences, blocks]")
    O, ldo, LSE = _out_rows(Q, O, LSE, return_lse, stream)
    workspace = _scratch(Q, workspace, lambda: mha_packed_workspace_bytes(T, S, H, H_kv, D), stream)
    held = [Q, K_cache, V_cache, cu_tokens, context_lens, block_table, O, workspace]
    lse = 0
    if LSE is not None:
        held.append(LSE)
        lse = LSE.data_ptr()
    _call("mlt_paged_attn_prefill", load().mlt_paged_attn_prefill, held,
          (Q.data_ptr(), K_cache.data_ptr(), V_cache.data_ptr(), cu_tokens.data_ptr(), context_lens.data_ptr(), block_table.data_ptr(),
           O.data_ptr(), lse, T, S, H, H_kv, D, block_size, block_table.shape[1], num_blocks, float(scale), _rows(Q, H, D), ldo,
           workspace.data_ptr(), workspace.numel() * workspace.element_size()), stream)
    return O, LSE


def paged_attn_decode_shared(Q, K_cache, V_cache, block_table, seq_lens, prefix_lens, cu_groups, *, scale: float, workspace=None, O=None,
                             LSE=None, return_lse: bool = True, stream=None):
    """paged_attn_decode for a batch whose sequences share prefixes, which are read once for all sequences behind them.

    Arguments as there, and prefix_lens [groups], cu_groups [groups + 1] int32: the sequences cu_groups[g] .. cu_groups[g + 1] - 1 have
    the first prefix_lens[g] // block_size entries of their block tables in common.  `workspace`: a contiguous
    uint8 CUDA tensor of paged_attn_shared_workspace_bytes (a new one without).
    Returns (O [S, H, D] bfloat16, LSE [S, H] float32 or None), those of paged_attn_decode.
    """
    import torch
    if Q.dtype != torch.bfloat16 or not Q.is_contiguous() or Q.dim() != 3:
        raise TypeError("Q must be a contiguous [S, H, D] bfloat16 tensor")
    for t in (K_cache, V_cache):
        if t.dtype != torch.bfloat16 or not t.is_contiguous() or t.dim() != 4:
            raise TypeError("the caches must be contiguous 4-D bfloat16 tensors")
    S, H, D = Q.shape
    _vectors(block_table, seq_lens, prefix_lens, cu_groups)
    num_blocks, H_kv, block_size, _ = K_cache.shape
    if V_cache.shape != K_cache.shape or K_cache.shape[3] != D:
        raise ValueError("shape mismatch")
    groups = prefix_lens.numel()
    if cu_groups.numel() != groups + 1 or seq_lens.numel() != S or block_table.dim() != 2 or block_table.shape[0] != S:
        raise ValueError("cu_groups must be [groups + 1], prefix_lens [groups], seq_lens [sequences], block_table [sequences, blocks]")
    O, _, LSE = _out_rows(Q, O, LSE, return_lse, stream)
    if not O.is_contiguous():
        raise ValueError("O must be contiguous")
    workspace = _scratch(Q, workspace, lambda: paged_attn_shared_workspace_bytes(S, groups, H, H_kv, D), stream)
    held = [Q, K_cache, V_cache, block_table, seq_lens, prefix_lens, cu_groups, O, workspace]
    lse = 0
    if LSE is not None:
        held.append(LSE)
        lse = LSE.data_ptr()
    _call("mlt_paged_attn_decode_shared", load().mlt_paged_attn_decode_shared, held,
          (Q.data_ptr(), K_cache.data_ptr(), V_cache.data_ptr(), block_table.data_ptr(), seq_lens.data_ptr(), prefix_lens.data_ptr(),
           cu_groups.data_ptr(), O.data_ptr(), lse, S, groups, H, H_kv, D, block_size, block_table.shape[1], num_blocks, float(scale),
           workspace.data_ptr(), workspace.numel() * workspace.element_size()), stream)
    return O, LSE


def gemm_w4(X, W, scales, zeros=None, C=None, *, stream=None):
    """C = X @ dequantised(W).T in bfloat16 for few rows X [M, K] bfloat16 and 4-bit weights (up to 8 rows faster than gemm_f8 and gemm,
    from 17 on slower than both).

    W [N, K / 2] uint8, two weights to a byte, the even k in the lower half; scales [N, K / group] bfloat16; zeros [N, K / group]
    uint8 (None: 8): weight (n, k) is scales[n, k / group] * (W(n, k) - zeros[n, k / group]).  group, 32, 64 or 128, follows from
    the shapes.  Row pitches come from the tensors' strides (X: a multiple of 8 elements, W: of 16 bytes).
    """
    import torch
    if X.dtype != torch.bfloat16 or scales.dtype != torch.bfloat16 or W.dtype != torch.uint8 or (zeros is not None and zeros.dtype != torch.uint8):
        raise TypeError("X and scales must be bfloat16, W and zeros uint8")
    (M, K), (N, half), (Ns, groups) = X.shape, W.shape, scales.shape
    if 2 * half != K or Ns != N or (K and (groups == 0 or K % groups)) or (zeros is not None and zeros.shape != scales.shape):
        raise ValueError("shape mismatch")
    group = K // groups if groups else 128
    if C is None:
        C = _new(X, (M, N), torch.bfloat16, stream)
    elif C.dtype != torch.bfloat16 or tuple(C.shape) != (M, N):
        raise ValueError("C must be bfloat16 [M, N]")
    held = [X, W, scales, C]
    z = ldz = 0
    if zeros is not None:
        held.append(zeros)
        z, ldz = zeros.data_ptr(), _pitch(zeros, groups)
    _call("mlt_gemm_w4", load().mlt_gemm_w4, held,
          (X.data_ptr(), W.data_ptr(), scales.data_ptr(), z, C.data_ptr(), M, N, K, group, _pitch(X, (K + 7) // 8 * 8), _pitch(W, (half + 15) // 16 * 16),
           _pitch(scales, groups), ldz, _pitch(C, N)), stream)
    return C
