"""B200 (sm_100a) dense hot path: BF16 GEMM, FlashAttention-2 style MHA forward, paged decode, and the 8-bit serving path
(E4M3 quantiser, scaled GEMM, cache append with rotation, decode over an E4M3 cache).

`binding` wraps the C ABI of include/mlt.h (libmlt.so, built by `build`);
`inputs` holds the seeded synthetic workloads.  Nothing here computes on the CPU.
"""
from . import inputs  # noqa: F401
from .binding import (MltError, debug_wait_timeout_selftest, gemm, gemm_ex_raw, gemm_f16_raw, gemm_plan, gemm_raw, gemm_workspace_bytes, last_clock_mhz, last_device_error, load, mha_fwd, mha_fwd_raw,  # noqa: F401
                      paged_attn_decode, paged_attn_decode_raw, paged_attn_decode_static_raw,
                      paged_attn_workspace_bytes, status_string, version,
                      gemm_f8, gemm_f8_plan, gemm_f8_raw, kv_append, kv_append_f8, kv_append_f8_raw, kv_append_raw, paged_attn_decode_f8,
                      paged_attn_decode_f8_raw, paged_attn_f8_workspace_bytes, quantize_f8, quantize_f8_raw)
