/*
 * mlt.h -- C ABI of the B200 (sm_100a) dense hot path: BF16 GEMM with FP32
 * accumulation and a FlashAttention-2 style multi-head-attention forward.
 *
 * Every pointer named "device" must be device memory of the CUDA device that
 * is current on the calling thread.  `stream` is a cudaStream_t passed as
 * void* (NULL = the legacy default stream).  All calls are asynchronous on
 * `stream`, allocate no device memory, keep no pointer after returning, and
 * return an mlt_status (never throw, never exit).  Argument validation runs
 * before any CUDA call.  Outputs must not alias inputs.
 *
 * BF16 values are passed as their 16-bit patterns.
 */
#ifndef MLT_H_
#define MLT_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    MLT_OK = 0,
    MLT_ERR_INVALID_ARG = 1, /* NULL pointer, negative size, pitch < row width, causal with Nq > Nk, Nk == 0, scale <= 0 */
    MLT_ERR_UNSUPPORTED = 2, /* head dimension other than 64 or 128; size beyond a TMA descriptor's range */
    MLT_ERR_ALIGNMENT = 3,   /* base pointer not 16-byte aligned, or pitch not a multiple of 8 elements */
    MLT_ERR_CUDA = 4,        /* a CUDA runtime / driver call failed */
    MLT_ERR_ARCH = 5,        /* current device is not compute capability 10.x */
    MLT_ERR_TIMEOUT = 6,     /* a bounded device-side wait expired (reported by mlt_last_device_error) */
    MLT_ERR_BAD_BLOCK = 7,   /* a block-table entry outside [0, num_blocks) was met (reported by mlt_last_device_error) */
    MLT_ERR_SCRATCH_LIMIT = 8, /* mlt_paged_attn_decode_static: the call needs more than MLT_PAGED_STATIC_SCRATCH_BYTES */
    MLT_ERR_BAD_POSITION = 9 /* mlt_kv_append*: a sequence's token offsets or positions lie outside the call's tokens or the
                                cos / sin tables (reported by mlt_last_device_error) */
} mlt_status;

/*
 * C = A * B  (paper Sec. 2: A in R^{m x k}, B in R^{k x n}, C in R^{m x n};
 * Listing 2: zero-initialised accumulator, K loop of tile dots, one store).
 * Reading taken: C is overwritten, its prior contents are ignored.
 *
 *   A  device, BF16, M x K row-major, A[i*lda + k]
 *   B  device, BF16, K x N row-major, B[k*ldb + j]
 *   C  device, BF16 out, M x N row-major, C[i*ldc + j]; products accumulate in
 *      FP32 and are rounded once, to nearest even
 *   lda, ldb, ldc  row pitches in ELEMENTS, each >= the row width and a multiple
 *      of 8 (16-byte rows for the TMA descriptors); base pointers 16-byte aligned
 *
 * M == 0 or N == 0: MLT_OK, nothing launched.  K == 0: C is zero-filled.
 * Any M, N, K otherwise (ragged tiles are zero-filled on load, clipped on store).
 */
int mlt_gemm(const void* A, const void* B, void* C,
             int64_t M, int64_t N, int64_t K,
             int64_t lda, int64_t ldb, int64_t ldc,
             void* stream);

/*
 * The GEMM in the data types of the paper's Listing 2 (FP16 operands, FP32 accumulator and FP32 result), with
 * the accumulate form of the problem statement of Sec. 2 (C += A * B) as an option.
 *
 *   A, B   device, FP16 (bit patterns), layouts and pitches as for mlt_gemm
 *   C      device, FP32, M x N row-major, pitch ldc in ELEMENTS, a multiple of 4; 16-byte aligned
 *   accumulate  0: C = A * B (prior contents ignored);  non-zero: C = C + A * B, the product summed in FP32 first
 *               and added to the prior C once
 * K == 0: C is zero-filled, or left as it is when accumulating.  Errors as for mlt_gemm.
 */
int mlt_gemm_f16(const void* A, const void* B, float* C,
                 int64_t M, int64_t N, int64_t K,
                 int64_t lda, int64_t ldb, int64_t ldc,
                 int accumulate, void* stream);

/*
 * mlt_gemm with caller-provided scratch, for the memory-bound shapes of paper Sec. 4.1 (next-token prediction:
 * few rows of A against large weight matrices, "large k" and "large n" cases).  Such a problem has too few output
 * tiles to occupy the GPU, so K is cut into slices (split-K) and every SM streams a part of B.  With at most one
 * 128 x 128 tile per two SMs the slices of a tile run as a thread-block cluster that sums its FP32 partial tiles
 * through distributed shared memory; this needs no scratch and mlt_gemm does the same.  With more tiles than that
 * the FP32 partial tiles go to the workspace and a second small kernel sums them.  Either way the sum runs in a
 * fixed order and is rounded once to BF16.  Same operation, arguments, layouts and errors as mlt_gemm; the result
 * can differ from an uncut sum in the last BF16 bit (the FP32 partial sums are added in a different order).
 *
 *   workspace        device scratch, 16-byte aligned, or NULL (then this is mlt_gemm)
 *   workspace_bytes  its size; mlt_gemm_workspace_bytes(M, N, K) is always enough (0 when K would not be cut; an
 *                    upper bound that does not depend on the device); with less, fewer slices are used.  Calls
 *                    that overlap on the GPU must not share it.
 */
size_t mlt_gemm_workspace_bytes(int64_t M, int64_t N, int64_t K);
int mlt_gemm_ex(const void* A, const void* B, void* C,
                int64_t M, int64_t N, int64_t K,
                int64_t lda, int64_t ldb, int64_t ldc,
                void* workspace, size_t workspace_bytes, void* stream);

/*
 * O = softmax(scale * Q K^T [+ causal mask]) V,  LSE = log-sum-exp of the
 * scaled, masked scores (natural log)  -- paper Sec. 2.5, Algorithm 1
 * (FlashAttention-2 forward: per Q block, loop over K/V blocks, S = Q K_j^T,
 * online softmax with running row max m and row sum l, O += P V_j, store O).
 * The scale, the mask, the final 1/l and the LSE output are the benchmark
 * configuration's; the algorithm box leaves them implicit.
 *
 *   Q      device, BF16, [B, H, Nq, D] contiguous (D fastest)
 *   K, V   device, BF16, [B, H, Nk, D] contiguous
 *   O      device, BF16 out, [B, H, Nq, D]
 *   LSE    device, FP32 out, [B, H, Nq], or NULL to skip it
 *   D      64 or 128
 *   causal non-zero: key j is visible to query i iff j <= i + (Nk - Nq)
 *          (bottom-right aligned; requires Nq <= Nk)
 *   scale  multiplies the raw dot products (typically 1/sqrt(D)); must be finite and > 0
 *
 * B*H*Nq == 0: MLT_OK, nothing launched.  Nk == 0: MLT_ERR_INVALID_ARG.
 * P is rounded to BF16 for the second product; S, m, l and O accumulate in FP32.
 */
int mlt_mha_fwd(const void* Q, const void* K, const void* V,
                void* O, float* LSE,
                int B, int H, int Nq, int Nk, int D,
                int causal, float scale, void* stream);

/*
 * Paged-attention decode: O[s,h,:] = softmax(scale * q[s,h] . K_s^T) V_s over the len[s] tokens of sequence s,
 * whose keys and values live in cache blocks reached through a block table -- paper Sec. 3.2 (Listings 6 and 7:
 * one query token per sequence, KV blocks split across warps, cross-warp max / sum / output reduction) and
 * Sec. 4.3.  The listings are schematic (they normalise per block); the operation is plain softmax attention.
 *
 *   Q            device, BF16, [num_seqs, H, D]
 *   K_cache, V_cache  device, BF16, [num_blocks, H_kv, block_size, D] (D fastest)
 *   block_table  device, int32, [num_seqs, max_blocks_per_seq]: physical block of each logical block; entries of
 *                logical blocks a sequence uses must lie in [0, num_blocks) (others are never read; a bad entry is
 *                skipped and reported through mlt_last_device_error, it is never dereferenced)
 *   seq_lens     device, int32, [num_seqs], 0 <= len <= max_blocks_per_seq * block_size; token i sits in logical
 *                block i / block_size at offset i % block_size (a length outside that range is cut to it: no
 *                table entry beyond a sequence's row is read)
 *   O            device, BF16 out, [num_seqs, H, D];  LSE device FP32 out [num_seqs, H] (natural log) or NULL
 *   H_kv         KV heads; H / H_kv in {1, 2, 4, 8}; query head h reads KV head h / (H / H_kv)
 *   D in {64, 128}; block_size in {8, 16, 32}; scale finite and > 0
 *   workspace    device scratch of workspace_bytes bytes (16-byte aligned) for the partial results when a
 *                sequence is split over several CTAs; mlt_paged_attn_workspace_bytes gives a size that is always
 *                enough.  With less (or NULL) fewer splits are used, down to one CTA per (sequence, KV head).
 *                Its contents are scratch; calls that overlap on the GPU must not share it.
 * A sequence of length 0 gives O = 0 and LSE = -inf.  num_seqs == 0: MLT_OK, nothing launched.
 */
size_t mlt_paged_attn_workspace_bytes(int num_seqs, int H, int D);
int mlt_paged_attn_decode(const void* Q, const void* K_cache, const void* V_cache,
                          const int32_t* block_table, const int32_t* seq_lens,
                          void* O, float* LSE,
                          int num_seqs, int H, int H_kv, int D,
                          int block_size, int max_blocks_per_seq, int num_blocks, float scale,
                          void* workspace, size_t workspace_bytes, void* stream);

/*
 * mlt_paged_attn_decode for callers that cannot supply scratch memory.  (The paper has no counterpart: this is a
 * library addition.)  Who needs it: an engine whose own pool already owns all device memory, a plug-in that
 * receives tensors but no allocator, a decode loop in which cudaMalloc -- it synchronises the device -- is ruled
 * out once the loop is running.  The partial results of split sequences go into an array of
 * MLT_PAGED_STATIC_SCRATCH_BYTES bytes that is part of the library's device image (every GPU that loads the
 * library carries it until the process exits).  The call allocates nothing, on host or device.
 *
 * Arguments, layouts, results and errors are those of mlt_paged_attn_decode, without the workspace pair.  The
 * split over CTAs is the one mlt_paged_attn_decode makes with a full workspace, so the outputs are the same;
 * it needs num_seqs * H * splits * (4 * D + 8) bytes with splits <= 32 (splits = ceil(max_blocks_per_seq / 16), / 32
 * with 4 or 8 query heads per KV head, half as many blocks per split for few sequences), and a call that needs more
 * than the array holds returns MLT_ERR_SCRATCH_LIMIT
 * and launches nothing.
 *
 * The first call on each device looks up the array's device address (with that device current); make that first
 * call before any stream capture begins.  All calls on a device share the one array and it keeps the last call's
 * contents: nothing in it has to be cleared between calls, but two calls that overlap on the GPU (different
 * streams, or one thread per stream) race on it -- serialise them, or use mlt_paged_attn_decode with separate
 * workspaces.
 */
#define MLT_PAGED_STATIC_SCRATCH_BYTES (16 * 1024 * 1024)
int mlt_paged_attn_decode_static(const void* Q, const void* K_cache, const void* V_cache,
                                 const int32_t* block_table, const int32_t* seq_lens,
                                 void* O, float* LSE,
                                 int num_seqs, int H, int H_kv, int D,
                                 int block_size, int max_blocks_per_seq, int num_blocks, float scale,
                                 void* stream);

/*
 * ---- The 8-bit serving path (library additions; the paper's workloads have no 8-bit form) ----
 *
 * These calls are launched so that a kernel's blocks may be placed while the kernel before it in the stream drains; they
 * wait for its completion before they touch memory, so nothing changes for the caller.
 *
 * E4M3 values are passed as bytes.  A decoding step runs them in this order: mlt_quantize_f8 (activations) ->
 * mlt_gemm_f8 (projections) -> mlt_kv_append_f8 -> mlt_paged_attn_decode_f8 -> mlt_quantize_f8 -> mlt_gemm_f8.
 *
 * Scales that the library makes are powers of two: s = 2^e with the smallest e >= -64 for which amax <= 448 * s (amax
 * over finite values; 2^-64 for a block of zeros).  E4M3's relative step does not depend on s, x / s is exact, and a
 * stored value has one rounding (to nearest even).  Infinities are stored as +-448 * s, NaN as NaN.  Scales that it
 * reads may be any FP32 values.
 */

/*
 * Q = round(X / s) in E4M3 with one scale s per block of `block_rows` x 128 elements.
 *
 *   X       device, BF16, M x K row-major, pitch ldx in elements, a multiple of 8; 16-byte aligned
 *   Q       device, E4M3 out, M x K row-major, pitch ldq in bytes, a multiple of 16; 16-byte aligned
 *   scales  device, FP32 out.  block_rows 1 (activations): scales[kb * lds + i] for row i and K block kb, lds >= M.
 *           block_rows 128 (weights): scales[rb * lds + kb] for row block rb, lds >= ceil(K / 128).
 * The last blocks may be ragged; nothing outside M x K (and its blocks' scales) is written.  M == 0 or K == 0: MLT_OK,
 * nothing launched.  MLT_ERR_UNSUPPORTED for another block_rows.
 */
int mlt_quantize_f8(const void* X, void* Q, float* scales, int64_t M, int64_t K, int64_t ldx, int64_t ldq, int64_t lds,
                    int block_rows, void* stream);

/*
 * C[i][j] = sum over K blocks kb of 128: sa[kb][i] * sb[j / 128][kb] * sum over k in kb of A[i][k] * B[j][k]
 * (B is stored with K contiguous, as the weights of a linear layer are).
 *
 *   A, B     device, E4M3, M x K and N x K, pitches lda, ldb in bytes, multiples of 16; 16-byte aligned
 *   scale_a  device, FP32, scale_a[kb * ldsa + i], ldsa >= M                    (mlt_quantize_f8 with block_rows 1)
 *   scale_b  device, FP32, scale_b[(j / 128) * ldsb + kb], ldsb >= ceil(K / 128)  (block_rows 128)
 *   C        device, BF16 out, M x N, pitch ldc in elements, a multiple of 8; 16-byte aligned
 * Products of a K block are summed in the tensor core's FP32, weighted, and summed over the blocks in FP32 in a fixed
 * order; one rounding to nearest even.  K need not be a multiple of 128.  M == 0 or N == 0: MLT_OK, nothing launched;
 * K == 0: C is zero-filled.  Needs no scratch.
 */
int mlt_gemm_f8(const void* A, const float* scale_a, const void* B, const float* scale_b, void* C,
                int64_t M, int64_t N, int64_t K, int64_t lda, int64_t ldb, int64_t ldc, int64_t ldsa, int64_t ldsb,
                void* stream);

/*
 * Appends the keys and values of new tokens to the paged cache that mlt_paged_attn_decode reads (mlt_kv_append, BF16) or
 * that mlt_paged_attn_decode_f8 reads (mlt_kv_append_f8, E4M3), and rotates queries and keys by their positions.
 *
 * Sequence s has the new tokens cu_tokens[s] .. cu_tokens[s + 1] - 1 (none is allowed), which follow the context_lens[s]
 * tokens that its cache holds: token t sits at position p = context_lens[s] + t - cu_tokens[s], in block
 * block_table[s][p / block_size] at offset p % block_size.
 *
 *   Q, K, V      device, BF16; token t, head h, element d at t * ld + h * D + d (pitches ldq, ldk, ldv in elements,
 *                multiples of 8; views of one fused projection work).  Q may be NULL: then only the cache is written.
 *   cos_table, sin_table  device, FP32, [max_position, rotary_dim / 2]: row p holds the angles of position p
 *   rotary_dim   elements of each head that are rotated, a multiple of 16, 0 (none: the tables may be NULL) .. D.
 *                Pair i is (i, i + rotary_dim / 2), or with `interleaved` (2 i, 2 i + 1); (a, b) becomes
 *                (a cos_i - b sin_i, b cos_i + a sin_i).  The other elements pass through.
 *   cu_tokens    device, int32, [num_seqs + 1], ascending from 0;  context_lens device, int32, [num_seqs]
 *   block_table  device, int32, [num_seqs, max_blocks_per_seq].  The entries that one call writes through must all differ,
 *                within a sequence and between sequences (a shared block is copied before a sequence appends to it);
 *                where two are equal all the same, what that block's tokens and scales hold afterwards is undefined.
 *   Q_out        device, BF16 out, pitch ldqo; may be Q itself with the same pitch
 *   K_cache, V_cache  device, [num_blocks, H_kv, block_size, D]
 *   k_scale, v_scale  device, FP32, [num_blocks, H_kv] (E4M3 cache).  A block's scale becomes the larger of the scale it
 *                had, if it holds tokens of the sequence already, and the power of two that its new tokens need; if it
 *                grows, the tokens already there are rescaled (exact for powers of two unless a value underflows).  Scales
 *                of blocks that hold tokens must be positive.
 * D in {64, 128}, block_size in {8, 16, 32}.  Tokens from cu_tokens[num_seqs] on (a padded batch), their rows of
 * Q_out and all cache positions without a new token are left as they were.  A block-table entry outside
 * [0, num_blocks) or beyond the table's row is not written and reported (MLT_ERR_BAD_BLOCK); a sequence whose
 * cu_tokens reach outside [0, num_tokens] or whose positions are negative or reach max_position is left out and
 * reported (MLT_ERR_BAD_POSITION), both through mlt_last_device_error.  num_tokens == 0 or num_seqs == 0: MLT_OK,
 * nothing launched.
 */
int mlt_kv_append(const void* Q, const void* K, const void* V, const float* cos_table, const float* sin_table,
                  const int32_t* cu_tokens, const int32_t* context_lens, const int32_t* block_table,
                  void* Q_out, void* K_cache, void* V_cache,
                  int num_tokens, int num_seqs, int H, int H_kv, int D, int rotary_dim, int interleaved,
                  int block_size, int max_blocks_per_seq, int num_blocks, int max_position,
                  int64_t ldq, int64_t ldk, int64_t ldv, int64_t ldqo, void* stream);
int mlt_kv_append_f8(const void* Q, const void* K, const void* V, const float* cos_table, const float* sin_table,
                     const int32_t* cu_tokens, const int32_t* context_lens, const int32_t* block_table,
                     void* Q_out, void* K_cache, void* V_cache, float* k_scale, float* v_scale,
                     int num_tokens, int num_seqs, int H, int H_kv, int D, int rotary_dim, int interleaved,
                     int block_size, int max_blocks_per_seq, int num_blocks, int max_position,
                     int64_t ldq, int64_t ldk, int64_t ldv, int64_t ldqo, void* stream);

/*
 * mlt_paged_attn_decode over an E4M3 cache: key element = k_scale[block][head] * K_cache value, and likewise for V.
 * Arguments as there, but
 *   K_cache, V_cache  device, E4M3, [num_blocks, H_kv, block_size, D];  k_scale, v_scale  device, FP32, [num_blocks, H_kv]
 *   workspace    device scratch, 16-byte aligned; mlt_paged_attn_f8_workspace_bytes is always enough.  With less the
 *                work is cut into fewer shares, with NULL (or less than num_seqs * H_kv + 2 partials of
 *                (H / H_kv) * (4 D + 8) + 8 bytes) one CTA works on each (sequence, KV head).  Calls that overlap on the
 *                GPU must not share it.
 * num_blocks * H_kv must be below 2^31.  The scales may be any FP32 values for which scores and outputs stay in FP32.
 * The tokens of a bad block-table entry are left out and reported.  The maximum, the sum and the output accumulate in
 * FP32.  Two operands are rounded to FP16: a token's weight p * |v_scale| for the second product, under a power of
 * two for the row's largest one, so that weights below 2^-28 of that lose bits and below 2^-39 are zero; and the
 * queries, under a power of two for each row's largest element, so that elements below 2^-28 of that lose bits.
 */
size_t mlt_paged_attn_f8_workspace_bytes(int num_seqs, int H, int H_kv, int D);
int mlt_paged_attn_decode_f8(const void* Q, const void* K_cache, const void* V_cache, const float* k_scale, const float* v_scale,
                             const int32_t* block_table, const int32_t* seq_lens,
                             void* O, float* LSE,
                             int num_seqs, int H, int H_kv, int D,
                             int block_size, int max_blocks_per_seq, int num_blocks, float scale,
                             void* workspace, size_t workspace_bytes, void* stream);

/*
 * The SM clock the last GEMM (which = 0) or attention (which = 1) launch on the current device really ran at, in
 * MHz: CTA 0 of those kernels notes the SM cycle counter and the nanosecond timer at its start and at its end.  (No
 * counterpart in the paper; a measurement aid: under tensor-core load this part runs well below the clock NVML
 * reports, and throughput is only comparable across runs together with it.)  Synchronises the device.  *mhz is 0
 * if no such kernel has run yet.  Concurrent launches of the same kind overwrite each other's notes.
 */
int mlt_debug_last_clock_mhz(int which, double* mhz);

/*
 * The launch plan of mlt_gemm / mlt_gemm_ex for an M x N x K problem with BF16 output (no counterpart in the paper;
 * lets tests pin which kernel a shape reaches).  sm_count >= 2: a device of that many SMs on which clusters can use
 * every SM (host arithmetic only, no CUDA call).  sm_count == 0: the current device, with the number of resident
 * clusters it reports (a cluster must fit one GPC); configures the device on first use like any other call.
 *   out4[0]  tile shape: 0 = CTA pairs on 256 x 256 tiles, 1 = 128 x 256 tiles, 2 = 128 x 128 tiles, 3 = 128 x 128
 *            tiles with the even K hand-out through the workspace (every CTA the same number of (tile, K block)
 *            units; then out4[1] = the most partial tiles one output tile can get, out4[3] = units per CTA)
 *   out4[1]  K slices through the workspace (1 = none);  workspace_bytes = 0 stands for no workspace
 *   out4[2]  CTAs per cluster that cut K for one tile (1 = none)
 *   out4[3]  K blocks of 64 per slice
 * MLT_ERR_INVALID_ARG for a null pointer, a non-positive size, sm_count 1 or negative.
 */
int mlt_debug_gemm_plan(int64_t M, int64_t N, int64_t K, size_t workspace_bytes, int sm_count, int* out4);

/*
 * The launch plan of mlt_gemm_f8 (likewise; sm_count as above).
 *   out4[0]  0 = one 128 x out4[1] tile per cluster, 1 = 128 x 256 tiles, 2 = CTA pairs on 256 x 256 tiles
 *   out4[1]  tile width    out4[2]  CTAs per cluster that cut K    out4[3]  shared memory of the first kind in bytes
 */
int mlt_debug_gemm_f8_plan(int64_t M, int64_t N, int64_t K, int sm_count, int* out4);

/*
 * Device-side health word.  Kernels never trap: a wait that exceeds its bound
 * records {code, barrier id, block} in a per-device status word and the kernel
 * drains and returns.  This call synchronises the current device, reads and
 * clears that word, and returns MLT_OK, MLT_ERR_TIMEOUT, MLT_ERR_BAD_BLOCK, MLT_ERR_BAD_POSITION or MLT_ERR_CUDA.
 * detail (host, may be NULL) receives 4 words: code, barrier id, block, aux.
 * (Library addition; the paper has no counterpart.)
 */
int mlt_last_device_error(uint32_t* detail);

/*
 * Self-test of the bounded device-side waits (library addition; the paper has no counterpart).  Launches one warp
 * that waits, with a budget of `budget_cycles` SM clocks (1 .. 1e9, i.e. at most about half a second), on a barrier
 * that nothing completes.  The wait gives up, the kernel returns normally, and the next mlt_last_device_error
 * reports MLT_ERR_TIMEOUT with detail = {code, barrier id 0x7E57, block 0, parity 0}.  Nothing traps; the context
 * stays usable.  Returns MLT_OK when the launch was made, MLT_ERR_INVALID_ARG for a budget outside the range.
 */
int mlt_debug_wait_timeout_selftest(uint64_t budget_cycles, void* stream);

/* Text for an mlt_status value (static storage). */
const char* mlt_status_string(int status);

/* Library version: major*10000 + minor*100 + patch. */
int mlt_version(void);

#ifdef __cplusplus
}
#endif
#endif /* MLT_H_ */
