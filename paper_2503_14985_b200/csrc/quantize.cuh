// BF16 -> E4M3 with one power-of-two scale per 1 x 128 block (activations) or per 128 x 128 block (weights): the
// operand formats of the scaled GEMM.  q = round(x / s), s from the block's largest finite magnitude (f8.cuh).
//
// Bound by HBM: 2 bytes read and 1 written per element, one pass; a block stays in registers between its maximum and
// its rounding.  Sixteen lanes own a row's 128 columns (16 bytes each), so the maximum is four shuffles away.
//
// Infinities and NaN do not set a scale.  The common path takes the maximum of the magnitude bits as packed 16-bit
// integers (BF16 magnitudes order like integers) and only redoes it with a per-element test when the result says that
// a non-finite value is there.
#pragma once

#include "f8.cuh"

namespace mlt {

struct QuantizeParams {
    const __nv_bfloat16* X;  // [M, K], pitch ldx
    uint8_t* Q;              // [M, K] E4M3, pitch ldq
    float* S;                // rows of 1: [K blocks][lds], element (kb, row); rows of 128: [row blocks][lds], element (rb, kb)
    int64_t ldx, ldq, lds;
    int M, K;
};

__device__ __forceinline__ uint4 quantize_load8(const __nv_bfloat16* p, int left) {  // 8 elements, zeros beyond `left`
    if (left >= 8) return *reinterpret_cast<const uint4*>(p);
    uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < left) w[i >> 1] |= static_cast<uint32_t>(__bfloat16_as_ushort(p[i])) << ((i & 1) * 16);
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint32_t quantize_absmax(const uint4& v) {  // largest magnitude pattern of the 8 elements (15 bits)
    const uint32_t m = 0x7FFF7FFFu;
    const uint32_t a = __vmaxu2(__vmaxu2(v.x & m, v.y & m), __vmaxu2(v.z & m, v.w & m));
    return max(a & 0xFFFFu, a >> 16);
}
__device__ __forceinline__ uint32_t quantize_absmax_finite(const uint4& v) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t a = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t b = (w[i >> 1] >> ((i & 1) * 16)) & 0x7FFFu;
        if (b < 0x7F80u) a = max(a, b);
    }
    return a;
}
__device__ __forceinline__ uint2 quantize_pack8(const uint4& v, float inv) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        o[i] = f8x2_from_f32(__uint_as_float(w[i] << 16) * inv, __uint_as_float(w[i] & 0xFFFF0000u) * inv);
    return make_uint2(o[0] | (o[1] << 16), o[2] | (o[3] << 16));
}
__device__ __forceinline__ void quantize_store8(uint8_t* p, const uint2& v, int left) {
    if (left >= 8) {
        *reinterpret_cast<uint2*>(p) = v;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) p[i] = static_cast<uint8_t>((i < 4 ? v.x : v.y) >> ((i & 3) * 8));
    }
}
__device__ __forceinline__ uint32_t max16lanes(uint32_t a) {
#pragma unroll
    for (int w = 1; w < 16; w <<= 1) a = max(a, __shfl_xor_sync(0xffffffffu, a, w));
    return a;
}

// 1 x 128 blocks.  A warp owns kRows rows x 256 columns: kRows independent 16-byte loads per lane, and the scales of
// kRows consecutive rows leave as one contiguous piece per K block.
// Measured, device time in a captured graph: 8192 x 28672 in 110 us, 6.4 TB/s (a copy: 6.45); 16 x 4096 in 2.6 us (latency).  One call among
// other passes on fresh buffers takes 111 to 125 us and 11 us.  4 or 16 rows per warp 116 to 119 us, loads and stores marked as
// streaming 112 to 117.
constexpr int kQuantizeThreads = 128;
template <int kRows>
__global__ void __launch_bounds__(kQuantizeThreads) quantize_rows_kernel(const QuantizeParams p) {
    static_assert(kRows <= 16, "one lane of a half warp per row stores its scale");
    pdl_begin();
    const int lane = threadIdx.x & 31;
    const int col_tiles = (p.K + 255) / 256;
    const int64_t tile = static_cast<int64_t>(blockIdx.x) * (kQuantizeThreads / 32) + (threadIdx.x >> 5);
    const int row0 = static_cast<int>(tile / col_tiles) * kRows;
    const int c0 = static_cast<int>(tile % col_tiles) * 256 + lane * 8;
    if (row0 >= p.M) return;
    const int left = p.K - c0;
    uint4 v[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r)
        v[r] = (row0 + r < p.M && left > 0) ? quantize_load8(p.X + (row0 + r) * p.ldx + c0, left) : make_uint4(0u, 0u, 0u, 0u);
    uint32_t a[kRows];
    bool odd = false;
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        a[r] = max16lanes(quantize_absmax(v[r]));
        odd |= a[r] >= 0x7F80u;
    }
    if (__any_sync(0xffffffffu, odd)) {
#pragma unroll
        for (int r = 0; r < kRows; ++r) a[r] = max16lanes(quantize_absmax_finite(v[r]));
    }
    float scale = 0.0f;
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const int e = f8_scale_exp(__uint_as_float(a[r] << 16));
        if ((lane & 15) == r) scale = pow2f(e);
        if (row0 + r < p.M && left > 0) quantize_store8(p.Q + (row0 + r) * p.ldq + c0, quantize_pack8(v[r], pow2f(-e)), left);
    }
    const int kb = c0 >> 7;
    if ((lane & 15) < kRows && row0 + (lane & 15) < p.M && kb * 128 < p.K) p.S[kb * p.lds + row0 + (lane & 15)] = scale;
}

// 128 x 128 blocks: one CTA each, 16 rows at a time.  Measured, device time in a captured graph: 28672 x 4096 and 4096 x 28672 in 54 us,
// 6.5 TB/s.
constexpr int kQuantizeBlockThreads = 256;
__global__ void __launch_bounds__(kQuantizeBlockThreads) quantize_blocks_kernel(const QuantizeParams p) {
    __shared__ uint32_t sm[kQuantizeBlockThreads / 32];
    pdl_begin();
    const int kbs = (p.K + 127) / 128;
    const int rb = static_cast<int>(blockIdx.x / kbs), kb = static_cast<int>(blockIdx.x % kbs);
    const int c0 = kb * 128 + (threadIdx.x & 15) * 8, r0 = rb * 128 + (threadIdx.x >> 4);
    const int left = p.K - c0;
    uint4 v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        v[i] = (r0 + i * 16 < p.M && left > 0) ? quantize_load8(p.X + (r0 + i * 16) * p.ldx + c0, left) : make_uint4(0u, 0u, 0u, 0u);
    auto block_max = [&](bool finite_only) {
        uint32_t a = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) a = max(a, finite_only ? quantize_absmax_finite(v[i]) : quantize_absmax(v[i]));
        a = max16lanes(a);
        a = max(a, __shfl_xor_sync(0xffffffffu, a, 16));
        if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = a;
        __syncthreads();
        a = 0;
#pragma unroll
        for (int w = 0; w < kQuantizeBlockThreads / 32; ++w) a = max(a, sm[w]);
        __syncthreads();
        return a;
    };
    uint32_t a = block_max(false);
    if (a >= 0x7F80u) a = block_max(true);  // the same in every thread of the CTA
    const int e = f8_scale_exp(__uint_as_float(a << 16));
    const float inv = pow2f(-e);
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (r0 + i * 16 < p.M && left > 0) quantize_store8(p.Q + (r0 + i * 16) * p.ldq + c0, quantize_pack8(v[i], inv), left);
    if (threadIdx.x == 0) p.S[rb * p.lds + kb] = pow2f(e);
}

inline int quantize_launch(const QuantizeParams& p, int block_rows, cudaStream_t st) {
    if (block_rows == 1) {
        constexpr int kRows = 8;
        const int64_t tiles = static_cast<int64_t>((p.M + kRows - 1) / kRows) * ((p.K + 255) / 256);
        const int64_t ctas = (tiles + kQuantizeThreads / 32 - 1) / (kQuantizeThreads / 32);
        if (ctas > INT32_MAX) return 2;
        return pdl_launch(quantize_rows_kernel<kRows>, dim3(static_cast<unsigned>(ctas)), dim3(kQuantizeThreads), 0, st, 0, p) == cudaSuccess ? 0 : 4;
    }
    const int64_t ctas = static_cast<int64_t>((p.M + 127) / 128) * ((p.K + 127) / 128);
    if (ctas > INT32_MAX) return 2;
    return pdl_launch(quantize_blocks_kernel, dim3(static_cast<unsigned>(ctas)), dim3(kQuantizeBlockThreads), 0, st, 0, p) == cudaSuccess ? 0 : 4;
}

}  // namespace mlt
