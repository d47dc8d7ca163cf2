// E4M3 helpers shared by the 8-bit kernels (quantiser, cache append, scaled GEMM, decode over an 8-bit cache).
//
// Scales made here are powers of two, s = 2^e with the smallest e >= -64 for which amax <= 448 * s.  E4M3 is a
// floating format: its relative step does not depend on s, so a power of two costs no precision against amax / 448,
// x / s is exact (the stored value has one rounding), and values that were stored under one scale move to a larger one
// without a second rounding unless they underflow.
#pragma once

#include "ptx.cuh"

namespace mlt {

constexpr int kF8MinExp = -64;

// The kernels of the 8-bit path follow one another in short calls, so they are launched with programmatic stream
// serialisation: a kernel's blocks may be placed while the one before it in the stream drains, and wait there
// (pdl_begin, before the first access to memory and before any tensor memory is allocated) until that one has completed and
// its writes are visible.  No load is a non-coherent one (ld.global.nc, __ldg): that asks for memory that does not change while
// the kernel is there, and it is there while the kernel before it still writes.  Every block executes pdl_begin, so a kernel's
// completion implies its predecessors'.
// Measured in captured graphs of one call after the other, against plain launches: 0.1 to 0.3 us less per call for single tokens
// (2.6 to 3.9 us), 0.4 to 0.8 for the next-token products, prompts and batches of decode, 1.3 for two long sequences, 1.9 for 777 x 5000 x 4200.
__device__ __forceinline__ void pdl_begin() {
    pdl_launch_dependents();
    cudaGridDependencySynchronize();
}
template <class... Params, class... Args>
cudaError_t pdl_launch(void (*kernel)(Params...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, int cluster, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attrs[2];
    attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attrs[0].val.programmaticStreamSerializationAllowed = 1;
    attrs[1].id = cudaLaunchAttributeClusterDimension;
    attrs[1].val.clusterDim.x = static_cast<unsigned>(cluster);
    attrs[1].val.clusterDim.y = attrs[1].val.clusterDim.z = 1;
    cfg.attrs = attrs;
    cfg.numAttrs = cluster > 0 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// {hi, lo} -> two E4M3 codes, round to nearest even; magnitudes beyond 448 (infinities too) become 448, NaN stays NaN
__device__ __forceinline__ uint32_t f8x2_from_f32(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t f8x4_from_f32(float a, float b, float c, float d) {
    return f8x2_from_f32(a, b) | (f8x2_from_f32(c, d) << 16);
}
// two E4M3 codes -> two FP16 values (exact: FP16 holds every E4M3 value), low code in the low half
__device__ __forceinline__ uint32_t f16x2_from_f8x2(uint16_t v) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(v));
    return r;
}
__device__ __forceinline__ void f16x2_from_f8x4(uint32_t v, uint32_t& lo, uint32_t& hi) {
    lo = f16x2_from_f8x2(static_cast<uint16_t>(v & 0xFFFFu));
    hi = f16x2_from_f8x2(static_cast<uint16_t>(v >> 16));
}
__device__ __forceinline__ float2 f32x2_from_f16x2(uint32_t v) {
    float2 f;
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.f32.f16 %0, l;\n\tcvt.f32.f16 %1, h;\n\t}" : "=f"(f.x), "=f"(f.y) : "r"(v));
    return f;
}

// Exponent e of the scale for a finite amax >= 0 (448 = 1.75 * 2^8).
__device__ __forceinline__ int f8_scale_exp(float amax) {
    const uint32_t b = __float_as_uint(amax);
    const int e = static_cast<int>(b >> 23) - 127 - 8 + ((b & 0x7FFFFFu) > 0x600000u ? 1 : 0);  // FP32 subnormals give e < -64
    return max(kF8MinExp, e);  // at most 127 - 8 + 1 = 120
}
__device__ __forceinline__ float pow2f(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }  // -126 <= e <= 127

__device__ __forceinline__ bool is_pow2(float s) { return (__float_as_uint(s) & 0x7FFFFFu) == 0u; }  // of a positive normal number

// a * b and a / b rounded to odd: toward zero, with the last bit set where something was cut off.  A later rounding to E4M3's four
// bits then gives what rounding the exact result gives (a rounding to nearest in between could land on the middle between two
// values).  The remainders are exact, or far too small to matter where they underflow.
__device__ __forceinline__ float to_odd(float cut, float rest) {
    const bool odd = rest != 0.0f && fabsf(cut) <= 3.402823466e38f;  // (infinities and NaN as they are)
    return __uint_as_float(__float_as_uint(cut) | (odd ? 1u : 0u));
}
__device__ __forceinline__ float mul_to_odd(float a, float b) {
    const float r = __fmul_rz(a, b);
    return to_odd(r, fmaf(a, b, -r));
}
__device__ __forceinline__ float div_to_odd(float a, float b) {
    const float r = __fdiv_rz(a, b);
    return to_odd(r, fmaf(-r, b, a));
}

__device__ __forceinline__ float abs_if_finite(float x) {
    const float a = fabsf(x);
    return a <= 3.402823466e38f ? a : 0.0f;  // infinities and NaN do not set a scale
}

}  // namespace mlt
