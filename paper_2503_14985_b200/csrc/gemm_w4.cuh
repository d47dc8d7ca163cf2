// Few rows times 4-bit weights:  C[i][n] = sum over groups j of scale[n][j] * sum over k in j of x[i][k] (q[n][k] - z[n][j]).
//
// Bound by the weights' bytes (N K / 2, read once).  At the copy bandwidth an SM gets about 46 weights per clock, so what
// counts besides keeping loads in flight is instructions per weight, above all on the integer pipe (one per two clocks and scheduler):
//  * The weights are the A operand (16 rows) of mma.sync m16n8k16, the rows of x the B operand (8 columns), both FP16 with FP32
//    accumulators.  The bits of a 4-bit weight are an FP16 number as they stand, the subnormal q 2^-24: a 32-bit word of 8 weights
//    becomes four FP16 pairs with one shift and four ANDs, v & 0x000F000F and v & 0x00F000F0 for v = w and v = w >> 8; the x that meet
//    the latter, 16 q 2^-24, are divided by 16.  The accumulator of a group starts at -z sum x (the sums are taken once per CTA),
//    products are exact, and the group's scale and the factors are applied once per group and output.
//  * x is BF16, whose range FP16 lacks: each group of a row is multiplied by the power of two that brings its largest element to
//    2^14 .. 2^15, and the inverse goes into the group's factor.  An element loses bits only below 2^-27 of that largest one.
//    (The smallest BF16 numbers would need more than an FP32 power of two, but 2^126 already makes whole multiples of 2^-7 of them.)
//  * Range.  The inverse times 2^24 need not fit FP32, so 2^12 of it are kept for the end: a group's sum times 2^-12 fits whatever x
//    is, and meets the scale only then (two columns at a time: one by one, 16 x 4096 x 28672 took 46.1 us instead of 43.6).  Sums over groups overflow where 2^12 times as much would.  What is smaller than 2^-114 is
//    rounded at 2^-138.  The sum of x itself is taken in units of 2^8.
//  * The order of the summation index of an MMA is free.  The pairs of a word are (k, k + 4); x is laid out in shared memory
//    in that order once per CTA, as the B fragments (16 bytes per lane, no bank conflicts).  A lane's words of a group lie side by
//    side, so that a quad covers whole groups.
//  * A warp works on pieces of 32 weight rows x 256 of K, so every B fragment serves two MMAs.  Pieces come by TMA in halves of 128 of
//    K (64-byte swizzle, zeros beyond N and K) into a ring of the warp's own, and a half is requested again as soon as it has been
//    read; which row of a piece a lane takes is chosen so that the swizzled reads of 16, 8 or 4 bytes (groups of 128, 64, 32)
//    meet no bank conflicts.
//  * CTAs are persistent (one per SM) and keep x in shared memory.  The pieces of all row tiles of a CTA, in order (row tile, then
//    K), are one list of which each of the 16 warps takes a sixteenth, wherever that cuts a tile's K; the sums of the runs meet
//    once, behind the only barrier.  (Against one set of row tiles at a time, K cut over the warps and a barrier per set:
//    16 x 28672 x 4096 38.7 -> 29.9 us, 16 x 4096 x 28672 56 -> 42.7, 1 x 28672 x 4096 18.6 -> 16.4; 1 x 4096 x 4096, one tile per CTA
//    either way, 5.3 -> 5.7.)  Where x does not fit or there are fewer tiles than SMs, a cluster cuts K and sums through
//    distributed shared memory, in a fixed order.  More than 16 rows run as several passes over the weights (from L2, mostly), one behind the
//    other: 28672 x 4096 with group 128 takes 32 us with 16 rows, 59 with 32, 112 with 64.
// Times are those of graphs of ten calls.  58.7 MB of weights (28672 x 4096) take 12.3 us to read by TMA or by plain loads and nothing
// else, 9 at the copy bandwidth.  With 1 row the kernel is 1.3 of that; with 16 the matrix instructions (m16n8k16 at 16 weights and 8
// columns) and what turns the words into them bound it.
#pragma once

#include <cuda_fp16.h>

#include <algorithm>

#include "paged.cuh"
#include "ptx.cuh"

namespace mlt {

constexpr int kW4Warps = 16;
constexpr int kW4Threads = kW4Warps * 32;
constexpr int kW4Step = 256;       // K per piece: 128 bytes of a weight row, in two halves
constexpr int kW4Tile = 32;        // weight rows per piece
constexpr int kW4PieceBytes = kW4Tile * kW4Step / 2, kW4HalfBytes = kW4PieceBytes / 2;
constexpr int kW4MaxRing = 3;      // pieces per warp in shared memory
constexpr int kW4ColPitch = 36;    // words per column of a warp's partial sums (no bank conflicts)
constexpr int kW4Smem = 227 * 1024;
constexpr float kW4SumUnit = 0.00390625f;  // 2^-8: 128 elements of any BF16 value add up to less than FP32's largest

struct W4Params {
    const __nv_bfloat16* X;       // [M, K], pitch ldx
    const __nv_bfloat16* scales;  // [N, K / group], pitch lds
    const uint8_t* zeros;         // [N, K / group], pitch ldz, or null (8)
    __nv_bfloat16* C;             // [M, N], pitch ldc
    int64_t ldx, lds, ldz, ldc;
    int M, N, K;
    int wide_scales;  // a piece's scales (zero points) of a row can be read at once
    int rows;         // rows of x per pass (R of the kernel)
    int steps;        // pieces of K per CTA
    int cluster;      // CTAs that cut K
    int tiles_each, tiles_over;  // row tiles of a CTA or cluster (the first tiles_over have one more)
    int sets;         // sets of row tiles that those are cut into
    int set_tiles;    // row tiles of a set, at most
    int ring;         // pieces per warp in flight
    // offsets in shared memory, in bytes
    int at_x, at_fac, at_sums;
};

// Row (0..7) of an 8-row group that lane group g reads: with the TMA's 64-byte swizzle (16-byte chunk c of row r at c ^ ((r >> 1) & 3))
// the lanes that one shared-memory phase serves (8 of 16 bytes, 16 of 8, 32 of 4) then hit different banks.
template <int VEC>
__device__ __forceinline__ int w4_row(int g) {
    return VEC == 2 ? (g & 1) | ((g & 2) << 1) | ((g & 4) >> 1) : g;
}

__device__ __forceinline__ void w4_mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// R: rows of x per pass, a power of two (those beyond the last are zeros);  VEC: words of a lane per group (group = 32 * VEC)
template <int R, int VEC>
__global__ void __launch_bounds__(kW4Threads, 1) gemm_w4_kernel(const __grid_constant__ CUtensorMap tmap_w, const W4Params p) {
    constexpr int kGroup = 32 * VEC;
    constexpr int kGroups = kW4Step / kGroup;  // groups per piece
    constexpr int MT = R > 8 ? 2 : 1;          // columns of x in units of 8
    constexpr int kColumns = R < 8 ? R : 8;    // of a unit
    extern __shared__ uint8_t w4_smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(w4_smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ uint64_t bars[kW4Warps][2 * kW4MaxRing];
    __shared__ uint32_t abort_word;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int rank = p.cluster > 1 ? static_cast<int>(cluster_ctarank()) : 0;
    const int m0 = blockIdx.y * R, rows = min(R, p.M - m0);
    const int step0 = rank * p.steps;                                  // first piece of K of this CTA
    const int all_steps = (p.K + kW4Step - 1) / kW4Step;
    const int steps = max(0, min(p.steps, all_steps - step0));         // (the last CTAs of a cluster may have fewer, or none)
    const int owner = static_cast<int>(blockIdx.x) >> (31 - __clz(p.cluster));  // (1, 2, 4 or 8 CTAs)
    const int first = owner * p.tiles_each + min(owner, p.tiles_over), end = first + p.tiles_each + (owner < p.tiles_over);
    uint8_t* ring = smem + warp * p.ring * kW4PieceBytes;
    uint4* xs = reinterpret_cast<uint4*>(smem + p.at_x);               // [piece][word][row][t]
    float2* fac = reinterpret_cast<float2*>(smem + p.at_fac);          // [group][row] {scaled sum of x times 2^-24, inverse factor times 2^12}
    float* sums = reinterpret_cast<float*>(smem + p.at_sums);          // [row tile of the set][row of x][kW4ColPitch]
    constexpr int kSums = R * kW4ColPitch;                             // floats per tile

    if (lane == 0) {
        for (int i = 0; i < 2 * kW4MaxRing; ++i) mbar_init(&bars[warp][i], 1);
        if (warp == 0) abort_word = 0;
        fence_mbar_init();
    }
    pdl_launch_dependents();
    __syncthreads();
    cudaGridDependencySynchronize();

    // A set of row tiles is n * steps pieces in order (row tile, then K), of which each warp takes a sixteenth.
    int sets_left = p.sets, tile0 = first, n = 0, u = 0, u_end = 0;
    int ld_tile = 0, ld_step = 0, ld_u = 0, ld_slot = 0;
    auto request = [&](int half) {  // half of the next piece, into its slot
        if (ld_u < u_end && lane == 0) {
            const int at = 2 * ld_slot + half;
            mbar_arrive_expect_tx(&bars[warp][at], kW4HalfBytes);
            tma_load_2d(ring + at * kW4HalfBytes, &tmap_w, &bars[warp][at], (step0 + ld_step) * (kW4Step / 2) + half * (kW4Step / 4), ld_tile * kW4Tile);
        }
    };
    auto next_request = [&]() {
        if (ld_u >= u_end) return;
        ++ld_u;
        if (++ld_slot == p.ring) ld_slot = 0;
        if (++ld_step == steps) {
            ld_step = 0;
            ++ld_tile;
        }
    };
    auto tile_of = [&](int unit) { return n == 1 || steps == 0 ? 0 : unit / steps; };
    auto run_start = [&](int w) { return n * steps * w / kW4Warps; };
    auto begin_set = [&]() {
        n = min(p.set_tiles, end - tile0);
        u = run_start(warp);
        u_end = run_start(warp + 1);
        ld_u = u;
        ld_tile = tile0 + tile_of(u);
        ld_step = u - (ld_tile - tile0) * steps;
        for (int i = 0; i < p.ring; ++i) {
            request(0);
            request(1);
            next_request();
        }
    };
    begin_set();

    // x, in fragment order: 8 consecutive k become (k, k + 4), (k + 1, k + 5), ...
    for (int k8 = threadIdx.x; k8 < steps * (kW4Step / 8); k8 += kW4Threads) {  // (whole warps)
        const int k = step0 * kW4Step + k8 * 8;
        const int in_step = k8 % 32, q = in_step / (4 * VEC), r = in_step % (4 * VEC);
        uint4* to = xs + ((k8 / 32) * 8 + q * VEC + r % VEC) * R * 4 + r / VEC;
        const __nv_bfloat16* from = p.X + m0 * p.ldx + k;
        uint4 v[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            v[i] = make_uint4(0u, 0u, 0u, 0u);
            if (i < rows && k < p.K) v[i] = *reinterpret_cast<const uint4*>(from + i * p.ldx);
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            float f[8];
            bf16x8_to_f32(v[i], f);
            float top = 0.0f, sum = f[0] * kW4SumUnit, sum1 = f[4] * kW4SumUnit;
#pragma unroll
            for (int e = 1; e < 4; ++e) {
                sum = fmaf(f[e], kW4SumUnit, sum);
                sum1 = fmaf(f[e + 4], kW4SumUnit, sum1);
            }
            sum += sum1;
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(f[e]));
#pragma unroll
            for (int w = 1; w < 4 * VEC; w <<= 1) {
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
                sum += __shfl_xor_sync(0xffffffffu, sum, w);
            }
            const int up = min(268 - static_cast<int>(__float_as_uint(top) >> 23), 253);  // exponent field of the factor
            const float mul = __uint_as_float(static_cast<uint32_t>(up) << 23), mul16 = mul * 0.0625f;
            const __half2 h0 = __floats2half2_rn(f[0] * mul, f[4] * mul), h1 = __floats2half2_rn(f[1] * mul16, f[5] * mul16);
            const __half2 h2 = __floats2half2_rn(f[2] * mul, f[6] * mul), h3 = __floats2half2_rn(f[3] * mul16, f[7] * mul16);
            to[i * 4] = make_uint4(*reinterpret_cast<const uint32_t*>(&h0), *reinterpret_cast<const uint32_t*>(&h1),
                                   *reinterpret_cast<const uint32_t*>(&h2), *reinterpret_cast<const uint32_t*>(&h3));
            if (r == 0)
                fac[((k8 / 32) * kGroups + q) * R + i] = make_float2(sum * mul * 1.52587890625e-5f, __uint_as_float(static_cast<uint32_t>(266 - up) << 23));
        }
    }
    __syncthreads();
    // scales and zero points of a piece, as they lie in memory: this lane holds those of row 8 t + w4_row(g)
    const int my_row = w4_row<VEC>(g);
    int sc_tile = 0, sc_step = 0, sc_u = 0;
    const uint16_t* scale_at = nullptr;
    const uint8_t* zero_at = nullptr;
    struct Scales {
        uint32_t s[kGroups / 2], z[(kGroups + 3) / 4];
    };
    auto load_scales = [&](Scales& sc) {
        if (sc_u < u_end) {
            const bool in_n = sc_tile * kW4Tile + 8 * t + my_row < p.N;
            if (p.wide_scales && (step0 + sc_step + 1) * kW4Step <= p.K) {
                if (in_n) {
                    if constexpr (kGroups == 8) {
                        const uint4 v = *reinterpret_cast<const uint4*>(scale_at);
                        sc.s[0] = v.x; sc.s[1] = v.y; sc.s[2] = v.z; sc.s[3] = v.w;
                    } else if constexpr (kGroups == 4) {
                        const uint2 v = *reinterpret_cast<const uint2*>(scale_at);
                        sc.s[0] = v.x; sc.s[1] = v.y;
                    } else {
                        sc.s[0] = *reinterpret_cast<const uint32_t*>(scale_at);
                    }
                    if (p.zeros) {
                        if constexpr (kGroups == 8) {
                            const uint2 v = *reinterpret_cast<const uint2*>(zero_at);
                            sc.z[0] = v.x; sc.z[1] = v.y;
                        } else if constexpr (kGroups == 4) {
                            sc.z[0] = *reinterpret_cast<const uint32_t*>(zero_at);
                        } else {
                            sc.z[0] = *reinterpret_cast<const uint16_t*>(zero_at);
                        }
                    }
                }
            } else {
                const int left = in_n ? p.K / kGroup - (step0 + sc_step) * kGroups : 0;
#pragma unroll
                for (int i = 0; i < kGroups / 2; ++i) sc.s[i] = 0;
#pragma unroll
                for (int q = 0; q < kGroups; ++q)
                    if (q < left) {
                        sc.s[q >> 1] |= static_cast<uint32_t>(scale_at[q]) << (16 * (q & 1));
                        if (p.zeros) sc.z[q >> 2] = (sc.z[q >> 2] & ~(0xFFu << (8 * (q & 3)))) | (static_cast<uint32_t>(zero_at[q]) << (8 * (q & 3)));
                    }
            }
        }
        ++sc_u;
        int64_t by = kGroups, z_by = kGroups;
        if (++sc_step == steps) {
            sc_step = 0;
            ++sc_tile;
            by += kW4Tile * p.lds - static_cast<int64_t>(steps) * kGroups;
            z_by += kW4Tile * p.ldz - static_cast<int64_t>(steps) * kGroups;
        }
        scale_at += by;
        zero_at += z_by;
    };
    float acc[2][MT][4];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[h][m][e] = 0.0f;
    // (columns beyond R repeat others; their sums go nowhere)
    const uint4* x_at = xs + (g & (kColumns - 1)) * 4 + t;
    const int col0 = (2 * t) & (kColumns - 1), col1 = (2 * t + 1) & (kColumns - 1);
    const int twist = (my_row >> 1) & 3;
    const int w_at = my_row * 64 + (VEC == 4 ? (t ^ twist) * 16 : VEC == 2 ? ((t >> 1) ^ twist) * 16 + (t & 1) * 8 : twist * 16 + t * 4);

    constexpr int kHalfGroups = kGroups / 2;
    // (One copy of this code, not one per half: unrolled, a row tile's pass runs through more instructions than the cache near
    // the schedulers holds.)
    auto compute = [&](int slot, int half, int step, const Scales& sc) {
        uint32_t s_half[(kHalfGroups + 1) / 2], z_half;  // the half's scales and zero points, from the lowest bits on
        if constexpr (kHalfGroups == 4) {
            s_half[0] = half ? sc.s[2] : sc.s[0];
            s_half[1] = half ? sc.s[3] : sc.s[1];
            z_half = half ? sc.z[1] : sc.z[0];
        } else if constexpr (kHalfGroups == 2) {
            s_half[0] = half ? sc.s[1] : sc.s[0];
            z_half = sc.z[0] >> (16 * half);
        } else {
            s_half[0] = sc.s[0] >> (16 * half);
            z_half = sc.z[0] >> (8 * half);
        }
        const uint8_t* w_half = ring + (2 * slot + half) * kW4HalfBytes;
        const uint4* x_half = x_at + (2 * step + half) * (4 * R * 4);
        const float2* fac_half = fac + (2 * step + half) * (kHalfGroups * R);
#pragma unroll
        for (int q = 0; q < kHalfGroups; ++q) {
            uint32_t w[4][VEC];  // rows w4_row(g) + 0, 8, 16, 24
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const uint8_t* at = w_half + (w_at ^ (q * 16 * VEC)) + r * 512;
                if constexpr (VEC == 4) {
                    const uint4 v = *reinterpret_cast<const uint4*>(at);
                    w[r][0] = v.x; w[r][1] = v.y; w[r][2] = v.z; w[r][3] = v.w;
                } else if constexpr (VEC == 2) {
                    const uint2 v = *reinterpret_cast<const uint2*>(at);
                    w[r][0] = v.x; w[r][1] = v.y;
                } else {
                    w[r][0] = *reinterpret_cast<const uint32_t*>(at);
                }
            }
            float s[4], z[4];
            // scale in the upper half, 128 + z in the lower, both BF16
            const uint32_t sz = __byte_perm(s_half[q >> 1], __byte_perm(z_half, 0x43u, 0x0040 + q), (q & 1) ? 0x3254 : 0x1054);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const uint32_t v = __shfl_sync(0xffffffffu, sz, (lane & 28) | r);
                s[r] = __uint_as_float(v & 0xFFFF0000u);
                z[r] = 128.0f - __uint_as_float(v << 16);  // -z
            }
            float c[2][MT][4], u0[MT], u1[MT];
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const float2 f0 = fac_half[q * R + m * 8 + col0], f1 = fac_half[q * R + m * 8 + col1];
                u0[m] = f0.y;
                u1[m] = f1.y;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    c[h][m][0] = z[2 * h] * f0.x;
                    c[h][m][1] = z[2 * h] * f1.x;
                    c[h][m][2] = z[2 * h + 1] * f0.x;
                    c[h][m][3] = z[2 * h + 1] * f1.x;
                }
            }
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                uint4 b[MT];
#pragma unroll
                for (int m = 0; m < MT; ++m) b[m] = x_half[(q * VEC + v) * (R * 4) + m * 32];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t a0 = w[2 * h][v], a1 = w[2 * h + 1][v], b0 = a0 >> 8, b1 = a1 >> 8;
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        w4_mma(c[h][m], a0 & 0x000F000Fu, a1 & 0x000F000Fu, a0 & 0x00F000F0u, a1 & 0x00F000F0u, b[m].x, b[m].y);
                        w4_mma(c[h][m], b0 & 0x000F000Fu, b1 & 0x000F000Fu, b0 & 0x00F000F0u, b1 & 0x00F000F0u, b[m].z, b[m].w);
                    }
                }
            }
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
#pragma unroll
                    for (int e = 0; e < 4; e += 2) {
                        const float sc_row = s[2 * h + e / 2];
                        const float2 sum = fmul2(make_float2(c[h][m][e], c[h][m][e + 1]), make_float2(u0[m], u1[m]));
                        const float2 to = ffma2(sum, make_float2(sc_row, sc_row), make_float2(acc[h][m][e], acc[h][m][e + 1]));
                        acc[h][m][e] = to.x;
                        acc[h][m][e + 1] = to.y;
                    }
                }
        }
    };

    // Sums.  A warp's pieces of a row tile are a run of K.  A run that ends with its tile while the warp has more to do leaves its
    // sums in the tile's place (there is at most one such run per tile), a warp's last run in the warp's ring, which is empty by
    // then.  Behind one barrier a warp per (tile, row of x) adds the runs up in the order of K, a lane per weight row.  With a
    // cluster the CTA's sums take the tile's place, and the CTAs' are added in order.
    auto put_sums = [&](float* to) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (2 * t + (e & 1) < kColumns) to[(8 * m + 2 * t + (e & 1)) * kW4ColPitch + h * 16 + (e >> 1) * 8 + my_row] = acc[h][m][e];
                    acc[h][m][e] = 0.0f;
                }
    };
    auto store = [&](int i, int row, float sum) {
        const int col = (tile0 + i) * kW4Tile + lane;
        if (col < p.N) p.C[(m0 + row) * p.ldc + col] = __float2bfloat16(sum * 4096.0f);
    };
    auto add_sums = [&]() {
        for (int item = warp; item < n * R; item += kW4Warps) {
            const int i = item / R, row = item % R, from = i * steps, to = from + steps;
            if (row >= rows) continue;
            float* place = sums + i * kSums + row * kW4ColPitch + lane;
            float sum = 0.0f;
            for (int w = n == 1 ? 0 : i * kW4Warps / n; w < kW4Warps && run_start(w) < to; w += 4) {
                float v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int a = run_start(w + j), b = run_start(w + j + 1);
                    v[j] = 0.0f;
                    if (w + j < kW4Warps && a < to && b > max(a, from))
                        v[j] = b > to ? *place : reinterpret_cast<const float*>(smem + (w + j) * p.ring * kW4PieceBytes)[row * kW4ColPitch + lane];
                }
                sum += v[0];
                sum += v[1];
                sum += v[2];
                sum += v[3];
            }
            if (p.cluster > 1) *place = sum;
            else store(i, row, sum);
        }
        if (p.cluster == 1) return;
        __syncwarp();
        cluster_sync_all();
        for (int item = rank * kW4Warps + warp; item < n * R; item += p.cluster * kW4Warps) {
            const int i = item / R, row = item % R;
            if (row >= rows) continue;
            const uint32_t at = smem_u32(sums + i * kSums + row * kW4ColPitch + lane);
            float v[8];
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                v[c] = 0.0f;
                if (c < p.cluster) asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v[c]) : "r"(map_to_cta(at, static_cast<uint32_t>(c))) : "memory");
            }
            store(i, row, ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7])));
        }
        __syncwarp();
        cluster_sync_all();  // the sums have been read
    };

    Scales sc, next_sc;
#pragma unroll
    for (int i = 0; i < (kGroups + 3) / 4; ++i) sc.z[i] = 0x08080808u;
#pragma unroll
    for (int i = 0; i < kGroups / 2; ++i) sc.s[i] = 0u;
    next_sc = sc;
    int slot = 0;
    uint32_t phase = 0;  // of the slot in turn
    bool ok = true;
#pragma unroll 1
    for (;;) {
        int i = tile_of(u), step = u - i * steps;  // row tile of the set, and piece of K, of unit u
        sc_u = u;
        sc_tile = tile0 + i;
        sc_step = step;
        const int64_t row = static_cast<int64_t>(sc_tile) * kW4Tile + 8 * t + my_row;
        scale_at = reinterpret_cast<const uint16_t*>(p.scales) + row * p.lds + (step0 + step) * kGroups;
        zero_at = p.zeros + row * p.ldz + (step0 + step) * kGroups;
        load_scales(sc);
#pragma unroll 1
        while (u < u_end) {
            load_scales(next_sc);
#pragma unroll 1
            for (int half = 0; half < 2; ++half) {
                if (ok) {
                    ok = __all_sync(0xffffffffu, mbar_wait(&bars[warp][2 * slot + half], phase, &abort_word, 0x800 + warp)) != 0;
                    if (ok) compute(slot, half, step, sc);
                }
                __syncwarp();
                if (ok) request(half);
            }
            next_request();
            sc = next_sc;
            if (++slot == p.ring) {
                slot = 0;
                phase ^= 1;
            }
            ++u;
            if (++step == steps || u == u_end) {
                put_sums(u == u_end ? reinterpret_cast<float*>(ring) : sums + i * kSums);
                step = 0;
                ++i;
            }
        }
        __syncthreads();
        add_sums();
        tile0 += n;
        if (--sets_left == 0) break;
        fence_proxy_async_smem();  // the rings have been written and read as sums
        __syncthreads();
        begin_set();
    }
}

template <int R, int VEC>
int w4_launch_one(const CUtensorMap& tw, const W4Params& p, int grid, int smem, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(grid), static_cast<unsigned>((p.M + R - 1) / R));
    cfg.blockDim = dim3(kW4Threads);
    cfg.dynamicSmemBytes = static_cast<size_t>(smem);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = static_cast<unsigned>(p.cluster);
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = p.cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, gemm_w4_kernel<R, VEC>, tw, p) == cudaSuccess ? 0 : 4;
}

template <int VEC>
int w4_launch_rows(const CUtensorMap& tw, const W4Params& p, int grid, int smem, cudaStream_t st) {
    switch (p.rows) {
        case 1: return w4_launch_one<1, VEC>(tw, p, grid, smem, st);
        case 2: return w4_launch_one<2, VEC>(tw, p, grid, smem, st);
        case 4: return w4_launch_one<4, VEC>(tw, p, grid, smem, st);
        case 8: return w4_launch_one<8, VEC>(tw, p, grid, smem, st);
        default: return w4_launch_one<16, VEC>(tw, p, grid, smem, st);
    }
}
inline int w4_launch(const CUtensorMap& tw, const W4Params& p, int group, int grid, int smem, cudaStream_t st) {
    return group == 32 ? w4_launch_rows<1>(tw, p, grid, smem, st) : group == 64 ? w4_launch_rows<2>(tw, p, grid, smem, st)
                                                                               : w4_launch_rows<4>(tw, p, grid, smem, st);
}

template <int R, int VEC>
bool w4_configure_one() {
    return cudaFuncSetAttribute(gemm_w4_kernel<R, VEC>, cudaFuncAttributeMaxDynamicSharedMemorySize, kW4Smem - 1024) == cudaSuccess;
}
template <int VEC>
bool w4_configure_rows() {
    return w4_configure_one<1, VEC>() && w4_configure_one<2, VEC>() && w4_configure_one<4, VEC>() && w4_configure_one<8, VEC>() &&
           w4_configure_one<16, VEC>();
}
inline bool w4_configure() { return w4_configure_rows<1>() && w4_configure_rows<2>() && w4_configure_rows<4>(); }

// Pieces per warp that fit beside `rows` rows of x and the sums of one row tile, K cut over c CTAs (0: not even one).
constexpr int kW4Limit = kW4Smem - 2048;  // 1 KB of static shared memory and its like, 1 KB for the ring's alignment
inline int w4_steps(int K, int c) {
    const int all_steps = (K + kW4Step - 1) / kW4Step;
    return std::max(1, (all_steps + c - 1) / c);
}
inline int64_t w4_fixed_bytes(int K, int group, int rows, int c) {  // x and its factors
    return static_cast<int64_t>(rows) * w4_steps(K, c) * (kW4Step * 2 + kW4Step / group * 8) + 16;
}
inline int w4_sum_bytes(int rows) { return rows * kW4ColPitch * 4; }  // of a row tile
inline int w4_ring(int K, int group, int rows, int c) {
    const int64_t left = kW4Limit - w4_fixed_bytes(K, group, rows, c) - w4_sum_bytes(rows);
    return left < 0 ? 0 : static_cast<int>(std::min<int64_t>(kW4MaxRing, left / (kW4Warps * kW4PieceBytes)));
}
// Whether M rows, as many at a time as a cluster of 8 holds, are no more passes than a grid has.
inline bool w4_fits(int64_t M, int K, int group) {
    int rows = 16;
    while (rows > 0 && w4_ring(K, group, rows, 8) == 0) rows /= 2;
    return rows > 0 && (M + rows - 1) / rows <= 65535;
}

// Rows per pass, CTAs per cluster, warps along K and the layout of shared memory; false if not even one row of x fits a cluster of 8, or
// there are more passes than a grid has.
// cluster_slots: resident CTAs in clusters of 2, 4, 8.
inline bool w4_plan(W4Params* p, int group, int sm_count, const int* cluster_slots, int* grid, int* smem) {
    const int all_steps = (p->K + kW4Step - 1) / kW4Step, tiles = (p->N + kW4Tile - 1) / kW4Tile;
    auto ring_of = [&](int rows, int c) { return w4_ring(p->K, group, rows, c); };
    auto slots = [&](int c) { return c == 1 ? sm_count : cluster_slots[c == 2 ? 0 : c == 4 ? 1 : 2]; };
    auto most_tiles = [&](int c) {  // of a cluster
        const int owners = std::max(1, std::min(slots(c) / c, tiles));
        return (tiles + owners - 1) / owners;
    };
    auto room = [&](int rows, int c) {  // row tiles that a set can have
        return static_cast<int>((kW4Limit - w4_fixed_bytes(p->K, group, rows, c) - ring_of(rows, c) * kW4Warps * kW4PieceBytes) / w4_sum_bytes(rows));
    };
    // The smallest cluster that x and one piece per warp fit, and beside them the sums of four row tiles, or of all that there are
    // (16 x 28672 x 4864: sets of one tile 54 us, a cluster of two 48).
    int rows = 1, c = 0;
    while (rows < 16 && rows < p->M) rows *= 2;
    for (; rows > 0; rows /= 2) {
        for (int k = 8; k >= 1; k /= 2)
            if (slots(k) >= k && ring_of(rows, k) > 0 && (c == 0 || room(rows, k) >= std::min(4, most_tiles(k)))) c = k;
        if (c > 0) break;
    }
    if (rows <= 0 || (p->M + rows - 1) / rows > 65535) return false;
    // fewer tiles than half the SMs: cut K further, while a CTA keeps four pieces
    while (c < 8 && slots(2 * c) >= 2 * c && static_cast<int64_t>(tiles) * 2 * c <= sm_count && all_steps >= 2 * c * 4) c *= 2;
    p->rows = rows;
    p->cluster = c;
    p->steps = w4_steps(p->K, c);
    p->ring = ring_of(rows, c);
    const int owners = std::max(1, std::min(slots(c) / c, tiles)), most = most_tiles(c);
    *grid = c * owners;
    p->at_x = kW4Warps * p->ring * kW4PieceBytes;
    p->at_fac = p->at_x + rows * p->steps * kW4Step * 2;
    p->at_sums = p->at_fac + (rows * p->steps * (kW4Step / group) * 8 + 15) / 16 * 16;
    p->tiles_each = tiles / owners;
    p->tiles_over = tiles % owners;
    const int at_most = (kW4Limit - p->at_sums) / w4_sum_bytes(rows);
    p->sets = (most + at_most - 1) / at_most;
    p->set_tiles = (most + p->sets - 1) / p->sets;
    *smem = p->at_sums + p->set_tiles * w4_sum_bytes(rows) + 1024;
    return true;
}

}  // namespace mlt
