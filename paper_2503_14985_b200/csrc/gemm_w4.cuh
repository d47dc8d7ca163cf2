// Few rows times 4-bit weights:  C[i][n] = sum over groups j of scale[n][j] * sum over k in j of x[i][k] (q[n][k] - z[n][j]).
//
// Bound by the weights' bytes (N K / 2, read once).  At the copy bandwidth an SM gets about 46 weights per clock, so what
// counts besides keeping loads in flight is instructions per weight:
//  * The weights are the A operand (16 rows) of mma.sync m16n8k16, the rows of x the B operand (8 columns).  A 32-bit word of 8
//    weights becomes four BF16 pairs by (w >> 4 i) & 0x000F000F | 0x43004300: 128 + q, exact, one shift and one three-input
//    logic operation per pair.  Nothing is subtracted per weight: the accumulator of a group starts at -(128 + z) sum x, with the
//    sums of x taken once per CTA, so products and sums stay in FP32 and scales are applied once per group and output.
//    (Starting value and sum are up to 143 sum |x|, so a group's rounding is 143 * 2^-23 of that at most per addition.)
//  * The order of the summation index of an MMA is free.  The pairs of a word are (k, k + 4); x is laid out in shared memory
//    in that order once per CTA, as the B fragments (16 bytes per lane, no bank conflicts).  A lane's words of a group lie side by
//    side, so that a quad covers whole groups: a load is 16, 8 or 4 bytes per lane for groups of 128, 64 or 32.
//  * A warp works on 32 weight rows x 128 of K at a time, so every B fragment serves two MMAs.  The 16 warps of a CTA cut K among
//    them (and row tiles, where K is short); their partial sums meet in shared memory.  Weights go from global memory straight to
//    registers, kW4Ahead pieces ahead of their use.
//  * CTAs are persistent (one per SM); x stays in shared memory for all row tiles of a CTA.  Where x does not fit or there are
//    fewer tiles than SMs, a cluster cuts K and sums through distributed shared memory, in a fixed order.  More than 16 rows run as
//    several passes over the weights (from L2, mostly).
#pragma once

#include <algorithm>

#include "paged.cuh"
#include "ptx.cuh"

namespace mlt {

constexpr int kW4Threads = 512;
constexpr int kW4Warps = kW4Threads / 32;
constexpr int kW4Ahead = 2;        // pieces of 32 rows x 128 of K that a warp has in flight
constexpr int kW4Step = 128;       // K per piece
constexpr int kW4Tile = 32;        // weight rows per piece
constexpr int kW4ColPitch = 36;    // words per column of a warp's partial sums (no bank conflicts)
constexpr int kW4Smem = 227 * 1024;

struct W4Params {
    const __nv_bfloat16* X;       // [M, K], pitch ldx
    const uint8_t* W;             // [N, K / 2], pitch ldw bytes
    const __nv_bfloat16* scales;  // [N, K / group], pitch lds
    const uint8_t* zeros;         // [N, K / group], pitch ldz, or null (8)
    __nv_bfloat16* C;             // [M, N], pitch ldc
    int64_t ldx, ldw, lds, ldz, ldc;
    int M, N, K;
    int rows;         // rows of x per pass
    int steps;        // pieces of K per CTA
    int k_warps;      // warps that cut them (a power of two); kW4Warps / k_warps row tiles at a time
    int cluster;      // CTAs that cut K
};

// bytes of shared memory in front of the partial sums: x, then the groups' sums
__host__ __device__ inline int w4_x_bytes(int rows, int steps) { return rows * steps * kW4Step * 2; }
__host__ __device__ inline int w4_sum_bytes(int rows, int steps, int group) { return (rows * steps * (kW4Step / group) * 4 + 15) / 16 * 16; }
template <int MT>
__host__ __device__ constexpr int w4_red_bytes() { return 2 * kW4Warps * MT * 8 * kW4ColPitch * 4; }
__host__ __device__ inline int w4_part_bytes(int rows, int k_warps, int cluster) {
    return cluster > 1 ? 2 * (kW4Warps / k_warps) * kW4Tile * rows * 4 : 0;
}

// MT: columns of x in units of 8;  VEC: words of a lane per group (group = 32 * VEC)
template <int MT, int VEC>
__global__ void __launch_bounds__(kW4Threads, 1) gemm_w4_kernel(const W4Params p) {
    constexpr int kGroup = 32 * VEC;
    constexpr int kGroups = kW4Step / kGroup;  // groups per piece
    extern __shared__ __align__(16) uint8_t w4_smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int k_warps = p.k_warps, tiles_at_once = kW4Warps / k_warps;
    const int kw = warp % k_warps, tw = warp / k_warps;
    const int rank = p.cluster > 1 ? static_cast<int>(cluster_ctarank()) : 0;
    const int m0 = blockIdx.y * p.rows, rows = min(p.rows, p.M - m0);
    const int step0 = rank * p.steps;                                  // first piece of K of this CTA
    const int all_steps = (p.K + kW4Step - 1) / kW4Step;
    const int steps = max(0, min(p.steps, all_steps - step0));         // (the last CTAs of a cluster may have fewer, or none)
    const int tiles = (p.N + kW4Tile - 1) / kW4Tile;
    const int stride = static_cast<int>(gridDim.x) / p.cluster * tiles_at_once;
    const int first = static_cast<int>(blockIdx.x) / p.cluster * tiles_at_once;
    uint4* xs = reinterpret_cast<uint4*>(w4_smem);                     // [piece][word][row][t]
    float* sums = reinterpret_cast<float*>(w4_smem + w4_x_bytes(p.rows, p.steps));  // [group][row]
    float* red = sums + w4_sum_bytes(p.rows, p.steps, kGroup) / 4;     // [2][warp][column][kW4ColPitch]
    float* part = red + w4_red_bytes<MT>() / 4;                        // [2][tile][column][row]

    pdl_launch_dependents();
    cudaGridDependencySynchronize();

    // pieces of this warp, in order: row tile, then K
    struct Piece {
        uint32_t w[4][4];      // rows g, g + 8, g + 16, g + 24
        uint32_t sz[kGroups];  // of row g + 8 t: scale in the upper half, 128 + z in the lower
    };
    Piece piece[kW4Ahead];
    int ld_tile = first + tw, ld_step = kw;
    const int n_groups = p.K / kGroup;
    auto load = [&](Piece& pc) {
        if (ld_tile < tiles && ld_step < steps) {
            const int k_step = (step0 + ld_step) * kW4Step;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int n = min(ld_tile * kW4Tile + 8 * r + g, p.N - 1);
                const uint8_t* row = p.W + n * p.ldw + k_step / 2 + t * 4 * VEC;
#pragma unroll
                for (int q = 0; q < kGroups; ++q) {
                    const bool in = k_step + q * kGroup < p.K;
                    if constexpr (VEC == 4) {
                        uint4 v = make_uint4(0u, 0u, 0u, 0u);
                        if (in) v = *reinterpret_cast<const uint4*>(row);
                        pc.w[r][0] = v.x; pc.w[r][1] = v.y; pc.w[r][2] = v.z; pc.w[r][3] = v.w;
                    } else if constexpr (VEC == 2) {
                        uint2 v = make_uint2(0u, 0u);
                        if (in) v = *reinterpret_cast<const uint2*>(row + q * 32);
                        pc.w[r][2 * q] = v.x; pc.w[r][2 * q + 1] = v.y;
                    } else {
                        pc.w[r][q] = in ? *reinterpret_cast<const uint32_t*>(row + q * 16) : 0u;
                    }
                }
            }
            const int n = min(ld_tile * kW4Tile + 8 * t + g, p.N - 1);
#pragma unroll
            for (int q = 0; q < kGroups; ++q) {
                const int j = k_step / kGroup + q;
                uint32_t s = 0, z = 8;
                if (j < n_groups) {
                    s = *reinterpret_cast<const uint16_t*>(p.scales + n * p.lds + j);
                    if (p.zeros) z = p.zeros[n * p.ldz + j];
                }
                pc.sz[q] = (s << 16) | z;
            }
        }
        ld_step += k_warps;
        if (ld_step >= steps) {
            ld_step = kw;
            ld_tile += stride;
        }
    };
#pragma unroll
    for (int i = 0; i < kW4Ahead; ++i) load(piece[i]);

    // x, in fragment order: 8 consecutive k become (k, k + 4), (k + 1, k + 5), ...
    for (int i = threadIdx.x; i < rows * steps * (kW4Step / 8); i += kW4Threads) {
        const int per_row = steps * (kW4Step / 8);
        const int row = i / per_row, k8 = i % per_row, k = step0 * kW4Step + k8 * 8;
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (k < p.K) v = *reinterpret_cast<const uint4*>(p.X + (m0 + row) * p.ldx + k);
        const int in_step = k8 % 16, q = in_step / (4 * VEC), r = in_step % (4 * VEC);
        const int word = q * VEC + r % VEC, tt = r / VEC;
        xs[(((k8 / 16) * 4 + word) * rows + row) * 4 + tt] =
            make_uint4(__byte_perm(v.x, v.z, 0x5410), __byte_perm(v.x, v.z, 0x7632), __byte_perm(v.y, v.w, 0x5410), __byte_perm(v.y, v.w, 0x7632));
    }
    __syncthreads();
    for (int i = threadIdx.x; i < rows * steps * kGroups; i += kW4Threads) {
        const int row = i % rows, j = i / rows;  // group j of the CTA's K
        float s = 0.0f;
        for (int e = 0; e < 4 * VEC; ++e) {
            const int word = j / kGroups * 4 + j % kGroups * VEC + e % VEC;
            const uint4 v = xs[(word * rows + row) * 4 + e / VEC];
            float f[8];
            bf16x8_to_f32(v, f);
            s += ((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]));
        }
        sums[j * rows + row] = s;
    }
    __syncthreads();

    float acc[2][MT][4];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[h][m][e] = 0.0f;
    int my_row[MT], col0[MT], col1[MT];  // columns beyond the rows of x repeat the last one; their sums go nowhere
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        my_row[m] = min(m * 8 + g, rows - 1);
        col0[m] = min(m * 8 + 2 * t, rows - 1);
        col1[m] = min(m * 8 + 2 * t + 1, rows - 1);
    }

    auto compute = [&](const Piece& pc, int step) {
#pragma unroll
        for (int q = 0; q < kGroups; ++q) {
            float s[4], z[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const uint32_t v = __shfl_sync(0xffffffffu, pc.sz[q], (lane & 28) | r);
                s[r] = __uint_as_float(v & 0xFFFF0000u);
                z[r] = -__uint_as_float((v << 16) | 0x43000000u);  // -(128 + z)
            }
            float c[2][MT][4];
            const float* sum = sums + (step * kGroups + q) * rows;
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const float s0 = sum[col0[m]], s1 = sum[col1[m]];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    c[h][m][0] = z[2 * h] * s0;
                    c[h][m][1] = z[2 * h] * s1;
                    c[h][m][2] = z[2 * h + 1] * s0;
                    c[h][m][3] = z[2 * h + 1] * s1;
                }
            }
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                const int word = q * VEC + v;
                uint4 b[MT];
#pragma unroll
                for (int m = 0; m < MT; ++m) b[m] = xs[((step * 4 + word) * rows + my_row[m]) * 4 + t];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t lo[4], hi[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        lo[i] = ((pc.w[2 * h][word] >> (4 * i)) & 0x000F000Fu) | 0x43004300u;
                        hi[i] = ((pc.w[2 * h + 1][word] >> (4 * i)) & 0x000F000Fu) | 0x43004300u;
                    }
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        mma_bf16_16816(c[h][m], lo[0], hi[0], lo[1], hi[1], b[m].x, b[m].y);
                        mma_bf16_16816(c[h][m], lo[2], hi[2], lo[3], hi[3], b[m].z, b[m].w);
                    }
                }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    acc[h][m][0] = fmaf(s[2 * h], c[h][m][0], acc[h][m][0]);
                    acc[h][m][1] = fmaf(s[2 * h], c[h][m][1], acc[h][m][1]);
                    acc[h][m][2] = fmaf(s[2 * h + 1], c[h][m][2], acc[h][m][2]);
                    acc[h][m][3] = fmaf(s[2 * h + 1], c[h][m][3], acc[h][m][3]);
                }
        }
    };

    // The warps' sums of one set of tiles meet in one of two buffers, which alternate: a buffer is written again only after a
    // barrier that every reader of it has passed.  With a cluster the CTAs' sums do the same.
    auto finish_tiles = [&](int tile, int round) {
        float* buf = red + (round & 1) * (kW4Warps * MT * 8 * kW4ColPitch);
        float* mine = buf + warp * (MT * 8 * kW4ColPitch);
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    mine[(m * 8 + 2 * t + (e & 1)) * kW4ColPitch + h * 16 + (e >> 1) * 8 + g] = acc[h][m][e];
                    acc[h][m][e] = 0.0f;
                }
        __syncthreads();
        const int outputs = tiles_at_once * rows * kW4Tile;  // (tile, row of x, weight row)
        float* dst = part + (round & 1) * outputs;
        for (int i = threadIdx.x; i < outputs; i += kW4Threads) {
            const int n_in = i % kW4Tile, m = i / kW4Tile % rows, tl = i / (kW4Tile * rows);
            const float* src = buf + tl * k_warps * (MT * 8 * kW4ColPitch) + m * kW4ColPitch + n_in;
            float sum = 0.0f;
            for (int w = 0; w < k_warps; ++w) sum += src[w * (MT * 8 * kW4ColPitch)];
            const int n = (tile + tl) * kW4Tile + n_in;
            if (p.cluster > 1) dst[i] = sum;
            else if (n < p.N) p.C[(m0 + m) * p.ldc + n] = __float2bfloat16(sum);
        }
        if (p.cluster > 1) {
            cluster_sync_all();
            const int lo = outputs * rank / p.cluster, hi = outputs * (rank + 1) / p.cluster;
            for (int i = lo + threadIdx.x; i < hi; i += kW4Threads) {
                const int n_in = i % kW4Tile, m = i / kW4Tile % rows, tl = i / (kW4Tile * rows);
                float sum = 0.0f;
                for (int c = 0; c < p.cluster; ++c) {
                    float v;
                    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(map_to_cta(smem_u32(dst + i), static_cast<uint32_t>(c))));
                    sum += v;
                }
                const int n = (tile + tl) * kW4Tile + n_in;
                if (n < p.N) p.C[(m0 + m) * p.ldc + n] = __float2bfloat16(sum);
            }
        }
    };

    int tile = first, step = kw, round = 0;
    while (tile < tiles) {
#pragma unroll
        for (int u = 0; u < kW4Ahead; ++u) {
            if (tile < tiles) {
                if (tile + tw < tiles && step < steps) compute(piece[u], step);
                load(piece[u]);
                step += k_warps;
                if (step >= steps) {
                    finish_tiles(tile, round++);
                    step = kw;
                    tile += stride;
                }
            }
        }
    }
    if (p.cluster > 1) cluster_sync_all();  // nobody leaves while its sums are being read
}

template <int MT, int VEC>
int w4_launch_one(const W4Params& p, int grid, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(grid), static_cast<unsigned>((p.M + p.rows - 1) / p.rows));
    cfg.blockDim = dim3(kW4Threads);
    cfg.dynamicSmemBytes = static_cast<size_t>(w4_x_bytes(p.rows, p.steps)) + w4_sum_bytes(p.rows, p.steps, 32 * VEC) + w4_red_bytes<MT>() +
                           w4_part_bytes(p.rows, p.k_warps, p.cluster);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = static_cast<unsigned>(p.cluster);
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = p.cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, gemm_w4_kernel<MT, VEC>, p) == cudaSuccess ? 0 : 4;
}

template <int MT>
int w4_launch(const W4Params& p, int group, int grid, cudaStream_t st) {
    switch (group) {
        case 32: return w4_launch_one<MT, 1>(p, grid, st);
        case 64: return w4_launch_one<MT, 2>(p, grid, st);
        default: return w4_launch_one<MT, 4>(p, grid, st);
    }
}

template <int MT, int VEC>
bool w4_configure_one() {
    return cudaFuncSetAttribute(gemm_w4_kernel<MT, VEC>, cudaFuncAttributeMaxDynamicSharedMemorySize, kW4Smem) == cudaSuccess;
}
inline bool w4_configure() {
    return w4_configure_one<1, 1>() && w4_configure_one<1, 2>() && w4_configure_one<1, 4>() && w4_configure_one<2, 1>() && w4_configure_one<2, 2>() &&
           w4_configure_one<2, 4>();
}

// Rows per pass, CTAs per cluster and warps along K; false if not even one row of x fits a cluster of 8.
// cluster_slots: resident CTAs in clusters of 2, 4, 8.
inline bool w4_plan(W4Params* p, int group, int sm_count, const int* cluster_slots, int* grid) {
    const int all_steps = (p->K + kW4Step - 1) / kW4Step, tiles = (p->N + kW4Tile - 1) / kW4Tile;
    auto steps_of = [&](int c) { return (all_steps + c - 1) / c; };
    auto warps_of = [&](int c) {
        int kw = 1;
        while (kw < kW4Warps && 2 * kw <= steps_of(c)) kw *= 2;
        return kw;
    };
    auto fits = [&](int rows, int c) {
        const int64_t bytes = static_cast<int64_t>(rows) * steps_of(c) * kW4Step * 2 + static_cast<int64_t>(rows) * steps_of(c) * (kW4Step / group) * 4 + 16 +
                              (rows > 8 ? w4_red_bytes<2>() : w4_red_bytes<1>()) + w4_part_bytes(rows, warps_of(c), c);
        return bytes <= kW4Smem;
    };
    auto slots = [&](int c) { return c == 1 ? sm_count : cluster_slots[c == 2 ? 0 : c == 4 ? 1 : 2]; };
    int rows = std::min(p->M, 16), c = 1;
    for (; rows > 0; rows = rows > 8 ? 8 : rows - 1) {
        for (c = 1; c <= 8 && !(fits(rows, c) && slots(c) >= c); c *= 2) {}
        if (c <= 8) break;
    }
    if (rows <= 0) return false;
    // fewer tiles than half the SMs: cut K further, while a warp of the CTAs keeps a piece
    while (c < 8 && slots(2 * c) >= 2 * c && static_cast<int64_t>(tiles) * 2 * c <= sm_count && all_steps >= 2 * c * 4) c *= 2;
    p->rows = rows;
    p->cluster = c;
    p->steps = steps_of(c);
    p->k_warps = warps_of(c);
    const int at_once = kW4Warps / p->k_warps;
    *grid = c * std::max(1, std::min(slots(c) / c, (tiles + at_once - 1) / at_once));
    return true;
}

}  // namespace mlt
