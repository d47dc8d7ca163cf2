// Scaled 8-bit GEMM: C[i][j] = sum over K blocks b of 128: sa[b][i] * sb[j / 128][b] * (sum over k in b: A[i][k] B[j][k]),
// A [M, K] and B [N, K] E4M3 with K contiguous, scales FP32 (any value), FP32 sums, one rounding to BF16.
//
// The scales change along K, so the tensor core may only accumulate 128 products (four tcgen05.mma of K = 32) before
// the partial sums have to be weighted: every K block goes into a fresh accumulator in tensor memory, and the
// promotion warps read it (tcgen05.ld), multiply by sa * sb and add it to FP32 registers while the tensor core fills the
// other accumulator.  A thread owns one row and its columns, so a K block needs one multiplication of scales per thread
// and one FMA per element.
//
//   warp 0      TMA producer: 128 bytes of K per stage for the tile's rows of A and of B (128-byte swizzle)
//   warp 1      UMMA issuer, owner of the tensor-memory allocation
//   warps 2..   promotion and epilogue
// gemm_f8_big_kernel (256 columns per tile, persistent) for problems with enough tiles, gemm_f8_kernel otherwise.
#pragma once

#include "f8.cuh"
#include "gemm.cuh"

namespace mlt {

constexpr int kF8BK = 128;  // elements (= bytes) of K per stage, and per scale

struct GemmF8Params {
    __nv_bfloat16* C;
    const float *sa, *sb;
    int64_t ldc, ldsa, ldsb;
    int M, N, K;
    int tiles_m, tiles_n, group_m;
    int kb_per_split;  // K blocks per CTA of a cluster
    int a_rows;        // rows of A per stage (a multiple of 8; fewer than 128 when M is smaller)
    int stages;
};

// ---------------------------------------------------------------------------------------------------------
// 128 x BN tiles, K cut over the S CTAs of a cluster (S = 1: none), one tile per cluster.  The CTAs' FP32 tiles are
// summed through distributed shared memory in ascending slice order (deterministic).
// ---------------------------------------------------------------------------------------------------------
constexpr int kF8MaxStages = 16;
constexpr int kF8Threads = 192;
template <int BN>
struct GemmF8Smem {
    static constexpr int kBBytes = BN * kF8BK;
    static constexpr int kBarrierBytes = 512;
    static constexpr int kPartPitch = BN + 4;  // FP32 words per row of the tile summed over the cluster
    // A stages | B stages | barriers; the A descriptor always spans 128 rows, of which the first a_rows are loaded: the
    // span may run on into whatever follows (rows that are never stored), so at least 16 KB follow the last A stage.
    static constexpr int bytes(int a_rows, int stages) { return stages * (a_rows * kF8BK + kBBytes) + kBarrierBytes + 1024; }
};

constexpr int kGemmF8NarrowSmem = 75 * 1024;  // per CTA of the 64-wide kernel (three on an SM)
constexpr int kGemmF8WideSmem = 200 * 1024;   // per CTA of the 128-wide kernel (one on an SM)

// A load that stays where it is written (a prefetch that the compiler would move down to its use); 0 where `there` is false.
__device__ __forceinline__ float ld_f32_if(const float* p, bool there) {
    float v;
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %2, 0;\n\tmov.f32 %0, 0f00000000;\n\t@q ld.global.nc.f32 %0, [%1];\n\t}"
                 : "=f"(v)
                 : "l"(p), "r"(static_cast<int>(there)));
    return v;
}

// One row's 32 consecutive results to BF16 C; a ragged right edge is stored element by element.
__device__ __forceinline__ void gemm_f8_store32(__nv_bfloat16* crow, int col0, int N, const float* v) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int col = col0 + q * 8;
        if (col + 8 <= N) {
            *reinterpret_cast<uint4*>(crow + col) = make_uint4(pack_bf16x2(v[q * 8], v[q * 8 + 1]), pack_bf16x2(v[q * 8 + 2], v[q * 8 + 3]),
                                                               pack_bf16x2(v[q * 8 + 4], v[q * 8 + 5]), pack_bf16x2(v[q * 8 + 6], v[q * 8 + 7]));
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (col + j < N) crow[col + j] = __float2bfloat16(v[q * 8 + j]);
        }
    }
}

// acc += s * (kCols accumulator columns of tensor memory), 16 columns at a time: the next 16 are on their way while these
// are added, two columns per instruction.  `drained` runs when the last ones are in registers.
template <int kCols, class F>
__device__ __forceinline__ void gemm_f8_promote(float2 (&acc)[kCols / 2], uint32_t taddr, float s, F drained) {
    const float2 s2 = make_float2(s, s);
    uint32_t v[2][16];
    tmem_ld_32x32b_x16(taddr, v[0]);
#pragma unroll
    for (int c = 0; c < kCols / 16; ++c) {
        tmem_wait_ld_of(v[c & 1]);
        if (c + 1 < kCols / 16)
            tmem_ld_32x32b_x16(taddr + (c + 1) * 16, v[(c + 1) & 1]);
        else
            drained();
#pragma unroll
        for (int i = 0; i < 8; ++i)
            acc[c * 8 + i] = ffma2(s2, make_float2(__uint_as_float(v[c & 1][2 * i]), __uint_as_float(v[c & 1][2 * i + 1])), acc[c * 8 + i]);
    }
}

template <int BN, int kCtasPerSm>
__global__ void __launch_bounds__(kF8Threads, kCtasPerSm)
gemm_f8_kernel(const __grid_constant__ CUtensorMap tmap_a, const __grid_constant__ CUtensorMap tmap_b, const GemmF8Params p) {
    using L = GemmF8Smem<BN>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const int a_bytes = p.a_rows * kF8BK;
    uint8_t* smem_b = smem + p.stages * a_bytes;
    uint64_t* full = reinterpret_cast<uint64_t*>(smem_b + p.stages * L::kBBytes);
    uint64_t* empty = full + kF8MaxStages;
    uint64_t* acc_full = empty + kF8MaxStages;  // [2]
    uint64_t* acc_empty = acc_full + 2;         // [2]
    uint32_t* tmem_base_slot = reinterpret_cast<uint32_t*>(acc_empty + 2);
    volatile uint32_t* abort_flag = tmem_base_slot + 1;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int S = static_cast<int>(cluster_nctarank());
    const int slice = static_cast<int>(cluster_ctarank());
    const int tile = static_cast<int>(blockIdx.x) / S;
    const int num_kb = (p.K + kF8BK - 1) / kF8BK;
    const int kb0 = slice * p.kb_per_split, kb1 = min(num_kb, kb0 + p.kb_per_split);  // no slice is empty (host)
    const int per_group = p.group_m * p.tiles_n;  // raster groups of group_m tile rows, rows fastest (L2 reuse)
    const int first_m = tile / per_group * p.group_m;
    const int rows_in_group = min(p.group_m, p.tiles_m - first_m);
    const int m0 = (first_m + tile % per_group % rows_in_group) * 128, n0 = tile % per_group / rows_in_group * BN;
    const int active = min(4, (p.M - m0 + 31) / 32);  // promotion warps whose rows exist
    constexpr uint32_t kTmemCols = 2 * BN;

    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(&acc_full[a], 1);
            mbar_init(&acc_empty[a], active);
        }
        *abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == 0 && lane == 0) {
        prefetch_tensormap(&tmap_a);
        prefetch_tensormap(&tmap_b);
    }
    if (warp == 1) {
        tmem_alloc(tmem_base_slot, kTmemCols);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_base_slot;
    const int quarter = warp & 3;  // tensor-memory lanes this warp may touch: 32 * quarter .. + 31
    const int r = quarter * 32 + lane;
    float2 acc[BN / 2];
#pragma unroll
    for (int i = 0; i < BN / 2; ++i) acc[i] = make_float2(0.0f, 0.0f);

    if (warp == 0) {
        if (lane == 0) {
            int stage = 0;
            uint32_t phase = 0;
            for (int kb = kb0; kb < kb1; ++kb) {
                if (!mbar_wait(&empty[stage], phase ^ 1, abort_flag, 0x100 + stage)) break;
                mbar_arrive_expect_tx(&full[stage], a_bytes + L::kBBytes);
                tma_load_2d(smem + stage * a_bytes, &tmap_a, &full[stage], kb * kF8BK, m0);
                tma_load_2d(smem_b + stage * L::kBBytes, &tmap_b, &full[stage], kb * kF8BK, n0);
                if (++stage == p.stages) { stage = 0; phase ^= 1; }
            }
        }
    } else if (warp == 1) {
        const bool leader = elect_one();
        constexpr uint32_t idesc = make_idesc_e4m3(128, BN);
        const uint32_t a_lo0 = sdesc_lo(smem_u32(smem), 16), b_lo0 = sdesc_lo(smem_u32(smem_b), 16);
        int stage = 0;
        uint32_t phase = 0;
        for (int kb = kb0; kb < kb1; ++kb) {
            const int buf = (kb - kb0) & 1;
            const uint32_t use = (kb - kb0) >> 1;  // uses of this accumulator before
            bool ok = mbar_wait(&acc_empty[buf], (use & 1) ^ 1, abort_flag, 0x300 + buf);
            ok = ok && mbar_wait(&full[stage], phase, abort_flag, 0x200 + stage);
            if (!__all_sync(0xffffffffu, ok)) break;
            tc_fence_after();
            if (leader) {
                const uint32_t a_lo = a_lo0 + stage * (a_bytes >> 4), b_lo = b_lo0 + stage * (L::kBBytes >> 4);
#pragma unroll
                for (int k = 0; k < kF8BK / 32; ++k)
                    umma_f8_ss_lo(tmem_base + buf * BN, a_lo + k * (32 >> 4), b_lo + k * (32 >> 4), idesc, k != 0);
                umma_commit(&empty[stage]);
                umma_commit(&acc_full[buf]);
            }
            __syncwarp();
            if (++stage == p.stages) { stage = 0; phase ^= 1; }
        }
    } else if (quarter < active) {
        const bool live = m0 + r < p.M;
        const float* sa = p.sa + m0 + r;
        const float* sb = p.sb + static_cast<int64_t>(n0 / 128) * p.ldsb;
        const uint32_t t_row = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16);
        float s_next = live ? __ldg(sa + kb0 * p.ldsa) * __ldg(sb + kb0) : 0.0f;
        for (int kb = kb0; kb < kb1; ++kb) {
            const int buf = (kb - kb0) & 1;
            const float s = s_next;
            if (live && kb + 1 < kb1) s_next = __ldg(sa + (kb + 1) * p.ldsa) * __ldg(sb + kb + 1);
            if (!__all_sync(0xffffffffu, mbar_wait(&acc_full[buf], ((kb - kb0) >> 1) & 1, abort_flag, 0x400 + buf))) break;
            tc_fence_after();
gemm_f8_promote<BN>(acc, t_row + buf * BN, s, [&] {  // the accumulator is in registers: the tensor core may refill it
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&acc_empty[buf]);
            });
        }
    }

    if (S == 1) {
        if (warp >= 2 && m0 + r < p.M) {
            __nv_bfloat16* crow = p.C + static_cast<int64_t>(m0 + r) * p.ldc;
#pragma unroll
            for (int c = 0; c < BN / 32; ++c) gemm_f8_store32(crow, n0 + c * 32, p.N, reinterpret_cast<const float*>(acc + c * 16));
        }
        tc_fence_before();
        __syncthreads();
    } else {
        // every UMMA of this CTA has read its operands once the last accumulator is full, which the promotion warps have
        // waited for; the producer issued no load beyond them: the stages are free
        float* part = reinterpret_cast<float*>(smem);
        __syncthreads();
        if (warp >= 2 && m0 + r < p.M) {
            float4* dst = reinterpret_cast<float4*>(part + r * L::kPartPitch);
#pragma unroll
            for (int q = 0; q < BN / 4; ++q) dst[q] = make_float4(acc[2 * q].x, acc[2 * q].y, acc[2 * q + 1].x, acc[2 * q + 1].y);
        }
        tc_fence_before();
        cluster_sync_all();
        const int groups = BN / S / 4;  // this CTA's share of the columns, four at a time
        const int rows = min(128, p.M - m0);
        const uint32_t part_addr = smem_u32(part);
        for (int idx = threadIdx.x; idx < rows * groups; idx += kF8Threads) {
            const int row = idx / groups, c = slice * (BN / S) + (idx % groups) * 4;
            float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            for (int s2 = 0; s2 < S; ++s2) {
                const float4 v = ld_shared_cluster_f32x4(map_to_cta(part_addr + (row * L::kPartPitch + c) * 4, s2));
                sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
            }
            const int col = n0 + c;
            __nv_bfloat16* dst = p.C + static_cast<int64_t>(m0 + row) * p.ldc + col;
            if (col + 4 <= p.N) {
                *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(sum.x, sum.y), pack_bf16x2(sum.z, sum.w));
            } else {
                const float a[4] = {sum.x, sum.y, sum.z, sum.w};
                for (int j = 0; j < 4 && col + j < p.N; ++j) dst[j] = __float2bfloat16(a[j]);
            }
        }
        cluster_sync_all();  // no CTA leaves while a peer may still read its shared memory
    }
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc(tmem_base, kTmemCols);
    }
}

// ---------------------------------------------------------------------------------------------------------
// Large problems: persistent, 256 columns per tile, eight promotion warps (a thread owns one row and 128 columns in
// registers).
//   kPair  a cluster of two CTAs owns a 256 x 256 tile (cta_group::2, each CTA loads its 128 rows of A and 128 rows of B;
//          the barriers as in gemm_bf16_pair_kernel)
//   else   one CTA owns a 128 x 256 tile
// The two accumulators in tensor memory (2 x 256 columns) belong to alternate K blocks, across tile borders: while the
// promotion warps round and store a tile, the tensor core is up to two K blocks into the next one.  Results leave through
// 4 KB of shared memory per warp (32 rows x 64 columns, 128-byte swizzle) and TMA stores.
// ---------------------------------------------------------------------------------------------------------
constexpr int kF8BigThreads = 320;  // 2 + 8 warps; 200 registers per thread
template <bool kPair>
struct GemmF8BigSmem {
    static constexpr int kABytes = 128 * kF8BK;
    static constexpr int kBBytes = (kPair ? 128 : 256) * kF8BK;
    static constexpr int kStageBytes = kABytes + kBBytes;
    static constexpr int kStages = kPair ? 6 : 4;
    static constexpr int kTotal = kStages * kStageBytes + 8 * 4096 + 256 + 1024;
};

template <bool kPair>
__global__ void __launch_bounds__(kF8BigThreads, 1)
gemm_f8_big_kernel(const __grid_constant__ CUtensorMap tmap_a, const __grid_constant__ CUtensorMap tmap_b,
                   const __grid_constant__ CUtensorMap tmap_c, const GemmF8Params p) {
    using L = GemmF8BigSmem<kPair>;
    constexpr int kStages = L::kStages;
    constexpr int kTileM = kPair ? 256 : 128;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* staging = smem + kStages * L::kStageBytes;
    uint64_t* full = reinterpret_cast<uint64_t*>(staging + 8 * 4096);
    uint64_t* empty = full + kStages;
    uint64_t* acc_full = empty + kStages;  // [2]
    uint64_t* acc_empty = acc_full + 2;    // [2]
    uint32_t* tmem_base_slot = reinterpret_cast<uint32_t*>(acc_empty + 2);
    volatile uint32_t* abort_flag = tmem_base_slot + 1;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (blockIdx.x == 0 && threadIdx.x == 0) clock_probe(0, 0);
    const int rank = kPair ? static_cast<int>(cluster_ctarank()) : 0;
    const int first = kPair ? blockIdx.x >> 1 : blockIdx.x, step = kPair ? gridDim.x >> 1 : gridDim.x;
    const int num_kb = (p.K + kF8BK - 1) / kF8BK;
    const int tiles = p.tiles_m * p.tiles_n;
    auto coords = [&](int tile, int& m0, int& n0) {  // raster groups of group_m tile rows, rows fastest (L2 reuse)
        const int per_group = p.group_m * p.tiles_n;
        const int first_m = tile / per_group * p.group_m;
        const int rows = min(p.group_m, p.tiles_m - first_m), r = tile % per_group;
        m0 = (first_m + r % rows) * kTileM + rank * 128;
        n0 = r / rows * 256;
    };

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(&acc_full[a], 1);
            mbar_init(&acc_empty[a], kPair ? 16 : 8);  // every promotion warp
        }
        *abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == 0 && lane == 0) {
        prefetch_tensormap(&tmap_a);
        prefetch_tensormap(&tmap_b);
        prefetch_tensormap(&tmap_c);
    }
    if (warp == 1) {
        if constexpr (kPair) {
            tmem_alloc_pair(tmem_base_slot, 512);
            tmem_relinquish_pair();
        } else {
            tmem_alloc(tmem_base_slot, 512);
            tmem_relinquish();
        }
    }
    tc_fence_before();
    if constexpr (kPair) cluster_sync_all(); else __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_base_slot;

    if (warp == 0) {
        if (lane == 0) {
            int stage = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int tile = first; tile < tiles && ok; tile += step) {
                int m0, n0;
                coords(tile, m0, n0);
                for (int kb = 0; kb < num_kb; ++kb) {
                    ok = mbar_wait(&empty[stage], phase ^ 1, abort_flag, 0x100 + stage);
                    if (!ok) break;
                    uint8_t* sa = smem + stage * L::kStageBytes;
                    uint8_t* sb = sa + L::kABytes;
                    if constexpr (kPair) {
                        if (rank == 0) mbar_arrive_expect_tx(&full[stage], 2 * L::kStageBytes);
                        const uint32_t bar = map_to_cta(smem_u32(&full[stage]), 0);
                        tma_load_2d_pair(sa, &tmap_a, bar, kb * kF8BK, m0);
                        tma_load_2d_pair(sb, &tmap_b, bar, kb * kF8BK, n0 + rank * 128);
                    } else {
                        mbar_arrive_expect_tx(&full[stage], L::kStageBytes);
                        tma_load_2d(sa, &tmap_a, &full[stage], kb * kF8BK, m0);
                        tma_load_2d(sb, &tmap_b, &full[stage], kb * kF8BK, n0);
                        tma_load_2d(sb + 128 * kF8BK, &tmap_b, &full[stage], kb * kF8BK, n0 + 128);
                    }
                    if (++stage == kStages) { stage = 0; phase ^= 1; }
                }
            }
        }
    } else if (warp == 1) {
        if (rank == 0) {
            const bool issuer = elect_one();
            constexpr uint32_t idesc = make_idesc_e4m3(kTileM, 256);
            const uint32_t a_lo0 = sdesc_lo(smem_u32(smem), 16), b_lo0 = sdesc_lo(smem_u32(smem + L::kABytes), 16);
            int stage = 0;
            uint32_t phase = 0, use = 0;  // use: K blocks so far
            bool ok = true;
            for (int tile = first; tile < tiles && ok; tile += step) {
                for (int kb = 0; kb < num_kb; ++kb, ++use) {
                    const int buf = use & 1;
                    ok = mbar_wait(&full[stage], phase, abort_flag, 0x200 + stage);
                    ok = ok && mbar_wait(&acc_empty[buf], ((use >> 1) & 1) ^ 1, abort_flag, 0x300 + buf);
                    ok = __all_sync(0xffffffffu, ok) != 0;
                    if (!ok) break;
                    tc_fence_after();
                    if (issuer) {
                        const uint32_t a_lo = a_lo0 + stage * (L::kStageBytes >> 4), b_lo = b_lo0 + stage * (L::kStageBytes >> 4);
#pragma unroll
                        for (int k = 0; k < kF8BK / 32; ++k) {
                            if constexpr (kPair)
                                umma_f8_ss_pair_lo(tmem_base + buf * 256, a_lo + k * (32 >> 4), b_lo + k * (32 >> 4), idesc, k != 0);
                            else
                                umma_f8_ss_lo(tmem_base + buf * 256, a_lo + k * (32 >> 4), b_lo + k * (32 >> 4), idesc, k != 0);
                        }
                        if constexpr (kPair) {
                            umma_commit_pair(&empty[stage], 3);
                            umma_commit_pair(&acc_full[buf], 3);
                        } else {
                            umma_commit(&empty[stage]);
                            umma_commit(&acc_full[buf]);
                        }
                    }
                    __syncwarp();
                    if (++stage == kStages) { stage = 0; phase ^= 1; }
                }
            }
        }
    } else {
        const int quarter = warp & 3, half = (warp - 2) >> 2;  // 32 rows, 128 columns
        uint8_t* stg = staging + (warp - 2) * 4096;
        const uint32_t t_row = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16) + half * 128;
        uint32_t use = 0;
        bool ok = true;
        for (int tile = first; tile < tiles && ok; tile += step) {
            int m0, n0;
            coords(tile, m0, n0);
            const int row0 = m0 + quarter * 32, col0 = n0 + half * 128;
            const bool live = row0 + lane < p.M && col0 < p.N;
            const float* sa = p.sa + row0 + lane;
            const float* sb = p.sb + static_cast<int64_t>(col0 / 128) * p.ldsb;
            float2 acc[64];
#pragma unroll
            for (int i = 0; i < 64; ++i) acc[i] = make_float2(0.0f, 0.0f);
            // the scales of two K blocks at a time, requested two K blocks ahead
            float s[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) s[u] = ld_f32_if(sa + u * p.ldsa, live && u < num_kb) * ld_f32_if(sb + u, live && u < num_kb);
            for (int kb2 = 0; kb2 < num_kb && ok; kb2 += 2) {
                float xa[2], xb[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const bool there = live && kb2 + 2 + u < num_kb;
                    xa[u] = ld_f32_if(sa + (kb2 + 2 + u) * p.ldsa, there);
                    xb[u] = ld_f32_if(sb + kb2 + 2 + u, there);
                }
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    if (kb2 + u < num_kb && ok) {
                        const int buf = use & 1;
                        ok = __all_sync(0xffffffffu, mbar_wait(&acc_full[buf], (use >> 1) & 1, abort_flag, 0x400 + buf)) != 0;
                        if (ok) {
                            tc_fence_after();
                            gemm_f8_promote<128>(acc, t_row + buf * 256, s[u], [&] {
                                tc_fence_before();
                                __syncwarp();
                                if (lane == 0) {
                                    if constexpr (kPair)
                                        mbar_arrive_peer(map_to_cta(smem_u32(&acc_empty[buf]), 0));
                                    else
                                        mbar_arrive(&acc_empty[buf]);
                                }
                            });
                            ++use;
                        }
                    }
                }
#pragma unroll
                for (int u = 0; u < 2; ++u) s[u] = xa[u] * xb[u];
            }
            if (!ok) break;
            // ---- round and store: 64 columns at a time ----
            const int n8 = p.N & ~7;  // the tensor map of C ends here (16-byte units)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (lane == 0) tma_store_wait_read<0>();
                __syncwarp();
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const float2* a = acc + h * 32 + q * 4;
                    *reinterpret_cast<uint4*>(stg + lane * 128 + ((q ^ (lane & 7)) << 4)) =
                        make_uint4(pack_bf16x2(a[0].x, a[0].y), pack_bf16x2(a[1].x, a[1].y), pack_bf16x2(a[2].x, a[2].y), pack_bf16x2(a[3].x, a[3].y));
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    if (row0 < p.M && col0 + h * 64 < n8) tma_store_2d(&tmap_c, stg, col0 + h * 64, row0);
                    tma_store_commit();
                }
                if (n8 != p.N && col0 + h * 64 <= n8 && n8 < col0 + h * 64 + 64 && row0 + lane < p.M) {  // the up to seven columns beyond
                    __nv_bfloat16* crow = p.C + static_cast<int64_t>(row0 + lane) * p.ldc;
#pragma unroll
                    for (int j = 0; j < 32; ++j) {
                        const int col = col0 + h * 64 + 2 * j;
                        if (col >= n8 && col < p.N) crow[col] = __float2bfloat16(acc[h * 32 + j].x);
                        if (col >= n8 && col + 1 < p.N) crow[col + 1] = __float2bfloat16(acc[h * 32 + j].y);
                    }
                }
            }
        }
        if (lane == 0) tma_store_wait_all<0>();  // shared memory must outlive the stores that read it
    }

    // common exit: no CTA of a pair leaves while its peer may still touch its memory
    tc_fence_before();
    if constexpr (kPair) cluster_sync_all(); else __syncthreads();
    if (blockIdx.x == 0 && threadIdx.x == 0) clock_probe(0, 1);
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        if constexpr (kPair) tmem_dealloc_pair(tmem_base, 512); else tmem_dealloc(tmem_base, 512);
    }
}

}  // namespace mlt
