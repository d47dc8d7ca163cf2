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
//   warps 4-11  promotion and epilogue
// gemm_f8_big_kernel (256 columns per tile, persistent) for problems with enough tiles, gemm_f8_split_kernel otherwise.
#pragma once

#include <algorithm>
#include <type_traits>

#include "f8.cuh"
#include "gemm.cuh"

namespace mlt {

constexpr int kF8BK = 128;  // elements (= bytes) of K per stage, and per scale
// Twelve warps: producer, issuer, two that only hand their registers over, eight promotion warps (warps 4 .. 11).  The 128
// sums and the 32 words on their way do not fit the 168 registers a thread starts with, and a spilled word costs an L2 access
// (shared memory leaves no L1): with setmaxnreg the promotion warps take 208 and the others 88 of the launch's registers.
constexpr int kF8Threads = 384;
constexpr int kF8PromoteRegs = 208, kF8OtherRegs = 88, kF8LaunchRegs = 168;
static_assert(8 * kF8PromoteRegs + 4 * kF8OtherRegs <= 12 * kF8LaunchRegs, "setmaxnreg budget exceeds the launch allocation");

struct GemmF8Params {
    __nv_bfloat16* C;
    const float *sa, *sb;
    int64_t ldc, ldsa, ldsb;
    int M, N, K;
    int tiles_m, tiles_n, group_m;
    // gemm_f8_split_kernel
    int bn, bufs;  // tile width (a multiple of 16), accumulators in tensor memory (2 .. 4, bufs * bn <= 512)
    int a_rows;    // rows of A per stage (a multiple of 8; fewer than 128 when M is smaller)
    int stages;
};

// Scales travel through a ring in shared memory, four K blocks to a slot, filled by a warp of its own with 4-byte asynchronous
// copies.  (Not by the producer: an arrival waits for the copies its thread has in flight.)
constexpr int kF8MaxStages = 16;
constexpr int kF8ScaleSlots = 4;
struct GemmF8Scales {
    float row[4][128];
    float col[4][4];
};
__device__ __forceinline__ void cp_async_f32(float* smem_dst, const float* src, bool there) {  // 0 where `there` is false
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_u32(smem_dst)), "l"(src), "r"(there ? 4 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_arrive(uint64_t* bar) {  // arrives once this thread's copies so far have landed
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// The scale warp's part for one tile: K blocks kb0 .. kb1 - 1, `sa` at the tile's first row, sb: this lane's column scale
// (lanes 0 .. 3).  `slot` and `phase` run on from tile to tile.
__device__ __forceinline__ bool gemm_f8_load_scales(GemmF8Scales* ring, uint64_t* full, uint64_t* empty, int& slot, uint32_t& phase,
                                                    const float* sa, int64_t ldsa, int rows, const float* sb, int kb0, int kb1, int lane,
                                                    volatile uint32_t* abort_flag) {
    for (int kb = kb0; kb < kb1; kb += 4) {
        if (!__all_sync(0xffffffffu, mbar_wait(&empty[slot], phase ^ 1, abort_flag, 0x600 + slot))) return false;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (kb + u < kb1) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (i * 32 < rows) cp_async_f32(&ring[slot].row[u][i * 32 + lane], sa + (kb + u) * ldsa + i * 32 + lane, i * 32 + lane < rows);
                if (lane < 4) cp_async_f32(&ring[slot].col[u][lane], sb + kb + u, true);
            }
        }
        cp_async_arrive(&full[slot]);
        if (++slot == kF8ScaleSlots) { slot = 0; phase ^= 1; }
    }
    return true;
}

// acc += scale * (16 * kChunks accumulator columns of tensor memory), 16 columns at a time: the next 16 are on their way while
// these are added, two columns per instruction.  The scale is s0 before chunk `cut` and s1 from it on.  `drained` runs when the
// last columns are in registers.
template <int kChunks, class F>
__device__ __forceinline__ void gemm_f8_promote(float2 (&acc)[kChunks * 8], uint32_t taddr, float s0, float s1, int cut, F drained) {
    uint32_t v[2][16];
    tmem_ld_32x32b_x16(taddr, v[0]);
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        tmem_wait_ld_of(v[c & 1]);
        if (c + 1 < kChunks)
            tmem_ld_32x32b_x16(taddr + (c + 1) * 16, v[(c + 1) & 1]);
        else
            drained();
        const float s = c < cut ? s0 : s1;
        const float2 s2 = make_float2(s, s);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            acc[c * 8 + i] = ffma2(s2, make_float2(__uint_as_float(v[c & 1][2 * i]), __uint_as_float(v[c & 1][2 * i + 1])), acc[c * 8 + i]);
    }
}

// ---------------------------------------------------------------------------------------------------------
// Problems with few tiles (next-token shapes above all): one 128 x bn tile per cluster, bn any multiple of 16 up to 256, K
// cut over the S CTAs of the cluster.  Such a problem is bound by how evenly the stream of B is spread over the SMs, so the
// host picks bn and S together such that tiles x S comes close to the SM count from below.  The CTAs' FP32 tiles meet in
// distributed shared memory (the stages are free by then) and are summed in ascending slice order (deterministic).
// Bound by HBM with many columns and short K; with few columns and long K by the promotion, of which a cluster's CTA does one K
// block after the other (with 16 rows in two of the eight warps only).  Measured, device time in a captured graph (one call among other
// passes takes about 3 us more): 16 x 28672 x 4096 in 25 us (4.7 TB/s; 18 us at the copy's rate, 3.5 until the first data, 3 from the last
// product to the last store), 16 x 4096 x 28672 in 28 us (56 K blocks at about 440 ns by the launch plan's model, 24.5 us),
// 512 x 4096 x 4096 in 18 us.  Without setmaxnreg 45, with a branch per 16 columns instead of the switch 33, without the scale warp 28.
// (ptxas reports 32 bytes of spill stores and 260 of spill loads for the kernel as it is, 88 of stores for the one that took 45.)
// ---------------------------------------------------------------------------------------------------------
constexpr int kF8SplitSmem = 208 * 1024;
// A stages | B stages.  The A descriptor always spans 128 rows, of which the first a_rows are loaded: the span may
// run on into whatever follows (rows that are never stored), so at least 16 KB follow the A stages.  The FP32 tile of up to
// a_rows rows takes the stages' place at the end.
inline int gemm_f8_split_smem(int bn, int a_rows, int stages) {
    return std::max({stages * (a_rows + bn) * kF8BK, stages * a_rows * kF8BK + 16384, a_rows * (bn + 4) * 4}) + 1024;
}

__global__ void __launch_bounds__(kF8Threads, 1)
gemm_f8_split_kernel(const __grid_constant__ CUtensorMap tmap_a, const __grid_constant__ CUtensorMap tmap_b, const GemmF8Params p) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ uint64_t full[kF8MaxStages], empty[kF8MaxStages], acc_full[4], acc_empty[4], scale_full[kF8ScaleSlots], scale_empty[kF8ScaleSlots];
    __shared__ GemmF8Scales scales[kF8ScaleSlots];
    __shared__ uint32_t tmem_base_slot, abort_word;
    volatile uint32_t* abort_flag = &abort_word;
    const int bn = p.bn, bufs = p.bufs;
    const int a_bytes = p.a_rows * kF8BK, b_bytes = bn * kF8BK;
    uint8_t* smem_b = smem + p.stages * a_bytes;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int S = static_cast<int>(cluster_nctarank());
    const int slice = static_cast<int>(cluster_ctarank());
    const int tile = static_cast<int>(blockIdx.x) / S;
    const int num_kb = (p.K + kF8BK - 1) / kF8BK;
    // slices differ by at most one K block (none is empty: S <= num_kb)
    const int kb0 = static_cast<int>(static_cast<int64_t>(num_kb) * slice / S), kb1 = static_cast<int>(static_cast<int64_t>(num_kb) * (slice + 1) / S);
    const int m0 = tile % p.tiles_m * 128, n0 = tile / p.tiles_m * bn;
    const int rows = min(128, p.M - m0);
    const int cols0 = (bn / 16 + 1) / 2 * 16;  // columns of the first four promotion warps; the others have the rest
    const int quarters = (rows + 31) / 32, halves = bn > cols0 ? 2 : 1;  // promotion warps with something to do

    // one barrier per thread (one thread would take a microsecond for all of them)
    if (threadIdx.x < kF8MaxStages) {
        mbar_init(&full[threadIdx.x], 1);
        mbar_init(&empty[threadIdx.x], 1);
        if (threadIdx.x < 4) {
            mbar_init(&acc_full[threadIdx.x], 1);
            mbar_init(&acc_empty[threadIdx.x], quarters * halves);
        }
        if (threadIdx.x < kF8ScaleSlots) {
            mbar_init(&scale_full[threadIdx.x], 32);
            mbar_init(&scale_empty[threadIdx.x], quarters * halves);
        }
        if (threadIdx.x == 0) abort_word = 0;
        fence_mbar_init();
    }
    if (warp == 0 && lane == 0) {
        prefetch_tensormap(&tmap_a);
        prefetch_tensormap(&tmap_b);
    }
    pdl_begin();
    if (blockIdx.x == 0 && threadIdx.x == 0) clock_probe(0, 0);
    if (warp == 1) {
        tmem_alloc(&tmem_base_slot, 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = tmem_base_slot;
    float* part = reinterpret_cast<float*>(smem);  // [rows][bn + 4], written after the main loop
    const int part_pitch = bn + 4;

    if (warp == 0) {
        setmaxnreg_dec<kF8OtherRegs>();
        if (lane == 0) {
            int stage = 0;
            uint32_t phase = 0;
            for (int kb = kb0; kb < kb1; ++kb) {
                if (!mbar_wait(&empty[stage], phase ^ 1, abort_flag, 0x100 + stage)) break;
                mbar_arrive_expect_tx(&full[stage], a_bytes + b_bytes);
                tma_load_2d(smem_b + stage * b_bytes, &tmap_b, &full[stage], kb * kF8BK, n0);
                tma_load_2d(smem + stage * a_bytes, &tmap_a, &full[stage], kb * kF8BK, m0);
                if (++stage == p.stages) { stage = 0; phase ^= 1; }
            }
        }
        __syncwarp();
        cluster_sync_all();
    } else if (warp == 1) {
        setmaxnreg_dec<kF8OtherRegs>();
        const bool leader = elect_one();
        const uint32_t idesc = make_idesc_e4m3(128, bn);
        const uint32_t a_lo0 = sdesc_lo(smem_u32(smem), 16), b_lo0 = sdesc_lo(smem_u32(smem_b), 16);
        int stage = 0, buf = 0;
        uint32_t phase = 0, acc_phase = 0;
        for (int kb = kb0; kb < kb1; ++kb) {
            bool ok = mbar_wait(&full[stage], phase, abort_flag, 0x200 + stage);
            ok = ok && mbar_wait(&acc_empty[buf], acc_phase ^ 1, abort_flag, 0x300 + buf);
            if (!__all_sync(0xffffffffu, ok)) break;
            tc_fence_after();
            if (leader) {
                const uint32_t a_lo = a_lo0 + stage * (a_bytes >> 4), b_lo = b_lo0 + stage * (b_bytes >> 4);
#pragma unroll
                for (int k = 0; k < kF8BK / 32; ++k)
                    umma_f8_ss_lo(tmem_base + buf * bn, a_lo + k * (32 >> 4), b_lo + k * (32 >> 4), idesc, k != 0);
                umma_commit(&empty[stage]);
                umma_commit(&acc_full[buf]);
            }
            __syncwarp();
            if (++stage == p.stages) { stage = 0; phase ^= 1; }
            if (++buf == bufs) { buf = 0; acc_phase ^= 1; }
        }
        cluster_sync_all();
    } else if (warp == 2) {
        setmaxnreg_dec<kF8OtherRegs>();
        // lane c < 4: the c-th column scale, of half c / 2: the first or second block of 128 its columns touch
        const int block = min((n0 + (lane >> 1 & 1) * cols0) / 128 + (lane & 1), (p.N - 1) / 128);  // (columns beyond N are not stored)
        int slot = 0;
        uint32_t phase = 0;
        gemm_f8_load_scales(scales, scale_full, scale_empty, slot, phase, p.sa + m0, p.ldsa, rows, p.sb + block * p.ldsb, kb0, kb1, lane, abort_flag);
        cluster_sync_all();
    } else if (warp == 3) {
        setmaxnreg_dec<kF8OtherRegs>();
        cluster_sync_all();
    } else {
        setmaxnreg_inc<kF8PromoteRegs>();
        const int quarter = warp & 3, half = (warp - 4) >> 2;
        const int col = half * cols0, chunks = ((half ? bn : cols0) - col) / 16;
        if (quarter < quarters && chunks > 0) {
            const int r = quarter * 32 + lane;
            const uint32_t t_row = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16) + col;
            float4* dst = reinterpret_cast<float4*>(part + r * part_pitch + col);
            // One unrolled loop per number of chunks: a branch around every chunk costs more than the chunk.
            auto promote = [&](auto count) {
                constexpr int kChunks = decltype(count)::value;
                // a warp's columns lie in one or two blocks of 128: the second begins at chunk `cut`
                const int cut = (128 - (n0 + col) % 128) / 16;
                float2 acc[kChunks * 8];
#pragma unroll
                for (int i = 0; i < kChunks * 8; ++i) acc[i] = make_float2(0.0f, 0.0f);
                int buf = 0, slot = 0;
                uint32_t acc_phase = 0, slot_phase = 0;
                for (int kb = kb0; kb < kb1; ++kb) {
                    const int u = (kb - kb0) & 3;
                    bool ok = true;
                    if (u == 0) ok = mbar_wait(&scale_full[slot], slot_phase, abort_flag, 0x500 + slot);
                    const float row_scale = scales[slot].row[u][r];
                    const float s0 = row_scale * scales[slot].col[u][half * 2], s1 = row_scale * scales[slot].col[u][half * 2 + 1];
                    ok = ok && mbar_wait(&acc_full[buf], acc_phase, abort_flag, 0x400 + buf);
                    if (!__all_sync(0xffffffffu, ok)) break;
                    tc_fence_after();
                    gemm_f8_promote<kChunks>(acc, t_row + buf * bn, s0, s1, cut, [&] {  // the tensor core may refill the accumulator
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) {
                            mbar_arrive(&acc_empty[buf]);
                            if (u == 3) mbar_arrive(&scale_empty[slot]);
                        }
                    });
                    if (u == 3 && ++slot == kF8ScaleSlots) { slot = 0; slot_phase ^= 1; }
                    if (++buf == bufs) { buf = 0; acc_phase ^= 1; }
                }
                // Every UMMA of this CTA has read its operands once the last accumulator is full, and the producer issued no load
                // beyond them: the stages are free when all promotion warps are here.
                asm volatile("bar.sync 1, %0;" ::"r"(32 * quarters * halves) : "memory");
                if (r < rows) {
#pragma unroll
                    for (int q = 0; q < kChunks * 4; ++q) dst[q] = make_float4(acc[2 * q].x, acc[2 * q].y, acc[2 * q + 1].x, acc[2 * q + 1].y);
                }
            };
            switch (chunks) {
                case 1: promote(std::integral_constant<int, 1>()); break;
                case 2: promote(std::integral_constant<int, 2>()); break;
                case 3: promote(std::integral_constant<int, 3>()); break;
                case 4: promote(std::integral_constant<int, 4>()); break;
                case 5: promote(std::integral_constant<int, 5>()); break;
                case 6: promote(std::integral_constant<int, 6>()); break;
                case 7: promote(std::integral_constant<int, 7>()); break;
                default: promote(std::integral_constant<int, 8>()); break;
            }
        }
        __syncwarp();
        // Every CTA's tile is in its shared memory (or a wait expired there: its rows are then garbage and the status word says
        // so): sum this CTA's share of the columns over the cluster.  (Only the promotion warps: code behind the roles' common
        // end would have to do with the registers of the others.)
        tc_fence_before();
        cluster_sync_all();
        const int g0 = bn / 4 * slice / S, groups = bn / 4 * (slice + 1) / S - g0;  // groups of four columns
        const int per_row = groups > 16 ? 32 : groups > 8 ? 16 : groups > 4 ? 8 : 4;  // lanes to a row
        const int rows_at_once = 32 / per_row * 8;                                       // of the eight warps
        const uint32_t part_addr = smem_u32(part);
        // four rows at a time, whose loads do not wait for one another; the CTA's own tile by plain loads
        auto finish = [&](auto alone) {
            for (int c = g0 + lane % per_row; c < g0 + groups; c += per_row) {
                const int out = n0 + c * 4;
                for (int row = (warp - 4) * (32 / per_row) + lane / per_row; row < rows; row += 4 * rows_at_once) {
                    float4 sum[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) sum[u] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                    if constexpr (decltype(alone)::value) {
#pragma unroll
                        for (int u = 0; u < 4; ++u)
                            if (row + u * rows_at_once < rows) sum[u] = *reinterpret_cast<const float4*>(part + (row + u * rows_at_once) * part_pitch + c * 4);
                    } else {
                        for (int s2 = 0; s2 < S; ++s2) {
                            const uint32_t peer = map_to_cta(part_addr + (row * part_pitch + c * 4) * 4, s2);
                            float4 v[4];
#pragma unroll
                            for (int u = 0; u < 4; ++u)
                                if (row + u * rows_at_once < rows) v[u] = ld_shared_cluster_f32x4(peer + u * rows_at_once * part_pitch * 4);
#pragma unroll
                            for (int u = 0; u < 4; ++u)
                                if (row + u * rows_at_once < rows) {
                                    sum[u].x += v[u].x; sum[u].y += v[u].y; sum[u].z += v[u].z; sum[u].w += v[u].w;
                                }
                        }
                    }
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        if (row + u * rows_at_once < rows) {
                            __nv_bfloat16* dst = p.C + static_cast<int64_t>(m0 + row + u * rows_at_once) * p.ldc + out;
                            if (out + 4 <= p.N) {
                                *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(sum[u].x, sum[u].y), pack_bf16x2(sum[u].z, sum[u].w));
                            } else {
                                const float a[4] = {sum[u].x, sum[u].y, sum[u].z, sum[u].w};
                                for (int k = 0; k < 4 && out + k < p.N; ++k) dst[k] = __float2bfloat16(a[k]);
                            }
                        }
                    }
                }
            }
        };
        if (S == 1) finish(std::true_type()); else finish(std::false_type());
        __syncwarp();
    }

    tc_fence_before();
    cluster_sync_all();  // no CTA leaves while a peer may still read its shared memory
    if (blockIdx.x == 0 && threadIdx.x == 0) clock_probe(0, 1);
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc(tmem_base, 512);
    }
}

// A load that stays where it is written (a prefetch that the compiler would move down to its use); 0 where `there` is false.
__device__ __forceinline__ float ld_f32_if(const float* p, bool there) {
    float v;
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %2, 0;\n\tmov.f32 %0, 0f00000000;\n\t@q ld.global.f32 %0, [%1];\n\t}"
                 : "=f"(v)
                 : "l"(p), "r"(static_cast<int>(there)));
    return v;
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
// Bound by the hand-over between tensor core and promotion warps: without any promotion the first case takes 671 us, at the same power
// cap.  Measured, device time in captured graphs: 8192 x 28672 x 4096 in 950 to 975 us, 2.0 PFLOP/s at 1.4 GHz (one call among other
// passes up to 1020; 850 to 900 in the first replays, before the clock comes down); 777 x 5000 x 4200 in 25 us, 4096^3 in 69 (84 call after
// call).  Four accumulators of 128 columns 1048 (A is read twice), tcgen05.ld of 64 columns 1230, scales through a ring in shared memory
// 1060, setmaxnreg 1065.
// ---------------------------------------------------------------------------------------------------------
constexpr int kF8BigThreads = 320;  // producer, issuer, eight promotion warps (168 registers per thread)
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

    if (threadIdx.x < kStages) {  // one barrier per thread
        mbar_init(&full[threadIdx.x], 1);
        mbar_init(&empty[threadIdx.x], 1);
        if (threadIdx.x < 2) {
            mbar_init(&acc_full[threadIdx.x], 1);
            mbar_init(&acc_empty[threadIdx.x], kPair ? 16 : 8);  // every promotion warp
        }
        if (threadIdx.x == 0) *abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == 0 && lane == 0) {
        prefetch_tensormap(&tmap_a);
        prefetch_tensormap(&tmap_b);
        prefetch_tensormap(&tmap_c);
    }
    pdl_begin();
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
            if (blockIdx.x == 0) clock_probe(0, 0);
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
                            gemm_f8_promote<8>(acc, t_row + buf * 256, s[u], s[u], 8, [&] {
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

// Once per device.  0: ready, 1: a CUDA call failed, 2: the split kernel was compiled with fewer registers than its hand-over
// moves (it would wait for registers that never come: nothing may be launched).
inline int gemm_f8_configure() {
    cudaFuncAttributes attr;
    if (cudaFuncSetAttribute(gemm_f8_split_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kF8SplitSmem) != cudaSuccess ||
        cudaFuncSetAttribute(gemm_f8_big_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, GemmF8BigSmem<true>::kTotal) != cudaSuccess ||
        cudaFuncSetAttribute(gemm_f8_big_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, GemmF8BigSmem<false>::kTotal) != cudaSuccess ||
        cudaFuncGetAttributes(&attr, gemm_f8_split_kernel) != cudaSuccess)
        return 1;
    return attr.numRegs >= kF8LaunchRegs ? 0 : 2;
}

}  // namespace mlt
