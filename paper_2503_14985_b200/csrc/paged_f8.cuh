// Paged-attention decode over an E4M3 cache with one FP32 scale per (cache block, KV head), for K and for V:
//   O = softmax(scale * q . (ks K)) (vs V),  LSE in natural log.
//
// Bound by HBM: 2 * len * D bytes per (sequence, KV head), half of the BF16 cache's.  At the copy bandwidth an SM gets
// about 23 cache elements per clock, too many for the FP32 pipe (convert, multiply, add for each query head), so both
// products run on warp-level tensor-core MMAs (m16n8k16, FP16) for every group size: S^T = K Q^T with 16 tokens as rows and
// the group's query heads as the 8 columns, O^T = V^T P^T with 16 elements of D as rows.  (Heads as rows would leave half of
// every MMA empty, and of the accumulators: 64 MMAs of 8 clocks per 32 tokens instead of 32 kept the streams waiting.)
// E4M3 to FP16 is exact (one conversion instruction per two elements).
//   * Q is scaled by a power of two per row into FP16's range (its 8 significant bits fit), exact but for elements more
//     than 2^28 below the row's largest.
//   * K's scale multiplies the scores of its block's tokens.  A tile of 8 tokens lies in one block.
//   * The second product's FP16 operand is the weight w = p * vs.  The scales may be anything, so the most likely token need not
//     have the largest weight: next to the running maximum m of the scores x (log2 units), which the sum l of the probabilities
//     goes by, a head keeps d = max(x + e) - m with vs = (1 .. 2) * 2^e, and its weights and accumulators are held times 2^14
//     relative to 2^(m + d).  The largest lies in 2^14 .. 2^15 whatever the scales are, and weights down to 2^-28 of it keep
//     FP16's full precision.  Partial results are means (divided by l): a sum over many tokens may lie beyond FP32 where
//     their mean does not.  That is a second exponential per score (16 MUFU cycles of the 350 that a unit's copies take) and
//     no division.
//   * Scores, maxima, sums and outputs are FP32; the sum takes the probabilities, which are not rounded to FP16.
//
// Data path: tensor copies (TMA) of whole (block, head) pieces into a three-deep ring of 32-token units per warp, swizzled so
// that the fragment loads meet no bank conflict at D = 128 (a lane's 16 bytes of K cover 16 elements of one token: the
// order of an MMA's summation index is free as long as both operands agree, as is the order of its output columns).
//
// Work split: the live units of 32 tokens of all (sequence, KV head) rows are numbered in row order and dealt in equal
// contiguous shares, one per warp (the lengths are only known on the device: every CTA scans them).  From there on warps do not
// wait for one another.  A row inside one share is finished by its warp; otherwise each warp that meets row r writes a
// partial into slot r + (its share) -- strictly increasing along the line, so rows + shares slots are enough -- and
// a second kernel combines them in ascending order.  Which rows those are the first kernel writes down, so that the second does
// not read the lengths at all.  Without scratch, or beyond 1024 sequences, one CTA works on each row and its warps' results meet in
// shared memory.
//
// Measured, both kernels, device time in a captured graph: 32 sequences of 2k to 4k tokens, 32 heads over 4, 30 us (3.4
// TB/s), 2 of 32k with 8 heads 32 us (4.1 TB/s); 256 of 500, 32 heads over 4, 37.5 us (3.6 TB/s), 1000 of 200 60 us (3.7
// TB/s); 16 of 2k to 4k with D = 64, 16 heads over 8, 22 us.  Around the streams lie 6 us of dependent latencies (lengths,
// table, first data) and 3 to 4 us of the combine kernel; that leaves 4 to 5 us of the first case not accounted for.
// Without scratch, one CTA per row: 54, 324, 44 and 101. Beyond 1024 sequences likewise (1100 of 200 111).  Alternatives, in
// the order of the first four: weights relative to the largest V scale, which lost the output where that scale's tokens were
// unlikely, 29, 30.5, 35.5 and 58 (D = 64: 23.5); on top of those, shares of 128-token chunks per CTA with a merge in shared
// memory 28.5, 29.5, 44 and 107; the same with copies issued ahead into the CTA's next row (longer loop) 30, 32, 47 and 116.
// The first two cases at earlier stages: heads as rows 37 and 37 instead of 30 and 32, units of 16 tokens 31 to 33, two
// stages and three CTAs per SM 30 and 32.5 instead of 29 and 30.  For the maximum of x + e: next to that of x in one pass,
// with a branch for scores beyond 2^23, where x + e loses e, 30, 32, 37.5 and 61.
#pragma once

#include "f8.cuh"
#include "paged.cuh"

namespace mlt {

struct PagedF8Params {
    const __nv_bfloat16* Q;  // [num_seqs, H, D]
    const float *ks, *vs;    // [num_blocks, H_kv]
    const int *block_table, *seq_lens;
    __nv_bfloat16* O;        // [num_seqs, H, D]
    float* LSE;              // [num_seqs, H] or null
    float* part_o;           // [num_seqs * H_kv + shares][G][D], divided by l
    float2* part_ml;         // [num_seqs * H_kv + shares][G] {m in log2 units, l}
    int2* splits;            // what to combine: [row] {first share, shares it lies in}, or [share] {row that begins in it and goes on, ...}
    bool by_row;             // which of the two (the shorter)
    int num_seqs, H, H_kv, max_blocks, num_blocks;
    int shares;              // warps that the live units are dealt to; 0: one CTA per row
    float scale_log2e;
};

constexpr int kPagedF8Unit = 32;   // tokens per warp and ring stage
constexpr int kPagedF8Ring = 3;    // stages: one in use, the others on their way
constexpr int kPagedF8CtasPerSm = 2;
constexpr int kPagedF8MaxShares = 2048;  // bound on the shares that the workspace formula uses
constexpr int kPagedF8MinShare = 2;  // units per share at least (128 sequences of 128 tokens, 4 KV heads: 11.7 us, with 1 14.2; 8 of 500: 10.4, 9.9, with 4 13.3)

template <int D>
constexpr int paged_f8_smem_bytes() {
    return kPagedWarps * kPagedF8Ring * 2 * kPagedF8Unit * D + 1024;
}

__device__ __forceinline__ void mma_f16_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t v) {  // lane (g, tg): row g, columns 2 tg, 2 tg + 1 -> the same of the transpose
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// v = m * 2^e with 1 <= |m| < 2 (0: m = 0, e = -inf; infinities and NaN stay in m, with e = 0)
__device__ __forceinline__ void split_scale(float v, float& m, float& e) {
    const uint32_t b = __float_as_uint(v);
    const int x = static_cast<int>(b >> 23 & 0xFFu);
    m = __uint_as_float((b & 0x807FFFFFu) | 0x3F800000u);
    e = static_cast<float>(x - 127);
    if (x == 0 || x == 255) {
        const uint32_t f = b & 0x7FFFFFu;
        const int up = __clz(f) - 8;  // a subnormal is f * 2^-149
        m = x == 255 ? v : f == 0u ? 0.0f : __uint_as_float((b & 0x80000000u) | 0x3F800000u | (f << up & 0x7FFFFFu));
        e = x == 255 ? 0.0f : f == 0u ? -INFINITY : static_cast<float>(-126 - up);
    }
}

__device__ __forceinline__ float finite_or_0(float x) { return x == -INFINITY ? 0.0f : x; }  // a reference where nothing was seen

__device__ __forceinline__ int paged_f8_len(const PagedF8Params& p, int s, int bs) {  // cut at the table's end
    return static_cast<int>(max(0ll, min(static_cast<long long>(p.seq_lens[s]), static_cast<long long>(p.max_blocks) * bs)));
}
__device__ __forceinline__ int paged_f8_units(const PagedF8Params& p, int s, int bs) {
    const int len = paged_f8_len(p, s, bs);
    return len / kPagedF8Unit + (len % kPagedF8Unit != 0);
}
// n units are dealt to min(shares, n / kPagedF8MinShare) shares: share c has the units c n / shares .. (c + 1) n / shares - 1,
// and unit x lies in share ((x + 1) shares - 1) / n.
__device__ __forceinline__ long long paged_f8_shares(long long n, int shares) {
    return max(1ll, min(static_cast<long long>(shares), n / kPagedF8MinShare));
}

template <int D, int G, int BS>
__global__ void __launch_bounds__(kPagedThreads, kPagedF8CtasPerSm)
paged_f8_decode_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v, const PagedF8Params p) {
    constexpr int U = kPagedF8Unit;
    constexpr int PP = D / 64;       // 16-byte pieces of a token's K per lane
    constexpr int MT = D / 16;       // row tiles of the output
    constexpr int kPiece = BS < U ? BS : U;  // tokens per tensor copy: a cache block, or the part of one that the unit covers
    constexpr int NB = U / kPiece;   // cache blocks per unit
    constexpr uint32_t kFull = U == 32 ? 0xFFFFFFFFu : (1u << (U & 31)) - 1u;  // all tokens of a unit
    constexpr int kUnitBytes = 2 * U * D;
    __shared__ float2 sm_ml[kPagedWarps][G];
    __shared__ int sm_pre[kPagedBalanceMaxSeqs + 1];
    __shared__ int sm_red[kPagedWarps];
    __shared__ uint64_t ring_bar[kPagedWarps][kPagedF8Ring];
    __shared__ uint32_t ring_abort;
    extern __shared__ uint8_t ring_raw[];
    uint8_t* ring_base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(ring_raw) + 1023) & ~uintptr_t(1023));

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g = lane >> 2, tg = lane & 3;
    uint8_t* my_ring = ring_base + warp * kPagedF8Ring * kUnitBytes;
    if (lane == 0) {
#pragma unroll
        for (int i = 0; i < kPagedF8Ring; ++i) mbar_init(&ring_bar[warp][i], 1);
        if (warp == 0) ring_abort = 0;
        fence_mbar_init();
        prefetch_tensormap(&tmap_k);
        prefetch_tensormap(&tmap_v);
    }

    pdl_begin();

    // ---- which segments (row, token range) this warp works on (with its CTA's others, where there is no scratch) ----
    int seg_s, seg_kvh = 0, seg_tok_begin = 0, seg_tok_end = 0;
    bool seg_whole = true;  // the row lies inside this warp's share
    long long bal_i = 0, bal_hi = 0, bal_n = 0, bal_shares = 0;
    const int share = warp * gridDim.x + blockIdx.x;  // (neighbouring shares on different SMs: few shares spread over all)
    if (p.shares == 0) {
        seg_s = blockIdx.x / p.H_kv;
        seg_kvh = blockIdx.x % p.H_kv;
        seg_tok_end = paged_f8_len(p, seg_s, BS);
        __syncthreads();  // the ring barriers are initialised
    } else {
        const int S = p.num_seqs;
        const int per = (S + kPagedThreads - 1) / kPagedThreads;
        const int s_lo = min(S, static_cast<int>(threadIdx.x) * per), s_hi = min(S, s_lo + per);
        int sum = 0;
        for (int s2 = s_lo; s2 < s_hi; ++s2) {
            const int c = paged_f8_units(p, s2, BS);
            sm_pre[s2 + 1] = c;
            sum += c;
        }
        int incl = sum;
#pragma unroll
        for (int w = 1; w < 32; w <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, incl, w);
            if (lane >= w) incl += v;
        }
        if (lane == 31) sm_red[warp] = incl;
        __syncthreads();  // also: the ring barriers are initialised
        int before = incl - sum, total = 0;
#pragma unroll
        for (int w = 0; w < kPagedWarps; ++w) {
            if (w < warp) before += sm_red[w];
            total += sm_red[w];
        }
        if (threadIdx.x == 0) sm_pre[0] = 0;
        for (int s2 = s_lo; s2 < s_hi; ++s2) sm_pre[s2 + 1] = before += sm_pre[s2 + 1];
        __syncthreads();
        const long long n = static_cast<long long>(total) * p.H_kv;
        const long long shares = paged_f8_shares(n, p.shares);
        for (int s2 = blockIdx.x; s2 < S; s2 += gridDim.x) {
            if (sm_pre[s2] != sm_pre[s2 + 1]) continue;
            for (int i = threadIdx.x; i < p.H * D / 8; i += kPagedThreads) reinterpret_cast<uint4*>(p.O + static_cast<int64_t>(s2) * p.H * D)[i] = make_uint4(0u, 0u, 0u, 0u);
            for (int i = threadIdx.x; i < p.H; i += kPagedThreads) {
                if (p.LSE) p.LSE[static_cast<int64_t>(s2) * p.H + i] = -INFINITY;
                if (p.by_row && i < p.H_kv) p.splits[static_cast<int64_t>(s2) * p.H_kv + i] = make_int2(0, 0);
            }
        }
        if (share >= shares || n == 0) {  // (from here on no warp waits for another)
            if (!p.by_row && share < p.shares && lane == 0) p.splits[share] = make_int2(0, 0);
            return;
        }
        bal_n = n;
        bal_shares = shares;
        bal_i = share * n / shares;
        bal_hi = (share + 1) * n / shares;
        int lo = 0, hi = S;  // H_kv * pre[lo] <= bal_i < H_kv * pre[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (static_cast<long long>(sm_pre[mid]) * p.H_kv <= bal_i) lo = mid; else hi = mid;
        }
        seg_s = lo;
    }
    auto next_segment = [&]() -> bool {
        if (bal_i >= bal_hi) return false;
        while (static_cast<long long>(sm_pre[seg_s + 1]) * p.H_kv <= bal_i) ++seg_s;  // skips empty sequences too
        const int n_s = sm_pre[seg_s + 1] - sm_pre[seg_s];
        const long long r = bal_i - static_cast<long long>(sm_pre[seg_s]) * p.H_kv;
        seg_kvh = static_cast<int>(r / n_s);
        const int ch0 = static_cast<int>(r % n_s);
        const int ch1 = static_cast<int>(min(static_cast<long long>(n_s), ch0 + (bal_hi - bal_i)));
        seg_tok_begin = ch0 * U;
        seg_tok_end = ch1 == n_s ? paged_f8_len(p, seg_s, BS) : ch1 * U;
        seg_whole = ch0 == 0 && ch1 == n_s;
        if (lane == 0) {  // the combine kernel's list
            const int used = ch0 != 0 ? 0 : ch1 == n_s ? 1 : static_cast<int>(((bal_i + n_s) * bal_shares - 1) / bal_n) - share + 1;
            const int row = seg_s * p.H_kv + seg_kvh;
            if (p.by_row) {
                if (ch0 == 0) p.splits[row] = make_int2(share, used);
            } else if (bal_i + (ch1 - ch0) == bal_hi) {
                p.splits[share] = make_int2(row, used);
            }
        }
        bal_i += ch1 - ch0;
        return true;
    };
    if (p.shares != 0 && !next_segment()) return;

    uint32_t kbase = 0;        // units this warp has been through (the ring stage follows it)
    uint32_t ring_parity = 0;  // bit st: parity of the next completion of stage st's barrier
    bool ok = true;
    for (;;) {
    // =============================== one segment ===============================
    const int s = seg_s, kvh = seg_kvh, tok_begin = seg_tok_begin, tok_end = seg_tok_end;
    const int head0 = kvh * G;

    uint4 q_raw[2 * PP];  // lane (g, tg): elements tg * D / 4 .. of head g
#pragma unroll
    for (int i = 0; i < 2 * PP; ++i) {
        q_raw[i] = make_uint4(0u, 0u, 0u, 0u);
        if (g < G) q_raw[i] = *reinterpret_cast<const uint4*>(p.Q + (static_cast<int64_t>(s) * p.H + head0 + g) * D + tg * (D / 4) + i * 8);
    }
    float oacc[MT][4];  // elements g * MT * 2 + 2 mt (0, 1) and + 1 (2, 3) of D for heads 2 tg (0, 2) and 2 tg + 1 (1, 3)
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int i = 0; i < 4; ++i) oacc[mt][i] = 0.0f;
    float m_run[2] = {-INFINITY, -INFINITY};  // of the two heads: running max of x (log2 units, the same in all lanes of a tg)
    float d_run[2] = {-INFINITY, -INFINITY};  // ... running max of x + e, less m_run: the accumulators hold sums of 2^(x - m_run - d_run + 14) vs V
    float l_part[2] = {0.0f, 0.0f};           // ... this lane's share of the sum

    const int* table = p.block_table + static_cast<int64_t>(s) * p.max_blocks;
    struct Meta {  // of a unit whose copies are under way: which of its tokens count, and its blocks' scales
        uint32_t vis;
        float ks[NB], vs[NB];
    };
    // Unit k of this warp starts at token first + k * kStep.  The table entries and scales of 32 units at a time are
    // read by one lane each and handed out by shuffles.
    const int kStep = p.shares ? U : kPagedWarps * U;
    const int first = p.shares ? tok_begin : tok_begin + warp * U;
    const int n_units = first < tok_end ? (tok_end - first - 1) / kStep + 1 : 0;
    int tab[NB];
    float tks[NB], tvs[NB];
    int tab_base = -64;
    auto issue_unit = [&](Meta& meta, int stage, int k) {  // (take_scales fills in the scales)
        const int u0 = first + k * kStep;
        bool fresh = false;
        if (k >= tab_base + 32) {
            tab_base = k;
            const int n = k + lane < n_units ? tok_end - (first + (k + lane) * kStep) : 0;  // tokens of unit k + lane and beyond
#pragma unroll
            for (int i = 0; i < NB; ++i) tab[i] = i * kPiece < n ? table[(first + (k + lane) * kStep) / BS + i] : 0;
            fresh = true;
        }
        const int left = tok_end - u0;
        meta.vis = left >= U ? kFull : (1u << left) - 1u;
        int phys[NB], blocks = 0;
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            phys[i] = __shfl_sync(0xffffffffu, tab[i], k - tab_base);
            if (i * kPiece >= left) {
                phys[i] = -1;
            } else if (phys[i] < 0 || phys[i] >= p.num_blocks) {  // never dereference a bad table entry: report, leave its tokens out
                if (lane == 0 && atomicCAS(&g_status[0], 0u, kStatusBadBlock) == 0u) {
                    g_status[1] = static_cast<unsigned int>(u0 / BS + i);
                    g_status[2] = static_cast<unsigned int>(s);
                    g_status[3] = static_cast<unsigned int>(phys[i]);
                }
                phys[i] = -1;
                meta.vis &= ~((kPiece == 32 ? 0xFFFFFFFFu : (1u << (kPiece & 31)) - 1u) << (i * kPiece));
            } else {
                ++blocks;
            }
        }
        if (blocks > 0) {
            __syncwarp();  // every lane is done reading the stage's previous contents
            uint64_t* bar = &ring_bar[warp][stage];
            if (lane == 0) mbar_arrive_expect_tx(bar, 2u * blocks * kPiece * D);
            __syncwarp();
            uint8_t* dst = my_ring + stage * kUnitBytes;
#pragma unroll
            for (int i = 0; i < NB; ++i)
                if (phys[i] >= 0 && (lane >> 1) == i)
                    tma_load_3d(dst + (lane & 1) * (U * D) + i * kPiece * D, (lane & 1) ? &tmap_v : &tmap_k, bar, 0, u0 % BS / kPiece * kPiece, phys[i] * p.H_kv + kvh);
            __syncwarp();
        }
        if (fresh) {  // (behind the copies: the scales are only needed when the unit is used)
            const int n = k + lane < n_units ? tok_end - (first + (k + lane) * kStep) : 0;
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                const bool there = i * kPiece < n && tab[i] >= 0 && tab[i] < p.num_blocks;
                const int64_t at = static_cast<int64_t>(tab[i]) * p.H_kv + kvh;
                tks[i] = there ? p.ks[at] : 0.0f;
                tvs[i] = there ? p.vs[at] : 0.0f;
            }
        }
    };
    auto take_scales = [&](Meta& meta, int k) {  // of unit k, while the lanes hold its batch
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            meta.ks[i] = __shfl_sync(0xffffffffu, tks[i], k - tab_base);
            meta.vs[i] = __shfl_sync(0xffffffffu, tvs[i], k - tab_base);
        }
    };
    Meta ahead[kPagedF8Ring];  // units k, k + 1, ..: ahead[0] is the one in use
#pragma unroll
    for (int i = 0; i < kPagedF8Ring - 1; ++i)
        if (i < n_units) issue_unit(ahead[i], (kbase + i) % kPagedF8Ring, i);  // under way before the queries are converted

    // Q^T as B fragments in FP16: lane (g, tg) holds elements tg * D / 4 .. of head g, scaled by 2^-qexp
    uint32_t qb[PP][4][2];
    float c_head[2];  // of heads 2 tg, 2 tg + 1: scores to log2 units, before K's scale
    {
        const uint4 (&v)[2 * PP] = q_raw;
        float amax = 0.0f;
#pragma unroll
        for (int i = 0; i < 2 * PP; ++i) {
            float f[8];
            bf16x8_to_f32(v[i], f);
#pragma unroll
            for (int e = 0; e < 8; ++e) amax = fmaxf(amax, abs_if_finite(f[e]));
        }
        amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
        amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
        const int qexp = max(-100, static_cast<int>(__float_as_uint(amax) >> 23) - 127 - 14);  // the largest element becomes 2^14 .. 2^15
        const float down = pow2f(-qexp);
        const float c_row = p.scale_log2e * pow2f(qexp);
        c_head[0] = __shfl_sync(0xffffffffu, c_row, 8 * tg);
        c_head[1] = __shfl_sync(0xffffffffu, c_row, 8 * tg + 4);
#pragma unroll
        for (int i = 0; i < 2 * PP; ++i) {
            float f[8];
            bf16x8_to_f32(v[i], f);
#pragma unroll
            for (int e = 0; e < 4; ++e) qb[i >> 1][(i & 1) * 2 + (e >> 1)][e & 1] = pack_f16x2(f[2 * e] * down, f[2 * e + 1] * down);
        }
    }
    // byte offset of 16-byte piece c of token row r in a swizzled [tokens][D] tile
    auto at16 = [](int r, int c) { return D == 128 ? r * 128 + ((c ^ (r & 7)) << 4) : r * 64 + ((c ^ ((r >> 1) & 3)) << 4); };
    auto compute_unit = [&](const Meta& meta, int stage) {
        const uint8_t* ku = my_ring + stage * kUnitBytes;
        const uint8_t* vu = ku + U * D;
        // ---- scores of tokens 8 e + g for heads 2 tg, 2 tg + 1 ----
        float x[U / 8][2];
#pragma unroll
        for (int h = 0; h < U / 16; ++h) {
            float sc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int pp = 0; pp < PP; ++pp) {
                const uint4 lo = *reinterpret_cast<const uint4*>(ku + at16(16 * h + g, PP * tg + pp));
                const uint4 hi = *reinterpret_cast<const uint4*>(ku + at16(16 * h + 8 + g, PP * tg + pp));
                const uint32_t wl[4] = {lo.x, lo.y, lo.z, lo.w}, wh[4] = {hi.x, hi.y, hi.z, hi.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t a0, a1, a2, a3;
                    f16x2_from_f8x4(wl[j], a0, a2);
                    f16x2_from_f8x4(wh[j], a1, a3);
                    mma_f16_16816(sc, a0, a1, a2, a3, qb[pp][j][0], qb[pp][j][1]);
                }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {  // tiles e = 2 h + i, each inside one cache block
                const int e = 2 * h + i;
                const float ks = meta.ks[8 * e / kPiece];
                x[e][0] = sc[2 * i] * (c_head[0] * ks);
                x[e][1] = sc[2 * i + 1] * (c_head[1] * ks);
            }
        }
        if (meta.vis != kFull) {
#pragma unroll
            for (int e = 0; e < U / 8; ++e)
                if (!((meta.vis >> (8 * e + g)) & 1u)) x[e][0] = x[e][1] = -INFINITY;
        }
        float vm[NB], ve[NB];
#pragma unroll
        for (int i = 0; i < NB; ++i) split_scale(meta.vs[i], vm[i], ve[i]);
        bool moved = false;
        float m_new[2], d_new[2], f_l[2], f_o[2], off[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float mb = x[0][i];
#pragma unroll
            for (int e = 1; e < U / 8; ++e) mb = fmaxf(mb, x[e][i]);
#pragma unroll
            for (int w = 4; w < 32; w <<= 1) mb = fmaxf(mb, __shfl_xor_sync(0xffffffffu, mb, w));
            m_new[i] = fmaxf(m_run[i], mb);
            const float ref = finite_or_0(m_new[i]);
            float db = -INFINITY;  // (of x - ref: e would be lost next to a large x)
#pragma unroll
            for (int e = 0; e < U / 8; ++e) {
                x[e][i] -= ref;
                db = fmaxf(db, x[e][i] + ve[8 * e / kPiece]);
            }
#pragma unroll
            for (int w = 4; w < 32; w <<= 1) db = fmaxf(db, __shfl_xor_sync(0xffffffffu, db, w));
            const float fall = m_run[i] - ref;  // -inf the first time
            d_new[i] = fmaxf(d_run[i] + fall, db);
            const float d_ref = finite_or_0(d_new[i]);
            moved |= m_new[i] != m_run[i] || d_new[i] != d_run[i];
            f_l[i] = fast_exp2(fall);
            f_o[i] = fast_exp2(fall + (d_run[i] - d_ref));
            off[i] = 14.0f - d_ref;
        }
        if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                oacc[mt][0] *= f_o[0];
                oacc[mt][1] *= f_o[1];
                oacc[mt][2] *= f_o[0];
                oacc[mt][3] *= f_o[1];
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                l_part[i] *= f_l[i];
                m_run[i] = m_new[i];
                d_run[i] = d_new[i];
            }
        }
        uint32_t pb[U / 8];  // P^T as B fragments: lane (g, tg) holds tokens 8 e + 2 tg, + 1 of head g
#pragma unroll
        for (int e = 0; e < U / 8; ++e) {
            const int i = 8 * e / kPiece;
            l_part[0] += fast_exp2(x[e][0]);
            l_part[1] += fast_exp2(x[e][1]);
            pb[e] = transpose_8x8(pack_f16x2(fast_exp2(x[e][0] + (ve[i] + off[0])) * vm[i], fast_exp2(x[e][1] + (ve[i] + off[1])) * vm[i]));
        }
        // ---- O^T += V^T P^T: row g of tile mt is element g * 2 MT + 2 mt, row g + 8 the one after it ----
#pragma unroll
        for (int h = 0; h < U / 16; ++h) {
            uint32_t w[4][D / 32];  // tokens 16 h + {2 tg, 2 tg + 1, 2 tg + 8, 2 tg + 9}
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int t = 16 * h + 2 * tg + (i & 1) + (i >> 1) * 8;
                if constexpr (D == 128) {
                    const uint4 q = *reinterpret_cast<const uint4*>(vu + at16(t, g));
                    w[i][0] = q.x; w[i][1] = q.y; w[i][2] = q.z; w[i][3] = q.w;
                } else {
                    const uint2 q = *reinterpret_cast<const uint2*>(vu + at16(t, g >> 1) + (g & 1) * 8);
                    w[i][0] = q.x; w[i][1] = q.y;
                }
            }
            if (meta.vis != kFull) {  // whatever lies there, weight 0 must not meet a NaN
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (!((meta.vis >> (16 * h + 2 * tg + (i & 1) + (i >> 1) * 8)) & 1u)) {
#pragma unroll
                        for (int j = 0; j < D / 32; ++j) w[i][j] = 0u;
                    }
            }
#pragma unroll
            for (int j = 0; j < D / 32; ++j) {
#pragma unroll
                for (int q = 0; q < 2; ++q) {  // elements 4 j + 2 q, + 1 of two tokens each
                    const uint32_t sel = q ? 0x7362u : 0x5140u;
                    uint32_t a0, a1, a2, a3;
                    f16x2_from_f8x4(__byte_perm(w[0][j], w[1][j], sel), a0, a1);
                    f16x2_from_f8x4(__byte_perm(w[2][j], w[3][j], sel), a2, a3);
                    mma_f16_16816(oacc[2 * j + q], a0, a1, a2, a3, pb[2 * h], pb[2 * h + 1]);
                }
            }
        }
    };
    for (int k = 0; k < n_units && ok; ++k) {
        const uint32_t st = (kbase + k) % kPagedF8Ring;
        const int kk = k + kPagedF8Ring - 1;
        if (kk == tab_base + 32) {  // that unit's entries will replace those of the units before it
#pragma unroll
            for (int i = 0; i < kPagedF8Ring - 1; ++i)
                if (k + i >= tab_base) take_scales(ahead[i], k + i);
        }
        if (kk < n_units) issue_unit(ahead[kPagedF8Ring - 1], (kbase + kk) % kPagedF8Ring, kk);
        if (k >= tab_base) take_scales(ahead[0], k);  // (the first time they are still on their way)
        if (ahead[0].vis != 0) {  // (a unit all of whose blocks are bad has no copies and does not use its stage)
            ok = __all_sync(0xffffffffu, mbar_wait(&ring_bar[warp][st], (ring_parity >> st) & 1, &ring_abort, 0x600 + warp)) != 0;
            if (!ok) break;
            ring_parity ^= 1u << st;
            compute_unit(ahead[0], st);
        }
#pragma unroll
        for (int i = 0; i < kPagedF8Ring - 1; ++i) ahead[i] = ahead[i + 1];
    }
    kbase += n_units;

#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int w = 4; w < 32; w <<= 1) l_part[i] += __shfl_xor_sync(0xffffffffu, l_part[i], w);
    // The accumulators become means by two factors (their product could lie outside FP32: d is -150 .. 128).
    float mean1[2], mean2[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        mean1[i] = d_run[i] == -INFINITY ? 0.0f : fast_exp2(0.5f * d_run[i]);
        mean2[i] = l_part[i] == 0.0f ? 0.0f : mean1[i] * (1.0f / 16384.0f) / l_part[i];
    }
    if (p.shares) {  // lane (g, tg) has 2 MT neighbouring elements of heads 2 tg, 2 tg + 1
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int gg = 2 * tg + i;
            if (gg < G) {
                const float l = l_part[i], f1 = mean1[i], f2 = mean2[i];
                if (seg_whole) {
                    const int64_t row = static_cast<int64_t>(s) * p.H + head0 + gg;
                    uint4* dst = reinterpret_cast<uint4*>(p.O + row * D + g * 2 * MT);
#pragma unroll
                    for (int q = 0; q < MT / 4; ++q) {
                        uint32_t w[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) w[j] = pack_bf16x2(oacc[4 * q + j][i] * f2 * f1, oacc[4 * q + j][2 + i] * f2 * f1);
                        dst[q] = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                    if (g == 0 && p.LSE) p.LSE[row] = l == 0.0f ? -INFINITY : (m_run[i] + log2f(l)) * 0.6931471805599453f;
                } else {
                    const int64_t slot = (static_cast<int64_t>(s) * p.H_kv + kvh + share) * G + gg;
                    float4* dst = reinterpret_cast<float4*>(p.part_o + slot * D + g * 2 * MT);
#pragma unroll
                    for (int q = 0; q < MT / 2; ++q)
                        dst[q] = make_float4(oacc[2 * q][i] * f2 * f1, oacc[2 * q][2 + i] * f2 * f1, oacc[2 * q + 1][i] * f2 * f1, oacc[2 * q + 1][2 + i] * f2 * f1);
                    if (g == 0) p.part_ml[slot] = make_float2(m_run[i], l);
                }
            }
        }
        if (!ok || !next_segment()) return;
        continue;
    }

    // ---- without shares: the warps' results meet in shared memory, where the ring was (all copies have landed and been read) ----
    __syncthreads();
    constexpr int kRow = D + 2;  // (the lanes' pairs meet two-way bank conflicts, with D they would meet eight-way ones)
    float (*sm_o)[8][kRow] = reinterpret_cast<float (*)[8][kRow]>(ring_base);
    static_assert(sizeof(float) * kPagedWarps * 8 * kRow <= kPagedWarps * kPagedF8Ring * kUnitBytes, "partials fit the ring");
    {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (2 * tg + i < G) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
                    *reinterpret_cast<float2*>(&sm_o[warp][2 * tg + i][g * 2 * MT + 2 * mt]) = make_float2(oacc[mt][i] * mean2[i] * mean1[i], oacc[mt][2 + i] * mean2[i] * mean1[i]);
                if (g == 0) sm_ml[warp][2 * tg + i] = make_float2(m_run[i], l_part[i]);
            }
        }
    }
    __syncthreads();
    // all loads of a thread's places before the first use: one round trip instead of one per place
    constexpr int kPlaces = (G * D + kPagedThreads - 1) / kPagedThreads;
    float ot[kPlaces], lt[kPlaces], mt[kPlaces];
#pragma unroll
    for (int it = 0; it < kPlaces; ++it) {
        const int idx = threadIdx.x + it * kPagedThreads;
        const int gg = idx / D < G ? idx / D : 0, at = idx % D;
        float2 ml[kPagedWarps];
        float o[kPagedWarps];
#pragma unroll
        for (int w = 0; w < kPagedWarps; ++w) {
            ml[w] = sm_ml[w][gg];
            o[w] = sm_o[w][gg][at];
        }
        mt[it] = finite_or_0(fmaxf(fmaxf(ml[0].x, ml[1].x), fmaxf(ml[2].x, ml[3].x)));
        lt[it] = ot[it] = 0.0f;
        float h[kPagedWarps];  // the weights' roots, as in the combine kernel
#pragma unroll
        for (int w = 0; w < kPagedWarps; ++w) {
            h[w] = fast_exp2(0.5f * (ml[w].x - mt[it]));
            lt[it] += ml[w].y * h[w] * h[w];
        }
        const float inv = lt[it] == 0.0f ? 0.0f : 1.0f / lt[it];
#pragma unroll
        for (int w = 0; w < kPagedWarps; ++w) ot[it] += o[w] * h[w] * (ml[w].y * inv * h[w]);
    }
#pragma unroll
    for (int it = 0; it < kPlaces; ++it) {
        const int idx = threadIdx.x + it * kPagedThreads;
        const int gg = idx / D, at = idx % D;
        if (gg < G) {
            const int64_t row = static_cast<int64_t>(s) * p.H + head0 + gg;
            p.O[row * D + at] = __float2bfloat16(ot[it]);
            if (at == 0 && p.LSE) p.LSE[row] = lt[it] == 0.0f ? -INFINITY : (mt[it] + log2f(lt[it])) * 0.6931471805599453f;
        }
    }
    static_assert(kPagedWarps == 4, "the maximum above is over four warps");
    break;
    }  // segments
}

// Rows that several warps worked on: sum of their partials, rescaled to the common maximum.  A CTA has kVec float4 columns of a
// row's group of heads, a thread one of them and every kSplits-th partial.  Few rows have many partials each: below 64 rows
// 512 threads with 32 columns, otherwise all columns and 256 threads.  Both sides measured, decode and combine together (us, the first
// form and the second): 1 row of 32k tokens 15 and 101, 16 rows of 16k 23 and 35, 32 of 4k 15 and 21 (of 500 11.2 and 10.4), 64 of 4k 25.3 and
// 25.5 (of 500 13.7 and 11.4), 128 of 3k 36 and 31.
template <int D, int G, int kVec, int kThreads>
__global__ void __launch_bounds__(kThreads) paged_f8_combine_kernel(const PagedF8Params p) {
    constexpr int kWarps = kThreads / 32;
    constexpr int kSlices = G * D / 4 / kVec, kSplits = kThreads / kVec;
    static_assert(kSplits >= 1 && kSplits * kVec == kThreads, "whole splits");
    __shared__ float2 sm_m[kWarps][G];
    __shared__ float4 sm_o[kThreads];
    __shared__ float sm_l[kThreads];
    pdl_launch_dependents();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int v = blockIdx.x % kSlices * kVec + tid % kVec, split = tid / kVec, gg = v * 4 / D;  // column, of the group's outputs
    const int item = blockIdx.x / kSlices;
    // Nothing before this wait: the decode kernel releases this launch before its own wait, so the kernel in front of it, which
    // may be the one that writes the lengths, can still be at work here.
    cudaGridDependencySynchronize();
    const int2 what = p.splits[item];
    const int row = p.by_row ? item : what.x, c0 = p.by_row ? what.x : item, used = what.y;
    if (used <= 1) return;  // one warp had the whole row and finished it, or there is none
    if (row < 0 || row >= p.num_seqs * p.H_kv || c0 < 0 || c0 >= p.shares || used > p.shares - c0) return;  // (after a wait that expired the list has gaps)
    const int64_t row0 = static_cast<int64_t>(row) * G;  // of the group's first head
    const int64_t slot0 = static_cast<int64_t>(row) + c0;
    const float2* ml = p.part_ml + slot0 * G;
    const float4* po = reinterpret_cast<const float4*>(p.part_o + slot0 * G * D) + v;
    constexpr int kFirst = kThreads / 64;  // requested before the maximum is known
    float4 first[kFirst];
#pragma unroll
    for (int i = 0; i < kFirst; ++i)
        first[i] = split + i * kSplits < used ? po[static_cast<int64_t>(split + i * kSplits) * (G * D / 4)] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    float mt = -INFINITY, l_all = 0.0f;  // of all partials: the largest m, and the sum of l as if every m were that
    for (int i = tid; i < used * G; i += kThreads) {  // head tid % G (G divides the stride)
        const float2 a = ml[i];
        mt = fmaxf(mt, a.x);
        l_all += a.y;
    }
#pragma unroll
    for (int w = 16; w >= G; w >>= 1) {
        mt = fmaxf(mt, __shfl_xor_sync(0xffffffffu, mt, w));
        l_all += __shfl_xor_sync(0xffffffffu, l_all, w);
    }
    if (lane < G) sm_m[warp][lane] = make_float2(mt, l_all);
    __syncthreads();
    mt = -INFINITY;
    l_all = 0.0f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        const float2 a = sm_m[w][gg];
        mt = fmaxf(mt, a.x);
        l_all += a.y;
    }
    mt = finite_or_0(mt);
    // The weights l 2^(m - mt) / l_all sum to 1 at most, so that no sum of means overflows.  They are applied by two factors of half the
    // exponent: a weight of 2^-200 alone would vanish, but not its product with a mean of 2^100.
    const float unit = l_all == 0.0f ? 0.0f : 1.0f / l_all;
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    float lt = 0.0f;
    auto add = [&](int i, const float4& x) {
        const float2 a = ml[static_cast<int64_t>(i) * G + gg];
        const float h = fast_exp2(0.5f * (a.x - mt)), w = a.y * unit * h;
        lt = fmaf(w, h, lt);
        o.x = fmaf(x.x * h, w, o.x);
        o.y = fmaf(x.y * h, w, o.y);
        o.z = fmaf(x.z * h, w, o.z);
        o.w = fmaf(x.w * h, w, o.w);
    };
#pragma unroll
    for (int i = 0; i < kFirst; ++i)
        if (split + i * kSplits < used) add(split + i * kSplits, first[i]);
#pragma unroll 4
    for (int i = split + kFirst * kSplits; i < used; i += kSplits) add(i, po[static_cast<int64_t>(i) * (G * D / 4)]);
    if constexpr (kSplits > 1) {
        sm_o[tid] = o;
        sm_l[tid] = lt;
        __syncthreads();
        if (split != 0) return;
#pragma unroll
        for (int k = 1; k < kSplits; ++k) {
            const float4 x = sm_o[k * kVec + tid];
            o.x += x.x; o.y += x.y; o.z += x.z; o.w += x.w;
            lt += sm_l[k * kVec + tid];
        }
    }
    const float inv = lt == 0.0f ? 0.0f : 1.0f / lt;
    *reinterpret_cast<uint2*>(p.O + row0 * D + v * 4) = make_uint2(pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv));
    if (v * 4 % D == 0 && p.LSE) p.LSE[row0 + gg] = lt == 0.0f ? -INFINITY : (mt + log2f(lt) + log2f(l_all)) * 0.6931471805599453f;
}

inline size_t paged_f8_slot_bytes(int G, int D) { return static_cast<size_t>(G) * (static_cast<size_t>(D) * 4 + 8) + 8; }

template <int D, int G, int BS>
int paged_f8_launch_one(const CUtensorMap& tk, const CUtensorMap& tv, const PagedF8Params& p, cudaStream_t st) {
    const int64_t grid = p.shares ? (p.shares + kPagedWarps - 1) / kPagedWarps : static_cast<int64_t>(p.num_seqs) * p.H_kv;
    if (grid > INT32_MAX || static_cast<int64_t>(p.num_seqs) * p.H > INT32_MAX) return 2;
    if (pdl_launch(paged_f8_decode_kernel<D, G, BS>, dim3(static_cast<unsigned>(grid)), dim3(kPagedThreads), paged_f8_smem_bytes<D>(), st, 0, tk, tv, p) != cudaSuccess)
        return 4;
    if (p.shares == 0) return 0;
    constexpr int kAll = G * D / 4, kFew = kAll < 32 ? kAll : 32;  // float4 columns per CTA
    const int items = p.by_row ? p.num_seqs * p.H_kv : p.shares;
    const bool few = items < 64;
    return pdl_launch(few ? paged_f8_combine_kernel<D, G, kFew, 512> : paged_f8_combine_kernel<D, G, kAll, 256>,
                      dim3(static_cast<unsigned>(items * (few ? kAll / kFew : 1))), dim3(few ? 512 : 256), 0, st, 0, p) == cudaSuccess ? 0 : 4;
}
template <int D, int G>
int paged_f8_launch_bs(const CUtensorMap& tk, const CUtensorMap& tv, const PagedF8Params& p, int block_size, cudaStream_t st) {
    switch (block_size) {
        case 8: return paged_f8_launch_one<D, G, 8>(tk, tv, p, st);
        case 16: return paged_f8_launch_one<D, G, 16>(tk, tv, p, st);
        case 32: return paged_f8_launch_one<D, G, 32>(tk, tv, p, st);
        default: return 2;
    }
}
template <int D>
int paged_f8_launch(const CUtensorMap& tk, const CUtensorMap& tv, const PagedF8Params& p, int block_size, cudaStream_t st) {
    switch (p.H / p.H_kv) {
        case 1: return paged_f8_launch_bs<D, 1>(tk, tv, p, block_size, st);
        case 2: return paged_f8_launch_bs<D, 2>(tk, tv, p, block_size, st);
        case 4: return paged_f8_launch_bs<D, 4>(tk, tv, p, block_size, st);
        case 8: return paged_f8_launch_bs<D, 8>(tk, tv, p, block_size, st);
        default: return 2;
    }
}

// Once per device: the ring is larger than the default shared-memory limit.
template <int D, int G>
bool paged_f8_configure_one() {
    const int bytes = paged_f8_smem_bytes<D>();
    return cudaFuncSetAttribute(paged_f8_decode_kernel<D, G, 8>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) == cudaSuccess &&
           cudaFuncSetAttribute(paged_f8_decode_kernel<D, G, 16>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) == cudaSuccess &&
           cudaFuncSetAttribute(paged_f8_decode_kernel<D, G, 32>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) == cudaSuccess;
}
inline bool paged_f8_configure() {
    return paged_f8_configure_one<64, 1>() && paged_f8_configure_one<64, 2>() && paged_f8_configure_one<64, 4>() && paged_f8_configure_one<64, 8>() &&
           paged_f8_configure_one<128, 1>() && paged_f8_configure_one<128, 2>() && paged_f8_configure_one<128, 4>() && paged_f8_configure_one<128, 8>();
}

}  // namespace mlt
