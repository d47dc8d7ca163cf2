// Attention of whole prompts, for sequences of different lengths packed one behind another and grouped heads:
//   row (token i of sequence s, head h) sees keys j <= lim(i);  p_j = exp(scale q.k_j - m),  O = sum p_j v_j / sum p_j.
// Keys come from packed rows or from the paged cache; a decode batch that shares a prefix is the same problem with the
// batch's sequences as the tokens.
//
// The softmax core is that of mha.cuh (two 128-row tiles that take turns on the tensor pipe, one thread per row, running
// reference maximum, P through tensor memory; its comments give the reasons).  What differs:
//  * Rows.  The G query heads of a KV head are rows of one tile: row r is token r / G, head r % G, W = 128 / G tokens per
//    tile (G that do not divide 128 leave up to G - 1 rows unused; these are zeroed once).  A few tokens of many heads then
//    fill a tile, and K and V are read once for all G heads.  The Q tile is one TMA box [64 of D, G heads, W tokens].
//  * Work.  Lengths are on the device, so a one-CTA kernel writes the list of work items (two tiles of a sequence, a range of
//    key blocks), longest first, and persistent CTAs (one per SM) draw from it by an atomic counter.  The loading warp draws
//    the next item as soon as it has requested the current one's last keys, so the list's latency hides behind the ring.
//    With too few items for the SMs (few tokens behind a long context) the plan cuts the key range; the parts go to scratch
//    as FP32 {m, l, O} and a second kernel joins them.
//  * Keys from the cache.  One lane per (cache block, 64 columns) issues its own TMA box, so a 128-key tile is one table load
//    and one issue for the warp.  A block-table entry out of range loads zeros (coordinate beyond the tensor map) and is
//    reported.  Rows beyond the sequence's last key may hold anything (another sequence, stale cache): scores there are
//    masked, and a spare warp zeroes those rows of V in shared memory, because a weight of 0 must not meet a NaN.
//  * Output rows of a tile may belong to a sequence only in part, so they leave as plain 16-byte stores (eight lanes per
//    128-byte piece of a row) instead of TMA boxes.
#pragma once

#include <utility>

#include "mha.cuh"
#include "paged.cuh"

namespace mlt {

constexpr unsigned int kStatusBadSequence = 9;  // a sequence's offsets or positions lie outside the call's tokens or keys
constexpr int kPackedPlanThreads = 1024;
constexpr int kPackedBuckets = 2048;
constexpr int kPackedMaxSplitTiles = 1024;  // key ranges are cut only when there are fewer tile pairs than this
constexpr int kPackedMaxSlots = 320;        // partial results (256 rows each) that scratch is sized for

struct PackedHeader {  // at the front of the scratch memory, written by the plan kernel
    int num_items;     // entries * H_kv
    int counter;       // items handed out beyond the first one of each CTA
    int split;         // key blocks per part, 0: no range is cut
    int pad;
};

struct PackedParams {
    // lengths (device): cu_q [S + 1] token offsets; keys per sequence from cu_k (packed), context_lens (paged) or, for a shared
    // prefix, prefix_lens (floored to whole blocks) with seq_lens as the rows' own limits
    const int* cu_q;
    const int* cu_k;
    const int* context_lens;
    const int* prefix_lens;
    const int* seq_lens;
    const int* block_table;  // [rows, max_blocks]
    int S, T, num_k, W, G, H, H_kv, causal;
    int block_size, max_blocks, num_blocks;
    float scale;
    // results
    __nv_bfloat16* O;
    float* LSE;  // [T, H] or null
    int64_t ldo;
    // scratch
    PackedHeader* hdr;
    int4* seqs;      // [S] {first token, tokens, keys, tile pairs before this sequence}
    int4* entries;   // [max_entries] {sequence, tile pair, first key block, key blocks}
    int* tile_first; // [max_tiles] first entry of a tile pair (cut ranges only)
    float* part_o;   // [slots][rows][D]
    float2* part_ml; // [slots][rows] {m in log2 units, l}
    int max_tiles, max_entries, slots, slot_rows;
    int sm_count;
    // shared prefix: the sequences' own tails, which the decode kernels of paged.cuh work on
    PagedParams tail;  // (its seq_lens and table_skip are written by the plan kernel)
    int* tail_lens;    // = tail.seq_lens
    int* tail_skip;    // = tail.table_skip
    int* tail_parts;   // [T, H_kv] partial results of a tail
};

__host__ __device__ __forceinline__ int packed_blocks(int keys) { return (keys + kMhaBlock - 1) / kMhaBlock; }

// Key blocks that tokens first .. first + n - 1 of a sequence (nq tokens, nk keys) see.
__device__ __forceinline__ int packed_tile_blocks(int nq, int nk, int causal, int first, int n) {
    if (n <= 0) return 0;
    const int last = causal ? nk - nq + first + n : nk;  // keys that the last of them sees
    return packed_blocks(max(0, last));
}

__device__ __forceinline__ void packed_report(unsigned int code, int a, int b, int c) {
    if (atomicCAS(&g_status[0], 0u, code) == 0u) {
        g_status[1] = static_cast<unsigned int>(a);
        g_status[2] = static_cast<unsigned int>(b);
        g_status[3] = static_cast<unsigned int>(c);
    }
}

// Tokens of a sequence and its keys; false (and no tokens) if they do not fit the call.
__device__ __forceinline__ bool packed_sequence(const PackedParams& p, int s, int& q0, int& nq, int& nk) {
    q0 = p.cu_q[s];
    const long long q1 = p.cu_q[s + 1];
    nq = 0;
    nk = 0;
    if (q0 < 0 || q1 < q0 || q1 > p.T) return false;
    long long keys;
    if (p.cu_k) {
        const long long k0 = p.cu_k[s], k1 = p.cu_k[s + 1];
        if (k0 < 0 || k1 < k0 || k1 > p.num_k) return false;
        keys = k1 - k0;
    } else {
        const long long most = static_cast<long long>(p.max_blocks) * p.block_size;
        if (p.prefix_lens) {
            keys = max(0ll, min(static_cast<long long>(p.prefix_lens[s]), most));
            keys -= keys % p.block_size;
        } else {
            keys = static_cast<long long>(p.context_lens[s]) + (q1 - q0);
            if (p.context_lens[s] < 0 || (q1 > q0 && keys > most)) return false;
        }
    }
    nq = static_cast<int>(q1 - q0);
    nk = static_cast<int>(keys);
    return true;
}

// The sequence that holds tile pair i: the last one with at most i pairs before it that has any.
__device__ __forceinline__ int packed_find_tile(const int4* seqs, int S, int i) {
    int lo = 0, hi = S;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (seqs[mid].w <= i) lo = mid; else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ int packed_bucket(int blocks) {  // monotone: exact below 512 blocks, then 64 steps per octave
    int key = blocks;
    if (blocks >= 512) {
        const int e = 31 - __clz(blocks);
        key = 512 + (e - 9) * 64 + ((blocks >> (e - 6)) & 63);
    }
    return kPackedBuckets - 1 - min(key, kPackedBuckets - 1);
}

// Inclusive scan over the CTA (1024 threads); `red` holds 32 words.  Ends with all threads past their use of `red`.
__device__ __forceinline__ int packed_scan(int v, int* red, int& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int w = 1; w < 32; w <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, v, w);
        if (lane >= w) v += o;
    }
    if (lane == 31) red[warp] = v;
    __syncthreads();
    int r = red[lane];
#pragma unroll
    for (int w = 1; w < 32; w <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, r, w);
        if (lane >= w) r += o;
    }
    total = __shfl_sync(0xffffffffu, r, 31);
    const int before = warp ? __shfl_sync(0xffffffffu, r, warp - 1) : 0;
    __syncthreads();
    return v + before;
}

// The group that sequence s is in, or -1; and the sequence's tokens behind the group's prefix.
__device__ __forceinline__ int packed_group(const PackedParams& p, int s, int& tail) {
    int lo = 0, hi = p.S;  // the last group that begins at or before s
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (p.cu_q[mid] <= s) lo = mid; else hi = mid;
    }
    const int4 q = p.seqs[lo];
    const int group = s >= q.x && s - q.x < q.y ? lo : -1;
    const long long most = static_cast<long long>(p.max_blocks) * p.block_size;
    const int len = static_cast<int>(max(0ll, min(static_cast<long long>(p.seq_lens[s]), most)));
    tail = max(0, len - (group >= 0 ? q.z : 0));
    return group;
}

// The tails behind the prefixes, and how many partial results the decode kernel makes of each (one CTA).
__device__ __forceinline__ void packed_plan_tails(const PackedParams& p, int* red) {
    const int tid = threadIdx.x;
    const int per = (p.T + kPackedPlanThreads - 1) / kPackedPlanThreads;
    const int lo = min(p.T, tid * per), hi = min(p.T, lo + per);
    int chunks = 0, most = 0;
    for (int s = lo; s < hi; ++s) {
        int tail;
        const int group = packed_group(p, s, tail);
        p.tail_lens[s] = tail;
        p.tail_skip[s] = group >= 0 ? p.seqs[group].z / p.block_size : 0;
        const int n = (tail + kPagedChunkTokens - 1) / kPagedChunkTokens;
        chunks += n;
        most = max(most, n);
    }
    int total;
    int before = packed_scan(chunks, red, total) - chunks;
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, w));
    if ((tid & 31) == 0) red[tid >> 5] = most;
    __syncthreads();
    for (int w = 0; w < 32; ++w) most = max(most, red[w]);
    __syncthreads();
    const int quota = paged_quota(static_cast<long long>(total) * p.H_kv, most, max(1, p.tail.balanced_ctas));
    for (int s = lo; s < hi; ++s) {
        const int tail = p.tail_lens[s];
        if (p.tail.balanced) {  // as in paged_decode_mma_kernel: pieces of `quota` chunks across all rows
            const int n = (tail + kPagedChunkTokens - 1) / kPagedChunkTokens;
            for (int h = 0; h < p.H_kv; ++h) {
                const long long start = static_cast<long long>(before) * p.H_kv + static_cast<long long>(h) * n;
                p.tail_parts[static_cast<int64_t>(s) * p.H_kv + h] = n > 0 ? static_cast<int>((start + n - 1) / quota - start / quota + 1) : 0;
            }
            before += n;
        } else {
            const int nblk = (tail + p.block_size - 1) / p.block_size, share = paged_split_blocks(p.tail, nblk);
            for (int h = 0; h < p.H_kv; ++h) p.tail_parts[static_cast<int64_t>(s) * p.H_kv + h] = (nblk + share - 1) / share;
        }
    }
}

// One CTA.  Sequences -> tile pairs -> work items.
__global__ void __launch_bounds__(kPackedPlanThreads) mha_packed_plan_kernel(const PackedParams p) {
    pdl_launch_dependents();
    __shared__ int red[32];
    __shared__ int hist[kPackedBuckets];
    __shared__ int blocks_of[kPackedMaxSplitTiles];
    __shared__ int best_sh, sum_sh;
    __shared__ unsigned long long pick_sh;
    const int tid = threadIdx.x;
    for (int i = tid; i < kPackedBuckets; i += kPackedPlanThreads) hist[i] = 0;
    if (tid == 0) { best_sh = 0; sum_sh = 0; pick_sh = ~0ull; }
    cudaGridDependencySynchronize();

    // sequences: tile pairs and their prefix sums
    const int W2 = 2 * p.W;
    const int per = (p.S + kPackedPlanThreads - 1) / kPackedPlanThreads;
    const int s_lo = min(p.S, tid * per), s_hi = min(p.S, s_lo + per);
    int mine = 0;
    for (int s = s_lo; s < s_hi; ++s) {
        int q0, nq, nk;
        packed_sequence(p, s, q0, nq, nk);
        mine += (nq + W2 - 1) / W2;
    }
    int tiles;
    int before = packed_scan(mine, red, tiles) - mine;
    for (int s = s_lo; s < s_hi; ++s) {
        int q0, nq, nk;
        bool ok = packed_sequence(p, s, q0, nq, nk);
        int n = (nq + W2 - 1) / W2;
        if (before > p.max_tiles - n) {  // more tokens than the call has: the offsets do not ascend
            ok = false;
            nq = n = 0;
        }
        if (!ok) packed_report(kStatusBadSequence, s, q0, nk);
        p.seqs[s] = make_int4(q0, nq, nk, before);
        before += n;
    }
    tiles = min(tiles, p.max_tiles);
    __syncthreads();

    // tile pairs: key blocks of each
    auto tile_of = [&](int i, int& s, int& pair) -> int {
        s = packed_find_tile(p.seqs, p.S, i);
        const int4 q = p.seqs[s];
        pair = i - q.w;
        const int first = pair * W2;
        return packed_tile_blocks(q.y, q.z, p.causal, first, min(W2, q.y - first));
    };
    const bool may_split = p.slots > 0 && tiles <= kPackedMaxSplitTiles;
    int most = 0, sum = 0;
    for (int i = tid; i < tiles; i += kPackedPlanThreads) {
        int s, pair;
        const int blocks = tile_of(i, s, pair);
        atomicAdd(&hist[packed_bucket(blocks)], 1);
        if (may_split) blocks_of[i] = blocks;
        most = max(most, blocks);
        sum += min(blocks, 1 << 20);
    }
    if (may_split) {
        atomicMax(&best_sh, most);
        atomicAdd(&sum_sh, sum);
    }
    __syncthreads();

    // Cut the key ranges?  Time in key blocks: an item of b blocks takes b + kItem (fill, drain, epilogue); whole ranges end with
    // the longest, or when the SMs have shared the sum; parts of at most c blocks run in rounds, and joining them costs kJoin.
    constexpr int kItem = 3, kJoin = 4;
    int chunk = 0;
    if (may_split) {
        const int longest = best_sh;
        if (longest > 1) {
            const int warp = tid >> 5, lane = tid & 31;
            for (int n = warp + 1; n <= 160 && n <= longest; n += kPackedPlanThreads / 32) {
                const int c = (longest + n - 1) / n;
                int parts = 0;
                for (int i = lane; i < tiles; i += 32) parts += max(1, (blocks_of[i] + c - 1) / c);
                parts = __reduce_add_sync(0xffffffffu, parts);
                const long long items = static_cast<long long>(max(parts, 1)) * p.H_kv;
                long long cost;
                if (n == 1 && !p.prefix_lens) {
                    const long long shared_out = (static_cast<long long>(sum_sh) * p.H_kv + kItem * items) / p.sm_count;
                    cost = max(static_cast<long long>(c + kItem), shared_out);
                } else {
                    cost = (items + p.sm_count - 1) / p.sm_count * (c + kItem) + kJoin;
                    if (items > p.slots) cost = 1ll << 40;
                }
                if (lane == 0) atomicMin(&pick_sh, (static_cast<unsigned long long>(cost) << 16) | static_cast<unsigned long long>(n));
            }
        }
        __syncthreads();
        const int n = pick_sh == ~0ull ? 1 : static_cast<int>(pick_sh & 0xffff);
        chunk = n == 1 ? 0 : (longest + n - 1) / n;
        if (p.prefix_lens && chunk == 0) chunk = max(1, longest);  // a prefix's results always go on to the join
    }

    int total;
    if (chunk > 0) {
        const int blocks = tid < tiles ? blocks_of[tid] : 0;
        const int parts = tid < tiles ? max(1, (blocks + chunk - 1) / chunk) : 0;
        const int first = packed_scan(parts, red, total) - parts;
        if (tid < tiles) {
            int s, pair;
            tile_of(tid, s, pair);
            p.tile_first[tid] = first;
            for (int k = 0; k < parts; ++k)
                if (first + k < p.max_entries) p.entries[first + k] = make_int4(s, pair, k * chunk, min(chunk, blocks - k * chunk));
        }
        total = min(total, p.max_entries);
    } else {
        // longest first: counting sort
        const int a = hist[2 * tid], b = hist[2 * tid + 1];
        const int end = packed_scan(a + b, red, total);
        __syncthreads();
        hist[2 * tid] = end - a - b;
        hist[2 * tid + 1] = end - b;
        __syncthreads();
        for (int i = tid; i < tiles; i += kPackedPlanThreads) {
            int s, pair;
            const int blocks = tile_of(i, s, pair);
            const int at = atomicAdd(&hist[packed_bucket(blocks)], 1);
            if (at < p.max_entries) p.entries[at] = make_int4(s, pair, 0, blocks);
        }
        total = tiles;
    }
    if (p.prefix_lens) packed_plan_tails(p, red);
    if (tid == 0) {
        p.hdr->num_items = total * p.H_kv;
        p.hdr->counter = 0;
        p.hdr->split = chunk;
    }
}

template <int D>
struct PackedSmem {
    static constexpr int kTileBytes = kMhaBlock * D * 2;
    static constexpr int kChunkBytes = kMhaBlock * 128;
    static constexpr int kStages = (D == 128) ? 4 : 8;
    static constexpr int kBarrierBytes = 512;
    static constexpr int kItemBytes = 2 * 48;
    static constexpr int kStageBytes = 8 * 4096;
    static constexpr int kTotal = 2 * kTileBytes + kStages * kTileBytes + kBarrierBytes + kItemBytes + kStageBytes + 1024;
};

struct PackedItem {  // 48 bytes in shared memory
    int valid;       // 0: no more items
    int tok0;        // first token of the pair (in the call's tokens)
    int ntok;        // tokens of the pair that belong to the sequence
    int kvh;
    int lim0;        // last visible key of token tok0 (causal: one more per token)
    int b0;          // first key block
    int J[2];        // key blocks of each tile from b0 on
    int slot;        // partial result, or -1: O and LSE are written
    int fix;         // rows of the last V tile to zero: first | (end << 8), or 0
    int pad[2];
};

template <int D>
__global__ void __launch_bounds__(kMhaThreads, 1)
mha_packed_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_k,
                  const __grid_constant__ CUtensorMap tmap_v, const PackedParams p) {
    using L = PackedSmem<D>;
    constexpr int kIssuers = (D == 64) ? 2 : 1;
    constexpr int kStages = L::kStages;
    constexpr int kChunks = D / 64;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* smem_q = smem;                                   // [2][tile]
    uint8_t* smem_kv = smem + 2 * L::kTileBytes;              // [kStages][tile]
    uint8_t* smem_stage = smem_kv + kStages * L::kTileBytes;  // [8 warps][4 KB]
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem_stage + L::kStageBytes);
    uint64_t* q_full = bars;                  // [1]
    uint64_t* kv_full = bars + 1;             // [kStages]
    uint64_t* kv_empty = kv_full + kStages;   // [kStages]
    uint64_t* s_full = kv_empty + kStages;    // [2]  UMMA -> softmax: S_t(j) complete
    uint64_t* p_full = s_full + 2;            // [2]  softmax -> UMMA: P_t(j) in TMEM, O_t rescaled
    uint64_t* o_full = p_full + 2;            // [2]  UMMA -> epilogue: O_t complete
    uint64_t* q_empty = o_full + 2;           // [1]  UMMA -> loader: the item's last Q K^T has read the Q tiles
    uint64_t* s_free = q_empty + 1;           // [2]  softmax -> UMMA (D = 64): S_t(j) is in registers
    uint64_t* p_free = s_free + 2;            // [2]  UMMA -> softmax (D = 64): P_t(j) V has completed
    uint64_t* item_full = p_free + 2;         // [2]  loader -> all: the item is in shared memory
    uint64_t* item_empty = item_full + 2;     // [2]  all -> loader: nobody needs the item any more
    uint64_t* v_fixed = item_empty + 2;       // [2]  spare warp -> UMMA: the item's last V tile has its tail zeroed
    uint64_t* v_asked = v_fixed + 2;          // [2]  loader -> spare warp: the item's last V tile has been requested
    uint32_t* tmem_base_slot = reinterpret_cast<uint32_t*>(v_asked + 2);
    volatile uint32_t* abort_flag = tmem_base_slot + 1;
    PackedItem* items = reinterpret_cast<PackedItem*>(reinterpret_cast<uint8_t*>(bars) + L::kBarrierBytes);
    static_assert(sizeof(PackedItem) == 48, "item slots");

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    pdl_launch_dependents();

    if (warp == 9 && lane == 0) {
        mbar_init(q_full, 1);
        mbar_init(q_empty, kIssuers);
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&kv_full[s], 1);
            mbar_init(&kv_empty[s], kIssuers);
        }
        for (int t = 0; t < 2; ++t) {
            mbar_init(&s_full[t], 1);
            mbar_init(&p_full[t], 4);
            mbar_init(&o_full[t], 1);
            mbar_init(&s_free[t], 4);
            mbar_init(&p_free[t], 1);
            mbar_init(&item_full[t], 1);
            mbar_init(&item_empty[t], 8 + kIssuers + 1);  // softmax warps, issuers, the warp that zeroes tails
            mbar_init(&v_fixed[t], 1);
            mbar_init(&v_asked[t], 1);
        }
        *abort_flag = 0;
        fence_mbar_init();
        prefetch_tensormap(&tmap_q);
        prefetch_tensormap(&tmap_k);
        prefetch_tensormap(&tmap_v);
    }
    if (warp == 8) {
        tmem_alloc(tmem_base_slot, 512);
        tmem_relinquish();
    }
    // rows that no token fills (128 - W * G of them): zero for good, so that their scores are finite
    {
        const int used = p.W * p.G;
        for (int i = threadIdx.x; i < (kMhaBlock - used) * 8 * 2 * kChunks; i += kMhaThreads) {
            const int piece = i & 7, row = used + (i >> 3) % (kMhaBlock - used), tile_chunk = (i >> 3) / (kMhaBlock - used);
            *reinterpret_cast<uint4*>(smem_q + tile_chunk * L::kChunkBytes + row * 128 + piece * 16) = make_uint4(0u, 0u, 0u, 0u);
        }
        fence_proxy_async_smem();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    cudaGridDependencySynchronize();  // the plan, and everything before it
    if (blockIdx.x == 0 && threadIdx.x == 0) clock_probe(1, 0);
    const uint32_t tmem_base = *tmem_base_slot;
    constexpr uint32_t kColS = 0;    // S_t at kColS + t*128
    constexpr uint32_t kColO = 256;  // O_t at kColO + t*D
    constexpr bool kEarlyQK = (D == 64);
    constexpr uint32_t kColP = kEarlyQK ? 384 : kColS;
    constexpr uint32_t kStrideP = kEarlyQK ? 64 : kMhaBlock;

    auto wait_all = [&](uint64_t* bar, uint32_t parity, uint32_t id) {
        return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, id)) != 0;
    };
    // item n of this CTA; false at the end of the list or after an aborted wait
    auto take_item = [&](int n, uint32_t id) -> bool {
        if (!wait_all(&item_full[n & 1], (n >> 1) & 1, id)) return false;
        return items[n & 1].valid != 0;
    };
    auto drop_item = [&](int n) {
        __syncwarp();
        if (lane == 0) mbar_arrive(&item_empty[n & 1]);
    };

    static_assert(8 * 32 * kMhaSoftmaxRegs + 4 * 32 * kMhaOtherRegs <= kMhaThreads * 168, "setmaxnreg budget exceeds the launch allocation");
    if (warp == 9) {
        // ------------------------------- loader and scheduler -------------------------------
        setmaxnreg_dec<kMhaOtherRegs>();
        const int num_items = p.hdr->num_items;
        const bool split = p.hdr->split != 0;
        const int chunk = p.hdr->split;
        const int W2 = 2 * p.W;
        const uint32_t q_bytes = static_cast<uint32_t>(p.W) * p.G * 128 * kChunks;  // per tile
        const int nb = p.cu_k ? 1 : kMhaBlock / p.block_size;                       // cache blocks per tile
        int ld_stage = 0;
        uint32_t ld_phase = 0;
        int q_loads = 0;
        bool ok = true;
        int idx = blockIdx.x;
        for (int n = 0; ok; ++n) {
            PackedItem it = {};
            int k_first = 0, trow = 0, nk = 0;
            if (idx < num_items) {
                const int4 e = p.entries[idx / p.H_kv];
                const int4 q = p.seqs[e.x];
                const int first = e.y * W2;
                it.valid = 1;
                it.kvh = idx % p.H_kv;
                it.tok0 = q.x + first;
                it.ntok = min(W2, q.y - first);
                nk = q.z;
                it.lim0 = p.causal ? nk - q.y + first : nk - 1;
                it.b0 = e.z;
#pragma unroll
                for (int t = 0; t < 2; ++t)
                    it.J[t] = min(max(packed_tile_blocks(q.y, nk, p.causal, first + t * p.W, min(p.W, it.ntok - t * p.W)) - e.z, 0), e.w);
                const bool parts = split && (p.prefix_lens || packed_tile_blocks(q.y, nk, p.causal, first, it.ntok) > chunk);
                it.slot = parts ? idx : -1;
                // V rows beyond the last key, up to the next cache block (the blocks after that load zeros)
                const int tail = nk % kMhaBlock;
                int tail_end = kMhaBlock;
                if (!p.cu_k) tail_end = (tail + p.block_size - 1) / p.block_size * p.block_size;
                const int Jm = max(it.J[0], it.J[1]);
                if (Jm > 0 && it.b0 + Jm == packed_blocks(nk) && tail != 0 && tail < tail_end) it.fix = tail | (tail_end << 8);
                if (p.cu_k) k_first = p.cu_k[e.x];
                trow = p.prefix_lens ? q.x : e.x;
            }
            if (n >= 2) {
                ok = wait_all(&item_empty[n & 1], ((n >> 1) - 1) & 1, 0x600);
                if (!ok) break;
            }
            if (lane == 0) {
                items[n & 1] = it;
                mbar_arrive(&item_full[n & 1]);
            }
            __syncwarp();
            if (!it.valid) break;
            const int Jmax = max(it.J[0], it.J[1]);

            // block-table entry of this lane's cache block of key block b, as a coordinate of the tensor map
            const int nblk = p.cu_k ? 0 : (nk + p.block_size - 1) / p.block_size;
            const int beyond = max(1, p.num_blocks * p.H_kv);  // loads zeros
            auto table_at = [&](int b) -> int {
                const int i = b * nb + lane % nb;
                return (b < it.b0 + Jmax && i < nblk) ? p.block_table[static_cast<int64_t>(trow) * p.max_blocks + i] : -1;
            };
            auto coord = [&](int b, int phys) -> int {
                if (phys >= 0 && phys < p.num_blocks) return phys * p.H_kv + it.kvh;
                if (b * nb + lane % nb < nblk && lane < nb) packed_report(kStatusBadBlock, b * nb + lane, trow, phys);
                return beyond;
            };
            int next_entry = p.cu_k ? 0 : table_at(it.b0);
            int z[2] = {0, 0};
            for (int i = 0; i < 2 * Jmax; ++i) {
                bool is_k = (i & 1) == 0;
                int blk = i >> 1;
                if (D == 64 && i > 0) {  // K_0, K_1, V_0, K_2, V_1, ..., V_{J-1}
                    if (i == 2 * Jmax - 1) {
                        is_k = false;
                        blk = Jmax - 1;
                    } else {
                        is_k = (i & 1) == 1;
                        blk = is_k ? (i + 1) >> 1 : (i >> 1) - 1;
                    }
                }
                if (i == 1) {  // Q: K_0 first, then the tiles once the previous item's last Q K^T has read them
                    if (q_loads > 0) {
                        ok = wait_all(q_empty, (q_loads - 1) & 1, 0x110);
                        if (!ok) break;
                    }
                    ++q_loads;
                    const int tiles = it.ntok > p.W ? 2 : 1;
                    if (lane == 0) mbar_arrive_expect_tx(q_full, tiles * q_bytes);
                    __syncwarp();
                    if (lane < tiles * kChunks) {
                        const int t = lane / kChunks, c = lane % kChunks;
                        tma_load_3d(smem_q + t * L::kTileBytes + c * L::kChunkBytes, &tmap_q, q_full, c * 64, it.kvh * p.G, it.tok0 + t * p.W);
                    }
                    __syncwarp();
                }
                ok = wait_all(&kv_empty[ld_stage], ld_phase ^ 1, 0x100 + ld_stage);
                if (!ok) break;
                uint8_t* dst = smem_kv + ld_stage * L::kTileBytes;
                if (lane == 0) mbar_arrive_expect_tx(&kv_full[ld_stage], L::kTileBytes);
                __syncwarp();
                const CUtensorMap* map = is_k ? &tmap_k : &tmap_v;
                const int b = it.b0 + blk;
                if (p.cu_k) {
                    if (lane < kChunks) tma_load_3d(dst + lane * L::kChunkBytes, map, &kv_full[ld_stage], lane * 64, it.kvh, k_first + b * kMhaBlock);
                } else {
                    if (is_k) {
                        const int zz = coord(b, next_entry);
                        if (blk & 1) z[1] = zz; else z[0] = zz;
                        next_entry = table_at(b + 1);
                    }
                    if (lane < nb * kChunks) {
                        const int c = lane / nb, piece = lane % nb;
                        tma_load_3d(dst + c * L::kChunkBytes + piece * p.block_size * 128, map, &kv_full[ld_stage], c * 64, 0, (blk & 1) ? z[1] : z[0]);
                    }
                }
                __syncwarp();
                if (++ld_stage == kStages) { ld_stage = 0; ld_phase ^= 1; }
            }
            if (!ok) break;
            if (it.fix && lane == 0) mbar_arrive(&v_asked[n & 1]);
            if (lane == 0) idx = static_cast<int>(gridDim.x) + atomicAdd(&p.hdr->counter, 1);
            idx = __shfl_sync(0xffffffffu, idx, 0);
        }
    } else if (warp == 8 || (warp == 10 && kIssuers == 2)) {
        // ------------------------------- UMMA issuer -------------------------------
        const int t_lo = (kIssuers == 2 && warp == 10) ? 1 : 0;
        const int t_hi = (kIssuers == 2 && warp == 8) ? 1 : 2;
        setmaxnreg_dec<kMhaOtherRegs>();
        const bool leader = elect_one();
        constexpr uint32_t idesc_qk = make_idesc_bf16(kMhaBlock, kMhaBlock, false, false);
        constexpr uint32_t idesc_pv = make_idesc_bf16(kMhaBlock, D, false, true);
        const uint32_t q_lo0 = sdesc_lo(smem_u32(smem_q), 16);
        const uint32_t kv_lo0 = sdesc_lo(smem_u32(smem_kv), 16);
        const uint32_t v_lbo = (static_cast<uint32_t>(L::kChunkBytes) >> 4) << 16;
        auto issue_qk = [&](int t, int slot) {
            const uint32_t d = tmem_base + kColS + t * kMhaBlock;
            const uint32_t a0 = q_lo0 + t * (L::kTileBytes >> 4);
            const uint32_t b0 = kv_lo0 + slot * (L::kTileBytes >> 4);
            if (leader) {
                umma_ss_lo<false>(d, a0, b0, idesc_qk);
#pragma unroll
                for (int kk = 1; kk < D / 16; ++kk) {
                    const uint32_t off = ((kk / 4) * L::kChunkBytes + (kk % 4) * 32) >> 4;
                    umma_ss_lo<true>(d, a0 + off, b0 + off, idesc_qk);
                }
                umma_commit(&s_full[t]);
            }
            __syncwarp();
        };
        auto issue_pv = [&](int t, int slot, bool first) {
            const uint32_t d = tmem_base + kColO + t * D;
            const uint32_t a0 = tmem_base + kColP + t * kStrideP;
            const uint32_t b0 = (kv_lo0 & 0xFFFFu) + slot * (L::kTileBytes >> 4) + v_lbo;
            if (leader) {
                umma_ts_lo(d, a0, b0, idesc_pv, first ? 0u : 1u);
#pragma unroll
                for (int kk = 1; kk < kMhaBlock / 16; ++kk)
                    umma_ts_lo(d, a0 + kk * 8, b0 + kk * (2048 >> 4), idesc_pv, 1u);
            }
            __syncwarp();
        };
        int stage = 0;
        uint32_t phase = 0;
        uint32_t n_p[2] = {0, 0}, n_qk[2] = {0, 0};
        uint32_t n_q = 0;                 // items with keys so far (parity of q_full)
        uint32_t fixed = 0;               // bit: parity of v_fixed of an item slot
        bool ok = true;
        for (int n = 0; ok && take_item(n, 0x210); ++n) {
            const PackedItem& it = items[n & 1];
            const int J0 = it.J[0], J1 = it.J[1], Jmax = max(J0, J1);
            if (Jmax > 0) {
                ok = wait_all(q_full, n_q & 1, 0x200);
                if (!ok) break;
                ++n_q;
            }
            const bool fix = it.fix != 0;
            const int fix_step = fix ? Jmax - 1 : -1;  // the step whose V tile has a tail
            if constexpr (kEarlyQK) {
                // Step j: Q_t K_{j+1}^T as soon as S_t(j) has been read, then P_t(j) V_j, for this warp's tile
#pragma unroll 1
                for (int j = -1; j < Jmax && ok; ++j) {
                    if (j + 1 < Jmax) {
                        const int kslot = stage;
                        ok = wait_all(&kv_full[kslot], phase, 0x240 + kslot);
                        if (!ok) break;
                        if (++stage == kStages) { stage = 0; phase ^= 1; }
                        tc_fence_after();
                        for (int t = t_lo; t < t_hi && ok; ++t) {
                            if (j + 1 >= (t ? J1 : J0)) continue;
                            if (n_qk[t] > 0) {
                                ok = wait_all(&s_free[t], (n_qk[t] - 1) & 1, 0x250 + t);
                                if (!ok) break;
                                tc_fence_after();
                            }
                            ++n_qk[t];
                            issue_qk(t, kslot);
                        }
                        if (!ok) break;
                        if (leader) {
                            umma_commit(&kv_empty[kslot]);
                            if (j + 2 == Jmax) umma_commit(q_empty);
                        }
                        __syncwarp();
                    }
                    if (j >= 0) {
                        const int vslot = stage;
                        ok = wait_all(&kv_full[vslot], phase, 0x220 + vslot);
                        if (!ok) break;
                        if (j == fix_step) {
                            ok = wait_all(&v_fixed[n & 1], (fixed >> (n & 1)) & 1, 0x260);
                            if (!ok) break;
                        }
                        if (++stage == kStages) { stage = 0; phase ^= 1; }
                        for (int t = t_lo; t < t_hi && ok; ++t) {
                            const int Jt = t ? J1 : J0;
                            if (j >= Jt) continue;
                            ok = wait_all(&p_full[t], n_p[t] & 1, 0x230 + t);
                            if (!ok) break;
                            ++n_p[t];
                            tc_fence_after();
                            issue_pv(t, vslot, j == 0);
                            if (leader) {
                                umma_commit(&p_free[t]);
                                if (j == Jt - 1) umma_commit(&o_full[t]);
                            }
                            __syncwarp();
                        }
                        if (!ok) break;
                        if (leader) umma_commit(&kv_empty[vslot]);
                        __syncwarp();
                    }
                }
            } else {
                // Step j issues P_t(j) V_j and then Q_t K_{j+1}^T for both tiles; step -1 only the first Q K^T products
#pragma unroll 1
                for (int j = -1; j < Jmax && ok; ++j) {
                    int vslot = 0;
                    if (j >= 0) {
                        vslot = stage;
                        ok = wait_all(&kv_full[vslot], phase, 0x220 + vslot);
                        if (!ok) break;
                        if (j == fix_step) {
                            ok = wait_all(&v_fixed[n & 1], (fixed >> (n & 1)) & 1, 0x260);
                            if (!ok) break;
                        }
                        if (++stage == kStages) { stage = 0; phase ^= 1; }
                    }
                    const int kslot = stage;  // K_{j+1}, if there is one
                    bool k_ready = false;
                    for (int t = 0; t < 2 && ok; ++t) {
                        const int Jt = t ? J1 : J0;
                        if (j >= 0 && j < Jt) {
                            ok = wait_all(&p_full[t], n_p[t] & 1, 0x230 + t);
                            if (!ok) break;
                            ++n_p[t];
                            tc_fence_after();
                            issue_pv(t, vslot, j == 0);
                            if (j == Jt - 1 && leader) umma_commit(&o_full[t]);
                        }
                        if (j + 1 < Jt) {
                            if (!k_ready) {
                                ok = wait_all(&kv_full[kslot], phase, 0x240 + kslot);
                                if (!ok) break;
                                tc_fence_after();
                                k_ready = true;
                            }
                            issue_qk(t, kslot);
                        }
                    }
                    if (!ok) break;
                    if (leader) {
                        if (j >= 0) umma_commit(&kv_empty[vslot]);
                        if (j + 1 < Jmax) umma_commit(&kv_empty[kslot]);
                        if (j + 2 == Jmax) umma_commit(q_empty);
                    }
                    __syncwarp();
                    if (j + 1 < Jmax) {
                        if (++stage == kStages) { stage = 0; phase ^= 1; }
                    }
                }
            }
            if (!ok) break;
            if (fix) fixed ^= 1u << (n & 1);
            drop_item(n);
        }
    } else if (warp == 11 || warp == 10) {
        setmaxnreg_dec<kMhaOtherRegs>();
        if (warp == 11) {
            // ------------------------------- zeroes the tail of V -------------------------------
            uint32_t pos = 0;    // ring tiles of all items before
            uint32_t fixed = 0;  // bit: parity of v_asked of an item slot
            for (int n = 0; take_item(n, 0x720); ++n) {
                const PackedItem& it = items[n & 1];
                const int Jmax = max(it.J[0], it.J[1]);
                pos += 2 * Jmax;
                if (it.fix) {  // the item's last ring tile is its last V tile
                    // (a barrier's parity says something only about the phase that is under way and the one before it: the stage's
                    // earlier uses are over once the loader has requested this one)
                    const uint32_t last = pos - 1, stage = last % kStages;
                    if (!wait_all(&v_asked[n & 1], (fixed >> (n & 1)) & 1, 0x700)) break;
                    fixed ^= 1u << (n & 1);
                    if (!wait_all(&kv_full[stage], (last / kStages) & 1, 0x710)) break;
                    const int first = it.fix & 255, pieces = ((it.fix >> 8) - first) * 8;
                    uint8_t* tile = smem_kv + stage * L::kTileBytes + first * 128;
                    for (int i = lane; i < pieces; i += 32)
#pragma unroll
                        for (int c = 0; c < kChunks; ++c)
                            *reinterpret_cast<uint4*>(tile + c * L::kChunkBytes + i * 16) = make_uint4(0u, 0u, 0u, 0u);
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&v_fixed[n & 1]);
                }
                drop_item(n);
            }
        }
    } else {
        // ------------------- softmax, O rescale and epilogue of tile t -------------------
        setmaxnreg_inc<kMhaSoftmaxRegs>();
        const int t = warp >> 2;
        const int quarter = warp & 3;
        const int row_in_tile = quarter * 32 + lane;
        const int row_tok = row_in_tile / p.G, row_head = row_in_tile % p.G;  // (rows from W * G on belong to no token)
        const uint32_t lane_addr = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16);
        const uint32_t s_addr = lane_addr + kColS + t * kMhaBlock;
        const uint32_t o_addr = lane_addr + kColO + t * D;
        const uint32_t p_addr = lane_addr + kColP + t * kStrideP;
        const float c = p.scale * kLog2e;
        uint8_t* stage_o = smem_stage + warp * 4096;
        uint32_t n_s = 0, n_o = 0;
        bool ok = true;
        for (int n = 0; ok && take_item(n, 0x320); ++n) {
            const PackedItem& it = items[n & 1];
            const int tile_tok = it.ntok - t * p.W;  // tokens of this tile, if positive
            if (tile_tok <= 0) {
                drop_item(n);
                continue;
            }
            const int Jt = it.J[t], first_block = it.b0;
            // last visible key; rows without a token take the last token's, so that they mask no more than their neighbours
            int limit = it.lim0;
            if (p.causal) limit += t * p.W + min(row_tok, min(tile_tok, p.W) - 1);
            if (p.seq_lens && row_tok < tile_tok) limit = min(limit, p.seq_lens[it.tok0 + t * p.W + min(row_tok, p.W - 1)] - 1);
            float m_run = -INFINITY, l_run = 0.0f;

            for (int j = 0; j < Jt; ++j) {
                ok = wait_all(&s_full[t], n_s & 1, 0x300 + t);
                if (!ok) break;
                ++n_s;
                tc_fence_after();
                uint32_t s[4][32];  // this thread's row of S
#pragma unroll
                for (int q = 0; q < 4; ++q) tmem_ld_32x32b_x32(s_addr + q * 32, s[q]);
                tmem_wait_ld();
                if constexpr (kEarlyQK) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&s_free[t]);
                }
                const int j0 = (first_block + j) * kMhaBlock;
                if (j0 + kMhaBlock - 1 > limit) {
#pragma unroll
                    for (int q = 0; q < 4; ++q)
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (j0 + q * 32 + i > limit) s[q][i] = 0xFF800000u;  // -inf
                }
                float2 acc0, acc1;
                auto row_max = [&]() {
                    float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int q = 0; q < 4; ++q)
#pragma unroll
                        for (int i = 0; i < 32; i += 4)
                            mx[(i >> 2) & 3] = fmaxf(mx[(i >> 2) & 3],
                                                     fmaxf(fmaxf(__uint_as_float(s[q][i]), __uint_as_float(s[q][i + 1])),
                                                           fmaxf(__uint_as_float(s[q][i + 2]), __uint_as_float(s[q][i + 3]))));
                    return fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
                };
                auto exp_pass = [&](float neg_mc) {
                    constexpr int kPolyMask = (D == 64) ? MLT_POLY_MASK_64 : MLT_POLY_MASK_128;
                    const float2 c2 = make_float2(c, c), n2 = make_float2(neg_mc, neg_mc);
                    const float cs = c * (1.0f / kPolySpan), ns = (neg_mc + kPolyLow) * (1.0f / kPolySpan);
                    acc0 = make_float2(0.0f, 0.0f);
                    acc1 = make_float2(0.0f, 0.0f);
                    uint32_t pk[16];
                    auto exp_pair = [&](int k, bool poly) {
                        const float s0 = __uint_as_float(s[k >> 5][k & 31]), s1 = __uint_as_float(s[k >> 5][(k & 31) + 1]);
                        if (poly) return exp2_poly2(s0, s1, cs, ns);
                        float2 x = ffma2(make_float2(s0, s1), c2, n2);
                        x.x = fast_exp2(x.x);
                        x.y = fast_exp2(x.y);
                        return x;
                    };
#pragma unroll
                    for (int w = 0; w < 8; ++w) {
#pragma unroll
                        for (int i = 0; i < 8; i += 2) {
                            const int k = w * 16 + 2 * i;
                            const float2 x0 = exp_pair(k, (kPolyMask >> i) & 1);
                            const float2 x1 = exp_pair(k + 2, (kPolyMask >> (i + 1)) & 1);
                            acc0 = fadd2(acc0, x0);
                            acc1 = fadd2(acc1, x1);
                            pk[(w & 1) * 8 + i] = pack_bf16x2(x0.x, x0.y);
                            pk[(w & 1) * 8 + i + 1] = pack_bf16x2(x1.x, x1.y);
                        }
                        if (kEarlyQK && w == 1 && n_s > 1) {
                            if (!wait_all(&p_free[t], n_s & 1, 0x310 + t)) ok = false;
                            tc_fence_after();
                        }
                        if (w & 1) tmem_st_32x32b_x16(p_addr + (w >> 1) * 16, pk);
                    }
                };
                if (j == 0) m_run = row_max();
                exp_pass((m_run == -INFINITY) ? 0.0f : -m_run * c);
                if (j > 0) {
                    const float blk = (acc0.x + acc0.y) + (acc1.x + acc1.y);
                    const bool moved = !(blk < kRescaleLimit);
                    if (__any_sync(0xffffffffu, moved)) {  // rare: a new reference maximum (see mha.cuh for why O_t may be rewritten here)
                        float alpha = 1.0f;
                        if (moved) {
                            const float mxr = fmaxf(row_max(), m_run);
                            alpha = m_run == -INFINITY ? 0.0f : fast_exp2((m_run - mxr) * c);
                            m_run = mxr;
                        }
#pragma unroll 1
                        for (int q = 0; q < D / 16; ++q) {
                            uint32_t o[16];
                            tmem_ld_32x32b_x16(o_addr + q * 16, o);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
                            tmem_st_32x32b_x16(o_addr + q * 16, o);
                        }
                        l_run *= alpha;
                        exp_pass((m_run == -INFINITY) ? 0.0f : -m_run * c);
                    }
                }
                if (!ok) break;
                l_run += (acc0.x + acc0.y) + (acc1.x + acc1.y);
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&p_full[t]);
            }
            if (!ok) break;
            if (Jt > 0) {
                ok = wait_all(&o_full[t], n_o & 1, 0x400 + t);
                if (!ok) break;
                ++n_o;
                tc_fence_after();
            }
            // Rows leave in pieces of 128 bytes: each thread puts its row's piece into the warp's staging area (16-byte chunk k of
            // row r at chunk k ^ (r & 7): no bank conflicts either way), then eight lanes at a time write a row's piece.
            auto put = [&](int k, uint32_t a, uint32_t b, uint32_t c2, uint32_t d) {
                *reinterpret_cast<uint4*>(stage_o + lane * 128 + ((k ^ (lane & 7)) * 16)) = make_uint4(a, b, c2, d);
            };
            auto send = [&](uint64_t dst) {  // dst: where this thread's row's piece goes, 0: nowhere
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int row = i * 4 + (lane >> 3), k = lane & 7;
                    const uint64_t to = __shfl_sync(0xffffffffu, dst, row);
                    const uint4 v = *reinterpret_cast<const uint4*>(stage_o + row * 128 + ((k ^ (row & 7)) * 16));
                    if (to) *reinterpret_cast<uint4*>(to + k * 16) = v;
                }
                __syncwarp();
            };
            const bool seen = m_run != -INFINITY;
            const bool valid = row_tok < min(it.ntok - t * p.W, p.W);
            const int tok = it.tok0 + t * p.W + row_tok, head = it.kvh * p.G + row_head;
            if (it.slot < 0) {
                const float inv_l = seen ? __fdividef(1.0f, l_run) : 0.0f;
                const uint64_t row_at = valid ? reinterpret_cast<uint64_t>(p.O + static_cast<int64_t>(tok) * p.ldo + head * D) : 0;
#pragma unroll 1
                for (int h = 0; h < D / 32; ++h) {  // 32 columns: half a piece
                    uint32_t o[32];
                    if (Jt > 0) {
                        tmem_ld_32x32b_x32(o_addr + h * 32, o);
                        tmem_wait_ld();
                    }
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        uint32_t w[4] = {0u, 0u, 0u, 0u};
                        if (Jt > 0 && seen) {
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                w[e] = pack_bf16x2(__uint_as_float(o[8 * k + 2 * e]) * inv_l, __uint_as_float(o[8 * k + 2 * e + 1]) * inv_l);
                        }
                        put((h & 1) * 4 + k, w[0], w[1], w[2], w[3]);
                    }
                    if (h & 1) send(row_at ? row_at + (h >> 1) * 128 : 0);
                }
                if (valid && p.LSE)
                    p.LSE[static_cast<int64_t>(tok) * p.H + head] = seen ? m_run * p.scale + __log2f(l_run) * 0.6931471805599453f : -INFINITY;
            } else if (Jt > 0) {
                const int64_t row = static_cast<int64_t>(it.slot) * p.slot_rows + t * kMhaBlock + row_in_tile;
                const uint64_t row_at = valid ? reinterpret_cast<uint64_t>(p.part_o + row * D) : 0;
#pragma unroll 1
                for (int h = 0; h < D / 32; ++h) {
                    uint32_t o[32];
                    tmem_ld_32x32b_x32(o_addr + h * 32, o);
                    tmem_wait_ld();
#pragma unroll
                    for (int k = 0; k < 8; ++k) put(k, o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]);
                    send(row_at ? row_at + h * 128 : 0);
                }
                if (valid) p.part_ml[row] = make_float2(seen ? m_run * c : -INFINITY, seen ? l_run : 0.0f);
            }
            drop_item(n);
        }
    }

    // common exit: every role reaches this, also after an aborted wait
    tc_fence_before();
    __syncthreads();
    if (blockIdx.x == 0 && threadIdx.x == 0) clock_probe(1, 1);
    if (warp == 8) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc(tmem_base, 512);
    }
}

// Joins the parts of cut key ranges, and of tails behind a shared prefix: one warp per (token, head).
constexpr int kPackedJoinWarps = 8;
template <int D>
__global__ void __launch_bounds__(kPackedJoinWarps * 32) mha_packed_join_kernel(const PackedParams p) {
    pdl_launch_dependents();
    constexpr int V = D / 32;  // elements per lane
    cudaGridDependencySynchronize();
    const int chunk = p.hdr->split;
    if (chunk == 0) return;
    const int lane = threadIdx.x & 31;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * kPackedJoinWarps + (threadIdx.x >> 5);
    if (row >= static_cast<int64_t>(p.T) * p.H) return;
    const int tok = static_cast<int>(row / p.H), h = static_cast<int>(row % p.H);
    int lo = 0, hi = p.S;  // the last sequence that begins at or before the token
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (p.cu_q[mid] <= tok) lo = mid; else hi = mid;
    }
    const int4 q = p.seqs[lo];
    const int i = tok - q.x;
    int parts = 0;
    int64_t part0 = 0;
    if (i >= 0 && i < q.y) {
        const int W2 = 2 * p.W, pair = i / W2, first = pair * W2, t = (i - first) / p.W;
        const int n = min(W2, q.y - first);
        // a range that is not cut was written by its item
        if (!p.prefix_lens && packed_tile_blocks(q.y, q.z, p.causal, first, n) <= chunk) return;
        const int blocks = packed_tile_blocks(q.y, q.z, p.causal, first + t * p.W, min(p.W, n - t * p.W));
        parts = (blocks + chunk - 1) / chunk;
        const int r = t * kMhaBlock + (i - first - t * p.W) * p.G + h % p.G;
        part0 = (static_cast<int64_t>(p.tile_first[q.w + pair]) * p.H_kv + h / p.G) * p.slot_rows + r;
    } else if (!p.prefix_lens) {
        return;  // a token of no sequence
    }
    const int64_t step = static_cast<int64_t>(p.H_kv) * p.slot_rows;
    const int tails = p.prefix_lens ? p.tail_parts[static_cast<int64_t>(tok) * p.H_kv + h / p.G] : 0;
    const int all = parts + tails;
    const int64_t tail0 = row * p.tail.splits;
    auto stat = [&](int k) { return k < parts ? p.part_ml[part0 + k * step] : p.tail.part_ml[tail0 + k - parts]; };
    float m = -INFINITY;
    for (int k = lane; k < all; k += 32) m = fmaxf(m, stat(k).x);
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, w));
    float l = 0.0f, o[V] = {};
    for (int k0 = 0; k0 < all; k0 += 32) {
        float weight = 0.0f;
        if (k0 + lane < all) {
            const float2 ml = stat(k0 + lane);
            weight = ml.x == -INFINITY ? 0.0f : fast_exp2(ml.x - m);
            l += weight * ml.y;
        }
        for (int k = 0; k < 32 && k0 + k < all; ++k) {
            const float w = __shfl_sync(0xffffffffu, weight, k);
            if (w == 0.0f) continue;  // (a part without a visible key)
            const float* src = (k0 + k < parts ? p.part_o + (part0 + (k0 + k) * step) * D : p.tail.part_o + (tail0 + k0 + k - parts) * D) + lane * V;
#pragma unroll
            for (int e = 0; e < V; ++e) o[e] = fmaf(src[e], w, o[e]);
        }
    }
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) l += __shfl_xor_sync(0xffffffffu, l, w);
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    uint32_t packed[V / 2];
#pragma unroll
    for (int e = 0; e < V / 2; ++e) packed[e] = pack_bf16x2(o[2 * e] * inv, o[2 * e + 1] * inv);
    __nv_bfloat16* dst = p.O + static_cast<int64_t>(tok) * p.ldo + h * D + lane * V;
#pragma unroll
    for (int e = 0; e < V / 2; ++e) reinterpret_cast<uint32_t*>(dst)[e] = packed[e];
    if (lane == 0 && p.LSE) p.LSE[row] = l > 0.0f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
}

// Scratch: header, sequences, entries, first entries, partial results.
struct PackedScratch {
    size_t seqs, entries, tile_first, part_ml, part_o;  // byte offsets
    size_t lists;                                       // bytes without partial results
    size_t slot_bytes;
    int64_t slots;                                      // parts that scratch is sized for
    int max_tiles, max_entries, slot_rows, W;
};
inline PackedScratch packed_scratch(int64_t T, int64_t S, int G, int H_kv, int D, bool prefix = false) {
    PackedScratch x;
    auto up = [](size_t v) { return (v + 255) & ~size_t(255); };
    x.W = kMhaBlock / G;
    const int64_t tiles = T / (2 * x.W) + S;
    x.max_tiles = static_cast<int>(tiles);
    x.slots = prefix ? std::max<int64_t>(kPackedMaxSlots, tiles * H_kv) : kPackedMaxSlots;  // (a prefix's results all go to the join)
    x.max_entries = static_cast<int>(std::max<int64_t>(tiles, x.slots / H_kv));
    x.slot_rows = static_cast<int>(T * G <= kMhaBlock ? T * G : 2 * kMhaBlock);
    x.seqs = 256;
    x.entries = up(x.seqs + static_cast<size_t>(S) * 16);
    x.tile_first = up(x.entries + static_cast<size_t>(x.max_entries) * 16);
    x.lists = up(x.tile_first + static_cast<size_t>(std::min<int64_t>(tiles, kPackedMaxSplitTiles)) * 4);
    x.slot_bytes = static_cast<size_t>(x.slot_rows) * (static_cast<size_t>(D) * 4 + 8);
    return x;
}

inline int packed_configure() {  // as mha_configure: 0, 1 (a CUDA call failed), 2 (too few registers for the hand-over)
    if (cudaFuncSetAttribute(mha_packed_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, PackedSmem<64>::kTotal) != cudaSuccess ||
        cudaFuncSetAttribute(mha_packed_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, PackedSmem<128>::kTotal) != cudaSuccess)
        return 1;
    cudaFuncAttributes a64, a128;
    if (cudaFuncGetAttributes(&a64, mha_packed_kernel<64>) != cudaSuccess || cudaFuncGetAttributes(&a128, mha_packed_kernel<128>) != cudaSuccess)
        return 1;
    return a64.numRegs < kMhaMinRegsPerThread || a128.numRegs < kMhaMinRegsPerThread ? 2 : 0;
}

template <class... Params, class... Args>
inline bool packed_launch_one(void (*kernel)(Params...), int64_t grid, int threads, int smem, cudaStream_t st, Args&&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(grid));
    cfg.blockDim = dim3(static_cast<unsigned>(threads));
    cfg.dynamicSmemBytes = static_cast<size_t>(smem);
    cfg.stream = st;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...) == cudaSuccess;
}

// plan, (behind a shared prefix: the tails,) attention, and (where key ranges may be cut) the join
template <int D>
int packed_launch(const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const PackedParams& p, cudaStream_t st) {
    if (!packed_launch_one(mha_packed_plan_kernel, 1, kPackedPlanThreads, 0, st, p)) return 4;
    if (p.prefix_lens) {
        const int rc = paged_launch_g<D>(p.tail, st);
        if (rc != 0) return rc;
    }
    const int64_t most = static_cast<int64_t>(p.slots > 0 ? p.max_entries : p.max_tiles) * p.H_kv;
    if (!packed_launch_one(mha_packed_kernel<D>, std::min<int64_t>(p.sm_count, most), kMhaThreads, PackedSmem<D>::kTotal, st, tq, tk, tv, p)) return 4;
    if (p.slots > 0) {
        const int64_t rows = static_cast<int64_t>(p.T) * p.H;
        if (!packed_launch_one(mha_packed_join_kernel<D>, (rows + kPackedJoinWarps - 1) / kPackedJoinWarps, kPackedJoinWarps * 32, 0, st, p)) return 4;
    }
    return 0;
}

}  // namespace mlt
