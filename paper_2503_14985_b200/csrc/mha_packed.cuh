// Attention of whole prompts, for sequences of different lengths packed one behind another and grouped heads:
//   row (token i of sequence s, head h) sees keys j <= lim(i);  p_j = exp(scale q.k_j - m),  O = sum p_j v_j / sum p_j.
// Keys come from packed rows or from the paged cache.  Decode of a batch with shared prefixes is the same problem: each group of
// sequences is one "sequence" whose tokens are the group's queries and whose keys are the prefix, and each query has a second one for
// the keys behind the prefix; the two are joined.
//
// The softmax core is that of mha.cuh (two 128-row tiles that take turns on the tensor pipe, one thread per row, running
// reference maximum, P through tensor memory; its comments give the reasons).  What differs:
//  * Rows.  The G query heads of a KV head are rows of one tile: row r is token r / G, head r % G, W = 128 / G tokens per
//    tile (G that do not divide 128 leave up to G - 1 rows unused).  A few tokens of many heads then fill a tile, and K and V are
//    read once for all G heads.  The Q tile is one TMA box [64 of D, G heads, W tokens] (one token, where there is one).
//  * Work.  Lengths are on the device, so a one-CTA kernel writes the list of work items (two tiles of a sequence, a range of
//    key blocks), longest first, and persistent CTAs (one per SM) draw from it by an atomic counter.  The loading warp draws
//    the next item while it requests the current one's keys, so the list's latency hides behind the ring.  A call of one short
//    sequence with an SM for each item needs no list: 37 tokens of 32 heads take 10.3 us without the plan kernel, 13.5 with it.
//  * Few rows.  With too few items for the SMs (few tokens behind a long context) the plan cuts the key range, and where the rows
//    fill one tile only, both tiles work on them, each on every other key block ("dual": 128 keys then take 1600 clocks instead of
//    3000, the latency of one tile's chain S -> softmax -> P V; at the copy bandwidth an SM gets 128 keys in 2800).  The parts go to
//    scratch as FP32 {m, l, O} and a second kernel joins them.  Warps without a valid row leave the exponentials out.
//  * Keys from the cache.  One lane per (cache block, 64 columns) issues its own TMA box, so a 128-key tile is one table load
//    and one issue for the warp.  A block-table entry out of range loads zeros (coordinate beyond the tensor map) and is
//    reported.  Rows beyond the sequence's last key may hold anything (another sequence, stale cache): scores there are
//    masked, and a spare warp zeroes those rows of V in shared memory, because a weight of 0 must not meet a NaN.
//  * Output rows of a tile may belong to a sequence only in part.  A warp whose 32 rows are all valid sends them as a TMA box
//    through shared memory, any other as 16-byte stores (eight lanes per 128-byte piece of a row): the epilogue took 4500 to
//    5200 clocks with plain stores alone, 3200 with boxes.
// Measured (32 heads over 8, D = 128, device time in graphs): 4 prompts of 4k to 8k, causal, 1090 to 1270 us (1.0 to 1.2 PFLOP/s; a pair
// of 128-row blocks takes 3250 clocks, 2048 of them products); 8 of 500 to 1500 102 us (720 TFLOP/s, tensor pipe 38 %, exponential unit
// 37 %); 24 sequences of 100 to 1024 with D = 64 173 us (360 TFLOP/s).  Behind long contexts the bytes of the cache bound it: 32 x 5 tokens,
// 32 heads over 4, 2k to 4k 77 us, 2.5 TB/s over the call, of which plan, first latencies, last parts and join are about 25 us.
#pragma once

#include <utility>

#include "mha.cuh"
#include "paged.cuh"

namespace mlt {

constexpr unsigned int kStatusBadSequence = 9;  // a sequence's offsets or positions lie outside the call's tokens or keys
constexpr int kPackedPlanThreads = 1024;
constexpr int kPackedBuckets = 2048;
constexpr int kPackedSeqs = 1024;        // sequences that the plan keeps in shared memory (more are read back from scratch)
constexpr int kPackedMaxTiles = 1 << 20;  // tile pairs of a call, so that 1024 threads' sums of that many fit 32 bits
constexpr int kPackedMaxKeys = INT32_MAX - 127;  // keys that a block table's row spans, so that positions in whole key blocks fit 32 bits
constexpr int kPackedSplitTiles = 4096;  // key ranges are cut only when there are no more tile pairs than this
constexpr int kPackedSplitRows = 320 * 2 * kMhaBlock;  // rows of partial results that scratch is sized for (and see packed_scratch)

struct alignas(16) PackedHeader {  // at the front of the scratch memory, written by the plan kernel
    int num_items;     // entries * H_kv
    int counter;       // items handed out beyond the first one of each CTA
    int split;         // key blocks per part, 0: no range is cut
    int irregular;     // a sequence is left out: the offsets need not ascend
};

struct PackedParams {
    // lengths (device): cu_q [S + 1] token offsets; keys per sequence from cu_k (packed), context_lens (paged) or, for shared
    // prefixes, prefix_lens (floored to whole blocks) and seq_lens
    const int* cu_q;
    const int* cu_k;
    const int* context_lens;
    const int* prefix_lens;
    const int* seq_lens;
    const int* block_table;  // [rows, max_blocks]
    int S;                   // sequences (shared prefixes: groups)
    int all;                 // S, and with shared prefixes the T tails behind them
    int T, num_k, W, G, H, H_kv, causal;
    int block_size, max_blocks, num_blocks;
    float scale;
    // results
    __nv_bfloat16* O;
    float* LSE;  // [T, H] or null
    int64_t ldo;
    // scratch
    PackedHeader* hdr;
    int4* seqs;           // [all] {first token, tokens, keys, tile pairs before this sequence}
    long long* key_base;  // [all] first key row (packed) or block-table index (paged)
    int4* entries;        // [max_entries] {sequence, tile pair, first key block, key blocks}
    int* entry_rows;      // [max_entries] first row of the entry's partial results (of KV head 0)
    int2* tile_info;      // [max_tiles] that of a tile pair's first entry, and the pair's entries
    float* part_o;        // [part_rows][D]
    float2* part_ml;      // [part_rows] {m in log2 units, l}
    int max_tiles, max_entries, part_rows;
    int sm_count;
    int single;  // one sequence, no cut ranges, an SM for each item: the items follow from its lengths, without a plan
    int boxes;  // the output tensor maps exist: whole warps' rows leave as TMA boxes (H / H_kv divides 32)
};

__host__ __device__ __forceinline__ int packed_blocks(int keys) { return (keys + kMhaBlock - 1) / kMhaBlock; }

// Key blocks that tokens first .. first + n - 1 of a sequence (nq tokens, nk keys) see.
__device__ __forceinline__ int packed_tile_blocks(int nq, int nk, int causal, int first, int n) {
    if (n <= 0) return 0;
    const int last = causal ? nk - nq + first + n : nk;  // keys that the last of them sees
    return packed_blocks(max(0, last));
}
// Rows of partial results of a tile pair with n tokens, per part and KV head: two tiles, or one tile's rows twice.
__device__ __forceinline__ int packed_part_rows(const PackedParams& p, int n) { return n <= p.W ? 2 * n * p.G : 2 * kMhaBlock; }

__device__ __forceinline__ void packed_report(unsigned int code, int a, int b, int c) {
    if (atomicCAS(&g_status[0], 0u, code) == 0u) {
        g_status[1] = static_cast<unsigned int>(a);
        g_status[2] = static_cast<unsigned int>(b);
        g_status[3] = static_cast<unsigned int>(c);
    }
}

// Tokens {first, count, keys} of a sequence and where its keys begin; false (and no tokens) if they do not fit the call.
__device__ __forceinline__ bool packed_sequence(const PackedParams& p, int s, int3& q, long long& base) {
    q.x = p.cu_q[s];
    const long long q1 = p.cu_q[s + 1];
    q.y = 0;
    q.z = 0;
    base = 0;
    if (q.x < 0 || q1 < q.x || q1 > p.T) return false;
    long long keys;
    if (p.cu_k) {
        const long long k0 = p.cu_k[s], k1 = p.cu_k[s + 1];
        if (k0 < 0 || k1 < k0 || k1 > p.num_k) return false;
        keys = k1 - k0;
        base = k0;
    } else {
        const long long most = static_cast<long long>(p.max_blocks) * p.block_size;
        if (p.prefix_lens) {
            keys = max(0ll, min(static_cast<long long>(p.prefix_lens[s]), most));
            keys -= keys % p.block_size;
            base = static_cast<long long>(q.x) * p.max_blocks;  // the group's first sequence
        } else {
            keys = static_cast<long long>(p.context_lens[s]) + (q1 - q.x);
            if (p.context_lens[s] < 0 || (q1 > q.x && keys > most)) return false;
            base = static_cast<long long>(s) * p.max_blocks;
        }
    }
    q.y = static_cast<int>(q1 - q.x);
    q.z = static_cast<int>(keys);
    return true;
}

// The group (or sequence) that token t is in, or -1.
__device__ __forceinline__ int packed_owner(const int* cu_q, int S, int t) {
    if (S == 0) return -1;
    int lo = 0, hi = S;  // the last one that begins at or before the token
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (cu_q[mid] <= t) lo = mid; else hi = mid;
    }
    return cu_q[lo] <= t && t < cu_q[lo + 1] ? lo : -1;
}

// The same by a whole warp: 33 parts per step instead of two.
__device__ __forceinline__ int packed_owner_warp(const PackedParams& p, int t) {
    if (p.S == 0) return -1;
    const int lane = threadIdx.x & 31;
    int lo = 0, hi = p.S;  // cu_q[lo] <= t (or lo = 0), cu_q[hi] > t (or hi = S)
    while (hi - lo > 1) {
        const int step = max(1, (hi - lo + 32) / 33), at = lo + (lane + 1) * step;
        const unsigned int below = __ballot_sync(0xffffffffu, at < hi && p.cu_q[at] <= t);
        const int n = below ? 32 - __clz(below) : 0;  // (sorted: the lanes below are the first n)
        hi = min(hi, lo + (n + 1) * step);
        lo += n * step;
    }
    return p.cu_q[lo] <= t && t < p.cu_q[lo + 1] ? lo : -1;
}

// The same where offsets need not ascend, so that no search by halves finds what is kept: behind shared prefixes (cu_q given) what the plan
// gave the token's tail, else the first sequence that is kept and has the token.  (A call of its own, and not with all parameters, which it
// would put on the stack: the join of 32 x 5 tokens took 5 us longer.)
__device__ __noinline__ int packed_owner_any(const int* cu_q, const int4* seqs, int S, int t) {
    if (cu_q) return packed_owner(cu_q, S, t);
    for (int s0 = 0; s0 < S; s0 += 32) {
        const int s = s0 + static_cast<int>(threadIdx.x & 31);
        const int4 q = s < S ? seqs[s] : make_int4(0, 0, 0, 0);
        const unsigned int has = __ballot_sync(0xffffffffu, q.x <= t && t - q.x < q.y);
        if (has) return s0 + __ffs(has) - 1;
    }
    return -1;
}

// The keys of decoded sequence t behind its group's prefix.
__device__ __forceinline__ void packed_tail(const PackedParams& p, int t, int3& q, long long& base) {
    int3 g;
    long long unused;
    const int group = packed_owner(p.cu_q, p.S, t);
    const int prefix = group >= 0 && packed_sequence(p, group, g, unused) ? g.z : 0;
    const long long most = static_cast<long long>(p.max_blocks) * p.block_size;
    const int len = static_cast<int>(max(0ll, min(static_cast<long long>(p.seq_lens[t]), most)));
    q.x = t;
    q.z = max(0, len - prefix);
    q.y = q.z > 0 ? 1 : 0;
    base = static_cast<long long>(t) * p.max_blocks + prefix / p.block_size;
}

__device__ __forceinline__ int packed_bucket(int blocks) {  // monotone: exact below 512 blocks, then 64 steps per octave
    int key = blocks;
    if (blocks >= 512) {
        const int e = 31 - __clz(blocks);
        key = 512 + (e - 9) * 64 + ((blocks >> (e - 6)) & 63);
    }
    return kPackedBuckets - 1 - min(key, kPackedBuckets - 1);
}

// Inclusive scan over the CTA (1024 threads); `red` holds 32 words.  Ends with all threads past their use of `red`.  (A function of its own:
// the plan runs once, and what it costs is fetching its instructions.)
__device__ __noinline__ int packed_scan(int v, int* red, int& total) {
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

// One CTA.  Sequences -> tile pairs -> work items.
__global__ void __launch_bounds__(kPackedPlanThreads) mha_packed_plan_kernel(const PackedParams p) {
    pdl_launch_dependents();
    extern __shared__ int4 plan_smem[];
    int4* near_seqs = plan_smem;                                          // [kPackedSeqs]
    int* hist = reinterpret_cast<int*>(plan_smem + kPackedSeqs);          // [kPackedBuckets], or with cut ranges
    int4* near_tiles = reinterpret_cast<int4*>(hist + kPackedBuckets);    // [kPackedSplitTiles] {sequence, pair, tokens, key blocks}
    int* near_rows = reinterpret_cast<int*>(near_tiles + kPackedSplitTiles);  // [kPackedSplitTiles]
    __shared__ int red[32];
    __shared__ int longest_sh, kept_sh, irregular_sh;
    __shared__ float best_cost[32];
    __shared__ int best_n[32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    for (int i = tid; i < kPackedBuckets; i += kPackedPlanThreads) hist[i] = 0;
    if (tid == 0) longest_sh = kept_sh = irregular_sh = 0;
    cudaGridDependencySynchronize();

    // sequences: tile pairs and their prefix sums
    const int W2 = 2 * p.W;
    const int per = (p.all + kPackedPlanThreads - 1) / kPackedPlanThreads;
    const int s_lo = min(p.all, tid * per), s_hi = min(p.all, s_lo + per);
    int3 q = make_int3(0, 0, 0);
    long long base = 0;
    bool ok = true;
    auto get = [&](int s) {
        if (s < p.S) ok = packed_sequence(p, s, q, base);
        else { ok = true; packed_tail(p, s - p.S, q, base); }
    };
    int mine = 0;
#pragma unroll 1
    for (int s = s_lo; s < s_hi; ++s) {
        get(s);
        mine = min(mine + (q.y + W2 - 1) / W2, p.max_tiles + 1);  // (offsets that do not ascend could sum up to more than 32 bits hold)
    }
    int pairs, kept = 0;
    int before = packed_scan(mine, red, pairs) - mine;
    // Offsets that do not ascend can have more tile pairs than the call's tokens make, which is what the lists and the scratch are sized
    // for.  The sequences from the one on that does not fit are left out; with shared prefixes, where a token's group and its tail
    // belong together, all are.
    const bool too_many = pairs > p.max_tiles;
#pragma unroll 1
    for (int s = s_lo; s < s_hi; ++s) {
        if (per > 1) get(s);
        int n = (q.y + W2 - 1) / W2;
        if (before > p.max_tiles - n) {
            ok = false;
            q.y = n = 0;
        }
        if (!ok) {
            packed_report(kStatusBadSequence, s, q.x, q.z);
            irregular_sh = 1;
        }
        const int4 e = make_int4(q.x, q.y, q.z, before);
        p.seqs[s] = e;
        p.key_base[s] = base;
        if (s < kPackedSeqs) near_seqs[s] = e;
        before += n;
        if (n > 0) kept = before;
    }
    kept = __reduce_max_sync(0xffffffffu, kept);
    if (lane == 0) atomicMax(&kept_sh, kept);
    __syncthreads();
    // (up to the end of the last sequence that is kept: the numbers behind it belong to no tile)
    const int tiles = too_many && p.prefix_lens ? 0 : kept_sh;

    // tile pair i: its sequence (the last one with at most i pairs before it), number in it, tokens and key blocks
    const int4* seqs = p.all <= kPackedSeqs ? near_seqs : p.seqs;
    struct Tile { int s, pair, n, blocks; };
    const bool near = tiles <= kPackedSplitTiles;
    auto find_tile = [&](int i) {
        Tile t;
        int lo = 0, hi = p.all;
#pragma unroll 1
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (seqs[mid].w <= i) lo = mid; else hi = mid;
        }
        const int4 e = seqs[lo];
        t.s = lo;
        t.pair = i - e.w;
        t.n = min(W2, e.y - t.pair * W2);
        t.blocks = packed_tile_blocks(e.y, e.z, p.causal, t.pair * W2, t.n);
        return t;
    };
    auto tile_at = [&](int i) {
        if (!near) return find_tile(i);
        const int4 t = near_tiles[i];
        return Tile{t.x, t.y, t.z, t.w};
    };
    const bool may_split = p.part_rows > 0 && near && !(too_many && p.prefix_lens);
    int most = 0;
#pragma unroll 1
    for (int i = tid; i < tiles; i += kPackedPlanThreads) {
        const Tile t = find_tile(i);
        atomicAdd(&hist[packed_bucket(t.blocks)], 1);
        if (near) near_tiles[i] = make_int4(t.s, t.pair, t.n, t.blocks);
        most = max(most, t.blocks);
    }
    if (may_split) {
        most = __reduce_max_sync(0xffffffffu, most);
        if (lane == 0) atomicMax(&longest_sh, most);
    }
    __syncthreads();

    // Cut the key ranges?  Time in halves of a key block's: an item of b blocks takes 2 b + 3 (fill, drain, epilogue), with one tile's
    // rows on both tiles b + 3; equal items run in rounds of one per SM, unequal ones stick out by half of what the longest has
    // over the average (whole ranges, longest first, by less).  Joining the parts costs kJoin.
    constexpr int kItem = 3;
    constexpr float kJoin = 5.0f, kNever = 1e12f;
    int chunk = 0;
    if (may_split) {
        const int longest = longest_sh;
        float mine_cost = 3e38f;
        // n parts of the longest range, a warp per n: 0 (whole and not joined), 1 .. 12, then 4 to 8 per octave up to 128
        constexpr unsigned char kParts[32] = {0, 1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13, 14, 15, 16, 18, 20, 22, 24, 28, 32, 36, 40, 48, 56, 64, 80, 96, 112, 128};
        const int mine_n = kParts[warp];
        if (mine_n <= longest && (mine_n > 0 || !p.prefix_lens)) {  // (a prefix's results always go to the join)
            const int n = mine_n, c = n ? (longest + n - 1) / n : max(longest, 1);
            const float per_block = 1.0f / c;
            float work = 0.0f, rows = 0.0f;
            int top = 0, entries = 0;
#pragma unroll 1
            for (int k = lane; k < tiles; k += 32) {
                const int tokens = near_tiles[k].z, blocks = near_tiles[k].w;
                const int parts = max(1, __float2int_rd((blocks + c - 0.5f) * per_block)), each = min(blocks, c);  // (rounded up)
                const bool dual = n > 0 && tokens <= p.W;
                work += static_cast<float>((dual ? blocks : 2 * blocks) + kItem * parts);
                rows += static_cast<float>(parts * packed_part_rows(p, tokens));
                top = max(top, (dual ? each : 2 * each) + kItem);
                entries += parts;
            }
#pragma unroll
            for (int w = 16; w > 0; w >>= 1) {
                work += __shfl_xor_sync(0xffffffffu, work, w);
                rows += __shfl_xor_sync(0xffffffffu, rows, w);
            }
            top = __reduce_max_sync(0xffffffffu, top);
            entries = __reduce_add_sync(0xffffffffu, entries);
            const float items = static_cast<float>(max(entries, 1)) * p.H_kv, average = work * p.H_kv / items;
            const float rounds = n ? ceilf(items / p.sm_count) : fmaxf(items / p.sm_count, 1.0f);
            mine_cost = fmaxf(static_cast<float>(top), rounds * average + (top - average) * (n ? 0.5f : 0.25f)) + (n ? kJoin : 0.0f);
            // (1.0001: the sum of the rows is rounded)
            if (n && (rows * p.H_kv * 1.0001f > static_cast<float>(p.part_rows) || entries > p.max_entries))
                mine_cost = n == 1 && p.prefix_lens ? kNever / 2 : kNever;
        }
        if (lane == 0) {
            best_cost[warp] = mine_cost;
            best_n[warp] = mine_n;
        }
        __syncthreads();
        const uint32_t key = __float_as_uint(best_cost[lane]);  // (costs are positive: their bits are in their order)
        const unsigned int at = __ballot_sync(0xffffffffu, key == __reduce_min_sync(0xffffffffu, key));
        const int n = best_n[__ffs(at) - 1];
        if (n > 0 || p.prefix_lens) chunk = max(1, n ? (longest + n - 1) / n : longest);
    }

    int total;
    if (chunk > 0) {
        // parts of equal length, longest first: a tile pair's whole parts and its last one are counted, then placed
        for (int i = tid; i < kPackedBuckets; i += kPackedPlanThreads) hist[i] = 0;
        __syncthreads();
        auto whole_of = [&](const Tile& t) { return packed_bucket((t.n <= p.W ? 1 : 2) * chunk); };
        auto last_of = [&](const Tile& t) { return packed_bucket((t.n <= p.W ? 1 : 2) * (t.blocks % chunk)); };
        int first = 0, first_row = 0;
#pragma unroll 1
        for (int i0 = 0; i0 < tiles; i0 += kPackedPlanThreads) {
            const int i = i0 + tid;
            int parts = 0, rows = 0;
            if (i < tiles) {
                const Tile t = tile_at(i);
                parts = max(1, (t.blocks + chunk - 1) / chunk);
                rows = packed_part_rows(p, t.n) * p.H_kv;
                if (t.blocks >= chunk) atomicAdd(&hist[whole_of(t)], t.blocks / chunk);
                if (t.blocks % chunk != 0 || t.blocks == 0) atomicAdd(&hist[last_of(t)], 1);
            }
            int sum_parts, sum_rows;
            packed_scan(parts, red, sum_parts);
            const int row = first_row + packed_scan(parts * rows, red, sum_rows) - parts * rows;
            if (i < tiles) p.tile_info[i] = make_int2(row, parts);
            if (i < tiles) near_rows[i] = row;
            // (only for groups that overlap: scratch is sized for groups that do not)
            const bool no_room = sum_rows > p.part_rows - first_row || sum_parts > p.max_entries - first;
            first += sum_parts;
            first_row += sum_rows;
            if (no_room) {
                if (tid == 0) packed_report(kStatusBadSequence, p.S, tiles, 0);
                first = 0;
                chunk = 0;
                break;
            }
        }
        total = first;
        if (total > 0) {
            int sum;
            __syncthreads();
            const int a = hist[2 * tid], b = hist[2 * tid + 1];
            const int end = packed_scan(a + b, red, sum);
            hist[2 * tid] = end - a - b;
            hist[2 * tid + 1] = end - b;
            __syncthreads();
#pragma unroll 1
            for (int i = tid; i < tiles; i += kPackedPlanThreads) {
                const Tile t = tile_at(i);
                const int rows = packed_part_rows(p, t.n) * p.H_kv, row = near_rows[i], whole = t.blocks / chunk;
                if (whole > 0) {
                    const int at = atomicAdd(&hist[whole_of(t)], whole);
#pragma unroll 1
                    for (int k = 0; k < whole; ++k) {
                        p.entries[at + k] = make_int4(t.s, t.pair, k * chunk, chunk);
                        p.entry_rows[at + k] = row + k * rows;
                    }
                }
                if (t.blocks % chunk != 0 || t.blocks == 0) {
                    const int at = atomicAdd(&hist[last_of(t)], 1);
                    p.entries[at] = make_int4(t.s, t.pair, whole * chunk, t.blocks - whole * chunk);
                    p.entry_rows[at] = row + whole * rows;
                }
            }
        }
    } else {
        // longest first: counting sort
        const int a = hist[2 * tid], b = hist[2 * tid + 1];
        const int end = packed_scan(a + b, red, total);
        hist[2 * tid] = end - a - b;
        hist[2 * tid + 1] = end - b;
        __syncthreads();
#pragma unroll 1
        for (int i = tid; i < tiles; i += kPackedPlanThreads) {
            const Tile t = tile_at(i);
            const int at = atomicAdd(&hist[packed_bucket(t.blocks)], 1);
            if (at < p.max_entries) p.entries[at] = make_int4(t.s, t.pair, 0, t.blocks);
        }
        total = tiles;
    }
    if (tid == 0) {
        p.hdr->num_items = total * p.H_kv;
        p.hdr->counter = 0;
        p.hdr->split = chunk;
        p.hdr->irregular = irregular_sh;
    }
}
constexpr int kPackedPlanSmem = kPackedSeqs * 16 + kPackedBuckets * 4 + kPackedSplitTiles * 20;

// exp2_poly2 (see mha.cuh) with a polynomial of degree 5 (minimax for the relative error on [-1/2, 1/2], 2.2e-7): what is left is the
// resolution of the exponent, 252 * 2^-25, 5e-6 of the result.  (The cubic's 7.5e-5 showed in the LSE of rows that see one or
// two keys; two more packed FMAs for one in eight or four exponentials.)
__device__ __forceinline__ float2 exp2_poly2_fine(float s0, float s1, float cs, float ns) {
    constexpr float kMagic = 12582912.0f - kPolyLow;  // 1.5 * 2^23 - 125
    const float2 u = make_float2(fma_sat(s0, cs, ns), fma_sat(s1, cs, ns));
    const float2 span = make_float2(kPolySpan, kPolySpan), magic = make_float2(kMagic, kMagic);
    const float2 t = ffma2(u, span, magic);
    const float2 f = ffma2(u, span, fsub2(magic, t));
    float2 y = ffma2(f, make_float2(0.0013276472f, 0.0013276472f), make_float2(0.009675541f, 0.009675541f));
    y = ffma2(y, f, make_float2(0.05550713f, 0.05550713f));
    y = ffma2(y, f, make_float2(0.2402212f, 0.2402212f));
    y = ffma2(y, f, make_float2(0.69314694f, 0.69314694f));
    y = ffma2(y, f, make_float2(1.0f, 1.0f));
    y.x = __int_as_float(__float_as_int(y.x) + (__float_as_int(t.x) << 23));
    y.y = __int_as_float(__float_as_int(y.y) + (__float_as_int(t.y) << 23));
    return y;
}

template <int D>
struct PackedSmem {
    static constexpr int kTileBytes = kMhaBlock * D * 2;
    static constexpr int kChunkBytes = kMhaBlock * 128;
    static constexpr int kStages = (D == 128) ? 4 : 8;
    static constexpr int kBarrierBytes = 512;
    static constexpr int kItemBytes = 2 * 48 + kMhaBlock * 4;  // two work items, and which token and head a row is
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
    int part_row;    // first row of the partial results, or -1: O and LSE are written
    int fix;         // rows of the last V tile to zero: first | (end << 8), or 0
    int dual;        // both tiles have the same rows, tile t works on blocks b0 + t, b0 + t + 2, ...
    int row_limits;  // rows see no key beyond their sequence's length either
};

// kParts: items may be parts of a key range or have both tiles on one tile's rows.  Calls with enough items without that run the
// kernel that leaves the code out: what the schedulers fetch is what bounds the softmax warps' neighbours (with it prompts
// ran 2 to 11 % slower, D = 64 the most).  kOne: PackedParams::single.
template <int D, bool kParts, bool kOne>
__global__ void __launch_bounds__(kMhaThreads, 1)
mha_packed_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_q1,
                  const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                  const __grid_constant__ CUtensorMap tmap_o, const __grid_constant__ CUtensorMap tmap_part, const PackedParams p) {
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
    int* row_of = reinterpret_cast<int*>(items + 2);  // [128] token in the tile << 16 | head in the group
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
        prefetch_tensormap(&tmap_q1);
        prefetch_tensormap(&tmap_k);
        prefetch_tensormap(&tmap_v);
    }
    if (warp == 8) {
        tmem_alloc(tmem_base_slot, 512);
        tmem_relinquish();
    }
    if (threadIdx.x < kMhaBlock) row_of[threadIdx.x] = (static_cast<int>(threadIdx.x) / p.G << 16) | (static_cast<int>(threadIdx.x) % p.G);
    // Rows that no token fills: their scores need not be right, but a NaN would send the warp through the slow path.  Later items find
    // rows of earlier ones there.
    for (int i = threadIdx.x; i < 2 * L::kTileBytes / 16; i += kMhaThreads) reinterpret_cast<uint4*>(smem_q)[i] = make_uint4(0u, 0u, 0u, 0u);
    fence_proxy_async_smem();
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
        const int W2 = 2 * p.W;
        int num_items, chunk = 0;
        int4 e = make_int4(0, 0, 0, 0), q = e;
        long long base = 0;
        if constexpr (kOne) {
            int3 only;
            if (!packed_sequence(p, 0, only, base) && blockIdx.x == 0 && lane == 0) packed_report(kStatusBadSequence, 0, only.x, only.z);
            q = make_int4(only.x, only.y, only.z, 0);
            num_items = (only.y + W2 - 1) / W2 * p.H_kv;
        } else {
            num_items = p.hdr->num_items;
            chunk = p.hdr->split;
        }
        const int nb = p.cu_k ? 1 : kMhaBlock / p.block_size;     // cache blocks per tile
        const int lane_block = lane % nb, lane_chunk = lane / nb;  // which this lane loads, and which 64 columns of it
        const int beyond = max(1, p.num_blocks * p.H_kv);          // coordinate that loads zeros
        int ld_stage = 0;
        uint32_t ld_phase = 0;
        int q_loads = 0;
        bool ok = true;
        // The next item is drawn while the current one's tiles are loaded, and its entry read: the list's latency (atomic, entry,
        // sequence, one behind the other) is then off the path.
        int idx = blockIdx.x, drawn = 0;
        int entry_row = 0;
        auto read_entry = [&]() {
            if (idx < num_items) {
                const int entry = idx / p.H_kv;
                if (kOne) {
                    e = make_int4(0, entry, 0, INT32_MAX);
                } else {
                    e = p.entries[entry];
                    if (kParts && chunk > 0) entry_row = p.entry_rows[entry];
                }
            }
        };
        auto draw = [&]() {
            if (!kOne && lane == 0) drawn = atomicAdd(&p.hdr->counter, 1);
        };
        auto read_sequence = [&]() {
            if (!kOne && idx < num_items) {
                q = p.seqs[e.x];
                base = p.key_base[e.x];
            }
        };
        read_entry();
        read_sequence();
        for (int n = 0; ok; ++n) {
            PackedItem it = {};
            int nk = 0, total = 0;  // keys of the sequence, key blocks of the item
            const long long key_base = base;
            if (idx < num_items) {
                const int first = e.y * W2;
                it.valid = 1;
                it.kvh = idx % p.H_kv;
                it.tok0 = q.x + first;
                it.ntok = min(W2, q.y - first);
                nk = q.z;
                it.lim0 = p.causal ? nk - q.y + first : nk - 1;
                it.b0 = e.z;
                it.row_limits = p.prefix_lens && e.x < p.S;
                const bool parts = kParts && chunk > 0 && (p.prefix_lens || it.ntok <= p.W || packed_tile_blocks(q.y, nk, p.causal, first, it.ntok) > chunk);
                it.part_row = parts ? entry_row + it.kvh * packed_part_rows(p, it.ntok) : -1;
                it.dual = parts && it.ntok <= p.W;
                if (kParts && it.dual) {
                    total = e.w;
                    it.J[0] = (total + 1) >> 1;
                    it.J[1] = total >> 1;
                } else {
#pragma unroll
                    for (int t = 0; t < 2; ++t)
                        it.J[t] = min(max(packed_tile_blocks(q.y, nk, p.causal, first + t * p.W, min(p.W, it.ntok - t * p.W)) - e.z, 0), e.w);
                    total = max(it.J[0], it.J[1]);
                }
                // V rows beyond the last key, up to the next cache block (the blocks after that load zeros)
                const int tail = nk % kMhaBlock;
                int tail_end = kMhaBlock;
                if (!p.cu_k) tail_end = (tail + p.block_size - 1) / p.block_size * p.block_size;
                if (total > 0 && it.b0 + total == packed_blocks(nk) && tail != 0 && tail < tail_end) it.fix = tail | (tail_end << 8);
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

            // block-table entry of this lane's cache block of the item's key block b, as a coordinate of the tensor map
            const int nblk = p.cu_k ? 0 : (nk + p.block_size - 1) / p.block_size;
            auto table_at = [&](int b) -> int {
                const int i = (it.b0 + b) * nb + lane_block;
                return (b < total && i < nblk) ? p.block_table[key_base + i] : -1;
            };
            int next_entry = p.cu_k ? 0 : table_at(0);
            constexpr int kHeld = kParts ? 4 : 2;
            int z[4] = {0, 0, 0, 0};  // coordinates of the last kHeld key blocks
            // key block b of the item, K or V (K blocks in order; V blocks less than kHeld behind)
            auto load = [&](bool is_k, int b) -> bool {
                if (!wait_all(&kv_empty[ld_stage], ld_phase ^ 1, 0x100 + ld_stage)) return false;
                uint8_t* dst = smem_kv + ld_stage * L::kTileBytes;
                if (lane == 0) mbar_arrive_expect_tx(&kv_full[ld_stage], L::kTileBytes);
                __syncwarp();
                const CUtensorMap* map = is_k ? &tmap_k : &tmap_v;
                if (p.cu_k) {
                    if (lane < kChunks)
                        tma_load_3d(dst + lane * L::kChunkBytes, map, &kv_full[ld_stage], lane * 64, it.kvh, static_cast<int>(key_base) + (it.b0 + b) * kMhaBlock);
                } else {
                    if (is_k) {
                        int zz = beyond;
                        if (next_entry >= 0 && next_entry < p.num_blocks) zz = next_entry * p.H_kv + it.kvh;
                        else if (lane < nb && (it.b0 + b) * nb + lane < nblk) packed_report(kStatusBadBlock, (it.b0 + b) * nb + lane, it.tok0, next_entry);
#pragma unroll
                        for (int i = 0; i < kHeld; ++i)
                            if ((b & (kHeld - 1)) == i) z[i] = zz;
                        next_entry = table_at(b + 1);
                    }
                    int at = (b & 1) ? z[1] : z[0];
                    if (kParts && (b & 2)) at = (b & 1) ? z[3] : z[2];
                    if (lane_chunk < kChunks)
                        tma_load_3d(dst + lane_chunk * L::kChunkBytes + lane_block * p.block_size * 128, map, &kv_full[ld_stage], lane_chunk * 64, 0, at);
                }
                __syncwarp();
                if (++ld_stage == kStages) { ld_stage = 0; ld_phase ^= 1; }
                return true;
            };
            // Q: after the first K, once the previous item's last Q K^T has read the tiles
            auto load_q = [&]() -> bool {
                if (q_loads > 0 && !wait_all(q_empty, (q_loads - 1) & 1, 0x110)) return false;
                ++q_loads;
                const int tiles = kParts && it.dual ? (total > 1 ? 2 : 1) : it.ntok > p.W ? 2 : 1;
                const bool one = it.ntok == 1;
                if (lane == 0) mbar_arrive_expect_tx(q_full, static_cast<uint32_t>(tiles) * (one ? 1 : p.W) * p.G * 128 * kChunks);
                __syncwarp();
                if (lane < tiles * kChunks) {
                    const int t = lane / kChunks, c = lane % kChunks;
                    tma_load_3d(smem_q + t * L::kTileBytes + c * L::kChunkBytes, one ? &tmap_q1 : &tmap_q, q_full, c * 64, it.kvh * p.G,
                                it.tok0 + (kParts && it.dual ? 0 : t * p.W));
                }
                __syncwarp();
                return true;
            };
            // Ring order (the issuing warps walk the same): K of the first step's blocks (one, with `dual` two), then V of a block and K
            // of the next step's in turn; D = 64: all of a step's next K, then its V.  (One copy of `load`: code that is not
            // in a loop is fetched cold every time.)
            const int width = kParts && it.dual ? 2 : 1;
            int n_k = 0, n_v = 0;
            for (int i = 0; i < 2 * total && ok; ++i) {
                const bool is_k = n_k < min(total, kEarlyQK ? (n_v & ~(width - 1)) + 2 * width : n_v + width);
                if (i == 1) {
                    ok = load_q();
                    draw();
                }
                ok = ok && load(is_k, is_k ? n_k : n_v);
                n_k += is_k;
                n_v += !is_k;
                if (i == min(3, 2 * total - 1)) {
                    idx = static_cast<int>(gridDim.x) + __shfl_sync(0xffffffffu, drawn, 0);
                    read_entry();
                }
            }
            if (!ok) break;
            if (it.fix && lane == 0) mbar_arrive(&v_asked[n & 1]);
            if (total == 0) {
                draw();
                idx = static_cast<int>(gridDim.x) + __shfl_sync(0xffffffffu, drawn, 0);
                read_entry();
            }
            read_sequence();
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
            const bool fix = it.fix != 0;
            const bool dual = kParts && it.dual;
            const int fix_step = fix ? (dual ? J0 + J1 : Jmax) - 1 : -1;  // the block whose V tile has a tail
            if (Jmax > 0) {
                ok = wait_all(q_full, n_q & 1, 0x200);
                if (!ok) break;
                ++n_q;
            }
            if (dual) {
                // As below, but every tile in the ring belongs to one query tile (tile t: blocks t, t + 2, ...).  D = 64: both issuing
                // warps walk the whole ring and release every slot.
#pragma unroll 1
                for (int j = -1; j < J0 && ok; ++j) {
#pragma unroll 1
                    for (int i = 0; i < 4 && ok; ++i) {
                        // D = 128: V and the next K of tile 0, then of tile 1;  D = 64: the next K of both tiles, then V of both
                        const int t = kEarlyQK ? i & 1 : i >> 1, Jt = t ? J1 : J0;
                        const bool is_k = kEarlyQK ? i < 2 : (i & 1);
                        if (is_k ? j + 1 >= Jt : (j < 0 || j >= Jt)) continue;
                        const int slot = stage;
                        ok = wait_all(&kv_full[slot], phase, 0x240 + slot);
                        if (!ok) break;
                        if (++stage == kStages) { stage = 0; phase ^= 1; }
                        if (t >= t_lo && t < t_hi) {
                            if (is_k) {
                                const uint32_t done = t ? n_qk[1] : n_qk[0];
                                if (kEarlyQK && done > 0) ok = wait_all(&s_free[t], (done - 1) & 1, 0x250 + t);
                                if (!ok) break;
                                if (t) ++n_qk[1]; else ++n_qk[0];
                                tc_fence_after();
                                issue_qk(t, slot);
                            } else {
                                if (2 * j + t == fix_step) ok = wait_all(&v_fixed[n & 1], (fixed >> (n & 1)) & 1, 0x260);
                                ok = ok && wait_all(&p_full[t], (t ? n_p[1] : n_p[0]) & 1, 0x230 + t);
                                if (!ok) break;
                                if (t) ++n_p[1]; else ++n_p[0];
                                tc_fence_after();
                                issue_pv(t, slot, j == 0);
                                if (leader) {
                                    if (kEarlyQK) umma_commit(&p_free[t]);
                                    if (j == Jt - 1) umma_commit(&o_full[t]);
                                }
                            }
                        }
                        if (leader) umma_commit(&kv_empty[slot]);
                        __syncwarp();
                    }
                    if (ok && j + 2 == J0 && leader) umma_commit(q_empty);  // the item's last Q K^T products are issued
                    __syncwarp();
                }
            } else {
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
                pos += 2 * (kParts && it.dual ? it.J[0] + it.J[1] : max(it.J[0], it.J[1]));
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
            const int dual = kParts ? it.dual : 0;
            const int tok_shift = dual ? 0 : t * p.W;           // first token of this tile in the pair
            const int tile_tok = min(it.ntok - tok_shift, p.W);  // its tokens, if positive
            const int Jt = it.J[t], first_block = it.b0 + (dual ? t : 0), block_step = dual ? 2 : 1;
            if (tile_tok <= 0) {
                drop_item(n);
                continue;
            }
            const bool busy = quarter * 32 < tile_tok * p.G;  // this warp has a row of a token
            // last visible key; rows without a token take the last token's, so that they mask no more than their neighbours
            int limit = it.lim0;
            if (p.causal) limit += tok_shift + min(row_tok, tile_tok - 1);
            if (kParts && it.row_limits && row_tok < tile_tok) limit = min(limit, p.seq_lens[it.tok0 + tok_shift + row_tok] - 1);
            float m_run = -INFINITY, l_run = 0.0f;

            if (kParts && !busy) {  // nobody reads this warp's rows: P_t may be anything there
                for (int j = 0; j < Jt && ok; ++j) {
                    ok = wait_all(&s_full[t], n_s & 1, 0x340 + t);
                    ++n_s;
                    if constexpr (kEarlyQK) {
                        if (ok && lane == 0) mbar_arrive(&s_free[t]);
                        // (not ahead of the busy warps: a second arrival in p_full's phase would stand for theirs)
                        if (n_s > 1) ok = ok && wait_all(&p_free[t], n_s & 1, 0x330 + t);
                    }
                    __syncwarp();
                    if (ok && lane == 0) mbar_arrive(&p_full[t]);
                }
                if (Jt > 0) ok = ok && wait_all(&o_full[t], n_o & 1, 0x410 + t);
                n_o += Jt > 0;
                if (!ok) break;
                drop_item(n);
                continue;
            }
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
                const int j0 = (first_block + j * block_step) * kMhaBlock;
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
                        if (poly) return exp2_poly2_fine(s0, s1, cs, ns);
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
            // Rows leave in pieces of 128 bytes (64 columns of O, 32 of a partial result): each thread puts its row's piece into the warp's
            // staging area (16-byte chunk k of row r at chunk k ^ (r & 7), the tensor maps' 128-byte swizzle).  A warp whose 32 rows
            // are all tokens' stores it as one TMA box; else eight lanes at a time write a row's piece.  (An epilogue of plain
            // stores alone took 5200 clocks at D = 128: 1600 to convert, 3100 to read the staging area back and store.)
            // Short loops throughout: what runs once per item is fetched cold.
            const bool direct = !kParts || it.part_row < 0;
            const bool seen = Jt > 0 && limit >= first_block * kMhaBlock;  // (by the mask: a row of NaN has no maximum either)
            const int shift = dual ? t * it.ntok * p.G : t * kMhaBlock;  // of a partial result's rows
            uint8_t* base;       // where the tile's token 0, head 0 goes, and the bytes from one token and from one head to the next
            int64_t tok_bytes;
            int head_bytes;
            if (direct) {
                base = reinterpret_cast<uint8_t*>(p.O + static_cast<int64_t>(it.tok0 + tok_shift) * p.ldo + it.kvh * p.G * D);
                tok_bytes = p.ldo * 2;
                head_bytes = D * 2;
            } else {
                base = reinterpret_cast<uint8_t*>(p.part_o + (static_cast<int64_t>(it.part_row) + shift) * D);
                tok_bytes = p.G * D * 4;
                head_bytes = D * 4;
            }
            base += (lane & 7) * 16;
            const float inv_l = seen ? __fdividef(1.0f, l_run) : 0.0f;
            const float2 factor = make_float2(inv_l, inv_l);
            const int columns = direct ? 64 : 32;  // of a piece
            const bool boxed = p.boxes && quarter * 32 + 32 <= tile_tok * p.G;
#pragma unroll 1
            for (int h = 0; (direct || Jt > 0) && h < D; h += 32) {
                uint32_t o[32];
                if (Jt > 0) tmem_ld_32x32b_x32(o_addr + h, o);
                if (lane == 0) tma_store_wait_read<0>();  // the staging area's previous box has been read out
                __syncwarp();
                tmem_wait_ld();
                if (Jt == 0) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) o[i] = 0u;
                }
                if (!direct) {
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        *reinterpret_cast<uint4*>(stage_o + lane * 128 + ((k ^ (lane & 7)) * 16)) = make_uint4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]);
                } else {
                    const int first = (h & 32) >> 3;  // chunk
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        uint32_t w[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {  // (a row that sees nothing: its O is finite, and times 0)
                            const float2 v = fmul2(make_float2(__uint_as_float(o[8 * k + 2 * e]), __uint_as_float(o[8 * k + 2 * e + 1])), factor);
                            w[e] = pack_bf16x2(v.x, v.y);
                        }
                        *reinterpret_cast<uint4*>(stage_o + lane * 128 + (((first + k) ^ (lane & 7)) * 16)) = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                    if ((h & 32) == 0) continue;
                }
                if (boxed) {
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        if (direct) tma_store_3d(&tmap_o, stage_o, h - 32, it.kvh * p.G, it.tok0 + tok_shift + quarter * 32 / p.G);
                        else tma_store_2d(&tmap_part, stage_o, h, it.part_row + shift + quarter * 32);
                        tma_store_commit();
                    }
                    continue;
                }
                __syncwarp();
                uint8_t* to = base + (h / columns) * 128;
#pragma unroll 2
                for (int i = 0; i < 32; i += 4) {
                    const int row = i + (lane >> 3), at = row_of[quarter * 32 + row];
                    const uint4 v = *reinterpret_cast<const uint4*>(stage_o + row * 128 + (((lane & 7) ^ (row & 7)) * 16));
                    if ((at >> 16) < tile_tok) *reinterpret_cast<uint4*>(to + (at >> 16) * tok_bytes + (at & 0xFFFF) * head_bytes) = v;
                }
                __syncwarp();
            }
            if (row_tok < tile_tok) {
                if (!direct) {
                    p.part_ml[static_cast<int64_t>(it.part_row) + shift + row_in_tile] = make_float2(seen ? m_run * c : -INFINITY, seen ? l_run : 0.0f);
                } else if (p.LSE) {
                    p.LSE[static_cast<int64_t>(it.tok0 + tok_shift + row_tok) * p.H + it.kvh * p.G + row_head] =
                        seen ? m_run * p.scale + __log2f(l_run) * 0.6931471805599453f : -INFINITY;
                }
            }
            drop_item(n);
        }
        if (lane == 0) tma_store_wait_all<0>();  // shared memory must outlive the stores that read it
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

// Joins the parts of cut key ranges, and a prefix with the tail behind it: one warp per (token, head).  Compact on purpose (short
// loops, no 64-bit division): most of its time is fetching its instructions and a chain of dependent loads.
constexpr int kPackedJoinWarps = 8;
template <int D>
__global__ void __launch_bounds__(kPackedJoinWarps * 32) mha_packed_join_kernel(const PackedParams p) {
    pdl_launch_dependents();
    constexpr int V = D / 32;  // elements per lane
    cudaGridDependencySynchronize();
    const PackedHeader hdr = *p.hdr;
    if (hdr.split == 0) return;
    const int lane = threadIdx.x & 31, tok = blockIdx.x, h = blockIdx.y * kPackedJoinWarps + (threadIdx.x >> 5);
    if (h >= p.H) return;
    const int kvh = h / p.G, W2 = 2 * p.W;
    // This row's parts: a run from its sequence's (or group's) tile pair and, behind a prefix, one from its tail.  Part k lies at
    // first + k * step, or, where both tiles had the same rows, at first + (k / 2) * step + (k % 2) * half.
    int first[2] = {0, 0}, step[2] = {0, 0}, half[2] = {0, 0}, count[2] = {0, 0};
    const int owner = hdr.irregular ? packed_owner_any(p.prefix_lens ? p.cu_q : nullptr, p.seqs, p.S, tok) : packed_owner_warp(p, tok);
    if (owner < 0 && !p.prefix_lens) return;  // a token of no sequence
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (i == 0 ? owner < 0 : p.prefix_lens == nullptr) continue;
        const int4 q = p.seqs[i == 0 ? owner : p.S + tok];
        const int at = tok - q.x;
        if (at >= q.y) {  // left out by the plan (not written), or no key behind the prefix
            if (!p.prefix_lens) return;
            continue;
        }
        const int pair = at / W2, in_pair = at - pair * W2, n = min(W2, q.y - pair * W2);
        const int2 info = p.tile_info[q.w + pair];
        const bool dual = n <= p.W;
        if (!p.prefix_lens && !dual && info.y == 1) return;  // not cut: written by its item
        const int rows = packed_part_rows(p, n), t = !dual && in_pair >= p.W;
        first[i] = info.x + kvh * rows + t * kMhaBlock + (in_pair - t * p.W) * p.G + h - kvh * p.G;
        step[i] = rows * p.H_kv;
        half[i] = n * p.G;
        count[i] = info.y << dual;
        if (!dual) half[i] = -1;
    }
    auto row_of = [&](int k) -> int {  // parts of both runs, one behind the other
        const int i = k >= count[0];
        if (i) k -= count[0];
        const int f = i ? first[1] : first[0], s = i ? step[1] : step[0], d = i ? half[1] : half[0];
        return d < 0 ? f + k * s : f + (k >> 1) * s + (k & 1) * d;
    };
    const int all = count[0] + count[1];
    float m = -INFINITY;
#pragma unroll 1
    for (int k = lane; k < all; k += 32) m = fmaxf(m, p.part_ml[row_of(k)].x);
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, w));
    float l = 0.0f, o[V] = {};
#pragma unroll 1
    for (int k0 = 0; k0 < all; k0 += 32) {
        float weight = 0.0f;
        int row = 0;
        if (k0 + lane < all) {
            row = row_of(k0 + lane);
            const float2 ml = p.part_ml[row];
            weight = ml.x == -INFINITY ? 0.0f : fast_exp2(ml.x - m);
            l += weight * ml.y;
        }
        const int n = min(32, all - k0);
#pragma unroll 1
        for (int k = 0; k < n; k += 8) {  // eight parts' loads in flight
            float v[8][V], w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                w[i] = __shfl_sync(0xffffffffu, weight, k + i);
                const float* src = p.part_o + static_cast<int64_t>(__shfl_sync(0xffffffffu, row, k + i)) * D + lane * V;
#pragma unroll
                for (int e = 0; e < V; ++e) v[i][e] = 0.0f;
                if (w[i] != 0.0f) {  // (0: a part without a visible key, or none)
                    if constexpr (V == 4) {
                        const float4 f = *reinterpret_cast<const float4*>(src);
                        v[i][0] = f.x; v[i][1] = f.y; v[i][2] = f.z; v[i][3] = f.w;
                    } else {
                        const float2 f = *reinterpret_cast<const float2*>(src);
                        v[i][0] = f.x; v[i][1] = f.y;
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int e = 0; e < V; ++e) o[e] = fmaf(v[i][e], w[i], o[e]);
        }
    }
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) l += __shfl_xor_sync(0xffffffffu, l, w);
    const float inv = l != 0.0f ? __fdividef(1.0f, l) : 0.0f;  // (NaN stays NaN)
    uint32_t packed[V / 2];
#pragma unroll
    for (int e = 0; e < V / 2; ++e) packed[e] = pack_bf16x2(o[2 * e] * inv, o[2 * e + 1] * inv);
    __nv_bfloat16* dst = p.O + static_cast<int64_t>(tok) * p.ldo + h * D + lane * V;
    if constexpr (V == 4) *reinterpret_cast<uint2*>(dst) = make_uint2(packed[0], packed[1]);
    else *reinterpret_cast<uint32_t*>(dst) = packed[0];
    if (lane == 0 && p.LSE) p.LSE[static_cast<int64_t>(tok) * p.H + h] = l != 0.0f ? (m + __log2f(l)) * 0.6931471805599453f : -INFINITY;
}

// Scratch: header, sequences, key bases, entries, their rows, the tile pairs' parts, partial results.
struct PackedScratch {
    size_t seqs, key_base, entries, entry_rows, tile_info;  // byte offsets
    size_t lists;                                           // bytes without partial results
    size_t row_bytes;
    int64_t part_rows;  // rows of partial results that it is sized for
    int64_t max_tiles, max_entries;
    int W;
};
// S sequences of T tokens in all; prefix: S groups, with a tail behind them for each of the T sequences.
inline PackedScratch packed_scratch(int64_t T, int64_t S, int G, int H_kv, int D, bool prefix = false) {
    PackedScratch x;
    auto up = [](size_t v) { return (v + 255) & ~size_t(255); };
    x.W = kMhaBlock / G;
    const int64_t pairs = T / (2 * x.W) + S, all = prefix ? S + T : S;
    x.max_tiles = prefix ? pairs + T : pairs;
    // A row needs two partial results at least where it is cut (one per tile), and few rows more parts than many.
    const int64_t rows = T * G * H_kv;
    x.part_rows = std::min<int64_t>(kPackedSplitRows, 320 * 2 * T * G);
    if (prefix) x.part_rows += pairs * 2 * kMhaBlock * H_kv + 2 * rows;
    x.max_entries = std::max<int64_t>(x.max_tiles, std::min<int64_t>(x.part_rows / (2 * H_kv), (1 << 17)));
    x.seqs = 256;
    x.key_base = up(x.seqs + static_cast<size_t>(all) * 16);
    x.entries = up(x.key_base + static_cast<size_t>(all) * 8);
    x.entry_rows = up(x.entries + static_cast<size_t>(x.max_entries) * 16);
    x.tile_info = up(x.entry_rows + static_cast<size_t>(x.max_entries) * 4);
    x.lists = up(x.tile_info + static_cast<size_t>(std::min<int64_t>(x.max_tiles, kPackedSplitTiles)) * 8);
    x.row_bytes = static_cast<size_t>(D) * 4 + 8;
    return x;
}

inline int packed_configure() {  // as mha_configure: 0, 1 (a CUDA call failed), 2 (too few registers for the hand-over)
    if (cudaFuncSetAttribute(mha_packed_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kPackedPlanSmem) != cudaSuccess) return 1;
    auto one = [](auto* kernel, int smem) {
        cudaFuncAttributes a;
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess || cudaFuncGetAttributes(&a, kernel) != cudaSuccess)
            return 1;
        return a.numRegs < kMhaMinRegsPerThread ? 2 : 0;
    };
    const int rc[6] = {one(mha_packed_kernel<64, false, false>, PackedSmem<64>::kTotal), one(mha_packed_kernel<128, false, false>, PackedSmem<128>::kTotal),
                       one(mha_packed_kernel<64, true, false>, PackedSmem<64>::kTotal), one(mha_packed_kernel<128, true, false>, PackedSmem<128>::kTotal),
                       one(mha_packed_kernel<64, false, true>, PackedSmem<64>::kTotal), one(mha_packed_kernel<128, false, true>, PackedSmem<128>::kTotal)};
    int worst = 0;
    for (int r : rc) worst = r == 1 || worst == 1 ? 1 : std::max(worst, r);
    return worst;
}

template <class... Params, class... Args>
inline bool packed_launch_one(void (*kernel)(Params...), dim3 grid, int threads, int smem, cudaStream_t st, Args&&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
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

struct PackedMaps {
    CUtensorMap q, q1, k, v, o, part;
};

// plan, attention, and (where key ranges may be cut) the join
template <int D>
int packed_launch(const PackedMaps& m, const PackedParams& p, cudaStream_t st) {
    if (!p.single && !packed_launch_one(mha_packed_plan_kernel, dim3(1), kPackedPlanThreads, kPackedPlanSmem, st, p)) return 4;
    const int64_t most = static_cast<int64_t>(p.part_rows > 0 ? p.max_entries : p.max_tiles) * p.H_kv;
    const auto kernel = p.part_rows > 0 ? mha_packed_kernel<D, true, false> : p.single ? mha_packed_kernel<D, false, true> : mha_packed_kernel<D, false, false>;
    if (!packed_launch_one(kernel, dim3(static_cast<unsigned>(std::min<int64_t>(p.sm_count, most))), kMhaThreads, PackedSmem<D>::kTotal, st, m.q, m.q1, m.k,
                           m.v, m.o, m.part, p))
        return 4;
    if (p.part_rows > 0) {
        if (!packed_launch_one(mha_packed_join_kernel<D>, dim3(p.T, (p.H + kPackedJoinWarps - 1) / kPackedJoinWarps), kPackedJoinWarps * 32, 0, st, p)) return 4;
    }
    return 0;
}

}  // namespace mlt
