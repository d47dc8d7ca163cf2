// Appending to the paged cache that the decode kernels read, with the rotary position embedding applied on the way:
// for the new token t of sequence s, at position p = ctx[s] + (t - cu[s]), the queries and keys are rotated by the
// angles of row p of the cos / sin tables, the queries go to Q_out, and the key and value of every KV head go to
// cache[table[s][p / BS]][head][p % BS] as BF16, or as E4M3 under one scale per (cache block, head).
//
//   halves       (x[i], x[i + R/2])   i < R/2      rotated by cos[p][i], sin[p][i]
//   interleaved  (x[2i], x[2i + 1])
//   (a, b) -> (a c - b s, b c + a s)               elements from R on pass through
// Each product is rounded to FP32 on its own and then added (no contraction), so that the value does not depend on which
// product a compiler fuses.
//
// 8-bit cache: the block's scale becomes max(the scale it had, if the block already holds tokens of the sequence; the
// power-of-two scale of the new tokens' largest finite magnitude).  If that is larger than before, the tokens already
// there are moved to it: q' = round(q * old / new), exact for powers of two unless a value underflows.  Every value is rounded
// once, also under a scale that is no power of two (set by someone else).
//
// Bound by HBM for prompts and by latency for single tokens: every input is read once, every output written once.
//   keys, values  one warp owns one head of the (at most BS) new tokens of one cache block, because the 8-bit block scale needs
//                 them together
//   queries       one warp owns a token, whose heads lie side by side: the angles are read once for all of them
// Measured, device time in captured graphs (32 query heads, 8 KV heads of 128): 8 prompts of 500 to 1500 tokens in 36 us (BF16 cache, 5.6 TB/s)
// or 35 us (E4M3, 5.3 TB/s), 43 us with queries by head like the keys; 32 single tokens in 3.1 and 3.6 us, a chain of memory
// latencies (a call from Python takes 15 to 17 us of host time).
// A lane owns two 8-element chunks of a head that hold both partners of its rotation pairs, so no exchange between lanes is
// needed but the maximum.
//
// Which cache block a warp works on: the host does not know the lengths, so blocks are numbered with gaps: sequence s
// has the slots cu[s] / BS + 2 s onwards.  n new tokens touch at most n / BS + 2 - 2 / BS blocks, and there are at least
// that many slots before the next sequence's first.  A warp finds its sequence by a 32-way search over cu.
#pragma once

#include "f8.cuh"

namespace mlt {

constexpr unsigned int kStatusBadPosition = 9;  // token offsets or positions outside [0, num_tokens) / the cos and sin tables

struct AppendParams {
    const __nv_bfloat16 *Q, *K, *V;  // [T, heads, D], token pitches ldq, ldk, ldv; Q may be null
    __nv_bfloat16* Qo;               // [T, H, D], token pitch ldqo
    const float *cosv, *sinv;        // [max_pos, R / 2]
    const int *cu, *ctx, *table;     // [S + 1], [S], [S, max_blocks]
    void *Kc, *Vc;                   // [num_blocks, H_kv, BS, D]
    float *ks, *vs;                  // [num_blocks, H_kv]   (8-bit cache)
    int64_t ldq, ldk, ldv, ldqo;
    int T, S, H, H_kv, R, max_blocks, num_blocks, max_pos;
};

constexpr int kAppendWarps = 4;

// The last s with at(s) <= x for an increasing at; whole warp.
template <class F>
__device__ __forceinline__ int append_find_seq(int S, int x, int lane, F at) {
    int lo = 0, hi = S;
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 32;
        const int i = lo + lane * step;
        const bool le = i < hi && at(i) <= x;
        const int n = max(1, __popc(__ballot_sync(0xffffffffu, le)));
        lo += (n - 1) * step;
        hi = min(hi, lo + step);
    }
    return lo;
}

__device__ __forceinline__ void append_report(unsigned int code, int a, int b, int c) {
    if (atomicCAS(&g_status[0], 0u, code) == 0u) {
        g_status[1] = static_cast<unsigned int>(a);
        g_status[2] = static_cast<unsigned int>(b);
        g_status[3] = static_cast<unsigned int>(c);
    }
}

__device__ __forceinline__ void bf16x8_unpack(const uint4& v, float* f) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ uint4 bf16x8_pack(const float* f) {
    return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
}
__device__ __forceinline__ void rotate_pair(float& a, float& b, float c, float s) {
    const float x = __fsub_rn(__fmul_rn(a, c), __fmul_rn(b, s));
    b = __fadd_rn(__fmul_rn(b, c), __fmul_rn(a, s));
    a = x;
}

// Whether sequence s lies inside the call's tokens and the tables' positions; reported where it does not (nothing of such a
// sequence is read or written).
__device__ __forceinline__ bool append_in_range(const AppendParams& p, int s, int t_begin, int t_end, int ctx, int lane) {
    const bool ok = t_begin >= 0 && t_end <= p.T && ctx >= 0 && (p.R == 0 || static_cast<int64_t>(ctx) + (t_end - t_begin) <= p.max_pos);
    if (!ok && lane == 0) append_report(kStatusBadPosition, s, t_begin, ctx);
    return ok;
}
// cos (first half) and sin of the 8 pairs of lane position j at position pos
__device__ __forceinline__ void append_angles(const AppendParams& p, int64_t pos, int j, float (&a)[16]) {
    const int64_t at = pos * (p.R / 2) + j * 8;
    *reinterpret_cast<float4*>(a) = *reinterpret_cast<const float4*>(p.cosv + at);
    *reinterpret_cast<float4*>(a + 4) = *reinterpret_cast<const float4*>(p.cosv + at + 4);
    *reinterpret_cast<float4*>(a + 8) = *reinterpret_cast<const float4*>(p.sinv + at);
    *reinterpret_cast<float4*>(a + 12) = *reinterpret_cast<const float4*>(p.sinv + at + 4);
}
template <bool kInterleaved>
__device__ __forceinline__ void append_rotate(float (&a)[8], float (&b)[8], const float (&cs)[16]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (kInterleaved) {
            float* f = e < 4 ? a : b;
            rotate_pair(f[2 * (e & 3)], f[2 * (e & 3) + 1], cs[e], cs[8 + e]);
        } else {
            rotate_pair(a[e], b[e], cs[e], cs[8 + e]);
        }
    }
}

// One token's queries: kUnroll steps of 32 / LPT heads on their way at a time.
template <int D, bool kInterleaved>
__device__ __forceinline__ void append_queries(const AppendParams& p, int t, int lane) {
    constexpr int LPT = D / 16, HPS = 32 / LPT, kUnroll = 4;
    const int j = lane % LPT, grp = lane / LPT;
    const bool rot = j * 16 < p.R;
    const int ca = !kInterleaved && rot ? j : 2 * j, cb = !kInterleaved && rot ? j + p.R / 16 : 2 * j + 1;
    const __nv_bfloat16* src = p.Q + static_cast<int64_t>(t) * p.ldq + grp * D;
    __nv_bfloat16* dst = p.Qo + static_cast<int64_t>(t) * p.ldqo + grp * D;
    uint4 va[kUnroll], vb[kUnroll];
    auto load = [&](int h0) {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (h0 + u * HPS + grp < p.H) {
                va[u] = *reinterpret_cast<const uint4*>(src + static_cast<int64_t>(h0 + u * HPS) * D + ca * 8);
                vb[u] = *reinterpret_cast<const uint4*>(src + static_cast<int64_t>(h0 + u * HPS) * D + cb * 8);
            }
    };
    load(0);  // (the queries do not depend on the sequence: they are on their way before it is looked up)
    const int s = append_find_seq(p.S, t, lane, [&](int i) { return p.cu[i]; });
    const int t_begin = p.cu[s], t_end = p.cu[s + 1], ctx = p.ctx[s];
    if (t < t_begin || t >= t_end || !append_in_range(p, s, t_begin, t_end, ctx, lane)) return;
    float cs[16];
    if (rot) append_angles(p, static_cast<int64_t>(ctx) + (t - t_begin), j, cs);
    for (int h0 = 0; h0 < p.H; h0 += kUnroll * HPS) {
        if (h0 > 0) load(h0);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            if (h0 + u * HPS + grp < p.H) {
                float a[8], b[8];
                bf16x8_unpack(va[u], a);
                bf16x8_unpack(vb[u], b);
                if (rot) append_rotate<kInterleaved>(a, b, cs);
                *reinterpret_cast<uint4*>(dst + static_cast<int64_t>(h0 + u * HPS) * D + ca * 8) = bf16x8_pack(a);
                *reinterpret_cast<uint4*>(dst + static_cast<int64_t>(h0 + u * HPS) * D + cb * 8) = bf16x8_pack(b);
            }
        }
    }
}

template <int D, int BS, bool kF8, bool kInterleaved>
__global__ void __launch_bounds__(kAppendWarps * 32) kv_append_kernel(const AppendParams p, int kv_ctas_per_slot, int q_ctas) {
    constexpr int LPT = D / 16;      // lanes per token: each owns two chunks of 8 elements
    constexpr int TPS = 32 / LPT;    // tokens per step of a warp
    constexpr int STEPS = BS / TPS;
    static_assert(BS % TPS == 0, "whole steps per block");
    pdl_begin();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (static_cast<int>(blockIdx.x) < q_ctas) {
        const int t = blockIdx.x * kAppendWarps + warp;
        if (t < p.T) append_queries<D, kInterleaved>(p, t, lane);
        return;
    }
    const int kv = blockIdx.x - q_ctas;
    const int slot = kv / kv_ctas_per_slot;
    const int task = kv % kv_ctas_per_slot * kAppendWarps + warp;  // K heads, then V heads
    if (task >= 2 * p.H_kv) return;
    const bool is_v = task >= p.H_kv;
    const int head = is_v ? task - p.H_kv : task;
    const int s = append_find_seq(p.S, slot, lane, [&](int i) { return p.cu[i] / BS + 2 * i; });
    const int t_begin = p.cu[s], t_end = p.cu[s + 1], ctx = p.ctx[s];
    if (t_end <= t_begin) return;
    const int rel = slot - (t_begin / BS + 2 * s);
    if (rel < 0 || !append_in_range(p, s, t_begin, t_end, ctx, lane)) return;
    const int64_t blk64 = static_cast<int64_t>(ctx / BS) + rel;
    const int64_t end64 = static_cast<int64_t>(ctx) + (t_end - t_begin);
    if (blk64 * BS >= end64) return;
    const int blk = static_cast<int>(blk64);                                      // logical block
    const int off0 = max(0, static_cast<int>(ctx - blk64 * BS));                  // new tokens sit at offsets off0 .. off1 - 1 of it
    const int off1 = static_cast<int>(min(static_cast<int64_t>(BS), end64 - blk64 * BS));
    const int tok0 = t_begin + static_cast<int>(blk64 * BS - ctx);                // token of offset 0 (may lie before the sequence's first)

    // this lane's two chunks: partners of the rotation inside the first R elements, neighbours elsewhere
    const int j = lane % LPT, grp = lane / LPT;
    const bool rot = !is_v && j * 16 < p.R;
    int ca = 2 * j, cb = 2 * j + 1;
    if (!kInterleaved && rot) {
        ca = j;
        cb = j + p.R / 16;
    }
    const __nv_bfloat16* src = (is_v ? p.V : p.K) + static_cast<int64_t>(head) * D;
    const int64_t ld = is_v ? p.ldv : p.ldk;

    float fa[STEPS][8], fb[STEPS][8];
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        const int off = i * TPS + grp;
        uint4 va = make_uint4(0u, 0u, 0u, 0u), vb = va;
        if (off >= off0 && off < off1) {
            const __nv_bfloat16* row = src + static_cast<int64_t>(tok0 + off) * ld;
            va = *reinterpret_cast<const uint4*>(row + ca * 8);
            vb = *reinterpret_cast<const uint4*>(row + cb * 8);
        }
        bf16x8_unpack(va, fa[i]);
        bf16x8_unpack(vb, fb[i]);
    }
    if (rot) {
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            const int off = i * TPS + grp;
            if (off >= off0 && off < off1) {
                float cs[16];
                append_angles(p, blk64 * BS + off, j, cs);
                append_rotate<kInterleaved>(fa[i], fb[i], cs);
            }
        }
    }
    // (the elements are on their way while the table is read)
    const int phys = blk < p.max_blocks ? p.table[static_cast<int64_t>(s) * p.max_blocks + blk] : -1;
    if (phys < 0 || phys >= p.num_blocks) {  // never write through a bad table entry: report and leave the block out
        if (lane == 0) append_report(7u /* bad block */, blk, s, phys);
        return;
    }

    if (!kF8) {
        __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(is_v ? p.Vc : p.Kc) + (static_cast<int64_t>(phys) * p.H_kv + head) * BS * D;
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            const int off = i * TPS + grp;
            if (off >= off0 && off < off1) {
                *reinterpret_cast<uint4*>(dst + off * D + ca * 8) = bf16x8_pack(fa[i]);
                *reinterpret_cast<uint4*>(dst + off * D + cb * 8) = bf16x8_pack(fb[i]);
            }
        }
        return;
    }

    // ---- 8-bit cache: one scale for the block's tokens of this head ----
    float amax = 0.0f;
#pragma unroll
    for (int i = 0; i < STEPS; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fmaxf(abs_if_finite(fa[i][e]), abs_if_finite(fb[i][e])));
#pragma unroll
    for (int w = 1; w < 32; w <<= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, w));
    const int64_t at = static_cast<int64_t>(phys) * p.H_kv + head;
    float* scale_at = (is_v ? p.vs : p.ks) + at;
    uint8_t* rows = static_cast<uint8_t*>(is_v ? p.Vc : p.Kc) + at * BS * D;
    float scale = pow2f(f8_scale_exp(amax));
    if (off0 > 0) {  // the block holds off0 tokens of this sequence already
        const float old = *scale_at;
        if (old >= scale) {
            scale = old;
        } else {
            const float ratio = old / scale;
#pragma unroll 1
            for (int i = 0; i < STEPS; ++i) {
                const int off = i * TPS + grp;
                if (off < off0) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint2* q = reinterpret_cast<uint2*>(rows + off * D + (h ? cb : ca) * 8);
                        const uint2 v = *q;
                        uint32_t o[2];
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            uint32_t lo, hi;
                            f16x2_from_f8x4(u ? v.y : v.x, lo, hi);
                            const float2 x = f32x2_from_f16x2(lo), y = f32x2_from_f16x2(hi);
                            o[u] = f8x4_from_f32(mul_to_odd(x.x, ratio), mul_to_odd(x.y, ratio), mul_to_odd(y.x, ratio), mul_to_odd(y.y, ratio));
                        }
                        *q = make_uint2(o[0], o[1]);
                    }
                }
            }
        }
    }
    __syncwarp();  // every lane has read the old scale
    if (lane == 0) *scale_at = scale;
    // x / scale is exact for a power of two; a scale that came from elsewhere (and only such a block's) goes through divisions
    float inv = 1.0f / scale;
    if (!is_pow2(scale)) {
        inv = 1.0f;
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                fa[i][e] = div_to_odd(fa[i][e], scale);
                fb[i][e] = div_to_odd(fb[i][e], scale);
            }
    }
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        const int off = i * TPS + grp;
        if (off >= off0 && off < off1) {
            uint8_t* row = rows + off * D;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float* f = h ? fb[i] : fa[i];
                *reinterpret_cast<uint2*>(row + (h ? cb : ca) * 8) =
                    make_uint2(f8x4_from_f32(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv),
                               f8x4_from_f32(f[4] * inv, f[5] * inv, f[6] * inv, f[7] * inv));
            }
        }
    }
}

template <int D, int BS, bool kF8>
int append_launch_r(const AppendParams& p, bool interleaved, cudaStream_t st) {
    const int per_slot = (2 * p.H_kv + kAppendWarps - 1) / kAppendWarps, q_ctas = p.Q ? (p.T + kAppendWarps - 1) / kAppendWarps : 0;
    const int64_t ctas = q_ctas + (p.T / BS + 2ll * p.S) * per_slot;
    if (ctas > INT32_MAX) return 2;
    const dim3 grid(static_cast<unsigned>(ctas)), block(kAppendWarps * 32);
    const cudaError_t e = interleaved ? pdl_launch(kv_append_kernel<D, BS, kF8, true>, grid, block, 0, st, 0, p, per_slot, q_ctas)
                                      : pdl_launch(kv_append_kernel<D, BS, kF8, false>, grid, block, 0, st, 0, p, per_slot, q_ctas);
    return e == cudaSuccess ? 0 : 4;
}
template <int D, bool kF8>
int append_launch_bs(const AppendParams& p, int block_size, bool interleaved, cudaStream_t st) {
    switch (block_size) {
        case 8: return append_launch_r<D, 8, kF8>(p, interleaved, st);
        case 16: return append_launch_r<D, 16, kF8>(p, interleaved, st);
        case 32: return append_launch_r<D, 32, kF8>(p, interleaved, st);
        default: return 2;
    }
}
inline int append_launch(const AppendParams& p, int D, int block_size, bool f8, bool interleaved, cudaStream_t st) {
    if (D == 64) return f8 ? append_launch_bs<64, true>(p, block_size, interleaved, st) : append_launch_bs<64, false>(p, block_size, interleaved, st);
    return f8 ? append_launch_bs<128, true>(p, block_size, interleaved, st) : append_launch_bs<128, false>(p, block_size, interleaved, st);
}

}  // namespace mlt
