// Runs the plan of the packed attention on the CPU: the kernel's own text, cut out of the source by packed_plan_util.py, with a CTA's
// threads as coroutines of one thread.  A barrier or a warp collective lets the others run until all have come to it.
#include <setjmp.h>
#include <ucontext.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>

using std::max;
using std::min;
struct __nv_bfloat16 {
    uint16_t x;
};
struct int2 {
    int x, y;
};
struct int3 {
    int x, y, z;
};
struct alignas(16) int4 {
    int x, y, z, w;
};
struct float2 {
    float x, y;
};
static int2 make_int2(int x, int y) { return {x, y}; }
static int3 make_int3(int x, int y, int z) { return {x, y, z}; }
static int4 make_int4(int x, int y, int z, int w) { return {x, y, z, w}; }

namespace host {

constexpr int kThreads = 1024, kStack = 64 * 1024;
struct Warp {
    uint32_t value[2][32];
    int arrived = 0;
    unsigned generation = 0;
};
struct Fiber {
    ucontext_t first;
    jmp_buf at;
    const unsigned* waits_for;  // a generation that has to differ from `seen`
    unsigned seen;
    bool started, finished;
};
static Fiber fibers[kThreads];
static jmp_buf scheduler;
static Warp warps[kThreads / 32];
static int arrived = 0;
static unsigned generation = 0;
static std::vector<char> stacks;
static struct {
    int x;
} thread;
static void (*entry)();

static void wait(const unsigned& generation, unsigned seen) {
    Fiber& f = fibers[thread.x];
    f.waits_for = &generation;
    f.seen = seen;
    if (_setjmp(f.at) == 0) _longjmp(scheduler, 1);
}
static void start() {
    entry();
    fibers[thread.x].finished = true;
    _longjmp(scheduler, 1);
}
static void barrier() {
    const unsigned mine = generation;
    if (++arrived == kThreads) {
        arrived = 0;
        ++generation;
    } else {
        wait(generation, mine);
    }
}
// all lanes' values (of the collective that all of them are at)
static const uint32_t* exchange(uint32_t v) {
    Warp& w = warps[thread.x / 32];
    const unsigned mine = w.generation;
    w.value[mine & 1][thread.x % 32] = v;
    if (++w.arrived == 32) {
        w.arrived = 0;
        ++w.generation;
    } else {
        wait(w.generation, mine);
    }
    return w.value[mine & 1];
}
static bool run(void (*f)()) {
    entry = f;
    stacks.resize(static_cast<size_t>(kThreads) * kStack);
    arrived = 0;
    for (Warp& w : warps) w.arrived = 0;
    for (int i = 0; i < kThreads; ++i) {
        Fiber& t = fibers[i];
        t.waits_for = nullptr;
        t.started = t.finished = false;
        getcontext(&t.first);
        t.first.uc_stack.ss_sp = stacks.data() + static_cast<size_t>(i) * kStack;
        t.first.uc_stack.ss_size = kStack;
        t.first.uc_link = nullptr;
        makecontext(&t.first, start, 0);
    }
    static int left;  // (not in a register: _longjmp comes back into this function)
    static int i;
    static bool moved;
    for (left = kThreads; left > 0;) {
        moved = false;
        for (i = 0; i < kThreads; ++i) {
            Fiber& t = fibers[i];
            if (t.finished || (t.waits_for && *t.waits_for == t.seen)) continue;
            moved = true;
            thread.x = i;
            t.waits_for = nullptr;
            if (_setjmp(scheduler) == 0) {
                if (t.started) _longjmp(t.at, 1);
                t.started = true;
                setcontext(&t.first);
            }
            left -= fibers[i].finished;
        }
        if (!moved) return false;  // some never come to a barrier that others wait at
    }
    return true;
}
template <class T>
static uint32_t bits(T v) {
    uint32_t b;
    memcpy(&b, &v, 4);
    return b;
}
template <class T>
static T as(uint32_t b) {
    T v;
    memcpy(&v, &b, 4);
    return v;
}

}  // namespace host

#define __host__
#define __device__
#define __global__
#define __noinline__
#define __forceinline__ inline
#define __launch_bounds__(...)
#define __shared__ static
#define threadIdx host::thread
static void __syncthreads() { host::barrier(); }
static void cudaGridDependencySynchronize() {}
static void pdl_launch_dependents() {}
template <class T>
static T __shfl_up_sync(unsigned, T v, int by) {
    const int lane = threadIdx.x & 31;
    const uint32_t* all = host::exchange(host::bits(v));
    return host::as<T>(all[lane >= by ? lane - by : lane]);
}
template <class T>
static T __shfl_sync(unsigned, T v, int lane) {
    return host::as<T>(host::exchange(host::bits(v))[lane & 31]);
}
template <class T>
static T __shfl_xor_sync(unsigned, T v, int by) {
    const int lane = threadIdx.x & 31;
    return host::as<T>(host::exchange(host::bits(v))[lane ^ by]);
}
static int __reduce_max_sync(unsigned, int v) {
    const uint32_t* all = host::exchange(host::bits(v));
    int r = host::as<int>(all[0]);
    for (int i = 1; i < 32; ++i) r = max(r, host::as<int>(all[i]));
    return r;
}
static int __reduce_add_sync(unsigned, int v) {
    const uint32_t* all = host::exchange(host::bits(v));
    uint32_t r = 0;
    for (int i = 0; i < 32; ++i) r += all[i];
    return host::as<int>(r);
}
static uint32_t __reduce_min_sync(unsigned, uint32_t v) {
    const uint32_t* all = host::exchange(v);
    return *std::min_element(all, all + 32);
}
static uint32_t __ballot_sync(unsigned, bool v) {
    const uint32_t* all = host::exchange(v);
    uint32_t r = 0;
    for (int i = 0; i < 32; ++i) r |= all[i] << i;
    return r;
}
static int __clz(int v) { return v ? __builtin_clz(static_cast<unsigned>(v)) : 32; }
static int __ffs(unsigned v) { return __builtin_ffs(static_cast<int>(v)); }
static int __float2int_rd(float v) { return static_cast<int>(std::floor(v)); }
static uint32_t __float_as_uint(float v) { return host::bits(v); }
static int atomicAdd(int* p, int v) {
    const int old = *p;
    *p += v;
    return old;
}
static int atomicMax(int* p, int v) {
    const int old = *p;
    *p = max(old, v);
    return old;
}
static unsigned atomicCAS(unsigned* p, unsigned expected, unsigned v) {
    const unsigned old = *p;
    if (old == expected) *p = v;
    return old;
}

static unsigned g_status[4];
constexpr int kMhaBlock = 128;
alignas(16) static char plan_memory[256 * 1024];
#include "packed_plan_source.inc"  // the plan, its scratch, and the rule for the rows of parts

static PackedParams params;
static void plan() { mha_packed_plan_kernel(params); }

// What mlt.cu fills in, for each entry point.  kind: 0 packed, 1 prefill, 2 shared.  Returns the bytes of lists, or < 0.
extern "C" long long packed_scratch_layout(int kind, long long T, long long S, int G, int H_kv, int D, long long* out) {
    const PackedScratch x = packed_scratch(T, S, G, H_kv, D, kind == 2);
    const long long v[] = {(long long)x.seqs, (long long)x.key_base, (long long)x.entries, (long long)x.entry_rows, (long long)x.tile_info, (long long)x.lists,
                           (long long)x.row_bytes, x.part_rows, x.max_tiles, x.max_entries, x.W};
    memcpy(out, v, sizeof(v));
    return static_cast<long long>(x.lists);
}

extern "C" int run_packed_plan(int kind, int T, int S, int num_k, int G, int H_kv, int D, int causal, int block_size, int max_blocks, int sm_count,
                               const int* cu_q, const int* cu_k, const int* context_lens, const int* prefix_lens, const int* seq_lens, uint8_t* workspace,
                               long long workspace_bytes, int* part_rows, unsigned* status) {
    const PackedScratch x = packed_scratch(T, S, G, H_kv, D, kind == 2);
    params = PackedParams{};
    PackedParams& p = params;
    p.S = p.all = S;
    p.T = T;
    p.G = G;
    p.W = x.W;
    p.H = G * H_kv;
    p.H_kv = H_kv;
    p.hdr = reinterpret_cast<PackedHeader*>(workspace);
    p.seqs = reinterpret_cast<int4*>(workspace + x.seqs);
    p.key_base = reinterpret_cast<long long*>(workspace + x.key_base);
    p.entries = reinterpret_cast<int4*>(workspace + x.entries);
    p.entry_rows = reinterpret_cast<int*>(workspace + x.entry_rows);
    p.tile_info = reinterpret_cast<int2*>(workspace + x.tile_info);
    p.max_tiles = static_cast<int>(x.max_tiles);
    p.max_entries = static_cast<int>(x.max_entries);
    p.sm_count = sm_count;
    p.cu_q = cu_q;
    p.causal = kind == 2 ? 0 : causal;
    p.block_size = block_size;
    p.max_blocks = max_blocks;
    if (kind == 0) {
        p.cu_k = cu_k;
        p.num_k = num_k;
        p.part_rows = static_cast<int>(packed_part_limit(x, T, num_k, H_kv, workspace_bytes, sm_count));
    } else if (kind == 1) {
        p.context_lens = context_lens;
        p.part_rows = static_cast<int>(packed_part_limit(x, T, static_cast<int64_t>(max_blocks) * block_size, H_kv, workspace_bytes, sm_count));
    } else {
        p.all = S + T;
        p.prefix_lens = prefix_lens;
        p.seq_lens = seq_lens;
        p.part_rows = static_cast<int>(x.part_rows);
    }
    *part_rows = p.part_rows;
    memset(g_status, 0, sizeof(g_status));
    const bool ok = host::run(plan);
    memcpy(status, g_status, sizeof(g_status));
    return ok ? 0 : 1;
}
