// A thread-block cluster on the host: its threads are fibers that change turns at every barrier, shuffle and ballot, in an order that the caller
// chooses.  What the barriers of a kernel leave open, one order or another brings out; shared memory begins as a byte of the caller's
// choice.  (Between two such points a thread runs undisturbed, so orders of single loads and stores are not tried.)
#pragma once
#include <stdint.h>
#include <stdlib.h>
#include <string.h>
#include <ucontext.h>

#include <algorithm>
#include <functional>
#include <set>
#include <utility>
#include <vector>

namespace simt {

struct Dim { unsigned x, y, z; };
struct Fiber;
struct Barrier {
    int need = 0, arrived = 0;
    uint64_t phase = 0;
    std::vector<Fiber *> waiting;
};
struct Fiber {
    ucontext_t context;
    int rank, tid;
    uint64_t key;      // runnable ones with the least go first
    long turns = 0;
    void *stack = nullptr;
};
enum Order { kUpperFirst, kLowerFirst, kOneByOne, kBackwards, kDrawn };

struct Cluster {
    int ctas, threads;
    Order order;
    uint64_t seed;
    ucontext_t back;
    Fiber *now = nullptr;
    std::vector<Fiber> fibers;
    std::set<std::pair<uint64_t, Fiber *>> ready;
    std::vector<Barrier> cta, warps;
    Barrier all;
    std::vector<uint32_t> deposits;       // of a warp two turns of 32 words
    std::vector<std::vector<uint8_t>> shared;
    std::function<void()> body;
    int finished = 0;
};
inline Cluster *g = nullptr;
inline Dim g_block;

inline void make_ready(Fiber *f)
{
    const uint64_t turns = f->turns, n = f->rank * 1024 + f->tid, half = f->tid >= g->threads / 2;
    switch (g->order) {
    case kUpperFirst: f->key = (half ^ 1) << 40 | turns; break;
    case kLowerFirst: f->key = half << 40 | turns; break;
    case kOneByOne: f->key = n; break;
    case kBackwards: f->key = ~n; break;
    default: f->key = g->seed = g->seed * 6364136223846793005ull + 1442695040888963407ull, f->key >>= 20;
    }
    g->ready.insert({f->key, f});
}
inline void pause() { swapcontext(&g->now->context, &g->back); }
// everybody else's turn; then this one's again
inline void yield()
{
    ++g->now->turns;
    make_ready(g->now);
    pause();
}
inline uint64_t arrive(Barrier &b)
{
    const uint64_t phase = b.phase;
    if (++b.arrived == b.need) {
        ++b.phase, b.arrived = 0;
        for (Fiber *f : b.waiting) make_ready(f);
        b.waiting.clear();
    }
    return phase;
}
inline void wait(Barrier &b, uint64_t phase)
{
    if (b.phase > phase) return yield();
    ++g->now->turns;
    b.waiting.push_back(g->now);
    pause();
}
inline void meet(Barrier &b) { wait(b, arrive(b)); }
// a word of every lane of the warp
inline const uint32_t *exchange(uint32_t word)
{
    const int w = g->now->rank * (g->threads / 32) + g->now->tid / 32;
    Barrier &b = g->warps[w];
    uint32_t *at = &g->deposits[(w * 2 + (b.phase & 1)) * 32];
    at[g->now->tid & 31] = word;
    meet(b);
    return at;
}
inline void start()
{
    g->body();
    ++g->finished;
    pause();
}
// false: threads wait for something that nobody does
inline bool run(Cluster &c)
{
    g = &c;
    c.fibers.resize(c.ctas * c.threads), c.cta.resize(c.ctas), c.warps.resize(c.ctas * c.threads / 32), c.deposits.resize(c.warps.size() * 64);
    for (Barrier &b : c.cta) b.need = c.threads;
    for (Barrier &b : c.warps) b.need = 32;
    c.all.need = c.ctas * c.threads;
    constexpr size_t kStack = 48 << 10;
    for (size_t i = 0; i < c.fibers.size(); ++i) {
        Fiber &f = c.fibers[i];
        f.rank = i / c.threads, f.tid = i % c.threads, f.stack = malloc(kStack);
        getcontext(&f.context);
        f.context.uc_stack.ss_sp = f.stack, f.context.uc_stack.ss_size = kStack, f.context.uc_link = nullptr;
        makecontext(&f.context, start, 0);
        make_ready(&f);
    }
    while (!c.ready.empty()) {
        c.now = c.ready.begin()->second;
        c.ready.erase(c.ready.begin());
        swapcontext(&c.back, &c.now->context);
    }
    for (Fiber &f : c.fibers) free(f.stack);
    return c.finished == (int)c.fibers.size();
}

template <class T>
T *shared(size_t offset = 0) { return reinterpret_cast<T *>(g->shared[g->now->rank].data() + offset); }

}  // namespace simt

#define __device__
#define __host__
#define __global__
#define __forceinline__ inline
#define __launch_bounds__(...)
#define __grid_constant__
#define threadIdx (simt::Dim{(unsigned)simt::g->now->tid, 0u, 0u})
#define blockIdx (simt::Dim{(unsigned)simt::g->now->rank, simt::g_block.y, simt::g_block.z})
using std::max;
using std::min;
struct uint2 { uint32_t x, y; };
struct uint4 { uint32_t x, y, z, w; };
struct float2 { float x, y; };
struct float4 { float x, y, z, w; };
inline uint4 make_uint4(uint32_t x, uint32_t y, uint32_t z, uint32_t w) { return {x, y, z, w}; }
inline float4 make_float4(float x, float y, float z, float w) { return {x, y, z, w}; }
inline float bits_to_float(uint32_t b) { float f; memcpy(&f, &b, 4); return f; }
inline uint32_t __float_as_uint(float f) { uint32_t b; memcpy(&b, &f, 4); return b; }
struct __nv_bfloat162 { uint16_t x, y; };
inline float2 __bfloat1622float2(__nv_bfloat162 v) { return {bits_to_float((uint32_t)v.x << 16), bits_to_float((uint32_t)v.y << 16)}; }
template <class T>
T __ldg(const T *p) { return *p; }
inline int __popc(uint32_t x) { return __builtin_popcount(x); }
template <class T>
T atomicAdd(T *p, T v) { const T old = *p; *p += v; return old; }
template <class T>
T atomicOr(T *p, T v) { const T old = *p; *p |= v; return old; }
inline void __syncthreads() { simt::meet(simt::g->cta[simt::g->now->rank]); }
inline uint32_t __shfl_sync(uint32_t, uint32_t v, int lane) { return simt::exchange(v)[lane & 31]; }
inline uint32_t __shfl_up_sync(uint32_t, uint32_t v, int d)
{
    const int lane = simt::g->now->tid & 31;
    const uint32_t *all = simt::exchange(v);
    return lane >= d ? all[lane - d] : v;
}
inline uint32_t __shfl_xor_sync(uint32_t, uint32_t v, int d) { return simt::exchange(v)[(simt::g->now->tid & 31) ^ d]; }
inline uint32_t __ballot_sync(uint32_t, bool v)
{
    const uint32_t *all = simt::exchange(v);
    uint32_t bits = 0;
    for (int i = 0; i < 32; ++i) bits |= all[i] << i;
    return bits;
}

namespace cooperative_groups {
struct cluster_group {
    int block_rank() const { return simt::g->now->rank; }
    uint64_t barrier_arrive() const
    {
        const uint64_t phase = simt::arrive(simt::g->all);
        simt::yield();
        return phase;
    }
    void barrier_wait(uint64_t &&phase) const { simt::wait(simt::g->all, phase); }
    void sync() const { simt::meet(simt::g->all); }
    template <class T>
    T *map_shared_rank(T *p, int rank) const
    {
        const size_t at = reinterpret_cast<const uint8_t *>(p) - simt::g->shared[simt::g->now->rank].data();
        return reinterpret_cast<T *>(simt::g->shared[rank].data() + at);
    }
};
inline cluster_group this_cluster() { return {}; }
}  // namespace cooperative_groups

namespace svk {
constexpr int kStatusIndex = 1;
inline void grid_dependency_wait() {}
inline void grid_launch_dependents() {}
}  // namespace svk
