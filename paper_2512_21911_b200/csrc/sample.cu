// sv_sample: temperature, top-k, top-p and min-p on rows of logits, the kept entries' distribution and a token drawn from it.
//
// Mathematics: e(x) = 2^((x - max) log2 e / temperature).  The entries are never sorted: what stays is everything up to one entry, the
// boundary (logit, index), in the order "larger logit first, then smaller index".  Search for the boundary by count (top-k) or mass
// (top-p): a histogram of the entries by their distance from the maximum, the bin in which the goal is reached, and the few entries of
// that bin, divided again in the same way until a warp has them.  A bin with too many of them is divided again by the bits of its keys;
// entries that are all equal are counted off by index.  For a short top-k the histogram holds the threads' maxima only: the k-th largest
// of these bounds the k-th entry from below, all entries up to its bin are ranked at once, and top-p, min-p and the token follow from
// that list.
//
// Sums of masses are sums of whole numbers, exact in any order.  Of the nucleus: multiples of 2^-32 of the largest entry's mass, so that a
// bin is two 32-bit words that shared-memory atomics add to (2^-32 is less than fp32 sums keep; what is lost are entries below 2^-33 of
// the largest, 2^-16 of its mass if there were 2^17 of them); they also do for the draw from a nucleus, whose histogram has them by CTA.
// Of other draws: multiples of 2^-40, added in registers.
//
// A cluster of 1 to 8 CTAs per row; a CTA keeps its part of the row in shared memory, so the logits are read once from HBM (19.5 MB of 19.4
// for 64 bfloat16 rows of 151,936).  Warps own contiguous parts: a token is found by sums per CTA, warp and lane.
//
// Bound by the instructions of the passes (some 27 an entry for the histogram, 11 to gather a bin, 19 for the probabilities) and by the
// steps between them (a barrier of the cluster is 1.8 us), two CTAs an SM overlapping one's steps with the other's passes: warps issue in
// half of the cycles, and HBM, whose floor for these cases is 3 to 12 us, idles.  Measured, with nothing in L2 before the call: one row of
// 128,256 with a top-k of 50 13.3 us; 64 bfloat16 rows of 151,936 with a nucleus 48.4 us, one round of clusters of four; 80 rows of
// 128,256 with a nucleus and their distributions 77 us, three rounds of clusters of eight (12 of them the load, 10 the probabilities); 256
// rows of 32,003 with top-k, min-p and distributions 44 us.  Of calls back to back, whose rows are in L2: tests of an entry are written
// without branches, of which a pass had 20 an entry before (13.7, 57, 84 and 40 us, with lists ranked entry against entry by every CTA;
// 12.8, 48, 75 and 37.5 then).  A histogram of its own for rows without a top-k takes 46 us for the 64 rows and 13.7 for the one, by
// more code to fetch.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <float.h>

#include <algorithm>
#include <type_traits>

#include "sv_host.h"
#include "sv_ptx.cuh"

namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kBins = 2048;
constexpr int kGroups = 64;                    // of 32 bins each
constexpr float kBinsPerBit = 2048.f / 36.f;   // bins of the first histogram: 36 powers of two below the maximum, beyond what has a mass
constexpr int kList = 768;                     // entries that are looked at one by one
constexpr int kGrain = kWarps * 128;           // a CTA's part of a row is a multiple of this: 32 lanes x 4 entries for each warp
constexpr int kMostPart = 24 * kGrain;         // entries that fit in shared memory
constexpr int kTwo = 80 * 1024;                // bytes of a part that leave room for a second CTA on the SM
constexpr int kMaxVocab = kMaxCluster * kMostPart;
static_assert((1ll << 16) * kMostPart < 1ll << 32 && (1ll << 15) * kMostPart < 1ll << 31, "words of a bin");

using Mass = unsigned long long;

struct Params {
    const void *logits;
    long long stride;
    const float *temperature, *top_p, *min_p, *u;
    const int32_t *top_k;
    int32_t *tokens;
    float *probs;
    int V, rows_per_param;
    int part;   // entries of a CTA
};

// Ascending in the logit; -0 equals +0.  (Not for -infinity, which stands for an entry that is not there.)
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t b = __float_as_uint(x) == 0x80000000u ? 0u : __float_as_uint(x);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }
// What a logit counts as: a NaN as -infinity, +infinity as the largest number.
__device__ __forceinline__ float taken(float x) { return fminf(fmaxf(x, -INFINITY), FLT_MAX); }

// e * 2^(2 N) to the nearest integer as high * 2^N + low, by adding numbers whose last place is 1 (0 <= e <= 1).
struct Parts {
    uint32_t high;   // <= 2^N
    int low;         // at most 2^(N - 1) either way
};
template <int N>
__device__ __forceinline__ Parts parts_of(float e)
{
    constexpr float kOne = (float)(1 << N);
    const float t = __fmaf_rn(e, kOne, 8388608.f), rest = __fmaf_rn(e, kOne, -__fsub_rn(t, 8388608.f));
    return {__float_as_uint(t) - 0x4b000000u, (int)(__float_as_uint(__fmaf_rn(rest, kOne, 12582912.f)) - 0x4b400000u)};
}
template <int N>
__device__ __forceinline__ Mass whole(uint32_t high, int low) { return ((Mass)high << N) + (long long)low; }
template <int N>
__device__ __forceinline__ Mass mass_of(float e)
{
    const Parts p = parts_of<N>(e);
    return whole<N>(p.high, p.low);
}
constexpr int kNucleus = 16, kDraw = 20;   // halves of the bits of a mass
constexpr int kEach = (kList + kThreads - 1) / kThreads;   // entries of a list for each thread

struct Boundary {
    float x;
    uint32_t index;   // the last entry that stays
    __device__ bool keeps(float y, uint32_t i) const { return (y > x) | ((y == x) & (i <= index)); }
};

struct alignas(16) Smem {
    uint32_t high[kBins];     // histogram: sums of masses in two words, or counts in the second; later the list's masses
    int low[kBins];
    Mass list[kList], sorted[kList];   // key << 32 | ~index: descending is the order of the rule
    Mass sums[kWarps], scan[kWarps];
    Mass of_cta[2][kMaxCluster];   // written by all CTAs of the cluster; two in turn, so that no CTA writes what another still reads
    float top_of_cta[kMaxCluster], of_warp[kWarps];
    uint32_t count_of_cta[kMaxCluster];
    uint32_t range[kMaxCluster][2];
    Mass found_ahead, found_goal;
    int found_bin, token;
    Boundary boundary;
    uint32_t n_list;
    // The sums of every CTA's groups of bins, written by it, where the sorted list is later.  (Between two uses the cluster has a barrier.)
    __device__ Mass *groups(int cta) { return sorted + cta * kGroups; }
    __device__ Mass *masses() { return reinterpret_cast<Mass *>(high); }
};
static_assert(kBins * 4 >= kList * 8 && kList >= kMaxCluster * kGroups, "");

template <class T, class Op>
__device__ __forceinline__ T over_warp(T v, Op op)
{
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, d));
    return v;
}
__device__ __forceinline__ Mass sum_over_warp(Mass v) { return over_warp(v, [](Mass a, Mass b) { return a + b; }); }
template <class T>
__device__ __forceinline__ T scan_warp(T v)   // inclusive
{
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const T o = __shfl_up_sync(0xffffffffu, v, d);
        if ((threadIdx.x & 31) >= d) v += o;
    }
    return v;
}

// (one instruction with a predicate: as a branch it was a quarter of a pass)
__device__ __forceinline__ void add_shared(uint32_t at, int v)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.s32 p, %1, 0;\n\t@p red.shared.add.u32 [%0], %1;\n\t}" ::"r"(at), "r"(v) : "memory");
}

// log2 e / temperature to more than the bits of a float, in two words neither of which is negative or zero (times an infinite distance the
// sum stays infinite).  Rounded to one float, the rate acts as a temperature 2^-24 beside the one asked for, which in a vocabulary of 128K
// moves the sums at a nucleus' edge by up to 1e-7 of the whole: 1 % of the mass of the entry there.  The second word takes up to 2 % of a
// call (64 rows 48.0 -> 48.4 to 49.2 us, 80 rows with their distributions 77.2 -> 76.4 to 78.8, nothing in L2).
struct Rate {
    float high, low;
};
__device__ __forceinline__ Rate rate_of(float temperature)
{
    constexpr float kHigh = 1.4426950216f, kLow = 1.92596299e-8f, kLeast = 1.2e-38f;   // (log2 e; an infinite temperature: all alike)
    const float high = __fdiv_rd(kHigh, temperature);
    if (!(high > kLeast)) return {kLeast, kLeast};
    return {high, fmaxf(__fdividef(__fmaf_rn(-high, temperature, kHigh) + kLow, temperature), kLeast)};
}
// -log2 e(x)
__device__ __forceinline__ float bits_below(float peak, float x, Rate rate)
{
    const float d = __fsub_rn(peak, x);
    return __fmaf_rn(d, rate.high, __fmul_rn(d, rate.low));
}

// The cluster's CTAs, and a word of this CTA's shared memory in each of them (one warp).
__device__ __forceinline__ int cluster_size() { return (int)cg::this_cluster().num_blocks(); }
__device__ __forceinline__ int cluster_rank() { return (int)cg::this_cluster().block_rank(); }
template <class T>
__device__ __forceinline__ void everywhere(T *at, T v)
{
    const int lane = threadIdx.x & 31;
    if (lane < cluster_size()) *cg::this_cluster().map_shared_rank(at, lane) = v;
}

// The steps between the passes are functions of their own: inlined where they are used, the kernel had 230 KB of code that is run through
// once, and the time was that of fetching it.

// Exclusive prefix and total over the CTA, in thread order.
struct Scan {
    Mass before, total;
};
__device__ __noinline__ Scan scan_block(Smem &sm, Mass v)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const Mass upto = scan_warp(v);
    __syncthreads();
    if (lane == 31) sm.scan[warp] = upto;
    __syncthreads();
    Scan s = {upto - v, 0};
#pragma unroll 1
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) s.before += sm.scan[w];
        s.total += sm.scan[w];
    }
    return s;
}
// Total over the cluster of a value of each thread; sums keeps the warps' totals, of_cta[turn] the CTAs'.
__device__ __noinline__ Mass sum_over_cluster(Smem &sm, int turn, Mass v)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    v = sum_over_warp(v);
    __syncthreads();
    if (lane == 0) sm.sums[warp] = v;
    __syncthreads();
    if (warp == 0) everywhere(&sm.of_cta[turn][cluster_rank()], sum_over_warp(lane < kWarps ? sm.sums[lane] : 0));
    cg::this_cluster().sync();
    return sum_over_warp(lane < cluster_size() ? sm.of_cta[turn][lane] : 0);
}
// The bin in which the sums over the cluster's histograms reach the goal (0: `of_all` of the sum of all), and what is in the bins ahead
// of it.  Every CTA tells all others the sums of its groups of bins, finds the group of the goal by itself and reads the bins of that
// group from all CTAs: one barrier of the cluster (1.8 us each, with what goes before it), where shares of the bins added up by different
// CTAs take three.  -1: there is not as much.  The bins have to stay until the cluster's next barrier.
struct Found {
    int bin;
    Mass goal, ahead;
};
__device__ __noinline__ Found find_in_bins(Smem &sm, Mass goal, float of_all)
{
    const cg::cluster_group cluster = cg::this_cluster();
    const int CL = cluster_size(), rank = cluster_rank(), tid = threadIdx.x, lane = tid & 31;
    static_assert(kBins == 4 * kThreads && kBins == 32 * kGroups, "");
    __syncthreads();
    Mass mine = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) mine += whole<kNucleus>(sm.high[4 * tid + i], sm.low[4 * tid + i]);
#pragma unroll
    for (int d = 4; d > 0; d >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, d);
    if ((lane & 7) < CL) *cluster.map_shared_rank(sm.groups(rank) + (tid >> 3), lane & 7) = mine;   // (lanes of a group: the CTA to tell)
    cluster.sync();
    if (tid < 32) {
        Mass g[2] = {0, 0};
#pragma unroll 1
        for (int c = 0; c < CL; ++c) g[0] += sm.groups(c)[2 * lane], g[1] += sm.groups(c)[2 * lane + 1];
        const Mass upto = scan_warp(g[0] + g[1]), total = __shfl_sync(0xffffffffu, upto, 31);
        if (goal == 0) goal = max((Mass)1, (Mass)ceil((double)fmaxf(of_all, 0.f) * (double)total));
        int bin = -1;
        Mass ahead = 0;
        if (goal <= total) {
            const Mass before = upto - g[0] - g[1];
            const bool here = before < goal && upto >= goal, second = before + g[0] < goal;
            const int at = __ffs(__ballot_sync(0xffffffffu, here)) - 1;
            const int group = 2 * at + __shfl_sync(0xffffffffu, (int)second, at);
            ahead = __shfl_sync(0xffffffffu, second ? before + g[0] : before, at);
            Mass v = 0;
#pragma unroll 1
            for (int c = 0; c < CL; c += 4) {
                uint32_t high[4];
                int low[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int from = min(c + k, CL - 1);
                    high[k] = *cluster.map_shared_rank(&sm.high[group * 32 + lane], from), low[k] = *cluster.map_shared_rank(&sm.low[group * 32 + lane], from);
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) v += c + k < CL ? whole<kNucleus>(high[k], low[k]) : 0;
            }
            const Mass sum = ahead + scan_warp(v);
            const int in = __ffs(__ballot_sync(0xffffffffu, sum >= goal)) - 1;   // (the group reaches the goal)
            bin = group * 32 + in;
            ahead = __shfl_sync(0xffffffffu, sum - v, in);
        }
        if (lane == 0) sm.found_bin = bin, sm.found_ahead = ahead, sm.found_goal = goal;
    }
    __syncthreads();
    return {sm.found_bin, sm.found_goal, sm.found_ahead};
}
// All CTAs' lists behind this one's own, and sorted where that is asked for; their length (over kList: there is no list).  mine: what the
// CTA tells the others, into of_cta[turn].  The lists have to stay until the cluster's next barrier.
__device__ __noinline__ uint32_t collect(Smem &sm, int turn, Mass mine, bool sort)
{
    const cg::cluster_group cluster = cg::this_cluster();
    const int CL = cluster_size(), rank = cluster_rank(), tid = threadIdx.x;
    mine = sum_over_warp(mine);
    __syncthreads();
    if ((tid & 31) == 0) sm.sums[tid >> 5] = mine;
    __syncthreads();
    if (tid < 32) everywhere(&sm.count_of_cta[rank], sm.n_list), everywhere(&sm.of_cta[turn][rank], sum_over_warp(tid < kWarps ? sm.sums[tid] : 0));
    cluster.sync();
    // 64 threads for every CTA's list, all of them at once: behind this CTA's own, in the order of the CTAs
    constexpr int kPull = kThreads / kMaxCluster;
    const int from = tid / kPull;
    uint32_t n = 0, at = 0;
#pragma unroll 1
    for (int c = 0; c < CL; ++c) {
        if (c == from) at = n;
        n += sm.count_of_cta[c];
    }
    if (n > kList) {
        cluster.sync();   // (the counts and the bins may be written again)
        return n;
    }
    if (from < CL && from != rank) {
        const uint32_t count = sm.count_of_cta[from];
        if (from < rank) at += sm.count_of_cta[rank];
#pragma unroll 1
        for (uint32_t i = tid % kPull; i < count; i += kPull) sm.list[at + i] = *cluster.map_shared_rank(&sm.list[i], from);
    }
    __syncthreads();
    if (!sort) return n;
#pragma unroll 1
    for (uint32_t i = tid; i < n; i += kThreads) {
        const uint64_t me = sm.list[i];
        int place = 0;
#pragma unroll 4
        for (uint32_t o = 0; o < n; ++o) place += sm.list[o] > me;
        sm.sorted[place] = me;
    }
    __syncthreads();
    return n;
}

// Of the list's n entries, in their order, the one that brings the sum of their weights to the goal (it exists): divided into 256 parts
// of their range by sums as in the large histogram, the part of the goal divided again until a warp has what is left of it.  (Ranked one
// against another by all CTAs, 300 to 700 entries were most of a row's instructions.)
__device__ __noinline__ Boundary pick(Smem &sm, uint32_t n, Mass goal, bool by_mass, float peak, Rate rate)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    constexpr int kParts = 256, kWarpHas = 32;
    Mass me[kEach];   // 0: none, or not in question any more
    Parts w[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const uint32_t at = i * kThreads + tid;
        me[i] = at < n ? sm.list[at] : 0;
        const float x = logit_of((uint32_t)(me[i] >> 32));
        w[i] = by_mass && me[i] ? parts_of<kNucleus>(svk::fast_exp2(-bits_below(peak, x, rate))) : Parts{0u, me[i] ? 1 : 0};
    }
    uint32_t left = n;
#pragma unroll 1
    while (left > kWarpHas) {   // (the entries are different numbers: a part of two or more has a smaller range)
        Mass most = 0, least = ~0ull;
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (me[i]) most = max(most, me[i]), least = min(least, me[i]);
        most = over_warp(most, [](Mass a, Mass b) { return max(a, b); }), least = over_warp(least, [](Mass a, Mass b) { return min(a, b); });
        __syncthreads();   // (what the round before has found is read)
        if (lane == 0) sm.sums[warp] = most, sm.scan[warp] = least;
        if (tid < kParts) sm.high[tid] = 0, sm.low[tid] = 0;
        __syncthreads();
        most = over_warp(sm.sums[lane & (kWarps - 1)], [](Mass a, Mass b) { return max(a, b); });
        least = over_warp(sm.scan[lane & (kWarps - 1)], [](Mass a, Mass b) { return min(a, b); });
        const int shift = max(0, 64 - 8 - __clzll((long long)(most - least)));   // (most - least) >> shift < kParts
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const uint32_t part = me[i] ? (uint32_t)((most - me[i]) >> shift) : 0u;
            if (me[i]) add_shared(svk::smem_u32(&sm.high[part]), (int)w[i].high), add_shared(svk::smem_u32(&sm.low[part]), w[i].low);
        }
        __syncthreads();
        if (warp == 0) {
            Mass v[kParts / 32], mine = 0;
#pragma unroll
            for (int i = 0; i < kParts / 32; ++i) mine += v[i] = whole<kNucleus>(sm.high[lane * (kParts / 32) + i], sm.low[lane * (kParts / 32) + i]);
            const Mass upto = scan_warp(mine);
            Mass before = upto - mine;
            if (before < goal && upto >= goal) {
                int part = lane * (kParts / 32);
#pragma unroll
                for (int i = 0; i < kParts / 32 - 1; ++i)
                    if (before + v[i] < goal && part == lane * (kParts / 32) + i) before += v[i], ++part;
                sm.found_bin = part, sm.found_ahead = before;
            }
        }
        __syncthreads();
        const uint32_t found = (uint32_t)sm.found_bin;
        goal -= sm.found_ahead;
        left = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            if (me[i] && (uint32_t)((most - me[i]) >> shift) != found) me[i] = 0;
            left += __syncthreads_count(me[i] != 0);
        }
    }
    __syncthreads();
    if (tid == 0) sm.n_list = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        if (!me[i]) continue;
        const uint32_t at = atomicAdd(&sm.n_list, 1u);
        sm.sorted[at] = me[i], sm.masses()[at] = whole<kNucleus>(w[i].high, w[i].low);
    }
    __syncthreads();
    if (warp == 0) {
        const Mass mine = lane < left ? sm.sorted[lane] : 0, weight = lane < left ? sm.masses()[lane] : 0;
        Mass before = 0;
#pragma unroll 1
        for (uint32_t o = 0; o < left; ++o) before += sm.sorted[o] > mine ? sm.masses()[o] : 0;
        if (lane < left && before < goal && before + weight >= goal) sm.boundary = Boundary{logit_of((uint32_t)(mine >> 32)), ~(uint32_t)mine};
    }
    __syncthreads();
    return sm.boundary;
}

template <bool kHalf>
__global__ void __launch_bounds__(kThreads, 2) sample_kernel(const __grid_constant__ Params p)
{
    extern __shared__ __align__(16) uint8_t raw[];
    Smem &sm = *reinterpret_cast<Smem *>(raw);
    // the CTA's part of the row as it is read, but for NaNs
    using Held = std::conditional_t<kHalf, __nv_bfloat16, float>;
    Held *const held = reinterpret_cast<Held *>(raw + sizeof(Smem));
    const auto held1 = [&](int at) { return kHalf ? fminf((float)held[at], FLT_MAX) : (float)held[at]; };
    const auto held4 = [&](int at) {
        if constexpr (kHalf) {
            const uint2 w = *reinterpret_cast<const uint2 *>(held + at);
            return make_float4(fminf(__uint_as_float(w.x << 16), FLT_MAX), fminf(__uint_as_float(w.x & 0xffff0000u), FLT_MAX),
                               fminf(__uint_as_float(w.y << 16), FLT_MAX), fminf(__uint_as_float(w.y & 0xffff0000u), FLT_MAX));
        } else {
            return *reinterpret_cast<const float4 *>(held + at);
        }
    };
    const cg::cluster_group cluster = cg::this_cluster();
    const int CL = (int)cluster.num_blocks(), rank = (int)cluster.block_rank(), r = blockIdx.x / CL, g = r / p.rows_per_param;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int first = rank * p.part, n_here = min(p.part, p.V - first);   // entries of this CTA (possibly none), from `first` on
    const int words = p.part / kGrain, w0 = warp * (p.part / kWarps) + lane * 4;   // a lane's words of four entries: w0, w0 + 128, ...
    svk::cluster_arrive();   // (waited for behind the load, which hides it)
    svk::grid_dependency_wait();
    svk::grid_launch_dependents();

    const float T = p.temperature ? p.temperature[g] : 1.f;
    // (no entry reaches more than the largest one's mass: the first one is left, as in a greedy draw)
    const bool greedy = !(T > 0.f) || (p.min_p && p.min_p[g] > 1.f);
    const int k = greedy ? 1 : p.top_k ? p.top_k[g] : 0;
    const float top_p = p.top_p && !greedy ? p.top_p[g] : 1.f;
    float min_e = p.min_p && !greedy ? p.min_p[g] : 0.f;
    if (!(min_e > 0.f)) min_e = 0.f;
    const float u = p.tokens ? fminf(fmaxf(p.u[r], 0.f), 1.f) : 0.f;

    // the row, its maximum, and the maximum of the entries that this thread has read
    float most = -INFINITY;
    {
        const Held *const row = static_cast<const Held *>(p.logits) + r * p.stride + first;
        constexpr int kWide = 16 / sizeof(Held), kAhead = 4;
        const int n_wide = (reinterpret_cast<uintptr_t>(row) & 15) == 0 ? max(0, n_here) / kWide * kWide : 0;   // read 16 bytes at a time
#pragma unroll 1
        for (int base = 0; base < n_wide; base += kAhead * kThreads * kWide) {
            uint4 v[kAhead];
#pragma unroll
            for (int a = 0; a < kAhead; ++a) {
                const int at = base + (a * kThreads + tid) * kWide;
                if (at < n_wide) v[a] = __ldg(reinterpret_cast<const uint4 *>(row + at));
            }
#pragma unroll
            for (int a = 0; a < kAhead; ++a) {
                const int at = base + (a * kThreads + tid) * kWide;
                if (at >= n_wide) continue;
                uint32_t w[4] = {v[a].x, v[a].y, v[a].z, v[a].w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (kHalf) {
                        const __nv_bfloat162 least = __float2bfloat162_rn(-INFINITY);
                        const __nv_bfloat162 kept = __hmax2(*reinterpret_cast<const __nv_bfloat162 *>(&w[i]), least);   // (a NaN: the other)
                        w[i] = *reinterpret_cast<const uint32_t *>(&kept);
                        most = fmaxf(most, fmaxf(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u)));
                    } else {
                        const float x = taken(__uint_as_float(w[i]));
                        w[i] = __float_as_uint(x);
                        most = fmaxf(most, x);
                    }
                }
                *reinterpret_cast<uint4 *>(held + at) = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
        // what is left, an entry at a time; entries behind the end are not there
        constexpr int kSingles = 8;
#pragma unroll 1
        for (int base = n_wide; base < p.part; base += kSingles * kThreads) {
            Held v[kSingles];
#pragma unroll
            for (int a = 0; a < kSingles; ++a) {
                const int at = base + a * kThreads + tid;
                v[a] = at < n_here ? row[at] : (Held)-INFINITY;
            }
#pragma unroll
            for (int a = 0; a < kSingles; ++a) {
                const int at = base + a * kThreads + tid;
                if (at >= p.part) continue;
                const float x = fmaxf((float)v[a], -INFINITY);
                held[at] = (Held)(kHalf ? x : taken(x));
                most = fmaxf(most, x);
            }
        }
        most = taken(most);
    }
    const float top_here = over_warp(most, [](float a, float b) { return fmaxf(a, b); });
    if (lane == 0) sm.of_warp[warp] = top_here;
#pragma unroll 1
    for (int i = tid; i < kBins; i += kThreads) sm.high[i] = 0, sm.low[i] = 0;
    if (tid == 0) sm.n_list = 0;
    __syncthreads();
    svk::cluster_wait();   // every CTA of the cluster is running: its shared memory may be written from here on
    if (warp == 0) {
        const float top = over_warp(sm.of_warp[lane & (kWarps - 1)], [](float a, float b) { return fmaxf(a, b); });
        everywhere(&sm.top_of_cta[rank], top);
    }
    cluster.sync();
    const float peak = over_warp(sm.top_of_cta[lane < CL ? lane : 0], [](float a, float b) { return fmaxf(a, b); });
    if (peak == -INFINITY) {   // no entry
        if (p.probs)
#pragma unroll 1
            for (int i = tid; i < n_here; i += kThreads) p.probs[(size_t)r * p.V + first + i] = 0.f;
        if (p.tokens && rank == 0 && tid == 0) p.tokens[r] = -1;
        return;
    }
    const Rate rate = rate_of(greedy ? 1.f : T);
    const auto bits_of = [&](float x) { return bits_below(peak, x, rate); };
    const auto e_of = [&](float x) { return svk::fast_exp2(-bits_of(x)); };
    constexpr float kPlace = 8388608.f;   // (the last place of a sum with it is 1)
    const auto place_of = [&](float bits) { return fminf(__fmaf_rn(bits, kBinsPerBit, kPlace), kPlace + (float)(kBins - 1)); };
    const auto bin_at = [](float place) { return __float_as_uint(place) & (kBins - 1); };
    const auto each = [&](auto f) {   // f(index, logit), all entries of this lane in ascending order
#pragma unroll 1
        for (int j = 0; j < words; ++j) {
            const int at = w0 + j * 128;
            const float4 v = held4(at);
            f(first + at, v.x), f(first + at + 1, v.y), f(first + at + 2, v.z), f(first + at + 3, v.w);
        }
    };

    int turn = 0;   // of of_cta
    Mass mine = 0;
    const auto sum_cluster = [&](Mass v) { return sum_over_cluster(sm, turn ^= 1, v); };
    const auto before_warp = [&] {   // ... of the CTAs and warps before this one
        Mass before = 0;
#pragma unroll 1
        for (int c = 0; c < rank; ++c) before += sm.of_cta[turn][c];
#pragma unroll 1
        for (int w = 0; w < warp; ++w) before += sm.sums[w];
        return before;
    };
    const auto find_bin = [&](Mass goal, float of_all) { return find_in_bins(sm, goal, of_all); };
    const auto clear = [&] {
        __syncthreads();
#pragma unroll 1
        for (int i = tid; i < kBins; i += kThreads) sm.high[i] = 0, sm.low[i] = 0;
        if (tid == 0) sm.n_list = 0;
        __syncthreads();
    };
    // Counts are kept in units that make them masses of the nucleus' kind.
    const uint32_t bins = svk::smem_u32(sm.high), lows = svk::smem_u32(sm.low);
    const auto add_one = [&](uint32_t bin, bool really) { add_shared(lows + 4 * bin, really); };
    const auto add_mass = [&](uint32_t bin, float bits, bool really) {
        const Parts q = parts_of<kNucleus>(really ? svk::fast_exp2(-bits) : 0.f);
        add_shared(bins + 4 * bin, (int)q.high), add_shared(lows + 4 * bin, q.low);
    };
    // Entries for which `in` holds, in every CTA, sorted where that is asked for; their number (over kList: there is no list).
    const auto gather = [&](bool sort, auto in) {
#pragma unroll 1
        for (int j = 0; j < words; ++j) {   // (four entries, a branch for all of them)
            const int at = w0 + j * 128;
            const float4 v = held4(at);
            uint32_t found = (uint32_t)in(v.x, first + at) | (uint32_t)in(v.y, first + at + 1) << 1 | (uint32_t)in(v.z, first + at + 2) << 2 |
                             (uint32_t)in(v.w, first + at + 3) << 3;
#pragma unroll 1
            for (; found; found &= found - 1) {
                const int e = __ffs(found) - 1;
                const uint32_t to = atomicAdd(&sm.n_list, 1u);
                if (to < kList) sm.list[to] = (Mass)key_of(held1(at + e)) << 32 | (uint32_t)~(first + at + e);
            }
        }
        return collect(sm, turn ^= 1, mine, sort);
    };

    Boundary last{-FLT_MAX, 0xffffffffu};   // all of them
    const bool by_count = k > 0 && k < p.V, by_mass = top_p < 1.f;
    bool listed = false;   // the sorted list begins with all entries that stay
    uint32_t n_listed = 0;
    bool drawn = false;    // of_cta[turn] is what stays of the CTAs but for the list, and the list up to `last` the rest, in masses of the nucleus
    for (int step = 0; step < 2 && !listed; ++step) {
        if (!(step ? by_mass : by_count)) continue;
        Found found;
        if (step == 0) {
            // the k-th largest of the threads' maxima
            add_one(bin_at(place_of(bits_of(most))), most > -INFINITY);
            found = find_bin((Mass)k, 0.f);
            if (found.bin >= 0) {
                const float place = kPlace + found.bin;
                const uint32_t n = gather(true, [&](float x, uint32_t) { return (x > -INFINITY) & (place_of(bits_of(x)) <= place); });
                if (n <= kList) {
                    listed = true, n_listed = n;
                    break;
                }
            }
        }
        const Boundary within = last;
        const auto weight = [&](float x) { return step ? mass_of<kNucleus>(e_of(x)) : 1ull; };
        const auto add = [&](uint32_t bin, float bits, bool really) {
            if (step == 0) add_one(bin, really);
            else add_mass(bin, bits, really);
        };
        // first histogram: by the distance from the maximum
        if (by_count) {   // (else it still is clear)
            if (step || found.bin < 0) cluster.sync();   // the list of the first step, and the sums of its groups, have been read
            clear();
        }
        if (step == 0) {
            each([&](int, float x) {
                add_one(bin_at(place_of(bits_of(x))), x > -INFINITY);
            });
        } else {
            each([&](int i, float x) {   // (an entry that is not there has no mass)
                const float bits = bits_of(x);
                add_mass(bin_at(place_of(bits)), bits, !by_count || within.keeps(x, i));
            });
        }
        found = find_bin(step ? 0 : (Mass)k, top_p);
        if (found.bin < 0) continue;   // (fewer entries than k)
        const Mass goal = found.goal;
        Mass ahead = found.ahead;
        const float place = kPlace + found.bin;
        drawn = !by_count && min_e == 0.f;
        if (drawn) {
#pragma unroll
            for (int i = 0; i < kBins / kThreads; ++i) {
                const int b = i * kThreads + tid;
                mine += b < found.bin ? whole<kNucleus>(sm.high[b], sm.low[b]) : 0;
            }
        }
        __syncthreads();
        if (tid == 0) sm.n_list = 0;
        __syncthreads();
        uint32_t n = step && by_count ? gather(false, [&](float x, uint32_t i) { return (place_of(bits_of(x)) == place) & within.keeps(x, i); })
                                      : gather(false, [&](float x, uint32_t) { return (place_of(bits_of(x)) == place) & (x > -INFINITY); });
        drawn = drawn && n <= kList;
        // too many: the keys of the bin, then of a part of them, divided evenly
        uint32_t lo = 0, hi = 0;
        if (n > kList) {
            lo = 0xffffffffu;
            each([&](int i, float x) {
                if (place_of(bits_of(x)) == place && within.keeps(x, i)) lo = min(lo, key_of(x)), hi = max(hi, key_of(x));
            });
            lo = __reduce_min_sync(0xffffffffu, lo), hi = __reduce_max_sync(0xffffffffu, hi);
            if (tid == 0) sm.range[rank][0] = 0xffffffffu, sm.range[rank][1] = 0;
            __syncthreads();
            if (lane == 0) atomicMin(&sm.range[rank][0], lo), atomicMax(&sm.range[rank][1], hi);
            __syncthreads();
            if (warp == 0) {
                const uint32_t a = sm.range[rank][0], b = sm.range[rank][1];
                everywhere(&sm.range[rank][0], a), everywhere(&sm.range[rank][1], b);
            }
            cluster.sync();
            lo = __reduce_min_sync(0xffffffffu, lane < CL ? sm.range[lane][0] : 0xffffffffu);
            hi = __reduce_max_sync(0xffffffffu, lane < CL ? sm.range[lane][1] : 0u);
        }
        while (n > kList && lo < hi) {
            const int shift = max(0, 32 - __clz(hi - lo) - 11);   // (hi - lo) >> shift < kBins
            const auto in = [&](float x, uint32_t i) { return (x > -INFINITY) & (key_of(x) >= lo) & (key_of(x) <= hi) & within.keeps(x, i); };
            clear();
            each([&](int i, float x) {
                const bool is = in(x, i);
                add(is ? (hi - key_of(x)) >> shift : 0u, bits_of(x), is);
            });
            found = find_bin(goal - ahead, 0.f);
            const int b = found.bin;
            ahead += found.ahead;
            const uint32_t below = (uint32_t)(((Mass)(b + 1) << shift) - 1);
            lo = hi - lo < below ? lo : hi - below, hi -= (uint32_t)b << shift;
            __syncthreads();
            if (tid == 0) sm.n_list = 0;
            __syncthreads();
            n = gather(false, in);
        }
        const auto is_last = [&](float x, uint32_t i) {
#pragma unroll 1
            for (int c = 0; c < CL; ++c) *cluster.map_shared_rank(&sm.boundary, c) = Boundary{x, i};
        };
        if (n <= kList) {   // by the list, which every CTA has
            last = pick(sm, n, goal - ahead, step != 0, peak, rate);
            n_listed = n;
        } else {   // all equal: counted off in the order of the vocabulary
            const float x_all = logit_of(hi);
            const Mass one = weight(x_all), nth = (goal - ahead + one - 1) / one;   // the nth of them (from 1) is the last
            uint32_t mine = 0;
            each([&](int i, float x) { mine += x == x_all && within.keeps(x, i); });
            (void)sum_cluster(mine);
            Mass before = before_warp();
#pragma unroll 1
            for (int j = 0; j < words && before < nth; ++j) {   // (uniform over a warp)
                const int at = w0 + j * 128;
                const float4 v = held4(at);
                const float x[4] = {v.x, v.y, v.z, v.w};
                uint32_t m = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) m += x[e] == x_all && within.keeps(x[e], first + at + e);
                const uint32_t upto = scan_warp(m);
                Mass place_in = before + upto - m;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (x[e] == x_all && within.keeps(x[e], first + at + e) && ++place_in == nth) is_last(x_all, first + at + e);
                before += __shfl_sync(0xffffffffu, upto, 31);
            }
            cluster.sync();
            last = sm.boundary;
        }
    }
    if (listed || drawn) svk::cluster_arrive();   // nobody leaves while another CTA reads its list

    const auto stays = [&](float x, uint32_t i) {   // e of an entry that stays, 0 of others
        const float e = e_of(x);
        return last.keeps(x, i) & (e >= min_e) ? e : 0.f;
    };
    Mass total;   // of the draw
    float scale = 1099511627776.f;   // ... and what the largest entry counts
    if (listed) {
        // of the sorted list: the first k, their nucleus, those that are likely enough; at most two entries a thread
        const uint32_t n_k = min(n_listed, (uint32_t)k);
        float e[kEach];
        Mass ahead[kEach], all = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const uint32_t at = i * kThreads + tid;
            e[i] = at < n_k ? e_of(logit_of((uint32_t)(sm.sorted[at] >> 32))) : 0.f;
            const Scan scan = scan_block(sm, mass_of<kNucleus>(e[i]));
            ahead[i] = all + scan.before;
            all += scan.total;
        }
        const Mass goal = by_mass ? max((Mass)1, (Mass)ceil((double)fmaxf(top_p, 0.f) * (double)all)) : all + 1;
        uint32_t n_keep = 0;
        Mass kept = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const uint32_t at = i * kThreads + tid;
            const bool keep = at < n_k && (at == 0 || (ahead[i] < goal && e[i] >= min_e));
            n_keep += __syncthreads_count(keep);
            kept += keep ? mass_of<kDraw>(e[i]) : 0;
        }
        total = scan_block(sm, kept).total;
        const uint64_t final_entry = sm.sorted[n_keep - 1];
        last = {logit_of((uint32_t)(final_entry >> 32)), ~(uint32_t)final_entry}, min_e = 0.f;
        if (p.tokens && rank == 0) {   // the first entry in the order of the vocabulary up to which the masses reach the target
            const Mass target = max((Mass)1, min(total, (Mass)ceil((double)u * (double)total)));
            Mass *const of = sm.masses();
            if (tid == 0) sm.token = 0x7fffffff;
#pragma unroll
            for (int i = 0; i < kEach; ++i)
                if (i * kThreads + tid < n_keep) of[i * kThreads + tid] = mass_of<kDraw>(e[i]);
            __syncthreads();
#pragma unroll 1
            for (uint32_t i = tid; i < n_keep; i += kThreads) {
                const uint32_t me = (uint32_t)sm.sorted[i];   // (complement of the index)
                Mass upto = 0;
#pragma unroll 2
                for (uint32_t o = 0; o < n_keep; ++o) upto += (uint32_t)sm.sorted[o] >= me ? of[o] : 0;
                if (of[i] && upto >= target) atomicMin(&sm.token, (int)~me);
            }
            __syncthreads();
            if (tid == 0) p.tokens[r] = sm.token;
        }
    } else {
        // the mass that stays, by CTA; of the CTA in which the target lies by warp, word and entry
        const auto mass = [&](float x, uint32_t i) -> Mass {
            const float e = stays(x, i);
            return drawn ? mass_of<kNucleus>(e) : mass_of<kDraw>(e);
        };
        if (!drawn) {
            uint32_t high = 0;   // (a lane has at most 96 entries)
            int low = 0;
            each([&](int i, float x) {
                const Parts q = parts_of<kDraw>(stays(x, i));
                high += q.high, low += q.low;
            });
            mine = whole<kDraw>(high, low);
        }
        scale = drawn ? 4294967296.f : 1099511627776.f;
        Mass before = 0, here;
        if (drawn) {   // a warp for each CTA adds up what the list has of it
            if (warp < CL) {
                Mass m = 0;
#pragma unroll 1
                for (uint32_t i = lane; i < n_listed; i += 32) {
                    const uint64_t entry = sm.list[i];
                    const uint32_t index = ~(uint32_t)entry;
                    if (index - (uint32_t)(warp * p.part) < (uint32_t)p.part) m += mass(logit_of((uint32_t)(entry >> 32)), index);
                }
                m = sum_over_warp(m);
                if (lane == 0) sm.sums[warp] = sm.of_cta[turn][warp] + m;
            }
            __syncthreads();
            total = 0;
#pragma unroll 1
            for (int c = 0; c < CL; ++c) {
                if (c < rank) before += sm.sums[c];
                total += sm.sums[c];
            }
            here = sm.sums[rank];
            __syncthreads();
        } else {
            total = sum_cluster(mine);
#pragma unroll 1
            for (int c = 0; c < rank; ++c) before += sm.of_cta[turn][c];
            here = sm.of_cta[turn][rank];
        }
        if (p.tokens) {
            const Mass target = max((Mass)1, min(total, (Mass)ceil((double)u * (double)total)));
            if (before < target && before + here >= target) {
                if (drawn) {
                    uint32_t high = 0;
                    int low = 0;
                    each([&](int i, float x) {
                        const Parts q = parts_of<kNucleus>(stays(x, i));
                        high += q.high, low += q.low;
                    });
                    mine = sum_over_warp(whole<kNucleus>(high, low));
                    if (lane == 0) sm.sums[warp] = mine;
                    __syncthreads();
                }
#pragma unroll 1
                for (int w = 0; w < warp; ++w) before += sm.sums[w];
                if (before < target && before + sm.sums[warp] >= target) {   // this warp has it
#pragma unroll 1
                    for (int j = 0; j < words && before < target; ++j) {
                        const int at = w0 + j * 128;
                        const float4 v = held4(at);
                        const float x[4] = {v.x, v.y, v.z, v.w};
                        Mass w[4], m = 0;
#pragma unroll
                        for (int e = 0; e < 4; ++e) w[e] = mass(x[e], first + at + e), m += w[e];
                        const Mass upto = scan_warp(m);
                        Mass sum = before + upto - m;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            if (sum < target && sum + w[e] >= target) p.tokens[r] = first + at + e;
                            sum += w[e];
                        }
                        before += __shfl_sync(0xffffffffu, upto, 31);
                    }
                }
            }
        }
    }

    if (!p.probs) {
        if (listed || drawn) svk::cluster_wait();
        return;
    }
    const float inv = scale / (float)total;
    const auto prob = [&](float x, uint32_t i) { return stays(x, i) * inv; };
    float *const to = p.probs + (size_t)r * p.V + first;
    const int n_wide = (reinterpret_cast<uintptr_t>(to) & 15) == 0 ? max(0, n_here) / 4 * 4 : 0;
#pragma unroll 2
    for (int at = tid * 4; at < n_wide; at += kThreads * 4) {
        const float4 v = held4(at);
        float4 out = make_float4(0.f, 0.f, 0.f, 0.f);
        if (fmaxf(fmaxf(v.x, v.y), fmaxf(v.z, v.w)) >= last.x)   // (of a short top-k hardly any)
            out = make_float4(prob(v.x, first + at), prob(v.y, first + at + 1), prob(v.z, first + at + 2), prob(v.w, first + at + 3));
        *reinterpret_cast<float4 *>(to + at) = out;
    }
#pragma unroll 4
    for (int at = n_wide + tid; at < n_here; at += kThreads) {
        const float x = held1(at);
        to[at] = x >= last.x ? prob(x, first + at) : 0.f;
    }
    if (listed || drawn) svk::cluster_wait();
}

int part_for(int vocab, int cluster) { return ((vocab + cluster - 1) / cluster + kGrain - 1) / kGrain * kGrain; }

}  // namespace

extern "C" sv_status sv_sample(int32_t n_rows, int32_t vocab, const void *logits, int32_t logits_bf16, int64_t row_stride,
                               int32_t rows_per_param, const float *temperature, const int32_t *top_k, const float *top_p,
                               const float *min_p, const float *u, int32_t *tokens, float *probs, void *stream)
{
    if (n_rows < 0 || vocab < 1 || rows_per_param < 1 || n_rows % rows_per_param || row_stride < vocab) return SV_ERR_SHAPE;
    if (vocab > kMaxVocab) return SV_ERR_UNSUPPORTED;
    if ((!tokens && !probs) || (n_rows > 0 && (!logits || (tokens && !u)))) return SV_ERR_NULL;
    if (!svh::aligned(logits, logits_bf16 ? 2 : 4) || !svh::aligned(probs, 4)) return SV_ERR_ALIGN;
    if (n_rows == 0) return SV_OK;
    if ((int64_t)n_rows * kMaxCluster > INT32_MAX) return SV_ERR_SHAPE;
    // the smallest cluster whose CTAs share an SM by two, and larger ones while they find SMs
    const int bytes = logits_bf16 ? 2 : 4;
    int cluster = 1;
    while (cluster < kMaxCluster && part_for(vocab, cluster) > kGrain &&
           (part_for(vocab, cluster) * bytes > kTwo || 2ll * cluster * n_rows <= svh::sm_count()))
        cluster *= 2;
    const int part = part_for(vocab, cluster);
    const Params p = {logits, row_stride, temperature, top_p, min_p, u, top_k, tokens, probs, vocab, rows_per_param, part};
    const auto kernel = logits_bf16 ? sample_kernel<true> : sample_kernel<false>;
    static svh::OncePerDevice once[2];
    if (once[logits_bf16 != 0].run([&] {
            return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(sizeof(Smem) + kMostPart * bytes));
        }) != cudaSuccess) {
        (void)cudaGetLastError();
        return SV_ERR_CUDA;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(n_rows * cluster));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = sizeof(Smem) + part * bytes;
    cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[2];
    svh::pdl_attribute(attr);
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster, attr[1].val.clusterDim.y = 1, attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, p) == cudaSuccess ? svh::launch_status() : SV_ERR_CUDA;
}
