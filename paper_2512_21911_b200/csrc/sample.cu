// sv_sample: temperature, top-k, top-p and min-p on rows of logits, the kept entries' distribution and a token drawn from it.
//
// Mathematics: e(x) = 2^((x - max) log2 e / temperature).  Masses are whole multiples of 2^-40 (e <= 1, at most 2^20 entries: 60 bits), so
// every sum is exact and no order of adding changes a result.  The entries are never sorted: what stays is everything up to one entry, the
// boundary (key, index), in the order "larger logit first, then smaller index".  Search for the boundary by count (top-k) or mass (top-p):
// a histogram of the entries by their distance from the maximum, the bin in which the goal is reached, and the few entries of that bin,
// ranked exactly.  A bin with too many of them is divided again by the bits of its keys; entries that are all equal are
// counted off by index.  With a short top-k all entries up to the bin are ranked at once and top-p, min-p and the token follow from the list.
//
// A cluster of 1 to 8 CTAs per row; a CTA keeps its part of the row in shared memory, so the logits are read once from HBM.  Warps
// own contiguous parts: a token is found by sums per CTA, warp and lane.
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include <algorithm>

#include "sv_host.h"
#include "sv_ptx.cuh"

namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxVocab = 1 << 20;
constexpr int kMaxCluster = 8;
constexpr int kBins = 2048;
constexpr float kBinsPerBit = 2048.f / 44.f;   // bins of the first histogram: 44 powers of two below the maximum, beyond what has a mass
constexpr int kList = 1024;                    // entries that are ranked one against another
constexpr int kGrain = kWarps * 128;           // a CTA's part of a row is a multiple of this: 32 lanes x 4 entries for each warp

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

// Ascending in the logit; -0 equals +0.  0: an entry that is not there (-infinity; a NaN is taken as one when it is read).
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t b = __float_as_uint(x) == 0x80000000u ? 0u : __float_as_uint(x);
    return x == -INFINITY ? 0u : b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }

// e * 2^40 to the nearest integer as high * 2^20 + low, by adding numbers whose last place is 1 (0 <= e <= 1).
struct Parts {
    uint32_t high;   // <= 2^20
    int low;         // at most 2^19 either way
};
__device__ __forceinline__ Parts parts_of(float e)
{
    const float f = __fmul_rn(e, 1048576.f), t = __fadd_rn(f, 8388608.f);
    const float rest = __fsub_rn(f, __fsub_rn(t, 8388608.f));
    return {__float_as_uint(t) - 0x4b000000u, (int)(__float_as_uint(__fmaf_rn(rest, 1048576.f, 12582912.f)) - 0x4b400000u)};
}
__device__ __forceinline__ Mass mass_of(Parts p) { return ((Mass)p.high << 20) + (long long)p.low; }

struct Boundary {
    uint32_t key, index;   // the last entry that stays; (1, any): all of them
    __device__ bool keeps(uint32_t k, uint32_t i) const { return k > key || (k == key && i <= index); }
};

struct Smem {
    Mass bins[kBins];
    uint64_t list[kList];     // key << 32 | ~index: descending is the order of the rule
    uint64_t sorted[kList];
    Mass sums[kWarps], scan[kWarps];
    Mass of_cta[2][kMaxCluster];   // written by all CTAs of the cluster; two in turn, so that no CTA writes what another still reads
    uint32_t top_of_cta[kMaxCluster], count_of_cta[kMaxCluster];
    uint32_t range[kMaxCluster][2];
    Mass found_ahead;           // written by the CTA that finds it
    int found_bin, token;
    Boundary boundary;
    uint32_t n_list;
    uint32_t words[kWarps];
};

template <class T, class Op>
__device__ __forceinline__ T over_warp(T v, Op op)
{
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, d));
    return v;
}
__device__ __forceinline__ Mass sum_over_warp(Mass v) { return over_warp(v, [](Mass a, Mass b) { return a + b; }); }

// kHeld: the CTA's part of the row is in shared memory; else (parts that do not fit) every pass reads it again.
template <bool kHalf, bool kHeld>
struct Row {
    const void *row;
    float *held;
    int V, part, rank, warp, lane;
    bool wide;   // rows start on 16 bytes

    __device__ float at(int i) const
    {
        const float x = kHalf ? __bfloat162float(static_cast<const __nv_bfloat16 *>(row)[i]) : __ldg(static_cast<const float *>(row) + i);
        return x == x ? x : -INFINITY;
    }
    __device__ float4 read(int i) const
    {
        float4 v;
        if (wide && i + 4 <= V) {
            if constexpr (kHalf) {
                const uint2 w = __ldg(reinterpret_cast<const uint2 *>(static_cast<const __nv_bfloat16 *>(row) + i));
                v = make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xffff0000u));
            } else {
                v = __ldg(reinterpret_cast<const float4 *>(static_cast<const float *>(row) + i));
            }
            v.x = v.x == v.x ? v.x : -INFINITY, v.y = v.y == v.y ? v.y : -INFINITY;
            v.z = v.z == v.z ? v.z : -INFINITY, v.w = v.w == v.w ? v.w : -INFINITY;
        } else {
            v.x = i < V ? at(i) : -INFINITY, v.y = i + 1 < V ? at(i + 1) : -INFINITY;
            v.z = i + 2 < V ? at(i + 2) : -INFINITY, v.w = i + 3 < V ? at(i + 3) : -INFINITY;
        }
        return v;
    }
    __device__ int words() const { return part / kGrain; }   // of a lane
    __device__ int first(int j) const { return warp * (part / kWarps) + (j * 32 + lane) * 4; }   // entry of a lane's word, in the CTA's part
    __device__ float4 word(int j) const
    {
        const int i = first(j);
        if constexpr (kHeld) return *reinterpret_cast<const float4 *>(held + i);
        else return read(rank * part + i);
    }
    template <class F>
    __device__ void each(F f) const   // f(index, logit), all entries of this thread in ascending order
    {
        for (int j = 0; j < words(); ++j) {
            const float4 v = word(j);
            const int i = rank * part + first(j);
            f(i, v.x), f(i + 1, v.y), f(i + 2, v.z), f(i + 3, v.w);
        }
    }
};

template <bool kHalf, bool kHeld>
__global__ void __launch_bounds__(kThreads) sample_kernel(const Params p)
{
    extern __shared__ __align__(16) uint8_t raw[];
    Smem &sm = *reinterpret_cast<Smem *>(raw);
    static_assert(sizeof(Smem) % 16 == 0, "");
    const cg::cluster_group cluster = cg::this_cluster();
    const int CL = (int)cluster.num_blocks(), rank = (int)cluster.block_rank(), r = blockIdx.x / CL, g = r / p.rows_per_param;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const auto everywhere = [&](auto *at, auto v) {   // (one warp) the same word of every CTA's shared memory
        if (lane < CL) *cluster.map_shared_rank(at, lane) = v;
    };
    svk::grid_dependency_wait();
    svk::grid_launch_dependents();
    Row<kHalf, kHeld> row;
    row.row = static_cast<const char *>(p.logits) + r * p.stride * (kHalf ? 2 : 4);
    row.held = reinterpret_cast<float *>(raw + sizeof(Smem));
    row.V = p.V, row.part = p.part, row.rank = rank, row.warp = warp, row.lane = lane;
    row.wide = (reinterpret_cast<uintptr_t>(row.row) & 15) == 0;

    // the row, and its maximum
    const float T = p.temperature ? p.temperature[g] : 1.f;
    const bool greedy = !(T > 0.f);
    const int k = greedy ? 1 : p.top_k ? p.top_k[g] : 0;
    const float top_p = p.top_p && !greedy ? p.top_p[g] : 1.f;
    float min_e = p.min_p && !greedy ? p.min_p[g] : 0.f;
    if (!(min_e > 0.f)) min_e = 0.f;
    const float u = p.tokens ? fminf(fmaxf(p.u[r], 0.f), 1.f) : 0.f;
    float most = -INFINITY;
    for (int j = 0; j < row.words(); ++j) {
        const float4 v = row.read(rank * p.part + row.first(j));
        if constexpr (kHeld) *reinterpret_cast<float4 *>(row.held + row.first(j)) = v;
        most = fmaxf(most, fmaxf(fmaxf(v.x, v.y), fmaxf(v.z, v.w)));
    }
    most = over_warp(most, [](float a, float b) { return fmaxf(a, b); });
    if (lane == 0) sm.words[warp] = key_of(most);
    for (int i = tid; i < kBins; i += kThreads) sm.bins[i] = 0;
    if (tid == 0) sm.n_list = 0;
    __syncthreads();
    if (warp == 0) {
        const uint32_t top = __reduce_max_sync(0xffffffffu, lane < kWarps ? sm.words[lane] : 0u);
        everywhere(&sm.top_of_cta[rank], top);
    }
    cluster.sync();
    const uint32_t top = __reduce_max_sync(0xffffffffu, lane < CL ? sm.top_of_cta[lane] : 0u);
    const float peak = logit_of(top), rate = fmaxf(1.4426950408889634f / (greedy ? 1.f : T), 1.2e-38f);   // (an infinite T: all alike)
    const auto bits_of = [&](float x) { return x == peak ? 0.f : (x - peak) * rate; };   // log2 e
    const auto e_of = [&](float x) { return x == peak ? 1.f : svk::fast_exp2((x - peak) * rate); };
    if (top == 0) {   // no entry
        if (p.probs)
            for (int i = rank * p.part + tid; i < min(p.V, (rank + 1) * p.part); i += kThreads) p.probs[(size_t)r * p.V + i] = 0.f;
        if (p.tokens && rank == 0 && tid == 0) p.tokens[r] = -1;
        return;
    }

    // exclusive prefix and total over the CTA, in thread order
    const auto scan_block = [&](Mass v, Mass &total) {
        Mass upto = v;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const Mass o = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += o;
        }
        __syncthreads();
        if (lane == 31) sm.scan[warp] = upto;
        __syncthreads();
        Mass before = upto - v;
        total = 0;
        for (int w = 0; w < kWarps; ++w) {
            if (w < warp) before += sm.scan[w];
            total += sm.scan[w];
        }
        return before;
    };
    int turn = 0;
    // total over the cluster of a value of each thread; of_cta[turn] keeps the CTAs' totals
    const auto sum_cluster = [&](Mass v) {
        turn ^= 1;
        v = sum_over_warp(v);
        __syncthreads();
        if (lane == 0) sm.sums[warp] = v;
        __syncthreads();
        if (warp == 0) everywhere(&sm.of_cta[turn][rank], sum_over_warp(lane < kWarps ? sm.sums[lane] : 0));
        cluster.sync();
        return sum_over_warp(lane < CL ? sm.of_cta[turn][lane] : 0);
    };
    // The bin in which the sums over the cluster's histograms reach the goal, and what is in the bins ahead of it.  A CTA adds up its share of the
    // bins of all CTAs; the CTA in whose share the goal lies finds the bin.  goal <= the sum of all.
    const auto find_bin = [&](Mass goal, Mass &ahead) {
        const int share = kBins / CL, per = (share + kThreads - 1) / kThreads;
        cluster.sync();
        Mass v[kBins / kThreads], mine = 0;
#pragma unroll
        for (int i = 0; i < kBins / kThreads; ++i) {
            v[i] = 0;
            const int b = tid * per + i;
            if (i < per && b < share)
                for (int c = 0; c < CL; ++c) v[i] += *cluster.map_shared_rank(&sm.bins[rank * share + b], c);
            mine += v[i];
        }
        Mass total;
        Mass before = scan_block(mine, total);
        turn ^= 1;
        if (warp == 0) everywhere(&sm.of_cta[turn][rank], total);
        cluster.sync();
        for (int c = 0; c < rank; ++c) before += sm.of_cta[turn][c];
        if (before < goal && before + mine >= goal) {
            int b = 0;
#pragma unroll
            for (int i = 0; i < kBins / kThreads; ++i) {
                if (before + v[i] >= goal) break;
                before += v[i], ++b;
            }
            for (int c = 0; c < CL; ++c) {
                *cluster.map_shared_rank(&sm.found_bin, c) = rank * share + tid * per + b;
                *cluster.map_shared_rank(&sm.found_ahead, c) = before;
            }
        }
        cluster.sync();
        ahead = sm.found_ahead;
        return sm.found_bin;
    };
    const auto clear = [&] {
        __syncthreads();
        for (int i = tid; i < kBins; i += kThreads) sm.bins[i] = 0;
        if (tid == 0) sm.n_list = 0;
        __syncthreads();
    };
    // Entries for which `in` holds, into the first CTA's list; their number (over kList: the list is not complete).
    const auto gather = [&](auto in) {
        row.each([&](int i, float x) {
            const uint32_t key = key_of(x);
            if (key && in(key, x, (uint32_t)i)) {
                const uint32_t at = atomicAdd(&sm.n_list, 1u);
                if (at < kList) sm.list[at] = (uint64_t)key << 32 | (uint32_t)~i;
            }
        });
        __syncthreads();
        if (warp == 0) everywhere(&sm.count_of_cta[rank], sm.n_list);
        cluster.sync();
        uint32_t n = 0;
        for (int c = 0; c < CL; ++c) n += sm.count_of_cta[c];
        if (rank == 0 && n <= kList) {
            uint32_t at = sm.count_of_cta[0];
            for (int c = 1; c < CL; ++c) {
                for (uint32_t i = tid; i < sm.count_of_cta[c]; i += kThreads) sm.list[at + i] = *cluster.map_shared_rank(&sm.list[i], c);
                at += sm.count_of_cta[c];
            }
            __syncthreads();
            for (uint32_t i = tid; i < n; i += kThreads) {
                const uint64_t me = sm.list[i];
                int place = 0;
                for (uint32_t o = 0; o < n; ++o) place += sm.list[o] > me;
                sm.sorted[place] = me;
            }
            __syncthreads();
        }
        if (n > kList) cluster.sync();   // (the counts may be written again)
        return n;
    };
    const auto bin_of = [&](float x) { return max(0, min(kBins - 1, (int)(-bits_of(x) * kBinsPerBit))); };

    Boundary last{1u, 0xffffffffu};
    const bool by_count = k > 0 && k < p.V, by_mass = top_p < 1.f;
    bool listed = false;   // the first CTA's sorted list begins with all entries that stay
    uint32_t n_listed = 0;
    for (int step = 0; step < 2 && !listed; ++step) {
        if (!(step ? by_mass : by_count)) continue;
        const Boundary within = last;
        const auto weight = [&](uint32_t key, float x) { return step ? mass_of(parts_of(e_of(x))) : 1ull; };
        // first histogram: by the distance from the maximum
        Mass all = 0;
        clear();
        row.each([&](int i, float x) {
            const uint32_t key = key_of(x);
            if (!key || !within.keeps(key, i)) return;
            const Mass w = weight(key, x);
            all += w;
            if (w) atomicAdd(&sm.bins[bin_of(x)], w);
        });
        all = sum_cluster(all);
        const Mass goal = step ? max((Mass)1, (Mass)ceil((double)fmaxf(top_p, 0.f) * (double)all)) : (Mass)k;
        if (goal > all) continue;   // (fewer entries than k)
        Mass ahead;
        const int bin = find_bin(goal, ahead);
        if (step == 0) {
            const uint32_t n = gather([&](uint32_t, float x, uint32_t) { return bin_of(x) <= bin; });
            if (n <= kList) {
                listed = true, n_listed = n;
                break;
            }
            clear();
        }
        uint32_t n = gather([&](uint32_t key, float x, uint32_t i) { return bin_of(x) == bin && within.keeps(key, i); });
        // too many: the keys of the bin, then of a part of them, divided evenly
        uint32_t lo = 1, hi = 0xffffffffu;
        if (n > kList) {
            uint32_t least = 0xffffffffu, greatest = 0;
            row.each([&](int i, float x) {
                const uint32_t key = key_of(x);
                if (key && bin_of(x) == bin && within.keeps(key, i)) least = min(least, key), greatest = max(greatest, key);
            });
            least = __reduce_min_sync(0xffffffffu, least), greatest = __reduce_max_sync(0xffffffffu, greatest);
            if (tid == 0) sm.range[rank][0] = 0xffffffffu, sm.range[rank][1] = 0;
            __syncthreads();
            if (lane == 0) atomicMin(&sm.range[rank][0], least), atomicMax(&sm.range[rank][1], greatest);
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
            clear();
            row.each([&](int i, float x) {
                const uint32_t key = key_of(x);
                if (key < lo || key > hi || !within.keeps(key, i)) return;
                const Mass w = weight(key, x);
                if (w) atomicAdd(&sm.bins[(hi - key) >> shift], w);
            });
            const int b = find_bin(goal - ahead, all);
            ahead += all;
            const uint32_t below = (uint32_t)(((Mass)(b + 1) << shift) - 1);
            lo = hi - lo < below ? lo : hi - below, hi -= (uint32_t)b << shift;
            clear();
            n = gather([&](uint32_t key, float, uint32_t i) { return key >= lo && key <= hi && within.keeps(key, i); });
        }
        if (n <= kList) {   // ranked by the first CTA
            if (rank == 0) {
                Mass sum = ahead;
                for (uint32_t base = 0; base < n; base += kThreads) {
                    const bool in = base + tid < n;
                    const uint64_t me = in ? sm.sorted[base + tid] : 0;
                    const Mass w = in ? weight((uint32_t)(me >> 32), logit_of((uint32_t)(me >> 32))) : 0;
                    Mass total;
                    const Mass before = sum + scan_block(w, total);
                    if (in && before < goal && before + w >= goal) {
                        for (int c = 0; c < CL; ++c) *cluster.map_shared_rank(&sm.boundary, c) = Boundary{(uint32_t)(me >> 32), ~(uint32_t)me};
                    }
                    sum += total;
                }
            }
        } else {   // all equal: counted off in the order of the vocabulary
            const Mass each = weight(hi, logit_of(hi)), nth = (goal - ahead + each - 1) / each;   // >= 1; the nth of them is the last
            uint32_t mine = 0;
            row.each([&](int i, float x) { mine += key_of(x) == hi && within.keeps(hi, i); });
            mine = __reduce_add_sync(0xffffffffu, mine);
            (void)sum_cluster(lane == 0 ? mine : 0);
            Mass before = 0;
            for (int c = 0; c < rank; ++c) before += sm.of_cta[turn][c];
            for (int w = 0; w < warp; ++w) before += sm.sums[w];
            for (int j = 0; j < row.words() && before < nth; ++j) {   // (uniform over a warp)
                const float4 v = row.word(j);
                const float x[4] = {v.x, v.y, v.z, v.w};
                const int i = rank * p.part + row.first(j);
                uint32_t m = 0;
                for (int e = 0; e < 4; ++e) m += key_of(x[e]) == hi && within.keeps(hi, i + e);
                uint32_t upto = m;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const uint32_t o = __shfl_up_sync(0xffffffffu, upto, d);
                    if (lane >= d) upto += o;
                }
                Mass at = before + upto - m;
                for (int e = 0; e < 4; ++e)
                    if (key_of(x[e]) == hi && within.keeps(hi, i + e) && ++at == nth)
                        for (int c = 0; c < CL; ++c) *cluster.map_shared_rank(&sm.boundary, c) = Boundary{hi, (uint32_t)(i + e)};
                before += __shfl_sync(0xffffffffu, upto, 31);
            }
        }
        cluster.sync();
        last = sm.boundary;
    }

    if (listed) {
        if (rank == 0) {
            // of the sorted list: the first k, their nucleus, those that are likely enough; at most two entries a thread
            const uint32_t n_k = min(n_listed, (uint32_t)k);
            Mass w[kList / kThreads], ahead[kList / kThreads], whole = 0;
#pragma unroll
            for (int i = 0; i < kList / kThreads; ++i) {
                const uint32_t at = i * kThreads + tid;
                w[i] = at < n_k ? mass_of(parts_of(e_of(logit_of((uint32_t)(sm.sorted[at] >> 32))))) : 0;
                Mass total;
                ahead[i] = whole + scan_block(w[i], total);
                whole += total;
            }
            const Mass goal = by_mass ? max((Mass)1, (Mass)ceil((double)fmaxf(top_p, 0.f) * (double)whole)) : whole + 1;
            uint32_t n_keep = 0;
#pragma unroll
            for (int i = 0; i < kList / kThreads; ++i) {
                const uint32_t at = i * kThreads + tid;
                const uint32_t key = at < n_k ? (uint32_t)(sm.sorted[at] >> 32) : 0;
                n_keep += __syncthreads_count(at < n_k && (at == 0 || (ahead[i] < goal && (key == top || e_of(logit_of(key)) >= min_e))));
            }
            Mass total = 0;
#pragma unroll
            for (int i = 0; i < kList / kThreads; ++i) total += i * kThreads + tid < n_keep ? w[i] : 0;
            Mass sum;
            (void)scan_block(total, sum);
            if (tid == 0) {
                const uint64_t at = sm.sorted[n_keep - 1];
                for (int c = 0; c < CL; ++c) {
                    *cluster.map_shared_rank(&sm.boundary, c) = Boundary{(uint32_t)(at >> 32), ~(uint32_t)at};
                    *cluster.map_shared_rank(&sm.found_ahead, c) = sum;
                }
                sm.token = 0x7fffffff;
            }
            __syncthreads();
            if (p.tokens) {   // the first entry in the order of the vocabulary up to which the masses reach the target
                const Mass target = max((Mass)1, min(sum, (Mass)ceil((double)u * (double)sum)));
                Mass *of = sm.bins;
                for (uint32_t i = tid; i < n_keep; i += kThreads) of[i] = mass_of(parts_of(e_of(logit_of((uint32_t)(sm.sorted[i] >> 32)))));
                __syncthreads();
                for (uint32_t i = tid; i < n_keep; i += kThreads) {
                    const uint32_t me = (uint32_t)sm.sorted[i];   // (complement of the index)
                    Mass upto = 0;
                    for (uint32_t o = 0; o < n_keep; ++o) upto += (uint32_t)sm.sorted[o] >= me ? of[o] : 0;
                    if (of[i] && upto >= target) atomicMin(&sm.token, (int)~me);
                }
                __syncthreads();
                if (tid == 0) p.tokens[r] = sm.token;
            }
        }
        cluster.sync();   // (nobody leaves while the first CTA reads its list)
        if (!p.probs) return;
        last = sm.boundary;
        const float inv = 1099511627776.f / (float)sm.found_ahead;
        for (int j = 0; j < row.words(); ++j) {
            const float4 v = row.word(j);
            const float x[4] = {v.x, v.y, v.z, v.w};
            const int i = rank * p.part + row.first(j);
            float *to = p.probs + (size_t)r * p.V + i;
            float o[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t key = key_of(x[e]);
                o[e] = key && last.keeps(key, i + e) ? e_of(x[e]) * inv : 0.f;
            }
            if (i + 4 <= p.V && (reinterpret_cast<uintptr_t>(to) & 15) == 0) *reinterpret_cast<float4 *>(to) = make_float4(o[0], o[1], o[2], o[3]);
            else
                for (int e = 0; e < 4; ++e)
                    if (i + e < p.V) to[e] = o[e];
        }
        return;
    }

    // the mass that stays, by CTA and warp
    const auto kept = [&](int i, float x, float &e) {
        const uint32_t key = key_of(x);
        e = e_of(x);
        return key && last.keeps(key, i) && (e >= min_e || key == top);
    };
    uint32_t high = 0;
    int low = 0;
    Mass mine = 0;
    int since = 0;
    row.each([&](int i, float x) {
        float e;
        if (kept(i, x, e)) {
            const Parts q = parts_of(e);
            high += q.high, low += q.low;
        }
        if (++since == 1024) mine += ((Mass)high << 20) + (long long)low, high = 0, low = 0, since = 0;   // (before 32 bits overflow)
    });
    mine += ((Mass)high << 20) + (long long)low;
    const Mass total = sum_cluster(mine);
    const Mass target = max((Mass)1, min(total, (Mass)ceil((double)u * (double)total)));
    const float inv = 1099511627776.f / (float)total;
    if (p.tokens) {
        Mass before = 0;
        for (int c = 0; c < rank; ++c) before += sm.of_cta[turn][c];
        for (int w = 0; w < warp; ++w) before += sm.sums[w];
        if (before < target && before + sm.sums[warp] >= target) {   // this warp has it
            for (int j = 0; j < row.words(); ++j) {
                const float4 v = row.word(j);
                const float x[4] = {v.x, v.y, v.z, v.w};
                const int i = rank * p.part + row.first(j);
                Mass w[4], m = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float ex;
                    w[e] = kept(i + e, x[e], ex) ? mass_of(parts_of(ex)) : 0;
                    m += w[e];
                }
                Mass upto = m;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const Mass o = __shfl_up_sync(0xffffffffu, upto, d);
                    if (lane >= d) upto += o;
                }
                Mass at = before + upto - m;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (at < target && at + w[e] >= target) p.tokens[r] = i + e;
                    at += w[e];
                }
                before += __shfl_sync(0xffffffffu, upto, 31);
                if (before >= target) break;
            }
        }
    }
    if (p.probs) {
        for (int j = 0; j < row.words(); ++j) {
            const float4 v = row.word(j);
            const float x[4] = {v.x, v.y, v.z, v.w};
            const int i = rank * p.part + row.first(j);
            float *to = p.probs + (size_t)r * p.V + i;
            float o[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float ex;
                o[e] = kept(i + e, x[e], ex) ? ex * inv : 0.f;
            }
            if (i + 4 <= p.V && (reinterpret_cast<uintptr_t>(to) & 15) == 0) *reinterpret_cast<float4 *>(to) = make_float4(o[0], o[1], o[2], o[3]);
            else
                for (int e = 0; e < 4; ++e)
                    if (i + e < p.V) to[e] = o[e];
        }
    }
}

constexpr int kMostSmem = 227 * 1024;

const void *kernel_for(bool half, bool held)
{
    return half ? held ? (const void *)sample_kernel<true, true> : (const void *)sample_kernel<true, false>
                : held ? (const void *)sample_kernel<false, true> : (const void *)sample_kernel<false, false>;
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
    // the smallest cluster that holds a row, and larger ones while they find SMs
    int cluster = 1;
    while (cluster < kMaxCluster && (part_for(vocab, cluster) * sizeof(float) + sizeof(Smem) > kMostSmem || 2 * cluster * n_rows <= svh::sm_count()) &&
           part_for(vocab, cluster) > kGrain)
        cluster *= 2;
    const int part = part_for(vocab, cluster);
    const bool held = part * sizeof(float) + sizeof(Smem) <= kMostSmem;
    const Params p = {logits, row_stride, temperature, top_p, min_p, u, top_k, tokens, probs, vocab, rows_per_param, part};
    const void *fn = kernel_for(logits_bf16, held);
    static svh::OncePerDevice once[2][2];
    if (once[logits_bf16 != 0][held].run([&] { return cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSmem); }) != cudaSuccess) {
        (void)cudaGetLastError();
        return SV_ERR_CUDA;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(n_rows * cluster));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = sizeof(Smem) + (held ? part * sizeof(float) : 0);
    cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[2];
    svh::pdl_attribute(attr);
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster, attr[1].val.clusterDim.y = 1, attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    void *args[] = {const_cast<Params *>(&p)};
    return cudaLaunchKernelExC(&cfg, fn, args) == cudaSuccess ? svh::launch_status() : SV_ERR_CUDA;
}
