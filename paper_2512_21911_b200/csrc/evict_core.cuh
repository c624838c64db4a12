// Which tokens of a KV head stay (sv_kv_evict): the n-th largest of their order keys, found by the CTAs of a cluster together, and the list
// of those that stay.  Every CTA has the keys of a slice in its shared memory.
#pragma once
#include <cooperative_groups.h>
#include <stdint.h>

#include "order_key.h"

namespace svev {

namespace cg = cooperative_groups;

constexpr int kThreads = 256, kRowGroups = kThreads / 16, kCluster = 8;
constexpr int kBins = 2048;
constexpr int kMostTokens = kCluster * 49152;   // that a cluster's shared memory holds the keys of

struct Shared {
    uint32_t hist[kBins];
    uint32_t sums[kThreads / 32];
    uint32_t digit, above;      // what a pass found
    uint32_t kept[2];           // of the slice: keys above the n-th largest, keys equal to it
    uint32_t first[kCluster + 1];   // where the slices' kept tokens begin
    int32_t source[128];        // of a round's block
    float part[kRowGroups][128];
};

// The sum over the threads below this one, and over all.
__device__ __forceinline__ uint32_t sum_below(uint32_t x, uint32_t *sums, uint32_t &all)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t upto = x;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const uint32_t o = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += o;
    }
    __syncthreads();
    if (lane == 31) sums[warp] = upto;
    __syncthreads();
    all = 0;
    for (int w = 0; w < kThreads / 32; ++w) {
        if (w < warp) upto += sums[w];
        all += sums[w];
    }
    return upto - x;
}

// Of tokens 0 .. L - 1 with these weights n stay: the first n_sink, the last n_recent, and the heaviest others.  keys: room for the CTA's
// slice, which becomes the list of its tokens that stay; token d of all of them is source_of(d).  All threads of the cluster; peers are
// reached behind its first barrier, and the last is up to the caller, who reaches them too.
__device__ __forceinline__ void keep_heaviest(const cg::cluster_group &cluster, const float *weights, int L, int n, int n_sink, int n_recent,
                                              uint32_t *keys, Shared &sh)
{
    const int rank = cluster.block_rank(), tid = threadIdx.x;
    // the keys of the slice
    const int per = ((L + kCluster - 1) / kCluster + 3) & ~3, t0 = min(rank * per, L), count = min(t0 + per, L) - t0;
    for (int i = tid; i < count; i += kThreads) {
        const int t = t0 + i;
        const uint32_t key = svsel::key_of_bits(__float_as_uint(weights[t]));
        keys[i] = t < n_sink || t >= L - n_recent ? svsel::kForcedKey : key;
    }
    // the n-th largest key, by digits from the top
    uint32_t prefix = 0, wanted = n;
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
        const int low = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11, bins = 1 << bits;
        for (int i = tid; i < kBins; i += kThreads) sh.hist[i] = 0;
        __syncthreads();
        for (int i = tid; i < count; i += kThreads) {
            const uint32_t key = keys[i];
            if (pass == 0 || key >> (low + bits) == prefix) atomicAdd(&sh.hist[key >> low & (bins - 1)], 1u);
        }
        cluster.sync();
        // bins of a thread, from the top; all CTAs find the same
        constexpr int kEach = kBins / kThreads;
        uint32_t mine[kEach], sum = 0;
#pragma unroll
        for (int j = 0; j < kEach; ++j) mine[j] = 0;
        const int each = bins / kThreads;
#pragma unroll 1
        for (int r = 0; r < kCluster; ++r) {
            const uint32_t *hist = cluster.map_shared_rank(sh.hist, r);
#pragma unroll
            for (int j = 0; j < kEach; ++j)
                if (j < each) mine[j] += hist[bins - 1 - (tid * each + j)];
        }
#pragma unroll
        for (int j = 0; j < kEach; ++j) sum += mine[j];
        uint32_t all, above = sum_below(sum, sh.sums, all);
        if (above < wanted && wanted <= above + sum) {
            int j = 0;
            while (above + mine[j] < wanted) above += mine[j++];
            sh.digit = bins - 1 - (tid * each + j), sh.above = above;
        }
        cluster.sync();   // (also: everybody has read this CTA's histogram)
        prefix = prefix << bits | sh.digit;
        wanted -= sh.above;
    }
    // prefix is the key; of those equal to it the first `wanted` of the sequence stay.  A warp has a run of the slice; lane u of it keeps the
    // ballots of the run's words u, 32 + u, ...
    constexpr int kWords = kMostTokens / kCluster / (kThreads / 32) / 32 / 32;
    const int lane = tid & 31, warp = tid >> 5;
    const int run = ((count + kThreads / 32 - 1) / (kThreads / 32) + 31) & ~31, i0 = min(warp * run, count), i1 = min(i0 + run, count);
    uint32_t more[kWords], equal[kWords], n_more = 0, n_equal = 0;
#pragma unroll
    for (int j = 0; j < kWords; ++j) {
        more[j] = equal[j] = 0;
        if (i0 + j * 1024 < i1) {
#pragma unroll 4
            for (int u = 0; u < 32; ++u) {
                const int i = i0 + (j * 32 + u) * 32 + lane;
                const uint32_t key = i < i1 ? keys[i] : 0u;
                const uint32_t m = __ballot_sync(0xffffffffu, i < i1 && key > prefix), e = __ballot_sync(0xffffffffu, i < i1 && key == prefix);
                if (u == lane) more[j] = m, equal[j] = e;
            }
        }
        n_more += __popc(more[j]), n_equal += __popc(equal[j]);
    }
    uint32_t all_more, all_equal;
    (void)sum_below(n_more, sh.sums, all_more);
    (void)sum_below(n_equal, sh.sums, all_equal);
    if (tid == 0) sh.kept[0] = all_more, sh.kept[1] = all_equal;
    cluster.sync();
    if (tid == 0) {
        uint32_t at = 0, ties = 0;
        for (int r = 0; r < kCluster; ++r) {
            const uint32_t *k = cluster.map_shared_rank(sh.kept, r);
            sh.first[r] = at;
            if (r == rank) sh.digit = ties;
            const uint32_t take = min(k[1], wanted - ties);
            at += k[0] + take, ties += take;
        }
        sh.first[kCluster] = at;
    }
    // the warp's words in order: of word (j, lane) the equal keys ahead of it, then the kept ones
    const auto warp_below = [&](uint32_t x, uint32_t &all) {
        uint32_t upto = x;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t o = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += o;
        }
        all = __shfl_sync(0xffffffffu, upto, 31);
        return upto - x;
    };
    uint32_t warp_equal = n_equal, ignored;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) warp_equal += __shfl_xor_sync(0xffffffffu, warp_equal, d);
    __syncthreads();
    uint32_t ties = sh.digit + sum_below(lane == 0 ? warp_equal : 0, sh.sums, ignored);
    ties = __shfl_sync(0xffffffffu, ties, 0);
    uint32_t n_kept = 0;
#pragma unroll
    for (int j = 0; j < kWords; ++j) {
        uint32_t all;
        const uint32_t ahead = ties + warp_below(__popc(equal[j]), all);
        ties += all;
        // of the word's equal keys the first that are still wanted
        uint32_t take = ahead < wanted ? wanted - ahead : 0u, e = equal[j];
        if (take < (uint32_t)__popc(e)) {
            uint32_t some = 0;
            for (; take > 0; --take) some |= e & -e, e &= e - 1;
            e = some;
        }
        more[j] |= e;
        n_kept += __popc(more[j]);
    }
    uint32_t warp_kept = n_kept;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) warp_kept += __shfl_xor_sync(0xffffffffu, warp_kept, d);
    uint32_t at = sum_below(lane == 0 ? warp_kept : 0, sh.sums, ignored);   // (its barriers: all keys have been read)
    at = __shfl_sync(0xffffffffu, at, 0);
#pragma unroll
    for (int j = 0; j < kWords; ++j) {
        if (i0 + j * 1024 >= i1) break;
        uint32_t all;
        const uint32_t ahead = at + warp_below(__popc(more[j]), all);
        at += all;
#pragma unroll 4
        for (int u = 0; u < 32; ++u) {
            const uint32_t word = __shfl_sync(0xffffffffu, more[j], u), first = __shfl_sync(0xffffffffu, ahead, u);
            if (word >> lane & 1) keys[first + __popc(word & ((1u << lane) - 1))] = t0 + i0 + (j * 32 + u) * 32 + lane;
        }
    }
    cluster.sync();
}

__device__ __forceinline__ int source_of(const cg::cluster_group &cluster, uint32_t *keys, const Shared &sh, int d)
{
    int r = 0;
    while (r + 1 < kCluster && sh.first[r + 1] <= (uint32_t)d) ++r;
    return (int)*cluster.map_shared_rank(keys + (d - sh.first[r]), r);
}

}  // namespace svev
