// Which tokens of a KV head stay (sv_kv_evict): the n-th largest of their order keys, found by the CTAs of a cluster together, and the list
// of those that stay.  Every CTA has the keys of a slice in its shared memory.
#pragma once
#include <cooperative_groups.h>
#include <stdint.h>

#include "order_key.h"

namespace svev {

namespace cg = cooperative_groups;

constexpr int kRowGroups = 16;
constexpr int kThreads = 512, kCluster = 8;
constexpr int kPasses = 4, kBins = 256;          // of a key's digits
constexpr int kSlice = 49152;                    // tokens that a CTA's shared memory holds the keys of
constexpr int kMostTokens = kCluster * kSlice;
constexpr int kRound = 256;                      // tokens that a CTA moves at a time

struct Shared {
    union {
        uint32_t hist[kPasses][kBins];
        alignas(16) float part[4][kRowGroups][128];   // (the moves) of four blocks sums of keys
    };
    uint32_t sums[kThreads / 32];
    uint32_t digit, above;      // what a pass found
    alignas(8) uint32_t kept[2];   // of the slice: keys above the n-th largest, keys equal to it
    uint32_t first[kCluster + 1];   // where the slices' kept tokens begin
    int32_t source[2][kRound];     // of a round's tokens and the next one's
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

// Of tokens 0 .. L - 1 with these weights n > 0 stay: the first n_sink, the last n_recent, and the heaviest others.  keys: room for the CTA's
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
        const uint32_t bits = __float_as_uint(weights[t]), key = svsel::key_of_bits(bits == 0x80000000u ? 0u : bits);   // (the zeros are equal)
        keys[i] = t < n_sink || t >= L - n_recent ? svsel::kForcedKey : key;
    }
    for (int i = tid; i < kPasses * kBins; i += kThreads) sh.hist[i / kBins][i % kBins] = 0;
    __syncthreads();
    // The n-th largest key, by digits from the top; all CTAs find the same.  (Three passes over 11, 11 and 10 bits have eight times the bins to
    // fetch from the peers, 2.3 us a pass.)
    uint32_t prefix = 0, wanted = n;
#pragma unroll 1
    for (int pass = 0; pass < kPasses; ++pass) {
        const int low = 24 - 8 * pass;
        for (int i = tid; i < count; i += kThreads) {
            const uint32_t key = keys[i];
            if (pass == 0 || key >> (low + 8) == prefix) atomicAdd(&sh.hist[pass][key >> low & (kBins - 1)], 1u);
        }
        cluster.sync();
        // A thread a bin, from the top.  (All peers' are asked for at once: one peer behind the other is a trip of half a microsecond each.)
        uint32_t sum = 0;
        if (tid < kBins) {
            uint32_t x[kCluster];
#pragma unroll
            for (int r = 0; r < kCluster; ++r) x[r] = cluster.map_shared_rank(sh.hist[pass], r)[kBins - 1 - tid];
#pragma unroll
            for (int r = 0; r < kCluster; ++r) sum += x[r];
        }
        uint32_t all, above = sum_below(sum, sh.sums, all);
        if (above < wanted && wanted <= above + sum) sh.digit = kBins - 1 - tid, sh.above = above;
        __syncthreads();
        prefix = prefix << 8 | sh.digit;
        wanted -= sh.above;
        __syncthreads();
    }
    // prefix is the key; of those equal to it the first `wanted` of the sequence stay.  A warp has a run of the slice; lane u of it keeps the
    // ballots of the run's words u, 32 + u, ...
    constexpr int kWords = kSlice / (kThreads / 32) / 32 / 32;
    const int lane = tid & 31, warp = tid >> 5;
    const int run = ((count + kThreads / 32 - 1) / (kThreads / 32) + 31) & ~31, i0 = min(warp * run, count), i1 = min(i0 + run, count);
    uint32_t more[kWords], equal[kWords], n_more = 0, n_equal = 0;
#pragma unroll
    for (int j = 0; j < kWords; ++j) {
        more[j] = equal[j] = 0;
        if (i0 + j * 1024 < i1) {
            const int words = min((i1 - i0 - j * 1024 + 31) / 32, 32);
#pragma unroll 4
            for (int u = 0; u < words; ++u) {
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
    if (tid < 32) {
        uint32_t above = 0, same = 0;   // of the slice of CTA `tid`
        if (tid < kCluster) {
            const uint2 k = *reinterpret_cast<const uint2 *>(cluster.map_shared_rank(sh.kept, tid));
            above = k.x, same = k.y;
        }
        uint32_t at = above, ties = same;   // up to and with that slice
#pragma unroll
        for (int d = 1; d <= kCluster; d <<= 1) {
            const uint32_t a = __shfl_up_sync(0xffffffffu, at, d), b = __shfl_up_sync(0xffffffffu, ties, d);
            if (tid >= d) at += a, ties += b;
        }
        const uint32_t before = min(ties - same, wanted);
        if (tid <= kCluster) sh.first[tid] = at - above + before;
        if (tid == rank) sh.digit = before;
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
        const int words = min((i1 - i0 - j * 1024 + 31) / 32, 32);
#pragma unroll 4
        for (int u = 0; u < words; ++u) {
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
