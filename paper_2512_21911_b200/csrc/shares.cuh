// Where the shares of a batch's workers begin (q4_shares.h), found by all threads of a CTA, and plain accesses of shared memory by address.
#pragma once
#include "q4_shares.h"
#include "sv_ptx.cuh"

namespace svk {

__device__ __forceinline__ uint32_t lds32(uint32_t a)
{
    uint32_t v;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a)
{
    uint2 v;
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint4 lds128(uint32_t a)
{
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void sts32(uint32_t a, uint32_t v) { asm volatile("st.shared.b32 [%0], %1;" ::"r"(a), "r"(v) : "memory"); }
__device__ __forceinline__ void sts64(uint32_t a, unsigned long long v) { asm volatile("st.shared.b64 [%0], %1;" ::"r"(a), "l"(v) : "memory"); }
__device__ __forceinline__ void sts128(uint32_t a, uint4 v)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ float ldsf(uint32_t a) { return __uint_as_float(lds32(a)); }
__device__ __forceinline__ void stsf(uint32_t a, float v) { sts32(a, __float_as_uint(v)); }
__device__ __forceinline__ long long lds_ll(uint32_t a)
{
    const uint2 v = lds64(a);
    return (long long)((unsigned long long)v.y << 32 | v.x);
}

// The batch's line, `entries` of cost cost(e), among gridDim.x * kWorkers workers; few shares go to as many CTAs as there are.  Of the
// CTA's shares blockIdx.x * per_cta + w: found + 16 w holds the entry that it begins in, and where that begins on the line.  scan: 8 bytes
// for each warp.  All threads; ends with a barrier.
template <int kThreads, int kWorkers, class Cost>
__device__ __forceinline__ svq::Line find_shares(int entries, int den, uint32_t scan, uint32_t found, int &per_cta, Cost cost)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int run = (entries + kThreads - 1) / kThreads, e0 = min(tid * run, entries), e1 = min(e0 + run, entries);
    long long mine = 0;
#pragma unroll 1
    for (int e = e0; e < e1; ++e) mine += cost(e);
    long long upto = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const long long o = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += o;
    }
    if (lane == 31) sts64(scan + warp * 8, (unsigned long long)upto);
    __syncthreads();
    long long total = 0;
#pragma unroll 1
    for (int w = 0; w < kThreads / 32; ++w) {
        const long long sum = lds_ll(scan + w * 8);
        if (w < warp) upto += sum;
        total += sum;
    }
    const svq::Line line(total, gridDim.x * kWorkers, den, svq::kUnit);
    per_cta = (line.shares + (int)gridDim.x - 1) / (int)gridDim.x;
#pragma unroll 1
    for (int w = 0; w < per_cta; ++w) {
        const int share = blockIdx.x * per_cta + w;
        if (share >= line.shares) break;
        const long long lo = line.bound(share);
        if (mine > 0 && upto - mine <= lo && lo < upto) {
            long long at = upto - mine;
            int e = e0;
#pragma unroll 1
            for (; e < e1; ++e) {
                const long long c = cost(e);
                if (lo < at + c) break;
                at += c;
            }
            sts64(found + w * 16, (unsigned long long)e);
            sts64(found + w * 16 + 8, (unsigned long long)at);
        }
    }
    __syncthreads();
    return line;
}

}  // namespace svk
