// sv_kv_evict: the tokens of least weight leave the cache; those that stay close up in their order.
//
// Mathematics: of a KV head's L tokens the first n_sink and the last n_recent stay, and of the others the heaviest until there are n of
// them (equal ones: the earlier first).  n is the same for all heads of a sequence, so that the block table and one length stay what the
// cache is described by.  Bound by HBM for long caches (weights once, 512 bytes of keys and values of a moved token read and written), by
// rendezvous for short ones.  8 K of 32 K tokens, 8 KV heads (70 MB): 41.0 us, 15 of them until the tokens are known; 16 sequences of 4 K to
// 16 K tokens halved (288 MB): 117 us, 38 % of a copy's rate.
//
// A cluster of CTAs has a (sequence, KV head).  Each CTA holds the order keys of a slice of the tokens in shared memory; the n-th largest
// is found by four passes of a histogram over eight bits, which the CTAs add up through distributed shared memory; each CTA then
// writes down the kept tokens of its slice in place of the keys.  The moves go in rounds: in a round every CTA takes a block of the
// result, reads its tokens -- all of them stand at their new place or behind it -- and writes them when all CTAs have read theirs.  What a
// round writes lies behind what earlier rounds wrote and ahead of what later ones read, so that the cache is compacted in place without
// scratch.
#include <cuda_bf16.h>

#include <type_traits>
#include <utility>

#include "attn_common.cuh"
#include "evict_core.cuh"
#include "sv_host.h"
#include "sv_ptx.cuh"

namespace {

using namespace svev;

struct Params {
    uint4 *k_pool, *v_pool;
    const int32_t *block_table, *seq_lens, *budget;
    const float *weights;
    float *weights_out, *reps;
    int32_t *seq_lens_out, *status;
    int Hkv, NBmax, n_pages, n_sink, n_recent;
};

template <int B>
__global__ void __launch_bounds__(kThreads) kv_evict_kernel(const __grid_constant__ Params p)
{
    extern __shared__ __align__(16) uint32_t keys[];   // of the slice; then its kept tokens
    __shared__ Shared sh;
    const cg::cluster_group cluster = cg::this_cluster();
    const int rank = blockIdx.x, h = blockIdx.y, s = blockIdx.z, tid = threadIdx.x;
    svk::grid_dependency_wait();
    svk::grid_launch_dependents();
    const int held = p.seq_lens[s], L = (int)min((long long)max(held, 0), (long long)p.NBmax * B);
    const long long ends = min((long long)p.n_sink + p.n_recent, (long long)L);
    const int n = (int)min((long long)L, max((long long)p.budget[s], ends));
    const size_t base = ((size_t)s * p.Hkv + h) * p.NBmax * B;
    if (rank == 0 && h == 0 && tid == 0) p.seq_lens_out[s] = n < L ? n : held;
    if (n >= L) {
        if (p.weights_out != p.weights)
            for (int t = rank * kThreads + tid; t < L; t += kCluster * kThreads) p.weights_out[base + t] = p.weights[base + t];
        return;
    }
    if (n > 0) keep_heaviest(cluster, p.weights + base, L, n, p.n_sink, p.n_recent, keys, sh);

    // The moves: 256 tokens of the result a CTA and round, a thread eight rows of them -- of the rows of a block those that sv_block_reps
    // gives it, so that the means are the same to the last bit.
    const int *pages = p.block_table + (size_t)s * p.NBmax;
    const int c = tid & 15, g = tid >> 4 & 15, w = tid >> 8;
    constexpr int kRows = 8, kPer = B / kRowGroups, kTurns = kRows / kPer;   // rows of a thread: kPer of a block, in kTurns blocks
    const auto place = [&](int i) { return (w + 2 * (i / kPer)) * B + g + kRowGroups * (i % kPer); };
    bool lost = false;
    const auto slot_of = [&](int t) {   // its row of the pools, or -1
        const int page = __ldg(pages + t / B);
        return (unsigned)page < (unsigned)p.n_pages ? ((long long)page * p.Hkv + h) * B + t % B : -1ll;
    };
    // A thread arrives at the cluster's barrier when its rows are there, finds the next round's sources and sums up the keys meanwhile, and
    // writes behind it; the next round's reads follow at once.  (One behind the other: 49.8 us instead of 47.2 for 8 K
    // of 32 K tokens.)
    const auto find_sources = [&](int t0, int turn) {
        const int first = t0 + rank * kRound;
        if (tid < min(n - first, kRound)) sh.source[turn][tid] = source_of(cluster, keys, sh, first + tid);
    };
    find_sources(0, 0);
    __syncthreads();
    int turn = 0;
#pragma unroll 1
    for (int t0 = 0; t0 < n; t0 += kCluster * kRound, turn ^= 1) {
        const int first = t0 + rank * kRound, rows = min(max(n - first, 0), kRound);
        const int32_t *source = sh.source[turn];
        const bool still = rows == 0 || source[rows - 1] == first + rows - 1;   // nothing moves
        uint4 k[kRows], v[kRows];
        float weight = 0.f;
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int r = place(i);
            k[i] = v[i] = make_uint4(0u, 0u, 0u, 0u);
            if (r < rows && (!still || p.reps)) {
                const long long from = slot_of(source[r]);
                lost |= from < 0;
                if (from >= 0) {
                    k[i] = p.k_pool[from * 16 + c];
                    if (!still) v[i] = p.v_pool[from * 16 + c];
                }
            }
        }
        if (tid < rows) weight = p.weights[base + source[tid]];
        auto arrived = cluster.barrier_arrive();
        find_sources(t0 + kCluster * kRound, turn ^ 1);
        if (p.reps) {
#pragma unroll
            for (int half = 0; half < kTurns; ++half) {
                float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = half * kPer; i < (half + 1) * kPer; ++i) {
                    const uint32_t x[4] = {k[i].x, k[i].y, k[i].z, k[i].w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float2 f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&x[e]));
                        acc[2 * e] += f.x, acc[2 * e + 1] += f.y;
                    }
                }
                float4 *part = reinterpret_cast<float4 *>(&sh.part[w + 2 * half][g][c * 8]);
                part[0] = make_float4(acc[0], acc[1], acc[2], acc[3]), part[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
            }
            __syncthreads();
            const int block = tid >> 7, dim = tid & 127, held = min(rows - block * B, B);
            if (block < kRound / B && held > 0) {
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < kRowGroups; ++i) sum += sh.part[block][i][dim];
                p.reps[(((size_t)s * p.Hkv + h) * p.NBmax + first / B + block) * 128 + dim] = sum / (float)held;
            }
        }
        cluster.barrier_wait(std::move(arrived));
        __syncthreads();   // (the next sources are there and the sums are through: both came after the thread had arrived)
        if (tid < rows) p.weights_out[base + first + tid] = weight;
        if (!still) {
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                const int r = place(i);
                if (r < rows) {
                    const long long to = slot_of(first + r);
                    lost |= to < 0;
                    if (to >= 0) p.k_pool[to * 16 + c] = k[i], p.v_pool[to * 16 + c] = v[i];
                }
            }
        }
    }
    if (lost && p.status) atomicOr(p.status, svk::kStatusIndex);
    cluster.sync();   // (the other CTAs have read this one's list, and all weights have been read)
    for (int t = n + rank * kThreads + tid; t < L; t += kCluster * kThreads) p.weights_out[base + t] = 0.f;
}

}  // namespace

extern "C" sv_status sv_kv_evict(const sv_geom *geom, void *k_pool, void *v_pool, int32_t n_pages, const int32_t *block_table,
                                 const int32_t *seq_lens, const float *weights, const int32_t *budget, int32_t n_sink, int32_t n_recent,
                                 int32_t *seq_lens_out, float *weights_out, float *reps, int32_t *status_word, void *stream)
{
    const sv_status st = svh::check_ragged(geom, 0);
    if (st != SV_OK) return st;
    const int Hkv = geom->n_kv_heads, B = geom->block_size;
    if (!k_pool || !v_pool || !block_table || !seq_lens || !weights || !budget || !seq_lens_out || !weights_out) return SV_ERR_NULL;
    if (n_pages < 1 || (int64_t)n_pages * Hkv * B >= (int64_t)1 << 31 || n_sink < 0 || n_recent < 0) return SV_ERR_SHAPE;
    if (seq_lens_out == seq_lens) return SV_ERR_SHAPE;   // other CTAs still read the old length
    if (!svh::aligned(k_pool, 128) || !svh::aligned(v_pool, 128) || !svh::aligned(weights, 16) || !svh::aligned(weights_out, 16) || !svh::aligned(reps, 16))
        return SV_ERR_ALIGN;
    const int64_t cap = (int64_t)geom->max_blocks * B;
    if (cap > kMostTokens) return SV_ERR_UNSUPPORTED;
    Params p = {};
    p.k_pool = static_cast<uint4 *>(k_pool), p.v_pool = static_cast<uint4 *>(v_pool);
    p.block_table = block_table, p.seq_lens = seq_lens, p.budget = budget, p.weights = weights, p.weights_out = weights_out, p.reps = reps;
    p.seq_lens_out = seq_lens_out, p.status = status_word;
    p.Hkv = Hkv, p.NBmax = geom->max_blocks, p.n_pages = n_pages, p.n_sink = n_sink, p.n_recent = n_recent;
    const auto kernel = B == 64 ? kv_evict_kernel<64> : kv_evict_kernel<128>;
    static svh::OncePerDevice once;
    if (once.run([] {
            const cudaError_t e = cudaFuncSetAttribute(kv_evict_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSlice * 4);
            return e != cudaSuccess ? e : cudaFuncSetAttribute(kv_evict_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSlice * 4);
        }) != cudaSuccess) {
        (void)cudaGetLastError();
        return SV_ERR_CUDA;
    }
    const size_t bytes = (size_t)(((cap + kCluster - 1) / kCluster + 3) & ~3ll) * 4;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(kCluster, Hkv, geom->n_seq);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[2];
    svh::pdl_attribute(attr);
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = kCluster, attr[1].val.clusterDim.y = 1, attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, p) == cudaSuccess ? svh::launch_status() : SV_ERR_CUDA;
}
