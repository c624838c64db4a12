// sv_chunk_attn: causal attention of a ragged batch of new tokens over the paged cache that holds them.
//
// Mathematics, for a row q at position p: running maximum m and sum l of 2^(s_t - m), s_t = q . k_t * scale * log2 e over the keys t <= p,
// and o = sum_t 2^(s_t - m) v_t, rescaled when m grows; the output is o / l.  Simple form: a warp per row (token, query head), four dims a
// lane, one pass over the keys.
#include <cuda_bf16.h>

#include "attn_common.cuh"
#include "sv_host.h"
#include "sv_ptx.cuh"

namespace {

constexpr int kThreads = 256;

struct Params {
    const uint2 *q, *k_pool, *v_pool;
    const int32_t *block_table, *seq_lens, *q_start;
    uint2 *out;
    float *lse;
    int32_t *status;
    int S, N, Hq, Hkv, B, NBmax, n_pages;
    float scale_log2;
};

__device__ __forceinline__ float4 four(uint2 w)
{
    const float2 a = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&w.x)), b = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&w.y));
    return make_float4(a.x, a.y, b.x, b.y);
}

__global__ void __launch_bounds__(kThreads) chunk_attn_kernel(const Params p)
{
    svk::grid_dependency_wait();
    svk::grid_launch_dependents();
    const int token = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const auto start = [&](int s) { return min(max(p.q_start[s], 0), p.N); };
    int s = 0, hi = p.S - 1;   // the last sequence that starts at or before the token
    while (s < hi) {
        const int mid = (s + hi + 1) / 2;
        if (start(mid) <= token) s = mid;
        else hi = mid - 1;
    }
    if (token < start(s) || token >= start(s + 1)) return;
    const int len = (int)min((long long)p.seq_lens[s], (long long)p.NBmax * p.B);
    const int pos = min(p.seq_lens[s] - start(s + 1) + token, len - 1);
    const int G = p.Hq / p.Hkv;
    for (int hq = warp; hq < p.Hq; hq += kThreads / 32) {
        const int h = hq / G;
        const size_t row = (size_t)token * p.Hq + hq;
        const float4 q = four(p.q[row * 32 + lane]);
        float m = -INFINITY, l = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int t = 0; t <= pos; ++t) {
            int page = p.block_table[(size_t)s * p.NBmax + t / p.B];
            if ((unsigned)page >= (unsigned)p.n_pages) {
                if (lane == 0 && p.status) atomicOr(p.status, svk::kStatusIndex);
                page = page < 0 ? 0 : p.n_pages - 1;
            }
            const size_t at = (((size_t)page * p.Hkv + h) * p.B + t % p.B) * 32 + lane;
            const float4 k = four(p.k_pool[at]);
            float x = q.x * k.x + q.y * k.y + q.z * k.z + q.w * k.w;
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
            x *= p.scale_log2;
            const float m_new = fmaxf(m, x), c = svk::fast_exp2(m - m_new), w = svk::fast_exp2(x - m_new);
            const float4 v = four(p.v_pool[at]);
            o.x = o.x * c + w * v.x, o.y = o.y * c + w * v.y, o.z = o.z * c + w * v.z, o.w = o.w * c + w * v.w;
            l = l * c + w, m = m_new;
        }
        const float inv = l > 0.f ? 1.f / l : 0.f;
        p.out[row * 32 + lane] = make_uint2(svk::pack_bf16(o.x * inv, o.y * inv), svk::pack_bf16(o.z * inv, o.w * inv));
        if (p.lse && lane == 0) p.lse[row] = l > 0.f ? (m + log2f(l)) * 0.69314718055994531f : -INFINITY;
    }
}

}  // namespace

extern "C" size_t sv_chunk_workspace_bytes(const sv_geom *geom, int32_t n_tokens)
{
    return svh::check_ragged(geom, n_tokens) == SV_OK ? 16 : 0;
}

extern "C" sv_status sv_chunk_attn(const sv_geom *geom, const void *q, const sv_kv *kv, const int32_t *q_start, int32_t n_tokens,
                                   float softmax_scale, void *out, float *lse, void *workspace, size_t workspace_bytes,
                                   int32_t *status_word, void *stream)
{
    sv_status st = svh::check_ragged(geom, n_tokens);
    if (st != SV_OK) return st;
    st = svh::check_kv(geom, kv, true);
    if (st != SV_OK) return st;
    if (!q_start || (n_tokens > 0 && (!q || !out))) return SV_ERR_NULL;
    if (!svh::aligned(q, 16) || !svh::aligned(out, 16) || !svh::aligned(workspace, 16)) return SV_ERR_ALIGN;
    if (workspace_bytes < sv_chunk_workspace_bytes(geom, n_tokens)) return SV_ERR_WORKSPACE;
    if (!workspace) return SV_ERR_NULL;
    if (n_tokens == 0) return SV_OK;
    Params p = {};
    p.q = static_cast<const uint2 *>(q), p.k_pool = static_cast<const uint2 *>(kv->k_pool), p.v_pool = static_cast<const uint2 *>(kv->v_pool);
    p.block_table = kv->block_table, p.seq_lens = kv->seq_lens, p.q_start = q_start;
    p.out = static_cast<uint2 *>(out), p.lse = lse, p.status = status_word;
    p.S = geom->n_seq, p.N = n_tokens, p.Hq = geom->n_q_heads, p.Hkv = geom->n_kv_heads, p.B = geom->block_size, p.NBmax = geom->max_blocks;
    p.n_pages = kv->n_pages;
    p.scale_log2 = (softmax_scale == 0.f ? 0.08838834764831845f : softmax_scale) * 1.4426950408889634f;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)n_tokens);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[1];
    svh::pdl_attribute(attr);
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, chunk_attn_kernel, p) == cudaSuccess ? svh::launch_status() : SV_ERR_CUDA;
}
