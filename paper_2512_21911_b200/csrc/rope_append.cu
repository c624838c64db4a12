// sv_rope_append: rotary positions on the queries and keys of new tokens, keys and values into the paged cache, representatives of
// the blocks that grew (the mean key of a block, Eq. 5) -- what happens to a projection's output before anything attends over it.
//
// Mathematics: a pair (a, b) of a head's dims at position p becomes (a cos - b sin, b cos + a sin), cos and sin from a table.  Bound by
// HBM: (Hq + 2 Hkv) * 256 bytes read and written per token, a table row of 512 bytes shared by all heads, no reuse.  A prompt of 32,768
// tokens with 32 query and 8 KV heads moves 826 MB in 167 us, 4.9 TB/s, 76 % of a plain copy's rate; a token for each of 64 sequences
// takes 6.9 us, three dependent loads (starts, length and table, rows) behind a launch.  (All figures here: nothing in L2 before the call.)
//
// One launch of two kinds of CTAs.  The first take a block of a sequence and a KV head: 16 threads hold a 256-byte row, so that the
// partner of a dim is in the same thread (neighbours) or 2 to 8 lanes away (halves), the rows of the block go to its page, and the mean
// of the keys, rounded as they are stored, is summed in the order of sv_block_reps.  The others take a few tokens and all their query
// heads.  (rope.cuh has what the append of a 4-bit cache shares with this one: the rotation, the way from a CTA's number to its block.)
#include <cuda_bf16.h>

#include <type_traits>

#include "attn_common.cuh"
#include "rope.cuh"
#include "sv_host.h"
#include "sv_ptx.cuh"

namespace {

using namespace svrope;

struct Params {
    uint4 *k_pool, *v_pool;
    const int32_t *block_table, *seq_lens, *q_start;
    const int32_t *positions;   // of the sequences' first new tokens, or null: seq_lens
    const uint4 *q, *k, *v;
    long long q_stride, k_stride, v_stride;   // 16-byte chunks between tokens
    const float *rope;
    uint4 *q_out;
    int32_t *seq_lens_out;
    float *reps;
    int32_t *status;
    int S, N, Hq, Hkv, NBmax, n_pages, rope_rows, rot;
    int slots;   // CTAs of the first kind: slots x Hkv
};

template <int B, bool kNeighbours>
__device__ __forceinline__ void append_block(const Params &p, int slot, int h)
{
    __shared__ float part[kRowGroups][128];
    const int tid = threadIdx.x, c = tid & 15, rg = tid >> 4;
    Grown grown;
    if (!grown_block<B>(p, slot, h, grown)) return;
    const int s = grown.s, L = grown.before, b = grown.block, end = grown.end, page = grown.page, first = grown.first;
    const long long ahead = p.positions ? (long long)p.positions[s] - L : 0;   // of a token's position to its place in the cache
    constexpr int kIter = B / kRowGroups;
    uint4 k[kIter], v[kIter];
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
        const int t = b * B + rg + i * kRowGroups;
        k[i] = v[i] = make_uint4(0u, 0u, 0u, 0u);
        const size_t in_pool = (((size_t)page * p.Hkv + h) * B + t % B) * 16 + c;
        if (t < L) {
            if (p.reps) k[i] = p.k_pool[in_pool];
        } else if (t < end) {
            const long long row = first + (t - L);
            k[i] = __ldg(p.k + row * p.k_stride + h * 16 + c), v[i] = __ldg(p.v + row * p.v_stride + h * 16 + c);
        }
    }
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
        const int t = b * B + rg + i * kRowGroups;
        const bool fresh = t >= L && t < end;
        if (p.rope && __any_sync(0xffffffffu, fresh)) {
            const long long pos = t + ahead;
            const int at = (int)min(max(pos, 0ll), (long long)p.rope_rows - 1);
            Turn turn;
            if (8 * c < p.rot) turn = load_turn<kNeighbours>(p.rope + (size_t)at * p.rot, c, p.rot);
            const uint4 turned = rotate<kNeighbours>(k[i], turn, c, p.rot);
            if (fresh) {
                k[i] = turned;
                if (at != pos && p.status) atomicOr(p.status, svk::kStatusIndex);
            }
        }
        if (fresh) {
            const size_t in_pool = (((size_t)page * p.Hkv + h) * B + t % B) * 16 + c;
            p.k_pool[in_pool] = k[i], p.v_pool[in_pool] = v[i];
        }
    }
    if (!p.reps) return;
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
        const uint32_t w[4] = {k[i].x, k[i].y, k[i].z, k[i].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 f = halves_of(w[e]);
            acc[2 * e] += f.x;
            acc[2 * e + 1] += f.y;
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) part[rg][c * 8 + e] = acc[e];
    __syncthreads();
    if (tid < 128) {
        float sum = 0.f;
#pragma unroll
        for (int g = 0; g < kRowGroups; ++g) sum += part[g][tid];
        p.reps[(((size_t)s * p.Hkv + h) * p.NBmax + b) * 128 + tid] = sum / (float)(end - b * B);
    }
}

// Three CTAs an SM (80 registers): a ragged batch of 3,512 tokens (28 query heads, cache blocks of 128) takes 16.3 us; without the bound
// it takes 128 registers, two CTAs an SM and 16.9 us; four CTAs (64 registers) take 23.6 us, since the rows of a cache block then no
// longer all start to load at once.
template <int B, bool kNeighbours, int kQTokens>
__global__ void __launch_bounds__(kThreads, 3) rope_append_kernel(const Params p)
{
    svk::grid_dependency_wait();
    svk::grid_launch_dependents();
    const int i = blockIdx.x, cache = p.slots * p.Hkv;
    if (i < cache) append_block<B, kNeighbours>(p, i / p.Hkv, i % p.Hkv);
    else turn_queries<kNeighbours, kQTokens>(p, i - cache);
}

}  // namespace

extern "C" sv_status sv_rope_append_at(const sv_geom *geom, void *k_pool, void *v_pool, int32_t n_pages, const int32_t *block_table,
                                       const int32_t *seq_lens, const int32_t *positions, const void *q, const void *k, const void *v,
                                       int64_t q_stride, int64_t k_stride, int64_t v_stride, const int32_t *q_start, int32_t n_tokens,
                                       const float *rope, int32_t rope_rows, int32_t rot_dim, int32_t interleaved, void *q_out,
                                       int32_t *seq_lens_out, float *reps, int32_t *status_word, void *stream)
{
    const sv_status st = svh::check_ragged(geom, n_tokens);
    if (st != SV_OK) return st;
    const int Hq = geom->n_q_heads, Hkv = geom->n_kv_heads, B = geom->block_size;
    if (!k_pool || !v_pool || !block_table || !seq_lens || !q_start || !seq_lens_out || (n_tokens > 0 && (!k || !v)) || (!q) != (!q_out))
        return SV_ERR_NULL;
    if (n_pages < 1 || (int64_t)n_pages * Hkv * B >= (int64_t)1 << 31) return SV_ERR_SHAPE;
    if (seq_lens_out == seq_lens) return SV_ERR_SHAPE;   // other CTAs still read the old length
    if (rope && (rope_rows < 1 || rot_dim < 16 || rot_dim > svh::kHeadDim || rot_dim % 16)) return SV_ERR_SHAPE;
    if (n_tokens > 1 && (k_stride < (int64_t)Hkv * svh::kHeadDim || v_stride < (int64_t)Hkv * svh::kHeadDim ||
                         (q && q_stride < (int64_t)Hq * svh::kHeadDim)))
        return SV_ERR_SHAPE;
    // (a row of q_out is written by a CTA that reads other rows of q: in place only where both have the same layout)
    if (q && q_out == q && n_tokens > 1 && q_stride != (int64_t)Hq * svh::kHeadDim) return SV_ERR_SHAPE;
    if (n_tokens > 1 && (q_stride % 8 || k_stride % 8 || v_stride % 8)) return SV_ERR_ALIGN;
    if (!svh::aligned(k_pool, 128) || !svh::aligned(v_pool, 128) || !svh::aligned(q, 16) || !svh::aligned(k, 16) || !svh::aligned(v, 16) ||
        !svh::aligned(q_out, 16) || !svh::aligned(rope, 16) || !svh::aligned(reps, 16))
        return SV_ERR_ALIGN;
    Params p = {};
    p.k_pool = static_cast<uint4 *>(k_pool), p.v_pool = static_cast<uint4 *>(v_pool);
    p.block_table = block_table, p.seq_lens = seq_lens, p.positions = positions, p.q_start = q_start;
    p.q = static_cast<const uint4 *>(q), p.k = static_cast<const uint4 *>(k), p.v = static_cast<const uint4 *>(v);
    p.q_stride = q_stride / 8, p.k_stride = k_stride / 8, p.v_stride = v_stride / 8;
    p.rope = rope, p.q_out = static_cast<uint4 *>(q_out), p.seq_lens_out = seq_lens_out, p.reps = reps, p.status = status_word;
    p.S = geom->n_seq, p.N = n_tokens, p.Hq = Hq, p.Hkv = Hkv, p.NBmax = geom->max_blocks, p.n_pages = n_pages;
    p.rope_rows = rope_rows, p.rot = rot_dim;
    const long long slots = (long long)n_tokens / B + 2ll * geom->n_seq;
    const int tokens = n_tokens <= kFew ? kTokensOfFew : kTokensOfMany;
    const long long ctas = slots * Hkv + (q ? ((long long)n_tokens + tokens - 1) / tokens : 0);
    if (ctas > 0x7fffffff) return SV_ERR_SHAPE;
    p.slots = (int)slots;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[1];
    svh::pdl_attribute(attr);
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const auto pick = [&](auto block, auto turned) {
        return tokens == kTokensOfFew ? rope_append_kernel<decltype(block)::value, decltype(turned)::value, kTokensOfFew>
                             : rope_append_kernel<decltype(block)::value, decltype(turned)::value, kTokensOfMany>;
    };
    const auto by_order = [&](auto block) { return interleaved ? pick(block, std::true_type{}) : pick(block, std::false_type{}); };
    const auto kernel = B == 64 ? by_order(std::integral_constant<int, 64>{}) : by_order(std::integral_constant<int, 128>{});
    return cudaLaunchKernelEx(&cfg, kernel, p) == cudaSuccess ? svh::launch_status() : SV_ERR_CUDA;
}

extern "C" sv_status sv_rope_append(const sv_geom *geom, void *k_pool, void *v_pool, int32_t n_pages, const int32_t *block_table,
                                    const int32_t *seq_lens, const void *q, const void *k, const void *v, int64_t q_stride, int64_t k_stride,
                                    int64_t v_stride, const int32_t *q_start, int32_t n_tokens, const float *rope, int32_t rope_rows,
                                    int32_t rot_dim, int32_t interleaved, void *q_out, int32_t *seq_lens_out, float *reps,
                                    int32_t *status_word, void *stream)
{
    return sv_rope_append_at(geom, k_pool, v_pool, n_pages, block_table, seq_lens, nullptr, q, k, v, q_stride, k_stride, v_stride, q_start,
                             n_tokens, rope, rope_rows, rot_dim, interleaved, q_out, seq_lens_out, reps, status_word, stream);
}
