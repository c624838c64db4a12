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
// heads.  The batch is ragged and its lengths are only on the device: the blocks that sequence s enters are at most n / B + 2, so that
// numbering them from q_start[s] / B + 2 s gives every sequence room of its own, and a CTA finds its sequence by counting the starts up to
// its number instead of by a prefix sum.
#include <cuda_bf16.h>

#include <type_traits>

#include "attn_common.cuh"
#include "sv_host.h"
#include "sv_ptx.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kRowGroups = kThreads / 16;
// Tokens of a CTA that rotates queries: two in calls of up to kFew tokens, where the query CTAs of many would not fill the machine and a
// CTA's own chain of loads is what counts; many beyond, where reading the batch's starts and lengths is shared by more rows.  With two and
// with eight tokens: 64 sequences of one token 6.8 and 9.2 us; chunks of four sequences, 256 tokens in all 5.1 and 6.0, 1,024 7.3 and 9.1,
// 1,536 11.5 either way, 2,048 14.9 and 15.7, 4,096 26.4 and 24.9; a prompt of 32,768 195 and 168.  512, 1,024 and 2,048 sequences of one
// token each: 43 and 47, 86 and 89, 191 and 190.  The edge is not sharp: the two cross between 1,536 and 4,096 tokens.
constexpr int kFew = 1024, kTokensOfFew = 2, kTokensOfMany = 8;

struct Params {
    uint4 *k_pool, *v_pool;
    const int32_t *block_table, *seq_lens, *q_start;
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

// cos and sin of the 8 dims of chunk c at a table row: for halves, of dims 8 c .. 8 c + 7 (of their pairs' numbers); for neighbours,
// of pairs 4 c .. 4 c + 3.
struct Turn {
    float c[8], s[8];
};
template <bool kNeighbours>
__device__ __forceinline__ Turn load_turn(const float *row, int c, int rot)
{
    Turn t;
    const int half = rot / 2, n = kNeighbours ? 4 : 8;
    const int j = kNeighbours ? 4 * c : 8 * c >= half ? 8 * c - half : 8 * c;
#pragma unroll
    for (int i = 0; i < n; i += 4) {
        const float4 a = __ldg(reinterpret_cast<const float4 *>(row + j + i)), b = __ldg(reinterpret_cast<const float4 *>(row + half + j + i));
        t.c[i] = a.x, t.c[i + 1] = a.y, t.c[i + 2] = a.z, t.c[i + 3] = a.w;
        t.s[i] = b.x, t.s[i + 1] = b.y, t.s[i + 2] = b.z, t.s[i + 3] = b.w;
    }
    return t;
}

__device__ __forceinline__ float2 halves_of(uint32_t w) { return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&w)); }
// Rounded one by one (no contraction to a fused product and sum): the rotated values are those of the formula in plain fp32.
__device__ __forceinline__ float minus(float a, float c, float b, float s) { return __fsub_rn(__fmul_rn(a, c), __fmul_rn(b, s)); }
__device__ __forceinline__ float plus(float a, float c, float b, float s) { return __fadd_rn(__fmul_rn(a, c), __fmul_rn(b, s)); }

// Chunk c of a rotated row.  Every lane of the 16 that hold the row calls it; chunks from rot on come back as they are.
template <bool kNeighbours>
__device__ __forceinline__ uint4 rotate(uint4 x, const Turn &t, int c, int rot)
{
    uint32_t w[4] = {x.x, x.y, x.z, x.w}, r[4];
    if constexpr (kNeighbours) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 v = halves_of(w[i]);
            r[i] = svk::pack_bf16(minus(v.x, t.c[i], v.y, t.s[i]), plus(v.y, t.c[i], v.x, t.s[i]));
        }
    } else {
        const int away = rot / 16;   // chunks between a dim and its partner
        const bool lower = c < away;
        const int partner = ((threadIdx.x & 31) & 16) | (c < 2 * away ? (lower ? c + away : c - away) : c);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 v = halves_of(w[i]), o = halves_of(__shfl_sync(0xffffffffu, w[i], partner));
            const float y0 = lower ? minus(v.x, t.c[2 * i], o.x, t.s[2 * i]) : plus(v.x, t.c[2 * i], o.x, t.s[2 * i]);
            const float y1 = lower ? minus(v.y, t.c[2 * i + 1], o.y, t.s[2 * i + 1]) : plus(v.y, t.c[2 * i + 1], o.y, t.s[2 * i + 1]);
            r[i] = svk::pack_bf16(y0, y1);
        }
    }
    return 8 * c < rot ? make_uint4(r[0], r[1], r[2], r[3]) : x;
}

__device__ __forceinline__ int start_of(const Params &p, int s) { return min(max(__ldg(p.q_start + s), 0), p.N); }

// The last sequence s whose number (of ascending ones) is not above x; all threads of the CTA.
template <class F>
__device__ __forceinline__ int last_not_above(int S, int x, F number)
{
    int n = 0;
    for (int base = 0; base < S; base += kThreads) n += __syncthreads_count(base + (int)threadIdx.x < S && number(base + threadIdx.x) <= x);
    return n - 1;
}

template <int B, bool kNeighbours>
__device__ __forceinline__ void append_block(const Params &p, int slot, int h)
{
    __shared__ float part[kRowGroups][128];
    const int tid = threadIdx.x, c = tid & 15, rg = tid >> 4;
    const int s = last_not_above(p.S, slot, [&](int i) { return start_of(p, i) / B + 2 * i; });
    if (s < 0) return;
    const int first = start_of(p, s), n_all = max(0, start_of(p, s + 1) - first);
    const int L = p.seq_lens[s];
    const int *pages = p.block_table + (size_t)s * p.NBmax;
    const int j = slot - (first / B + 2 * s);   // the block's place among those that the sequence enters
    const int b0 = max(L, 0) / B;
    // Tokens that the table has pages for: a block behind its end, or whose entry is not a page of the pool, ends it.
    const auto bad = [&](int b) { return b >= p.NBmax || (unsigned)__ldg(pages + b) >= (unsigned)p.n_pages; };
    const auto room = [&](int b_last) {   // the first bad block of b0 .. b_last, or b_last + 1
        int found = b_last + 1;
        for (int base = b0; base <= b_last && found > b_last; base += kThreads) {
            const int b = base + tid;
            const bool is = b <= b_last && bad(b);
            if (__syncthreads_or(is)) {
                __shared__ int least;
                if (tid == 0) least = b_last + 1;
                __syncthreads();
                if (is) atomicMin(&least, b);
                __syncthreads();
                found = least;
            }
        }
        return found;
    };
    if (j == 0 && h == 0) {
        int Ln = L;
        if (L >= 0 && n_all > 0) {
            const int end = (int)min((long long)L + n_all, (long long)p.NBmax * B);
            Ln = end <= L ? L : max(L, min(end, room((end - 1) / B) * B));
        }
        if (tid == 0) {
            p.seq_lens_out[s] = Ln;
            if (p.status && Ln != (long long)L + n_all) atomicOr(p.status, svk::kStatusIndex);   // tokens were dropped
        }
    }
    const int b = b0 + j;
    if (L < 0 || n_all == 0 || b >= p.NBmax || (long long)b * B >= (long long)L + n_all || room(b) <= b) return;
    const int end = (int)min((long long)L + n_all, (long long)(b + 1) * B);   // behind the block's last token
    const int page = pages[b];
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
            const int at = min(max(t, 0), p.rope_rows - 1);
            Turn turn;
            if (8 * c < p.rot) turn = load_turn<kNeighbours>(p.rope + (size_t)at * p.rot, c, p.rot);
            const uint4 turned = rotate<kNeighbours>(k[i], turn, c, p.rot);
            if (fresh) {
                k[i] = turned;
                if (t >= p.rope_rows && p.status) atomicOr(p.status, svk::kStatusIndex);
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

// Query heads of kQTokens tokens: a token's heads are dealt to kStep groups of 16 threads; a thread has kAhead of them on their way at
// once and keeps its part of the token's table row for all of them.
template <bool kNeighbours, int kQTokens>
__device__ __forceinline__ void turn_queries(const Params &p, int tile)
{
    const int c = threadIdx.x & 15, rg = threadIdx.x >> 4;
    const int t0 = tile * kQTokens, token = t0 + (rg & (kQTokens - 1));
    int s = last_not_above(p.S, t0, [&](int i) { return start_of(p, i); });
    while (s + 1 < p.S && start_of(p, s + 1) <= token) ++s;
    const bool mine = s >= 0 && token < start_of(p, s + 1);
    Turn turn;
    if (p.rope && mine) {
        const long long pos = (long long)p.seq_lens[s] + (token - start_of(p, s));
        const int at = (int)min(max(pos, 0ll), (long long)p.rope_rows - 1);
        if (at != pos && p.status) atomicOr(p.status, svk::kStatusIndex);
        if (8 * c < p.rot) turn = load_turn<kNeighbours>(p.rope + (size_t)at * p.rot, c, p.rot);
    }
    constexpr int kStep = kRowGroups / kQTokens, kAhead = kQTokens == kTokensOfFew ? 4 : 8;
    for (int h0 = rg / kQTokens; h0 < p.Hq; h0 += kStep * kAhead) {   // (uniform over a warp: rotate exchanges between lanes)
        uint4 x[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            x[i] = mine && h0 + kStep * i < p.Hq ? p.q[token * p.q_stride + (h0 + kStep * i) * 16 + c] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (p.rope) x[i] = rotate<kNeighbours>(x[i], turn, c, p.rot);
            if (mine && h0 + kStep * i < p.Hq) p.q_out[((size_t)token * p.Hq + h0 + kStep * i) * 16 + c] = x[i];
        }
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

extern "C" sv_status sv_rope_append(const sv_geom *geom, void *k_pool, void *v_pool, int32_t n_pages, const int32_t *block_table,
                                    const int32_t *seq_lens, const void *q, const void *k, const void *v, int64_t q_stride, int64_t k_stride,
                                    int64_t v_stride, const int32_t *q_start, int32_t n_tokens, const float *rope, int32_t rope_rows,
                                    int32_t rot_dim, int32_t interleaved, void *q_out, int32_t *seq_lens_out, float *reps,
                                    int32_t *status_word, void *stream)
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
    p.block_table = block_table, p.seq_lens = seq_lens, p.q_start = q_start;
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
