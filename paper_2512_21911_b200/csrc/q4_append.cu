// sv_rope_append_q4, sv_kv_append_q4, sv_kv_read_q4: rows of keys and values into a paged cache held in 4 bits (q4.cuh), and back.
//
// Mathematics: the rotation of sv_rope_append; a row's two groups of 64 values as scale, offset and codes; the representatives are the means
// of what the cache then holds.  A prompt of 16,384 tokens (32 query heads, 8 KV heads; 450 MB) takes 154 us with its reading back, 45 % of a
// copy's rate: neither HBM (28 %) nor the issue slots (63 %) is full, a slab's loads, coding and turn come one behind the other.  A token each of 64
// sequences takes 20 us, a chain of loads and of the coding's steps.
//
// A CTA has a block of a sequence and a KV head, as in sv_rope_append: 16 threads hold a row, eight of them a group, so that its smallest
// and largest value are three shuffles away and a thread's eight codes are one word.  The keys' words go to the page as they are; those of
// the values, which the cache holds by dim, turn in shared memory, and join the nibbles of the tokens that were there.  No other CTA
// writes to the block, so nothing is atomic.
#include <cuda_bf16.h>

#include <type_traits>

#include "attn_common.cuh"
#include "q4.cuh"
#include "rope.cuh"
#include "sv_host.h"
#include "sv_ptx.cuh"

namespace {

using namespace svrope;
using svq::kSlabBytes;

struct Params {
    uint8_t *pool;
    const int32_t *block_table, *seq_lens, *q_start;
    const int32_t *positions;   // (null: seq_lens)
    const uint4 *q, *k, *v;
    long long q_stride, k_stride, v_stride;   // 16-byte chunks between tokens
    const float *rope;
    uint4 *q_out;
    int32_t *seq_lens_out;
    float *reps;
    int32_t *status;
    int S, N, Hq, Hkv, NBmax, n_pages, rope_rows, rot;
    int slots;   // CTAs of the first kind: slots x Hkv
    // of a commit: rows s * T + accept_idx[s][i]
    const int32_t *accept_idx, *n_accept;
    int T, max_accept;
};

__device__ __forceinline__ int shift_of(int e) { return 4 * (e & 1 ? 4 + e / 2 : e / 2); }   // where code e of eight lies in a word

// Eight values of a group (the 16 threads of a row, all of them): their codes as a word; scale and offset, low and high half.
__device__ __forceinline__ uint32_t code_row(uint4 x, uint32_t &scale)
{
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    float v[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = halves_of(w[i]);
        v[2 * i] = f.x, v[2 * i + 1] = f.y;
    }
    float low = v[0], high = v[0];
    bool odd = false;   // a NaN or an infinite value, which the extrema may lose
#pragma unroll
    for (int i = 0; i < 4; ++i) odd |= (w[i] & 0x7f80u) == 0x7f80u || (w[i] & 0x7f800000u) == 0x7f800000u;
#pragma unroll
    for (int i = 1; i < 8; ++i) low = svq::lesser(low, v[i]), high = svq::greater(high, v[i]);
#pragma unroll
    for (int d = 1; d < 8; d <<= 1)
        low = svq::lesser(low, __shfl_xor_sync(0xffffffffu, low, d)), high = svq::greater(high, __shfl_xor_sync(0xffffffffu, high, d));
    odd = __ballot_sync(0xffffffffu, odd) >> (threadIdx.x & 24) & 0xffu;
    svq::Scale s = svq::scale_of(low, high);
    if (odd) s.d = s.m = __ushort_as_bfloat16(0x7fff);
    scale = (uint32_t)__bfloat16_as_ushort(s.d) | (uint32_t)__bfloat16_as_ushort(s.m) << 16;
    const float d = __bfloat162float(s.d), m = __bfloat162float(s.m);
    return svq::codes_of(v, d, m);
}

// Tokens [before, end) of block b of a KV head, from rows k_row(t), v_row(t) of this thread's chunk; the block's mean.
template <int B, bool kNeighbours, class Row>
__device__ __forceinline__ void append_block(const Params &p, int s, int h, int b, int before, int end, int page, Row row)
{
    __shared__ float part[kRowGroups][128];
    __shared__ uint32_t codes[64][17];   // of a slab's values (a row and a word: no two threads of a warp in one bank)
    const int tid = threadIdx.x, c = tid & 15, rg = tid >> 4, group = c >> 3, dim = tid & 127;
    constexpr int kIter = 64 / kRowGroups, kSlabs = B / 64;
    const int r0 = max(before - b * B, 0), r1 = end - b * B;   // rows of the block that are new
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    // (slab by slab: the rows of 128 tokens in registers leave an SM one CTA, and a prompt of 16 K tokens in blocks of 128 takes 306 us
    // instead of 161, 64 single tokens 44 instead of 32)
#pragma unroll 1
    for (int j = 0; j < kSlabs; ++j) {
        const int first = j * 64;
        if (first >= r1) break;
        if (first + 64 <= r0 && !p.reps) continue;
        uint8_t *const slab = p.pool + (((size_t)page * p.Hkv + h) * kSlabs + j) * kSlabBytes;
        const auto key_word = [&](int r) { return reinterpret_cast<uint32_t *>(slab + (c >> 2) * 1024 + (r - first) * 16 + (c & 3) * 4); };
        const auto key_scale = [&](int r) { return reinterpret_cast<uint32_t *>(slab + svq::kOffKScale + (r - first) * 8 + group * 4); };
        // the values' words of this thread's dim and 32 tokens, some of whose nibbles may stay
        uint4 *const value_words = reinterpret_cast<uint4 *>(slab + svq::kOffV + (tid >> 7) * 2048 + dim * 16);
        const int t0 = first + (tid >> 7) * 32;
        const bool touched = t0 < r1 && t0 + 32 > r0;
        uint4 held = make_uint4(0u, 0u, 0u, 0u), k[kIter], v[kIter];
        uint32_t old_word[kIter], old_scale[kIter];
#pragma unroll
        for (int i = 0; i < kIter; ++i) {
            const int r = first + rg + i * kRowGroups;
            k[i] = v[i] = make_uint4(0u, 0u, 0u, 0u);
            old_word[i] = old_scale[i] = 0u;
            if (r < r0) {
                if (p.reps) old_word[i] = *key_word(r), old_scale[i] = *key_scale(r);
            } else if (r < r1) {
                row(b * B + r, k[i], v[i]);
            }
        }
        if (touched && (t0 < r0 || t0 + 32 > r1)) held = *value_words;
#pragma unroll
        for (int i = 0; i < kIter; ++i) {
            const int r = first + rg + i * kRowGroups;
            const bool fresh = r >= r0 && r < r1;
            if (__any_sync(0xffffffffu, fresh)) {
                if (p.rope) {
                    const int t = b * B + r, at = min(max(t, 0), p.rope_rows - 1);
                    Turn turn;
                    if (8 * c < p.rot) turn = load_turn<kNeighbours>(p.rope + (size_t)at * p.rot, c, p.rot);
                    k[i] = rotate<kNeighbours>(k[i], turn, c, p.rot);
                    if (fresh && t >= p.rope_rows && p.status) atomicOr(p.status, svk::kStatusIndex);
                }
                uint32_t ks, vs;
                const uint32_t kw = code_row(k[i], ks), vw = code_row(v[i], vs);
                if (fresh) {
                    old_word[i] = kw, old_scale[i] = ks;
                    *key_word(r) = kw;
                    codes[r - first][c] = vw;
                    if ((c & 7) == 0) {
                        *key_scale(r) = ks;
                        unsigned short *const to = reinterpret_cast<unsigned short *>(slab + svq::kOffVScale) + group * 128 + (r - first);
                        to[0] = (unsigned short)vs, to[64] = (unsigned short)(vs >> 16);
                    }
                }
            }
            if (r < r1) {
                uint32_t x[4];
                svq::decode(old_word[i], svq::both_low(old_scale[i]), svq::both_high(old_scale[i]), x);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 f = halves_of(x[e]);
                    acc[2 * e] += f.x, acc[2 * e + 1] += f.y;
                }
            }
        }
        __syncthreads();
        if (touched) {
            uint32_t w[4] = {held.x, held.y, held.z, held.w};
#pragma unroll
            for (int e = 0; e < 32; ++e) {
                const int r = t0 + e;
                if (r < r0 || r >= r1) continue;
                const uint32_t nibble = codes[r - first][dim >> 3] >> shift_of(dim & 7) & 15u;
                const int at = 4 * (e & 1 ? 4 + (e & 7) / 2 : (e & 7) / 2);
                w[e >> 3] = (w[e >> 3] & ~(15u << at)) | nibble << at;
            }
            *value_words = make_uint4(w[0], w[1], w[2], w[3]);
        }
        if (j + 1 < kSlabs) __syncthreads();   // (the codes have been read)
    }
    if (!p.reps) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) part[rg][c * 8 + e] = acc[e];
    __syncthreads();
    if (tid < 128) {
        float sum = 0.f;
#pragma unroll
        for (int g = 0; g < kRowGroups; ++g) sum += part[g][tid];
        p.reps[(((size_t)s * p.Hkv + h) * p.NBmax + b) * 128 + tid] = sum / (float)r1;
    }
}

// Three CTAs an SM: with two a prompt of 16 K tokens takes 175 us instead of 159 (alone, its reading back included).
template <int B, bool kNeighbours, int kQTokens>
__global__ void __launch_bounds__(kThreads, 3) q4_rope_append_kernel(const __grid_constant__ Params p)
{
    svk::grid_dependency_wait();
    svk::grid_launch_dependents();
    const int i = blockIdx.x, cache = p.slots * p.Hkv;
    if (i >= cache) return turn_queries<kNeighbours, kQTokens>(p, i - cache);
    const int h = i % p.Hkv, c = threadIdx.x & 15;
    Grown g;
    if (!grown_block<B>(p, i / p.Hkv, h, g)) return;
    append_block<B, kNeighbours>(p, g.s, h, g.block, g.before, g.end, g.page, [&](int t, uint4 &k, uint4 &v) {
        const long long row = g.first + (t - g.before);
        k = __ldg(p.k + row * p.k_stride + h * 16 + c), v = __ldg(p.v + row * p.v_stride + h * 16 + c);
    });
}

// A CTA per KV head, sequence and block of the two that at most 64 tokens can enter.
template <int B>
__global__ void __launch_bounds__(kThreads) q4_commit_kernel(const __grid_constant__ Params p)
{
    svk::grid_dependency_wait();
    svk::grid_launch_dependents();
    const int h = blockIdx.x, s = blockIdx.y, c = threadIdx.x & 15;
    const int L = p.seq_lens[s], b0 = max(L, 0) / B, b = b0 + blockIdx.z;
    const int *pages = p.block_table + (size_t)s * p.NBmax;
    const int page0 = b0 < p.NBmax ? pages[b0] : -1, page1 = b0 + 1 < p.NBmax ? pages[b0 + 1] : -1;
    int n = min(max(p.n_accept[s], 0), p.max_accept);
    n = L < 0 ? 0 : (int)max(0ll, min((long long)n, (long long)p.NBmax * B - L));
    // (a block whose entry is not a page of the pool ends the table)
    if ((unsigned)page0 >= (unsigned)p.n_pages) n = 0;
    if ((unsigned)page1 >= (unsigned)p.n_pages) n = min(n, (b0 + 1) * B - L);
    if (h == 0 && blockIdx.z == 0 && threadIdx.x == 0) p.seq_lens_out[s] = L + n;
    const int end = min(L + n, (b + 1) * B);
    if (n <= 0 || b * B >= end) return;
    append_block<B, false>(p, s, h, b, L, end, blockIdx.z ? page1 : page0, [&](int t, uint4 &k, uint4 &v) {
        const int j = min(max(p.accept_idx[(size_t)s * p.max_accept + (t - L)], 0), p.T - 1);
        const size_t at = (((size_t)s * p.T + j) * p.Hkv + h) * 16 + c;
        k = __ldg(p.k + at), v = __ldg(p.v + at);
    });
}

// A slab in shared memory, in 16-byte pieces, with gaps: a row's 16 threads read words that are 128 bytes apart (values) or 1024 (keys), and find
// them in different banks.  A word of values is read for four of its tokens.  (With neither a verification over 40
// blocks of four sequences takes 64 us instead of 48, 1,024 tokens over a cache of 30 K 552 instead of 509.)
constexpr int kValues = 264, kScales = kValues + 288, kPieces = kScales + 64;
__device__ __forceinline__ void fetch_slab(const uint4 *from, uint4 *slab)
{
    static_assert(kThreads == 256 && svq::kOffV == 256 * 16 && svq::kOffKScale == 512 * 16, "");
    const int tid = threadIdx.x;
    slab[tid + (tid >> 6) * 2] = __ldg(from + tid);                // keys: two pieces behind each chunk
    slab[kValues + tid + (tid >> 3)] = __ldg(from + 256 + tid);    // values: one behind each eight dims
    if (tid < 64) slab[kScales + tid] = __ldg(from + 512 + tid);
}
// Rows of eight dims, by key(token, eight dims, values) and value(...).  All threads of the CTA.
template <class Key, class Value>
__device__ __forceinline__ void decode_slab(const uint4 *slab, Key key, Value value)
{
    const int tid = threadIdx.x, c = tid & 15;
    const uint32_t *const words = reinterpret_cast<const uint32_t *>(slab);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = (tid >> 4) + 16 * i;
        const uint32_t sc = words[kScales * 4 + r * 2 + (c >> 3)];
        uint32_t x[4];
        svq::decode(words[(c >> 2) * 264 + r * 4 + (c & 3)], svq::both_low(sc), svq::both_high(sc), x);
        key(r, c, make_uint4(x[0], x[1], x[2], x[3]));
    }
    // four tokens of eight words: codes 2 j, 2 j + 1 of eight in nibble j of the halves of a word
    const int part = tid >> 4 & 1, o = tid >> 5, r = 8 * o + 4 * part;
    const uint2 *const scales = reinterpret_cast<const uint2 *>(slab + kScales + 32) + (c >> 3) * 32 + r / 4;
    const uint2 d = scales[0], m = scales[16];
    const uint32_t *const w = words + (kValues + (o >> 2) * 144 + c * 9) * 4 + (o & 3);
    uint32_t x[4][4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t a = w[8 * e] >> (8 * part), b = w[8 * e + 4] >> (8 * part);
        const uint32_t even = __byte_perm(a, b, 0x5410), odd = __byte_perm(a, b, 0x7632);
        x[0][e] = svq::fma_bf16x2(svq::steps<0>(even), svq::both_low(d.x), svq::both_low(m.x));
        x[1][e] = svq::fma_bf16x2(svq::steps<0>(odd), svq::both_high(d.x), svq::both_high(m.x));
        x[2][e] = svq::fma_bf16x2(svq::steps<1>(even), svq::both_low(d.y), svq::both_low(m.y));
        x[3][e] = svq::fma_bf16x2(svq::steps<1>(odd), svq::both_high(d.y), svq::both_high(m.y));
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) value(r + t, c, make_uint4(x[t][0], x[t][1], x[t][2], x[t][3]));
}

// Tokens back: row i of sequence s is the token at first[s] + i.  A CTA has a slab of them and a KV head.
__global__ void __launch_bounds__(kThreads) q4_read_kernel(const uint8_t *pool, const int32_t *block_table, const int32_t *seq_lens,
                                                           const int32_t *first, const int32_t *q_start, uint4 *k_out, uint4 *v_out, int S,
                                                           int N, int Hkv, int NBmax, int B, int n_pages, int32_t *status)
{
    __shared__ uint4 slab[kPieces];
    svk::grid_dependency_wait();
    svk::grid_launch_dependents();
    const int tid = threadIdx.x, h = blockIdx.y, slot = blockIdx.x;
    const struct { const int32_t *q_start; int N; } batch = {q_start, N};
    const int s = last_not_above(S, slot, [&](int i) { return start_of(batch, i) / 64 + 2 * i; });
    if (s < 0) return;
    const int row0 = start_of(batch, s), n = max(0, start_of(batch, s + 1) - row0);
    const long long at = first[s];
    const long long len = min((long long)max(seq_lens[s], 0), (long long)NBmax * B);
    // (floor division: a token before the first is nobody's, as is one behind the last)
    const long long j0 = at >= 0 ? at / 64 : -((63 - at) / 64), j = j0 + slot - (row0 / 64 + 2 * s);
    const long long t0 = max(j * 64, at), t1 = min((j + 1) * 64, at + n);   // tokens of this CTA
    if (t0 >= t1) return;
    const bool there = j >= 0 && j * 64 < len;
    bool bad = t0 < 0 || t1 > len;
    if (there) {
        const int b = (int)(j * 64 / B);
        int page = __ldg(block_table + (size_t)s * NBmax + b);
        bad = bad || (unsigned)page >= (unsigned)n_pages;
        page = min(max(page, 0), n_pages - 1);
        fetch_slab(reinterpret_cast<const uint4 *>(pool + (((size_t)page * Hkv + h) * (B / 64) + (j * 64 % B) / 64) * kSlabBytes), slab);
    }
    if (bad && tid == 0 && status) atomicOr(status, svk::kStatusIndex);
    __syncthreads();
    const auto put = [&](uint4 *out, int r, int c, uint4 x) {   // (of positions that the sequence does not hold: zeros)
        const long long t = j * 64 + r;
        if (t >= t0 && t < t1) out[((size_t)(row0 + (t - at)) * Hkv + h) * 16 + c] = there && t >= 0 && t < len ? x : make_uint4(0u, 0u, 0u, 0u);
    };
    decode_slab(slab, [&](int r, int c, uint4 x) { put(k_out, r, c, x); }, [&](int r, int c, uint4 x) { put(v_out, r, c, x); });
}

// The cache of a batch, or its listed blocks, as bfloat16 pages, block b of sequence s on page s * NBmax + b, and the table that says so: where there are many
// query rows, whose attention is bound by its products, decoding every key once is cheaper than once for every 64 of them (q4_attn.cu).
// A CTA has a slab; bound by HBM (144 bytes read and 512 written a token and head).
__global__ void __launch_bounds__(kThreads) q4_spread_kernel(const uint8_t *pool, const int32_t *block_table, const int32_t *seq_lens, const int32_t *sel_idx, const int32_t *sel_cnt,
                                                             int max_sel, uint4 *k_out, uint4 *v_out, int32_t *table_out, int Hkv, int NBmax, int B, int n_pages,
                                                             int32_t *status)
{
    __shared__ uint4 slab[kPieces];
    svk::grid_dependency_wait();
    svk::grid_launch_dependents();
    const int tid = threadIdx.x, per = B / 64, h = blockIdx.y, s = blockIdx.z, sub = blockIdx.x % per;
    int b = blockIdx.x / per;
    if (sel_idx) {   // a listed block; the table in turns
        for (int i = blockIdx.x * kThreads + tid; i < NBmax && h == 0; i += gridDim.x * kThreads) table_out[(size_t)s * NBmax + i] = (int32_t)((size_t)s * NBmax + i);
        if (b >= min(__ldg(sel_cnt + s * Hkv + h), max_sel)) return;
        b = __ldg(sel_idx + ((size_t)s * Hkv + h) * max_sel + b);
        b = min(max(b, 0), NBmax - 1);   // (the attention, which clamps it as well, says so)
    } else if (h == 0 && sub == 0 && tid == 0) {
        table_out[(size_t)s * NBmax + b] = (int32_t)((size_t)s * NBmax + b);
    }
    const size_t entry = (size_t)s * NBmax + b;
    if ((long long)b * B + sub * 64 >= min((long long)max(seq_lens[s], 0), (long long)NBmax * B)) return;
    int page = __ldg(block_table + entry);
    if ((unsigned)page >= (unsigned)n_pages) {
        if (tid == 0 && status) atomicOr(status, svk::kStatusIndex);
        page = min(max(page, 0), n_pages - 1);
    }
    const uint4 *from = reinterpret_cast<const uint4 *>(pool + (((size_t)page * Hkv + h) * per + sub) * kSlabBytes);
    fetch_slab(from, slab);
    __syncthreads();
    const size_t row0 = (entry * Hkv + h) * B + sub * 64;
    decode_slab(slab, [&](int r, int c, uint4 x) { k_out[(row0 + r) * 16 + c] = x; }, [&](int r, int c, uint4 x) { v_out[(row0 + r) * 16 + c] = x; });
}

cudaLaunchConfig_t config(dim3 grid, void *stream, cudaLaunchAttribute *attr)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(kThreads);
    cfg.stream = static_cast<cudaStream_t>(stream);
    svh::pdl_attribute(attr);
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cfg;
}

}  // namespace

sv_status svh::spread_q4(const sv_geom *geom, const sv_kv_q4 *kv, const int32_t *sel_idx, const int32_t *sel_cnt, int32_t max_sel, void *k_out, void *v_out,
                         int32_t *table_out, int32_t *status_word, void *stream)
{
    cudaLaunchAttribute attr[1];
    const int blocks = sel_idx ? max_sel : geom->max_blocks;
    const cudaLaunchConfig_t cfg = config(dim3((unsigned)(blocks * (geom->block_size / 64)), geom->n_kv_heads, geom->n_seq), stream, attr);
    const cudaError_t e = cudaLaunchKernelEx(&cfg, q4_spread_kernel, static_cast<const uint8_t *>(kv->pool), kv->block_table, kv->seq_lens, sel_idx, sel_cnt,
                                             (int)max_sel, static_cast<uint4 *>(k_out), static_cast<uint4 *>(v_out), table_out, (int)geom->n_kv_heads,
                                             (int)geom->max_blocks, (int)geom->block_size, (int)kv->n_pages, status_word);
    return e == cudaSuccess ? SV_OK : SV_ERR_CUDA;
}

extern "C" sv_status sv_rope_append_q4(const sv_geom *geom, void *pool, int32_t n_pages, const int32_t *block_table, const int32_t *seq_lens,
                                       const void *q, const void *k, const void *v, int64_t q_stride, int64_t k_stride, int64_t v_stride,
                                       const int32_t *q_start, int32_t n_tokens, const float *rope, int32_t rope_rows, int32_t rot_dim,
                                       int32_t interleaved, void *q_out, int32_t *seq_lens_out, float *reps, int32_t *status_word, void *stream)
{
    const sv_status st = svh::check_ragged(geom, n_tokens);
    if (st != SV_OK) return st;
    const int Hq = geom->n_q_heads, Hkv = geom->n_kv_heads, B = geom->block_size;
    if (!pool || !block_table || !seq_lens || !q_start || !seq_lens_out || (n_tokens > 0 && (!k || !v)) || (!q) != (!q_out)) return SV_ERR_NULL;
    if (n_pages < 1 || (int64_t)n_pages * Hkv * B >= (int64_t)1 << 31) return SV_ERR_SHAPE;
    if (seq_lens_out == seq_lens) return SV_ERR_SHAPE;   // other CTAs still read the old length
    if (rope && (rope_rows < 1 || rot_dim < 16 || rot_dim > svh::kHeadDim || rot_dim % 16)) return SV_ERR_SHAPE;
    if (n_tokens > 1 && (k_stride < (int64_t)Hkv * svh::kHeadDim || v_stride < (int64_t)Hkv * svh::kHeadDim ||
                         (q && q_stride < (int64_t)Hq * svh::kHeadDim)))
        return SV_ERR_SHAPE;
    // (a row of q_out is written by a CTA that reads other rows of q: in place only where both have the same layout)
    if (q && q_out == q && n_tokens > 1 && q_stride != (int64_t)Hq * svh::kHeadDim) return SV_ERR_SHAPE;
    if (n_tokens > 1 && (q_stride % 8 || k_stride % 8 || v_stride % 8)) return SV_ERR_ALIGN;
    if (!svh::aligned(pool, 128) || !svh::aligned(q, 16) || !svh::aligned(k, 16) || !svh::aligned(v, 16) || !svh::aligned(q_out, 16) ||
        !svh::aligned(rope, 16) || !svh::aligned(reps, 16))
        return SV_ERR_ALIGN;
    Params p = {};
    p.pool = static_cast<uint8_t *>(pool);
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
    cudaLaunchAttribute attr[1];
    const cudaLaunchConfig_t cfg = config(dim3((unsigned)ctas), stream, attr);
    const auto pick = [&](auto block, auto turned) {
        return tokens == kTokensOfFew ? q4_rope_append_kernel<decltype(block)::value, decltype(turned)::value, kTokensOfFew>
                                      : q4_rope_append_kernel<decltype(block)::value, decltype(turned)::value, kTokensOfMany>;
    };
    const auto by_order = [&](auto block) { return interleaved ? pick(block, std::true_type{}) : pick(block, std::false_type{}); };
    const auto kernel = B == 64 ? by_order(std::integral_constant<int, 64>{}) : by_order(std::integral_constant<int, 128>{});
    return cudaLaunchKernelEx(&cfg, kernel, p) == cudaSuccess ? svh::launch_status() : SV_ERR_CUDA;
}

extern "C" sv_status sv_kv_append_q4(const sv_geom *geom, void *pool, int32_t n_pages, const int32_t *block_table, const int32_t *seq_lens,
                                     const void *draft_k, const void *draft_v, const int32_t *accept_idx, const int32_t *n_accept,
                                     int32_t max_accept, int32_t *seq_lens_out, float *reps, void *stream)
{
    const sv_status st = svh::check_geom(geom);
    if (st != SV_OK) return st;
    if (!pool || !block_table || !seq_lens || !draft_k || !draft_v || !accept_idx || !n_accept || !seq_lens_out) return SV_ERR_NULL;
    if (n_pages < 1 || (int64_t)n_pages * geom->n_kv_heads * geom->block_size >= (int64_t)1 << 31) return SV_ERR_SHAPE;
    if ((int64_t)geom->max_blocks * geom->block_size >= (int64_t)1 << 31) return SV_ERR_SHAPE;
    if (max_accept < 1 || max_accept > geom->n_draft || seq_lens_out == seq_lens) return SV_ERR_SHAPE;
    if (!svh::aligned(pool, 128) || !svh::aligned(draft_k, 16) || !svh::aligned(draft_v, 16) || !svh::aligned(reps, 16)) return SV_ERR_ALIGN;
    Params p = {};
    p.pool = static_cast<uint8_t *>(pool), p.block_table = block_table, p.seq_lens = seq_lens;
    p.k = static_cast<const uint4 *>(draft_k), p.v = static_cast<const uint4 *>(draft_v);
    p.accept_idx = accept_idx, p.n_accept = n_accept, p.max_accept = max_accept, p.T = geom->n_draft;
    p.seq_lens_out = seq_lens_out, p.reps = reps;
    p.S = geom->n_seq, p.Hkv = geom->n_kv_heads, p.NBmax = geom->max_blocks, p.n_pages = n_pages;
    cudaLaunchAttribute attr[1];
    const cudaLaunchConfig_t cfg = config(dim3(p.Hkv, p.S, 2), stream, attr);
    const auto kernel = geom->block_size == 64 ? q4_commit_kernel<64> : q4_commit_kernel<128>;
    return cudaLaunchKernelEx(&cfg, kernel, p) == cudaSuccess ? svh::launch_status() : SV_ERR_CUDA;
}

extern "C" sv_status sv_kv_read_q4(const sv_geom *geom, const sv_kv_q4 *kv, const int32_t *first, const int32_t *q_start, int32_t n_tokens,
                                   void *k_out, void *v_out, int32_t *status_word, void *stream)
{
    const sv_status st = svh::check_ragged(geom, n_tokens);
    if (st != SV_OK) return st;
    if (!kv || !kv->pool || !kv->block_table || !kv->seq_lens || !first || !q_start || (n_tokens > 0 && (!k_out || !v_out))) return SV_ERR_NULL;
    if (kv->n_pages < 1 || (int64_t)kv->n_pages * geom->n_kv_heads * geom->block_size >= (int64_t)1 << 31) return SV_ERR_SHAPE;
    if (!svh::aligned(kv->pool, 128) || !svh::aligned(k_out, 16) || !svh::aligned(v_out, 16)) return SV_ERR_ALIGN;
    if (n_tokens == 0) return SV_OK;
    cudaLaunchAttribute attr[1];
    const cudaLaunchConfig_t cfg = config(dim3((unsigned)(n_tokens / 64 + 2 * geom->n_seq), geom->n_kv_heads), stream, attr);
    const cudaError_t e = cudaLaunchKernelEx(&cfg, q4_read_kernel, static_cast<const uint8_t *>(kv->pool), kv->block_table, kv->seq_lens, first, q_start,
                                             static_cast<uint4 *>(k_out), static_cast<uint4 *>(v_out), (int)geom->n_seq, (int)n_tokens,
                                             (int)geom->n_kv_heads, (int)geom->max_blocks, (int)geom->block_size, (int)kv->n_pages, status_word);
    return e == cudaSuccess ? svh::launch_status() : SV_ERR_CUDA;
}
