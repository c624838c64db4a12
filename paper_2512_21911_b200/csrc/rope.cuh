// Rotary positions: what the kernels that append new tokens to a cache share.  16 threads hold a 256-byte row, so that the partner of a dim
// is in the same thread (neighbours) or 2 to 8 lanes away (halves).
#pragma once
#include <cuda_bf16.h>
#include <stdint.h>

#include "attn_common.cuh"
#include "sv_ptx.cuh"

namespace svrope {

constexpr int kThreads = 256;
constexpr int kRowGroups = kThreads / 16;
// Tokens of a CTA that rotates queries: two in calls of up to kFew tokens, where the query CTAs of many would not fill the machine and a
// CTA's own chain of loads is what counts; many beyond, where reading the batch's starts and lengths is shared by more rows.  With two and
// with eight tokens: 64 sequences of one token 6.8 and 9.2 us; chunks of four sequences, 256 tokens in all 5.1 and 6.0, 1,024 7.3 and 9.1,
// 1,536 11.5 either way, 2,048 14.9 and 15.7, 4,096 26.4 and 24.9; a prompt of 32,768 195 and 168.  512, 1,024 and 2,048 sequences of one
// token each: 43 and 47, 86 and 89, 191 and 190.  The edge is not sharp: the two cross between 1,536 and 4,096 tokens.
constexpr int kFew = 1024, kTokensOfFew = 2, kTokensOfMany = 8;

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

template <class Params>
__device__ __forceinline__ int start_of(const Params &p, int s) { return min(max(__ldg(p.q_start + s), 0), p.N); }

// The last sequence s whose number (of ascending ones) is not above x; all threads of the CTA.
template <class F>
__device__ __forceinline__ int last_not_above(int S, int x, F number)
{
    int n = 0;
    for (int base = 0; base < S; base += kThreads) n += __syncthreads_count(base + (int)threadIdx.x < S && number(base + threadIdx.x) <= x);
    return n - 1;
}

// The blocks that sequence s enters are at most n / B + 2, so that numbering them from q_start[s] / B + 2 s gives every sequence room of
// its own, and a CTA finds its sequence by counting the starts up to its number instead of by a prefix sum.
struct Grown {
    int s, first;            // sequence, its first row of the batch
    int before;              // tokens that it held
    int block, end, page;    // the block, the position behind its last token, its page
};
// The block of this number, by all threads of the CTA; false: there is none, or no room for it.  Head 0 of a sequence's first block writes
// its new length.
template <int B, class Params>
__device__ __forceinline__ bool grown_block(const Params &p, int slot, int h, Grown &g)
{
    const int tid = threadIdx.x;
    const int s = last_not_above(p.S, slot, [&](int i) { return start_of(p, i) / B + 2 * i; });
    if (s < 0) return false;
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
    if (L < 0 || n_all == 0 || b >= p.NBmax || (long long)b * B >= (long long)L + n_all || room(b) <= b) return false;
    g = {s, first, L, b, (int)min((long long)L + n_all, (long long)(b + 1) * B), pages[b]};
    return true;
}

// Query heads of kQTokens tokens: a token's heads are dealt to kStep groups of 16 threads; a thread has kAhead of them on their way at
// once and keeps its part of the token's table row for all of them.
template <bool kNeighbours, int kQTokens, class Params>
__device__ __forceinline__ void turn_queries(const Params &p, int tile)
{
    const int c = threadIdx.x & 15, rg = threadIdx.x >> 4;
    const int t0 = tile * kQTokens, token = t0 + (rg & (kQTokens - 1));
    int s = last_not_above(p.S, t0, [&](int i) { return start_of(p, i); });
    while (s + 1 < p.S && start_of(p, s + 1) <= token) ++s;
    const bool mine = s >= 0 && token < start_of(p, s + 1);
    Turn turn;
    if (p.rope && mine) {
        const long long pos = (long long)(p.positions ? p.positions[s] : p.seq_lens[s]) + (token - start_of(p, s));
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

}  // namespace svrope
