// sv_verify_attn_q4, sv_chunk_attn_q4: attention over a paged cache held in 4 bits (q4.cuh), of draft tokens over kept blocks and their
// own keys, or of a ragged batch of new tokens over the cache that holds them.
//
// Mathematics, for a row q and the keys t that it sees: s_t = q . k_t * scale * log2 e, a reference m not far below the running maximum,
// l = sum 2^(s_t - m), o = sum 2^(s_t - m) v_t; the output is o / l.  When the maximum outgrows the reference by more than 24, m moves and
// l and o are multiplied by 2^(old - new).
//
// A quarter of the bytes of a bfloat16 cache, but every value has to be decoded: what counts is instructions per value and that decoded
// values go nowhere but to the tensor cores.  So the cache is operand A, read from tensor memory, and the roles of rows and keys are
// exchanged: both products are of 128 (keys, then dims) x N (query rows) with N = 16, 32 or 64,
//   S^T[128 keys x N] = K . Q^T      a thread decodes a key's 128 dims into its lane of tensor memory
//   O^T[128 dims x N] += V^T . P^T   a warp decodes 32 dims' 128 keys, a thread four dims and four keys of every 16
// and a few query rows cost what they are instead of a tile of 128.  A thread then has a key's scores against all rows: masks are its own
// affair, sums of weights stay in registers until the end, and the running maximum, which would have to go across lanes, is only
// looked for when a score outgrows the reference.
//
// A worker is a warpgroup that decodes and does the softmax, and a warp that copies and issues its products; it has everything to itself --
// a ring of slabs filled by bulk copies (one of 9216 bytes for 64 tokens, no tensor maps), queries, P, tensor memory -- and takes a share of
// the batch (q4_shares.h), so that workers never wait for one another: while one waits for a product the others decode.  An item that is
// cut is written as partial sums and merged by a second kernel.
//
// Eight sequences of 16 K to 131 K tokens, five draft tokens each (20 rows a KV head, 790 MB): 263 us, 46 % of a copy's rate; bound by a worker's
// chain of decoding, products and softmax (two thirds of the issue slots).  One token over 4 K tokens of a small model: 20 us, latency.
#include <cuda_bf16.h>
#include <stddef.h>

#include <algorithm>

#include "attn_common.cuh"
#include "q4.cuh"
#include "shares.cuh"
#include "sv_host.h"
#include "sv_ptx.cuh"

namespace {

using namespace svk;
using svq::kSlabBytes;
using svq::kUnit;

// What a score may exceed its reference by (log2).  Weights up to 2^24 cost no precision (o / l does not depend on the reference, and bf16 and
// fp32 have the same exponents), and a reference that moves costs as much as a unit.
constexpr float kLag = 24.f;
// Query rows of a sequence and KV head, on average, beyond which the cache is decoded first.  Both ways with nothing in L2, here and decoded first: 64 blocks of a
// 32 K sequence, 68 rows 33 and 18 us, 256 rows 49 and 22; 256 blocks 55 and 33, 90 and 44; all of 4 K tokens 33 and 17, 49 and 21.  One tile of rows
// is where measuring began: at 64 rows over 64 blocks 38 us here, and decoding (3.6) and the attention of its pages (13.5) are less, too.
constexpr int kSpreadRows = 64;

struct Params {
    const uint8_t *pool;
    const int32_t *block_table, *seq_lens, *sel_idx, *sel_cnt, *q_start, *parent;
    const __nv_bfloat16 *q, *draft_k, *draft_v;
    __nv_bfloat16 *out;
    float *lse;
    float *ws_o;     // [2 * workers][N][128]: of a worker, the part of an item that began before and of one that goes on behind
    float2 *ws_ml;   // [2 * workers][N]
    int4 *cuts;      // [workers][2] the cut item that begins in a worker's share: first token, first row, KV head and rows, parts (0: none); rows without a key
    int32_t *status;
    int S, Hq, Hkv, G, T, n_tokens, B, NBmax, n_pages, max_sel;
    float scale_log2;
};

// Sizes that follow from the rows of a tile.
template <int N>
struct Form {
    static constexpr int kWorkers = N == 64 ? 2 : 4;             // of a CTA
    static constexpr int kThreads = kWorkers * 128 + 128;        // (a warp of the last four for each worker)
    static constexpr int kStages = N == 64 ? 4 : 2;              // units of a worker's ring
    static constexpr int kUnitBytes = 2 * kSlabBytes;
    static constexpr int kQBytes = N * 256;                      // [2 halves of the dims][N rows][128 bytes]
    static constexpr int kPTile = 128 * 128;                     // [128 keys][128 bytes], of which N * 2 are one worker's
    static constexpr int kSharers = 64 / N < kWorkers ? 64 / N : kWorkers;
    static constexpr int kOffQ = 0;
    static constexpr int kOffP = kWorkers * kQBytes;
    static constexpr int kOffRing = kOffP + kWorkers / kSharers * kPTile;
    static constexpr int kOffMisc = kOffRing + kWorkers * kStages * kUnitBytes;
    // per worker: reference, its negative where there is one, factors, maxima and sums of four warps, row masks; barriers; tokens of the
    // slabs in the ring; the item and the next one
    static constexpr int kMRef = 0, kNeg = kMRef + N * 4, kFactor = kNeg + N * 4, kParts = kFactor + N * 4, kMasks = kParts + 4 * N * 4,
                         kBars = kMasks + 64 * 8, kValid = kBars + (kStages + 8) * 8, kItems = (kValid + kStages * 8 + 15) / 16 * 16, kMiscBytes = (kItems + 2 * 64 + 127) / 128 * 128;
    static constexpr int kOffShared = kOffMisc + kWorkers * kMiscBytes;   // tensor memory's address, the abort flag, the scan
    static constexpr int kSharedBytes = 512;
    static constexpr int kSmem = 1024 + kOffShared + kSharedBytes;
    // registers: the warpgroups that compute take what the warps that issue leave
    static constexpr int kRegs = N == 64 ? 168 : 96, kRegsFew = 64, kRegsMany = N == 64 ? 216 : 104;
    static_assert((kWorkers * kRegsMany + kRegsFew) * 128 <= kRegs * kThreads, "registers of the launch");
    static constexpr int kColumns = 64 + 2 * N;                  // of tensor memory: decoded keys or values, S, O
    static_assert(kWorkers * kColumns <= 512 && kSmem <= 232448, "");
};

// A (sequence, KV head) and what its items cost.
struct Place {
    int s, h;
    int len;          // cached tokens that may be seen, at most what the table has room for
    int slabs;        // verify: of the list, or of the sequence
    int tok0, n;      // chunk: first new token, new tokens; verify: s * T, T
    int pos0;         // chunk: position of the first new token
    svq::Entry cost;
};

template <bool kChunk, int N>
__device__ __forceinline__ Place place(const Params &p, int e)
{
    Place r;
    r.s = e / p.Hkv, r.h = e - r.s * p.Hkv;
    const int cap = (int)min((long long)p.NBmax * p.B, 0x7fffffffll);
    const int len = __ldg(p.seq_lens + r.s);
    r.len = min(max(len, 0), cap);
    if constexpr (kChunk) {
        const int first = min(max(__ldg(p.q_start + r.s), 0), p.n_tokens), end = min(max(__ldg(p.q_start + r.s + 1), 0), p.n_tokens);
        r.tok0 = first, r.n = max(end - first, 0), r.pos0 = (int)max((long long)len - r.n, -(1ll << 30));   // (further below zero than a call has tokens)
        r.slabs = 0;
        const int seen = min(max(r.pos0, 0), cap);
        r.cost.tiles = (int)(((long long)r.n * p.G + N - 1) / N);
        r.cost.a = (long long)p.G * (seen + svq::kItemCost), r.cost.b = N;
    } else {
        r.tok0 = r.s * p.T, r.n = p.T, r.pos0 = 0;
        if (p.sel_idx) {
            const int cnt = min(max(__ldg(p.sel_cnt + e), 0), min(p.max_sel, svq::kMostBlocks));
            r.slabs = cnt * (p.B / 64);
        } else {
            r.slabs = (r.len + 63) / 64;
        }
        r.cost.tiles = (p.G * p.T + N - 1) / N;
        r.cost.a = svq::kItemCost + (long long)kUnit * ((r.slabs + 1) / 2 + 1), r.cost.b = 0;
    }
    return r;
}

// A part of an item, as the warp that issues hands it to the warpgroup (which has no registers to walk the batch itself).
struct Item {
    int s, h, tok0;          // sequence, KV head, first token
    int row0, rows;          // rows of the tile (0: there are no more items)
    int n_units, u0;         // units of cached keys, the first of them
    int drafts, whole;       // the draft's own keys are part of it; nothing is cut
    int pos0, blind;         // (chunk) position of token 0; rows of the sequence that see no key
    int parts, begins;       // parts of the cut item that begins here; whether the part is an item's first
};
static_assert(sizeof(Item) <= 64, "");

template <int N, bool kChunk>
struct Worker {
    using F = Form<N>;
    const Params &p;
    uint32_t q_tile, p_tile, ring, misc, shared, tmem;   // shared memory and tensor memory of this worker
    const uint8_t *slabs;                                // the ring, for reading
    const float *refs;                                   // minus the references
    int wg, tid, lane, warp, worker;
    uint32_t parity = 0;            // of the next unit's barriers
    int taken = 0, asked = 0;       // units of the ring consumed and requested, ever
    int units_done = 0, items = 0;  // (the warp that issues) units and items so far

    __device__ uint32_t bar_full(int i) const { return misc + F::kBars + i * 8; }
    // of a unit: its keys are in tensor memory, its scores, its weights and values are, its product with them is through
    __device__ uint32_t bar_k() const { return bar_full(F::kStages); }
    __device__ uint32_t bar_s() const { return bar_full(F::kStages + 1); }
    __device__ uint32_t bar_p() const { return bar_full(F::kStages + 2); }
    __device__ uint32_t bar_o() const { return bar_full(F::kStages + 3); }
    // an item has been handed out; it has been read (two places in turn)
    __device__ uint32_t bar_item(int n) const { return bar_full(F::kStages + 4 + (n & 1)); }
    __device__ uint32_t bar_taken(int n) const { return bar_full(F::kStages + 6 + (n & 1)); }
    __device__ uint32_t item_at(int n) const { return misc + F::kItems + (n & 1) * 64; }
    __device__ void sync() const { named_bar_sync(1 + wg, 128); }
    __device__ bool aborted() const
    {
        uint32_t v;
        asm volatile("ld.volatile.shared.b32 %0, [%1];" : "=r"(v) : "r"(shared + 4) : "memory");
        return v != 0;
    }
    // Bounded.  Where it gives up it says so, later waits of the CTA look once, and everybody goes on to the end with what there is.
    __device__ __forceinline__ static void wait_long(uint32_t bar, uint32_t parity, uint32_t shared, int32_t *status, int bit)
    {
#pragma unroll 1
        for (int n = 0; n < 1 << 19; ++n) {
            if (mbar_try_wait(bar, parity)) return;
            if ((n & 63) == 0) {
                uint32_t v;
                asm volatile("ld.volatile.shared.b32 %0, [%1];" : "=r"(v) : "r"(shared + 4) : "memory");
                if (v) return;
            }
        }
        sts32(shared + 4, 1);
        if (status) atomicOr(status, bit);
    }
    __device__ void wait(uint32_t bar, uint32_t par, int bit) const
    {
        if (!mbar_try_wait(bar, par)) wait_long(bar, par, shared, p.status, bit);
    }
    __device__ void arrive(uint32_t bar) const
    {
        __syncwarp();
        if (lane == 0) mbar_arrive(bar);
    }

    // ------------------------------------------------------------------ the warp that copies and issues
    int list_base = -1, known = 0, known_valid = 0;   // a slab a lane, from list_base on: its page's slab number, its tokens
    __device__ void look_up(const Place &pl, int end, int n_slabs, int from)
    {
        list_base = from;
        const int j = from + lane, per = p.B / 64;
        known = 0, known_valid = 0;
        if (j >= n_slabs) return;
        int b = j / per;
        const int sub = j - b * per;
        bool bad = false;
        if (!kChunk && p.sel_idx) {
            b = __ldg(p.sel_idx + ((size_t)pl.s * p.Hkv + pl.h) * p.max_sel + b);
            bad = (unsigned)b >= (unsigned)p.NBmax;
            b = min(max(b, 0), p.NBmax - 1);
        }
        int page = __ldg(p.block_table + (size_t)pl.s * p.NBmax + b);
        known_valid = (int)min(max((long long)end - (long long)b * p.B - sub * 64, 0ll), 64ll);
        if (known_valid > 0) bad = bad || (unsigned)page >= (unsigned)p.n_pages;
        page = min(max(page, 0), p.n_pages - 1);
        if (bad && p.status) atomicOr(p.status, kStatusIndex);
        known = (page * p.Hkv + pl.h) * per + sub;
    }
    // unit u of the item
    __device__ void ask(const Place &pl, int end, int n_slabs, int u, uint64_t policy)
    {
        if (list_base < 0 || 2 * u >= list_base + 32) look_up(pl, end, n_slabs, 2 * u);
        const int i = 2 * u - list_base;
        const int a = __shfl_sync(0xffffffffu, known, i), b = __shfl_sync(0xffffffffu, known, (i + 1) & 31);
        const int va = __shfl_sync(0xffffffffu, known_valid, i), vb = __shfl_sync(0xffffffffu, known_valid, (i + 1) & 31);
        const int stage = asked % F::kStages;
        if (elect_one()) {
            const uint32_t full = bar_full(stage), dst = ring + stage * F::kUnitBytes;
            sts64(misc + F::kValid + stage * 8, (unsigned long long)(uint32_t)vb << 32 | (uint32_t)va);
            const bool second = 2 * u + 1 < n_slabs;
            mbar_arrive_expect_tx(full, second ? F::kUnitBytes : kSlabBytes);
            bulk_load(dst, p.pool + (size_t)a * kSlabBytes, kSlabBytes, full, policy);
            if (second) bulk_load(dst + kSlabBytes, p.pool + (size_t)b * kSlabBytes, kSlabBytes, full, policy);
        }
        __syncwarp();
        ++asked;
    }
    __device__ void hand_out(const Item &it)
    {
        if (items > 1) wait(bar_taken(items), ((items >> 1) - 1) & 1, 32);
        if (__any_sync(0xffffffffu, aborted())) return;   // (nothing is written under the eyes of those who still read)
        if (lane < (int)(sizeof(Item) / 4)) sts32(item_at(items) + lane * 4, reinterpret_cast<const uint32_t *>(&it)[lane]);
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_item(items));
        ++items;
    }
    __device__ void copy_and_issue(const Place &pl, int tile, const svq::Part &part, int units)
    {
        Item it{pl.s, pl.h, pl.tok0, tile * N, min(N, p.G * pl.n - tile * N), 0, part.u0, 0, part.u0 == 0 && part.u1 == units, pl.pos0, 0, part.parts, part.u0 == 0};
        int end = pl.len, n_slabs = pl.slabs;   // keys that any of the rows sees, and the slabs that hold them
        if constexpr (kChunk) {
            end = min(max(pl.pos0 + (it.row0 + it.rows - 1) / p.G + 1, 0), pl.len);
            n_slabs = (end + 63) / 64;
            it.blind = min(max(-pl.pos0, 0), pl.n) * p.G;
        } else {
            it.drafts = part.u1 == units;
        }
        it.n_units = max(min(part.u1, (n_slabs + 1) / 2) - part.u0, 0);
        hand_out(it);
        const uint64_t policy = policy_evict_first();
        constexpr uint32_t idesc_s = umma_idesc_bf16(128, N, false), idesc_o = umma_idesc_bf16(128, N, true);
        const uint64_t dq = umma_desc_sw128(q_tile, 16, 1024), dp = umma_desc_sw128(p_tile, 8192, 1024);
        list_base = -1;
        for (int u = 0; u < min(it.n_units, F::kStages); ++u) ask(pl, end, n_slabs, part.u0 + u, policy);
#pragma unroll 1
        for (int k = it.drafts ? -1 : 0, n = 0; k < it.n_units; ++k, ++n) {
            wait(bar_k(), units_done & 1, 4);
            tc_fence_after_sync();
            if (elect_one()) {
#pragma unroll
                for (int ks = 0; ks < 8; ++ks)
                    tc_mma_bf16_ta(tmem + 64, tmem + ks * 8, dq + (uint64_t)((ks & 3) * 2 + (ks >> 2) * (N * 128 >> 4)), idesc_s, ks > 0);
                tc_commit(bar_s());
            }
            __syncwarp();
            wait(bar_p(), units_done & 1, 8);
            tc_fence_after_sync();
            if (elect_one()) {
#pragma unroll
                for (int ks = 0; ks < 8; ++ks)
                    tc_mma_bf16_ta(tmem + 64 + N, tmem + ks * 8, dp + (uint64_t)(ks * 2048 >> 4), idesc_o, ks > 0 || n > 0);
                tc_commit(bar_o());
            }
            __syncwarp();
            ++units_done;
            // (the unit's slot has been read)
            if (k >= 0 && k + F::kStages < it.n_units) ask(pl, end, n_slabs, part.u0 + k + F::kStages, policy);
        }
    }
    // Copies and products that nobody waited for, when a wait gave up: this CTA's memory stays until they are through.
    __device__ void drain() const
    {
        if (!aborted()) return;
#pragma unroll 1
        for (int i = 0; i < F::kStages; ++i) {
            const int n = asked > i ? (asked - i + F::kStages - 1) / F::kStages : 0;
            if (n > 0) (void)mbar_wait_bounded(bar_full(i), (n - 1) & 1);
        }
        if (units_done == 0) return;
        (void)mbar_wait_bounded(bar_s(), (units_done - 1) & 1);
        (void)mbar_wait_bounded(bar_o(), (units_done - 1) & 1);
    }

    // ------------------------------------------------------------------ the warpgroup: operands, 16 columns of tensor memory at a time
    // (rolled: what the four workers run through at different places is to stay in the instruction caches)
    __device__ void put_keys(uint32_t at, int stage) const   // this thread's key
    {
        const uint8_t *slab = slabs + stage * F::kUnitBytes + (tid >> 6) * kSlabBytes;
        const int t = tid & 63;
        const uint2 sc = *reinterpret_cast<const uint2 *>(slab + svq::kOffKScale + t * 8);
        uint4 v[4];   // (all asked for at once: a store into tensor memory orders what is around it)
#pragma unroll
        for (int c = 0; c < 4; ++c) v[c] = *reinterpret_cast<const uint4 *>(slab + c * 1024 + t * 16);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const uint32_t w = c < 2 ? sc.x : sc.y, d = svq::both_low(w), m = svq::both_high(w);
            uint32_t x[16];
            svq::decode(v[c].x, d, m, x);
            svq::decode(v[c].y, d, m, x + 4);
            svq::decode(v[c].z, d, m, x + 8);
            svq::decode(v[c].w, d, m, x + 12);
            tmem_st_x16(at + 16 * c, x);
        }
    }
    // 128 tokens of the warp's 32 dims.  A thread has four dims (d0 + 8 i) and four tokens of every 16, so that it needs a quarter of the
    // scales: a thread with a dim's 128 tokens of its own, all of whose scales come from shared memory, moves 2.5 times the bytes there, and
    // they are what bounds the decoding.  Tokens that are not there are zero: whatever a slab holds for them, a weight of zero times it is
    // to be zero.
    __device__ void put_values(uint32_t at, int stage, const int (&valid)[2]) const
    {
        const int q = lane & 3, d0 = warp * 32 + (lane >> 2);
        const uint32_t turn = 29 + 8 * (q & 1);   // of a word, that brings the first of the thread's two pairs to where steps() has them
#pragma unroll 1
        for (int b = 0; b < 2; ++b) {   // slabs
            const uint8_t *slab = slabs + stage * F::kUnitBytes + b * kSlabBytes, *sc = slab + svq::kOffVScale + (warp >> 1) * 256 + q * 8;
            uint2 d[4], m[4];   // of tokens 16 j + 4 q ..
#pragma unroll
            for (int j = 0; j < 4; ++j) d[j] = *reinterpret_cast<const uint2 *>(sc + 32 * j), m[j] = *reinterpret_cast<const uint2 *>(sc + 128 + 32 * j);
            uint32_t words[16];   // of dims d0 + 8 i, then by j
#pragma unroll
            for (int i = 0; i < 16; ++i)
                words[i] = *reinterpret_cast<const uint32_t *>(slab + svq::kOffV + (i >> 1 & 1) * 2048 + (d0 + 8 * (i >> 2)) * 16 + (2 * (i & 1) + (q >> 1)) * 4);
            const int n = b ? valid[1] : valid[0];
            if (n < 64) {
                const auto cut = [](uint32_t w, int left) { return left >= 2 ? w : left == 1 ? w & 0xffffu : 0u; };
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int left = n - 16 * j - 4 * q;
                    d[j] = make_uint2(cut(d[j].x, left), cut(d[j].y, left - 2)), m[j] = make_uint2(cut(m[j].x, left), cut(m[j].y, left - 2));
                }
            }
#pragma unroll
            for (int half = 0; half < 2; ++half) {   // dims d0 + 16 half and 8 more
                uint32_t x[16];   // word 4 j + 2 h + e: dim + 8 h, tokens 16 j + 4 q + 2 e and the next
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t w = words[8 * half + 4 * h + j];
                        x[4 * j + 2 * h] = svq::fma_bf16x2(svq::steps_at(w, turn), d[j].x, m[j].x);
                        x[4 * j + 2 * h + 1] = svq::fma_bf16x2(svq::steps_at(w, turn + 4), d[j].y, m[j].y);
                    }
                tmem_st_16x256b_x4(at + ((uint32_t)half << 20) + 32 * b, x);   // (16 lanes further)
            }
        }
    }
    __device__ void put_draft_keys(uint32_t at, int tok0, int h) const
    {
        const uint4 *row = reinterpret_cast<const uint4 *>(p.draft_k + ((size_t)(tok0 + tid) * p.Hkv + h) * 128);
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
            uint32_t x[16];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint4 w = tid < p.T ? __ldg(row + 4 * c + i) : make_uint4(0, 0, 0, 0);
                x[4 * i] = w.x, x[4 * i + 1] = w.y, x[4 * i + 2] = w.z, x[4 * i + 3] = w.w;
            }
            tmem_st_x16(at + 16 * c, x);
        }
    }
    __device__ void put_draft_values(uint32_t at, int tok0, int h) const
    {
        const unsigned short *col = reinterpret_cast<const unsigned short *>(p.draft_v + ((size_t)tok0 * p.Hkv + h) * 128 + tid);
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
            uint32_t x[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int j = 32 * c + 2 * i;
                const uint32_t a = j < p.T ? __ldg(col + (size_t)j * p.Hkv * 128) : 0u;
                const uint32_t b = j + 1 < p.T ? __ldg(col + (size_t)(j + 1) * p.Hkv * 128) : 0u;
                x[i] = a | b << 16;
            }
            tmem_st_x16(at + 16 * c, x);
        }
    }

    // New references for the rows whose maximum over the unit's scores (of four warps, less the old ones) has outgrown theirs; the factors
    // for what was summed by the old ones, and O by them.  fresh: whether there are rows without a reference still.
    __device__ __forceinline__ void move_references(int rows, bool started, uint32_t t_o, bool &fresh) const
    {
        bool none = false;
        if (tid < rows) {
            float m = ldsf(misc + F::kParts + tid * 4);
#pragma unroll
            for (int w = 1; w < 4; ++w) m = fmaxf(m, ldsf(misc + F::kParts + (w * N + tid) * 4));
            const float old = ldsf(misc + F::kMRef + tid * 4);
            m -= ldsf(misc + F::kNeg + tid * 4);   // (of the scores themselves)
            float c = 1.f;
            if (m > old + kLag) {
                c = fast_exp2(old - m);
                stsf(misc + F::kMRef + tid * 4, m), stsf(misc + F::kNeg + tid * 4, -m);
            } else {
                none = old == -INFINITY;
            }
            stsf(misc + F::kFactor + tid * 4, c);
        }
        fresh = named_bar_or(1 + wg, 128, none);
        if (!started) return;
        // (the last product is through, the next not issued: O is at rest)
#pragma unroll 1
        for (int c0 = 0; c0 < N; c0 += 16) {
            uint32_t o[16];
            tmem_ld_x16(t_o + c0, o);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * ldsf(misc + F::kFactor + (c0 + i) * 4));
            tmem_st_x16(t_o + c0, o);
        }
    }

    // ------------------------------------------------------------------ the warpgroup: a part of an item
    __device__ int word(int n, size_t offset) const { return (int)lds32(item_at(n) + (uint32_t)offset); }
#define ITEM(name) word(n, offsetof(Item, name))
    __device__ void attend(int n)
    {
        const int rows = ITEM(rows);

        sync();   // (the last item's rows have been read)
        const bool drafts = ITEM(drafts) != 0;
        {
        const int row0 = ITEM(row0), tok0 = ITEM(tok0), h = ITEM(h);
#pragma unroll 4
        for (int i = 0; i < N / 8; ++i) {
            const int c = i * 128 + tid, r = c >> 4, ch = c & 15, row = row0 + r;
            uint4 v = make_uint4(0, 0, 0, 0);
            if (r < rows) v = __ldg(reinterpret_cast<const uint4 *>(p.q + ((size_t)(tok0 + row / p.G) * p.Hq + h * p.G + row % p.G) * 128) + ch);
            sts128(q_tile + (ch >> 3) * (N * 128) + r * 128 + (((ch & 7) ^ (r & 7)) << 4), v);
        }
        if (tid < N) {
            stsf(misc + F::kMRef + tid * 4, -INFINITY), stsf(misc + F::kNeg + tid * 4, 0.f);
            if (drafts) {
                // which drafts the row's token sees: itself and its ancestors, or all up to it
                unsigned long long seen = 0;
                const int i = min((row0 + tid) / p.G, p.T - 1);
                if (p.parent) {
                    const int32_t *parent = p.parent + (size_t)ITEM(s) * p.T;
                    int j = i;
#pragma unroll 1
                    for (int n = 0; n < 64 && j >= 0; ++n) {
                        seen |= 1ull << j;
                        const int up = __ldg(parent + j);
                        j = up < j ? up : -1;
                    }
                } else {
                    seen = (2ull << i) - 1;
                }
                sts64(misc + F::kMasks + tid * 8, seen);
            }
        }
        }
        fence_proxy_async();
        sync();

        unsigned long long l2[N / 2];   // sums of the weights, rows 2 i and 2 i + 1
#pragma unroll
        for (int i = 0; i < N / 2; ++i) l2[i] = 0ull;
        bool fresh = true, started = false;
        const unsigned long long scale2 = f2_pack(p.scale_log2, p.scale_log2);
        const uint32_t t_op = tmem + ((uint32_t)(warp * 32) << 16), t_s = t_op + 64, t_o = t_s + N;

        const int n_units = ITEM(n_units);
#pragma unroll 1
        for (int k = drafts ? -1 : 0; k < n_units; ++k) {
            const int stage = taken % F::kStages;
            int valid[2] = {0, 0};
            if (k >= 0) {
                wait(bar_full(stage), (taken / F::kStages) & 1, 1);
                const uint2 v = lds64(misc + F::kValid + stage * 8);
                valid[0] = (int)v.x, valid[1] = (int)v.y;
            }
            if (started) {   // the place of the operand is that of the last unit's values
                wait(bar_o(), parity ^ 1, 2);
                tc_fence_after_sync();
            }
            if (k < 0) put_draft_keys(t_op, ITEM(tok0), ITEM(h));
            else put_keys(t_op, stage);
            tmem_st_wait();
            tc_fence_before_sync();
            arrive(bar_k());
            // from which row on this thread's key is seen
            int first = N;
            if (k >= 0 && (tid & 63) < valid[tid >> 6]) {
                first = 0;
                if constexpr (kChunk) first = (int)min(max((long long)((ITEM(u0) + k) * kUnit + tid - ITEM(pos0)) * p.G - ITEM(row0), 0ll), (long long)N);
            }
            const bool some_hidden = __any_sync(0xffffffffu, first > 0);
            wait(bar_s(), parity, 4);
            tc_fence_after_sync();
            if (k < 0) put_draft_values(t_op, ITEM(tok0), ITEM(h));
            else put_values(t_op, stage, valid);
            // 16 rows' scores less their references; the scores are read twice, for the largest and for the weights, since there are no
            // registers to keep those of all rows beside the sums
            const auto scores = [&](int c, float (&y)[16]) {
                uint32_t s[16];
                tmem_ld_x16(t_s + c, s);
                tmem_ld_wait();
                if (k < 0) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const uint2 seen = lds64(misc + F::kMasks + (c + i) * 8);
                        const uint32_t w = tid & 32 ? seen.y : seen.x;
                        if (tid >= 64 || !(w >> (tid & 31) & 1)) s[i] = 0xff800000u;
                    }
                } else if (some_hidden) {
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (c + i < first) s[i] = 0xff800000u;
                }
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const float4 neg = *reinterpret_cast<const float4 *>(refs + c + i);
                    f2_unpack(f2_fma(f2_pack(__uint_as_float(s[i]), __uint_as_float(s[i + 1])), scale2, f2_pack(neg.x, neg.y)), y[i], y[i + 1]);
                    f2_unpack(f2_fma(f2_pack(__uint_as_float(s[i + 2]), __uint_as_float(s[i + 3])), scale2, f2_pack(neg.z, neg.w)), y[i + 2], y[i + 3]);
                }
            };
            float top = -INFINITY;
#pragma unroll 1
            for (int c = 0; c < rows; c += 16) {
                float y[16];
                scores(c, y);
#pragma unroll
                for (int i = 0; i < 16; i += 2) top = max3f(top, y[i], y[i + 1]);   // (rows that there are not have scores of zero)
            }
            // a score that outgrows its row's reference, or a row without one: references move
            if (named_bar_or(1 + wg, 128, fresh || top > kLag)) {
#pragma unroll 1
                for (int c = 0; c < rows; c += 16) {
                    float y[16], mine = 0.f;
                    scores(c, y);
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float m = warp_max(y[i]);
                        if (lane == i) mine = m;
                    }
                    if (lane < 16) stsf(misc + F::kParts + (warp * N + c + lane) * 4, mine);
                }
                sync();
                move_references(rows, started, t_o, fresh);
#pragma unroll
                for (int r = 0; r < N; r += 2) {
                    const uint2 c = lds64(misc + F::kFactor + r * 4);
                    float a, b;
                    f2_unpack(l2[r / 2], a, b);
                    l2[r / 2] = f2_pack(a * __uint_as_float(c.x), b * __uint_as_float(c.y));
                }
            }
            // Weights.  (bf16 because the matrix instruction takes both operands in one type; the sums are of what they were before.)
            const uint32_t p_row = (p_tile & ~1023u) + tid * 128;
            const int p_chunk = (p_tile >> 4) & 7;
#pragma unroll
            for (int c = 0; c < N; c += 16) {
                if (c >= rows) continue;   // (what is in the columns of rows that there are not is nobody's)
                float y[16];
                scores(c, y);
#pragma unroll
                for (int r = 0; r < 16; r += 8) {
                    if (c + r >= rows) continue;
                    uint32_t w[4];
#pragma unroll
                    for (int i = 0; i < 8; i += 2) {
                        const float a = fast_exp2(y[r + i]), b = fast_exp2(y[r + i + 1]);
                        l2[(c + r + i) / 2] = f2_add(l2[(c + r + i) / 2], f2_pack(a, b));
                        w[i / 2] = pack_bf16(a, b);
                    }
                    sts128(p_row + (((p_chunk + (c + r) / 8) ^ (tid & 7)) << 4), make_uint4(w[0], w[1], w[2], w[3]));
                }
            }
            fence_proxy_async();
            tmem_st_wait();
            tc_fence_before_sync();
            arrive(bar_p());
            if (k >= 0) ++taken;
            parity ^= 1;
            started = true;
        }

        // sums of the weights over the keys: lanes, then warps
        {
            float v[N];
#pragma unroll
            for (int i = 0; i < N / 2; ++i) f2_unpack(l2[i], v[2 * i], v[2 * i + 1]);
            int n = N;
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) {
                if (n > 1) {
                    n /= 2;
#pragma unroll
                    for (int i = 0; i < N / 2; ++i)
                        if (i < n) {
                            const bool up = lane & d;
                            const float send = up ? v[i] : v[i + n], keep = up ? v[i + n] : v[i];
                            v[i] = keep + __shfl_xor_sync(0xffffffffu, send, d);
                        }
                } else {
                    v[0] += __shfl_xor_sync(0xffffffffu, v[0], d);
                }
            }
            if constexpr (N == 64) stsf(misc + F::kParts + (warp * N + 2 * lane) * 4, v[0]), stsf(misc + F::kParts + (warp * N + 2 * lane + 1) * 4, v[1]);
            else if constexpr (N == 32) stsf(misc + F::kParts + (warp * N + lane) * 4, v[0]);
            else if (!(lane & 1)) stsf(misc + F::kParts + (warp * N + (lane >> 1)) * 4, v[0]);
        }
        if (started) {
            wait(bar_o(), parity ^ 1, 2);
            tc_fence_after_sync();
        }
        sync();
        const int row0 = ITEM(row0), blind = kChunk ? ITEM(blind) : 0;
        const bool whole = ITEM(whole) != 0;
        const size_t slot = (size_t)2 * worker + ITEM(begins), out_row = (size_t)ITEM(tok0) * p.Hq + ITEM(h) * p.G;   // (of row 0 of token 0)
        if (tid < N) {
            float l = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) l += ldsf(misc + F::kParts + (w * N + tid) * 4);
            const float m = ldsf(misc + F::kMRef + tid * 4);
            const int row = row0 + tid;
            const bool sees = row >= blind;
            stsf(misc + F::kFactor + tid * 4, sees ? 1.f / l : 0.f);
            if (tid < rows) {
                if (!whole) p.ws_ml[slot * N + tid] = make_float2(m, l);
                else if (p.lse) p.lse[out_row + (size_t)(row / p.G) * p.Hq + row % p.G] = sees ? (m + log2f(l)) * 0.69314718055994531f : -INFINITY;
            }
        }
        if (tid == 0 && ITEM(parts)) {
            p.cuts[2 * worker] = make_int4(ITEM(tok0), row0, ITEM(h) << 8 | rows, ITEM(parts));
            p.cuts[2 * worker + 1] = make_int4(blind, 0, 0, 0);
        }
        sync();
#pragma unroll 1
        for (int c0 = 0; c0 < rows; c0 += 16) {
            uint32_t o[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i] = 0u;
            if (started) {
                tmem_ld_x16(t_o + c0, o);
                tmem_ld_wait();
            }
            int row = row0 + c0, token = row / p.G, g = row - token * p.G;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                if (c0 + i < rows) {
                    const float v = __uint_as_float(o[i]);
                    if (whole) {
                        const float f = ldsf(misc + F::kFactor + (c0 + i) * 4);
                        p.out[(out_row + (size_t)token * p.Hq + g) * 128 + tid] = __float2bfloat16_rn(row + i < blind ? 0.f : v * f);
                    } else {
                        p.ws_o[(slot * N + c0 + i) * 128 + tid] = v;
                    }
                }
                if (++g == p.G) g = 0, ++token;
            }
        }
        tc_fence_before_sync();
    }
#undef ITEM
};

template <int N, bool kChunk>
__global__ void __launch_bounds__(Form<N>::kThreads, 1) q4_attn_kernel(const __grid_constant__ Params p)
{
    using F = Form<N>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem0 = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t shared = smem0 + F::kOffShared;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const bool issuer = tid >= F::kWorkers * 128;
    const int wg = issuer ? warp & 3 : tid >> 7;   // the worker
    const int workers = gridDim.x * F::kWorkers;

    if (tid == 0) {
#pragma unroll 1
        for (int w = 0; w < F::kWorkers; ++w)
#pragma unroll 1
            for (int i = 0; i < F::kStages + 8; ++i)   // (one lane of each warp says that keys, or weights and values, are there, and that an item is read)
                mbar_init(smem0 + F::kOffMisc + w * F::kMiscBytes + F::kBars + i * 8, i == F::kStages || i == F::kStages + 2 || i >= F::kStages + 6 ? 4 : 1);
        mbar_fence_init();
        sts32(shared + 4, 0);
    }
    if (warp == 0) tmem_alloc(shared, 512);
    grid_dependency_wait();

    const int entries = p.S * p.Hkv, den = kChunk ? p.G : 1;
    int per_cta;
    bool no_list = false;
    tc_fence_before_sync();
    const svq::Line line = find_shares<F::kThreads, F::kWorkers>(entries, den, shared + 64, shared + 256, per_cta, [&](int e) {
        if (!kChunk && p.sel_idx) no_list |= __ldg(p.sel_cnt + e) < 0;
        return place<kChunk, N>(p, e).cost.all();
    });
    tc_fence_after_sync();
    if (no_list && blockIdx.x == 0 && p.status) atomicOr(p.status, kStatusNoList);
    const uint32_t tmem = lds32(shared);
    // no cuts yet: of the CTA's own shares, and of those that there are not
    if (tid < per_cta && blockIdx.x * per_cta + tid < line.shares) p.cuts[2 * (blockIdx.x * per_cta + tid)] = make_int4(0, 0, 0, 0);
    for (int i = line.shares + blockIdx.x * F::kThreads + tid; i < workers; i += gridDim.x * F::kThreads) p.cuts[2 * i] = make_int4(0, 0, 0, 0);
    __syncthreads();
    const int share = blockIdx.x * per_cta + wg;
    const bool some = wg < min(per_cta, F::kWorkers) && share < line.shares && line.total > 0;
    const auto worker = [&] {
        Worker<N, kChunk> w{p};
        w.wg = wg, w.tid = tid & 127, w.lane = lane, w.warp = warp & 3, w.worker = share;
        w.q_tile = smem0 + F::kOffQ + wg * F::kQBytes;
        w.p_tile = smem0 + F::kOffP + wg / F::kSharers * F::kPTile + wg % F::kSharers * (N * 2);
        w.misc = smem0 + F::kOffMisc + wg * F::kMiscBytes;
        w.ring = smem0 + F::kOffRing + wg * F::kStages * F::kUnitBytes;
        w.slabs = smem_raw + (w.ring - smem_u32(smem_raw));
        w.refs = reinterpret_cast<const float *>(smem_raw + (w.misc + F::kNeg - smem_u32(smem_raw)));
        w.shared = shared;
        w.tmem = tmem + wg * F::kColumns;
        return w;
    };
    if (issuer) {
        reg_dealloc<F::kRegsFew>();
        if (some) {
            Worker<N, kChunk> w = worker();
            int e = (int)lds_ll(shared + 256 + wg * 16);
            long long at = lds_ll(shared + 256 + wg * 16 + 8);
            const long long lo = line.bound(share), hi = line.bound(share + 1);
            Place pl = place<kChunk, N>(p, e);
            int t = pl.cost.item_at(lo - at);
            at += pl.cost.before(t);
#pragma unroll 1
            while (at < hi) {
                const long long cost = pl.cost.cost(t);
                int units = (pl.slabs + 1) / 2 + 1;
                if constexpr (kChunk) {
                    const int rows = min(N, p.G * pl.n - t * N);
                    const int end = min(max(pl.pos0 + (t * N + rows - 1) / p.G + 1, 0), pl.len);
                    units = (end + kUnit - 1) / kUnit;
                }
                const svq::Part part = svq::part_of(line, share, at, cost, units, den);
                if (part.mine) w.copy_and_issue(pl, t, part, units);
                at += cost;
                if (++t == pl.cost.tiles) {
                    t = 0;
                    do {
                        if (++e < entries) pl = place<kChunk, N>(p, e);
                    } while (e < entries && pl.cost.tiles == 0);
                    if (e >= entries) break;
                }
            }
            w.hand_out(Item{});
            w.drain();
        }
    } else {
        reg_alloc<F::kRegsMany>();
        if (some) {
            Worker<N, kChunk> w = worker();
#pragma unroll 1
            for (int n = 0;; ++n) {
                w.wait(w.bar_item(n), (n >> 1) & 1, 32);
                if (named_bar_or(1 + wg, 128, w.aborted()) || w.word(n, offsetof(Item, rows)) == 0) break;   // (all or nobody)
                w.attend(n);
                w.arrive(w.bar_taken(n));
            }
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (warp == 0) tmem_dealloc(tmem, 512);
    grid_launch_dependents();
}

// A cut item: the sums of its parts, which are numbered from the worker that it begins with.  A warp a row, four dims a lane.
constexpr int kMergeRows = 8;
__global__ void __launch_bounds__(kMergeRows * 32) q4_merge_kernel(const __grid_constant__ Params p, int N)
{
    grid_dependency_wait();
    const int worker = blockIdx.x, lane = threadIdx.x & 31;
    const int4 cut = p.cuts[2 * worker];
    if (cut.w == 0) return;
    const int r = blockIdx.y * kMergeRows + (int)(threadIdx.x >> 5), rows = cut.z & 255, h = cut.z >> 8;
    if (r >= rows) return;
    const int blind = p.cuts[2 * worker + 1].x;
    SplitSum sum;
    constexpr int U = 8;
    for (int base = 0; base < cut.w; base += U) {
        float2 ml[U];
        float4 o[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const size_t at = ((size_t)(worker + base + k) * 2 + (base + k == 0)) * N + r;
            const bool in = base + k < cut.w;
            ml[k] = in ? __ldcg(p.ws_ml + at) : make_float2(-INFINITY, 0.f);
            o[k] = in ? __ldcg(reinterpret_cast<const float4 *>(p.ws_o + at * 128) + lane) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
        sum.add(ml, o);
    }
    const int row = cut.y + r;
    const bool sees = row >= blind;
    const size_t at = ((size_t)cut.x + row / p.G) * p.Hq + h * p.G + row % p.G;
    reinterpret_cast<uint2 *>(p.out + at * 128)[lane] = sees ? sum.out() : make_uint2(0u, 0u);
    if (p.lse && lane == 0) p.lse[at] = sees ? sum.lse() : -INFINITY;
}

sv_status check_kv_q4(const sv_geom *g, const sv_kv_q4 *kv)
{
    if (!kv || !kv->pool || !kv->block_table || !kv->seq_lens) return SV_ERR_NULL;
    if (kv->n_pages < 1) return SV_ERR_SHAPE;
    if ((int64_t)kv->n_pages * g->n_kv_heads * g->block_size >= (int64_t)1 << 31) return SV_ERR_SHAPE;
    if (!svh::aligned(kv->pool, 128) || !svh::aligned(kv->block_table, 4) || !svh::aligned(kv->seq_lens, 4)) return SV_ERR_ALIGN;
    return SV_OK;
}

// Query rows of a tile: as few as hold all rows of a KV head, at most 64.
int tile_rows(int64_t rows) { return rows <= 16 ? 16 : rows <= 32 ? 32 : 64; }
int workers_of(int n) { return svh::sm_count() * (n == 64 ? 2 : 4); }

template <int N, bool kChunk>
sv_status launch(Params &p, void *workspace, void *stream)
{
    using F = Form<N>;
    const int workers = workers_of(N);
    p.cuts = static_cast<int4 *>(workspace);
    p.ws_ml = reinterpret_cast<float2 *>(p.cuts + 2 * workers);
    p.ws_o = reinterpret_cast<float *>(p.ws_ml + (size_t)2 * workers * N);
    static svh::OncePerDevice once;
    if (once.run([] {
            // (the warpgroups that compute wait for the registers that they ask for: there have to be as many)
            cudaFuncAttributes a;
            const cudaError_t e = cudaFuncGetAttributes(&a, q4_attn_kernel<N, kChunk>);
            if (e != cudaSuccess) return e;
            if (a.numRegs < F::kRegs) return cudaErrorInvalidConfiguration;
            return cudaFuncSetAttribute(q4_attn_kernel<N, kChunk>, cudaFuncAttributeMaxDynamicSharedMemorySize, F::kSmem);
        }) != cudaSuccess) {
        (void)cudaGetLastError();
        return SV_ERR_CUDA;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(svh::sm_count());
    cfg.blockDim = dim3(F::kThreads);
    cfg.dynamicSmemBytes = F::kSmem;
    cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[1];
    svh::pdl_attribute(attr);
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, q4_attn_kernel<N, kChunk>, p) != cudaSuccess) {
        (void)cudaGetLastError();
        return SV_ERR_CUDA;
    }
    const int64_t rows = std::min<int64_t>(N, (int64_t)p.G * (kChunk ? p.n_tokens : p.T));
    cfg.gridDim = dim3(workers, (unsigned)((rows + kMergeRows - 1) / kMergeRows));
    cfg.blockDim = dim3(kMergeRows * 32);
    cfg.dynamicSmemBytes = 0;
    return cudaLaunchKernelEx(&cfg, q4_merge_kernel, p, N) == cudaSuccess ? svh::launch_status() : SV_ERR_CUDA;
}
// What the kernel itself needs, with the most rows.
size_t own_bytes()
{
    size_t most = 0;
    for (int n : {16, 32, 64}) most = std::max(most, (size_t)workers_of(n) * (2 * sizeof(int4) + 2 * (size_t)n * 130 * sizeof(float)));
    return (most + 127) / 128 * 128;
}
// Behind that, in a workspace that has room: the cache as bfloat16 pages, their table, and what the attention over such pages needs.  Not for
// caches of more than 256 MB of pages.
struct Spread {
    size_t pool, table, scratch, bytes;   // of one pool, the table, that attention's workspace; of all of it (0: there is none)
    explicit Spread(const sv_geom *g)
    {
        const int64_t pages = (int64_t)g->n_seq * g->max_blocks, rows = pages * g->n_kv_heads * g->block_size;
        pool = table = scratch = bytes = 0;
        if (rows > ((int64_t)256 << 20) / 512) return;
        pool = (size_t)rows * 256, table = ((size_t)pages * 4 + 127) / 128 * 128;
        scratch = std::max(sv_chunk_workspace_bytes(g, 129), sv_workspace_bytes(g, g->max_blocks));   // (of a geometry that does not verify: 0)
        bytes = 2 * pool + table + scratch + 128;
    }
};
// Whether a call of this many query rows a sequence and KV head goes over the decoded cache, and where it is then.  A tile of 64 rows here
// takes as long as one of 128 there, and every tile decodes all its keys: 1,024 tokens behind 30,001 (32 heads) take 1,490 us here, 505 there
// with the decoding; 12 sequences, three of them chunks of some 500 tokens, 290 and 128; trees of 60 tokens of four sequences (420 rows,
// 40 blocks) 98 and 48.
struct Decoded {
    bool use = false;
    uint8_t *k, *v, *scratch;
    int32_t *table;
    Decoded(const sv_geom *g, const Spread &s, int64_t rows, void *workspace, size_t workspace_bytes, size_t need)
    {
        if (!s.bytes || need > s.scratch || workspace_bytes < own_bytes() + s.bytes || rows <= kSpreadRows) return;
        use = true;
        k = static_cast<uint8_t *>(workspace) + own_bytes();
        k += (128 - (reinterpret_cast<uintptr_t>(k) & 127)) & 127;   // (pools stand on 128 bytes)
        v = k + s.pool, table = reinterpret_cast<int32_t *>(v + s.pool), scratch = v + s.pool + s.table;
    }
};

template <bool kChunk>
sv_status launch_rows(Params &p, int64_t rows, void *workspace, void *stream)
{
    const int n = tile_rows(rows);
    return n == 16 ? launch<16, kChunk>(p, workspace, stream) : n == 32 ? launch<32, kChunk>(p, workspace, stream) : launch<64, kChunk>(p, workspace, stream);
}

sv_status common(const sv_geom *g, const sv_kv_q4 *kv, const void *q, float softmax_scale, void *out, float *lse, void *workspace,
                 size_t workspace_bytes, int32_t *status_word, Params &p)
{
    if (!(softmax_scale >= 0.f && softmax_scale < INFINITY)) return SV_ERR_SHAPE;
    if (!svh::aligned(q, 16) || !svh::aligned(out, 16) || !svh::aligned(workspace, 16)) return SV_ERR_ALIGN;
    if ((int64_t)g->n_seq * g->n_kv_heads >= (int64_t)1 << 31) return SV_ERR_SHAPE;
    if (workspace_bytes < own_bytes()) return SV_ERR_WORKSPACE;
    if (!workspace) return SV_ERR_NULL;
    p = Params{};
    p.pool = static_cast<const uint8_t *>(kv->pool), p.block_table = kv->block_table, p.seq_lens = kv->seq_lens, p.n_pages = kv->n_pages;
    p.q = static_cast<const __nv_bfloat16 *>(q), p.out = static_cast<__nv_bfloat16 *>(out), p.lse = lse, p.status = status_word;
    p.S = g->n_seq, p.Hq = g->n_q_heads, p.Hkv = g->n_kv_heads, p.G = p.Hq / p.Hkv, p.B = g->block_size, p.NBmax = g->max_blocks;
    p.scale_log2 = (softmax_scale == 0.f ? 0.08838834764831845f : softmax_scale) * 1.4426950408889634f;
    return SV_OK;
}

}  // namespace

extern "C" size_t sv_workspace_bytes_q4(const sv_geom *geom)
{
    if (svh::check_ragged(geom, 0) != SV_OK) return 0;
    return own_bytes() + Spread(geom).bytes;
}

extern "C" sv_status sv_verify_attn_q4(const sv_geom *geom, const void *q, const sv_kv_q4 *kv, const void *draft_k, const void *draft_v,
                                       const int32_t *parent, const int32_t *sel_idx, const int32_t *sel_cnt, int32_t max_sel,
                                       float softmax_scale, void *out, float *lse, void *workspace, size_t workspace_bytes, int32_t *status_word,
                                       void *stream)
{
    sv_status st = svh::check_geom(geom);
    if (st != SV_OK) return st;
    st = svh::check_ragged(geom, 0);
    if (st != SV_OK) return st;
    st = check_kv_q4(geom, kv);
    if (st != SV_OK) return st;
    if (!q || !draft_k || !draft_v || !out || (sel_idx && !sel_cnt)) return SV_ERR_NULL;
    if (sel_idx && max_sel < 1) return SV_ERR_SHAPE;
    if (!svh::aligned(draft_k, 16) || !svh::aligned(draft_v, 16)) return SV_ERR_ALIGN;
    Params p;
    st = common(geom, kv, q, softmax_scale, out, lse, workspace, workspace_bytes, status_word, p);
    if (st != SV_OK) return st;
    p.draft_k = static_cast<const __nv_bfloat16 *>(draft_k), p.draft_v = static_cast<const __nv_bfloat16 *>(draft_v), p.parent = parent;
    p.sel_idx = sel_idx, p.sel_cnt = sel_cnt, p.max_sel = max_sel, p.T = geom->n_draft;
    const Spread spread(geom);
    const Decoded d(geom, spread, (int64_t)p.G * p.T, workspace, workspace_bytes, sv_workspace_bytes(geom, sel_idx ? max_sel : geom->max_blocks));
    if (d.use && (!sel_idx || max_sel <= geom->max_blocks)) {
        st = svh::spread_q4(geom, kv, sel_idx, sel_cnt, max_sel, d.k, d.v, d.table, status_word, stream);
        if (st != SV_OK) return st;
        const sv_kv pages = {d.k, d.v, d.table, kv->seq_lens, geom->n_seq * geom->max_blocks};
        return sv_verify_attn(geom, q, &pages, draft_k, draft_v, parent, sel_idx, sel_cnt, max_sel, softmax_scale, out, lse, d.scratch, spread.scratch,
                              status_word, stream);
    }
    return launch_rows<false>(p, (int64_t)p.G * p.T, workspace, stream);
}

extern "C" sv_status sv_chunk_attn_q4(const sv_geom *geom, const void *q, const sv_kv_q4 *kv, const int32_t *q_start, int32_t n_tokens,
                                      float softmax_scale, void *out, float *lse, void *workspace, size_t workspace_bytes,
                                      int32_t *status_word, void *stream)
{
    sv_status st = svh::check_ragged(geom, n_tokens);
    if (st != SV_OK) return st;
    st = check_kv_q4(geom, kv);
    if (st != SV_OK) return st;
    if (!q_start || (n_tokens > 0 && (!q || !out))) return SV_ERR_NULL;
    Params p;
    st = common(geom, kv, q, softmax_scale, out, lse, workspace, workspace_bytes, status_word, p);
    if (st != SV_OK || n_tokens == 0) return st;
    p.q_start = q_start, p.n_tokens = n_tokens;
    const Spread spread(geom);
    const Decoded d(geom, spread, (int64_t)p.G * n_tokens / geom->n_seq, workspace, workspace_bytes, sv_chunk_workspace_bytes(geom, n_tokens));
    if (d.use) {
        st = svh::spread_q4(geom, kv, nullptr, nullptr, 0, d.k, d.v, d.table, status_word, stream);
        if (st != SV_OK) return st;
        const sv_kv pages = {d.k, d.v, d.table, kv->seq_lens, geom->n_seq * geom->max_blocks};
        return sv_chunk_attn(geom, q, &pages, q_start, n_tokens, softmax_scale, out, lse, d.scratch, spread.scratch, status_word, stream);
    }
    // (By the mean rows of a sequence, which is what the host knows: a chunk among many single tokens has their narrow tiles.  One of 513 tokens behind 30,000
    // among 127 single tokens behind 1,000 takes 771 us, over bf16 pages 376.)
    return launch_rows<true>(p, (int64_t)p.G * ((n_tokens + geom->n_seq - 1) / geom->n_seq), workspace, stream);
}
