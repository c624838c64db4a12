// sv_chunk_attn: causal attention of a ragged batch of new tokens over the paged cache that holds them, on the 5th-generation tensor
// cores (tcgen05 + TMEM).
//
// Mathematics, for a row q at position p and its keys t <= p: s_t = q . k_t * scale * log2 e, a reference m not far below their running
// maximum, l = sum 2^(s_t - m), o = sum 2^(s_t - m) v_t; the output is o / l.  When the maximum outgrows the reference by more than 8,
// m moves and l and o are multiplied by 2^(old - new); o / l does not depend on m, and bf16 and fp32 have the same exponents.
//
// A row tile is 128 of the G * n rows (token-major: token r / G, head r % G) of a (sequence, KV head); an item is two neighbouring row
// tiles of TT = 128 / G tokens each, or the one that is left (always the case for single tokens).  A CTA runs two streams, each with
// eight softmax warps and S and O of its own in TMEM (4 x 128 columns), over units of 128 keys:
//   two tiles   stream g has tile g and takes every unit; K and V of a unit are fetched once for both
//   one tile    the streams take the units in turn and add their sums at the end
//   S[128 x 128] = Q . K^T      8 x tcgen05.mma (M128 N128 K16), both operands from shared memory (TMA, 128-byte swizzle)
//   P = 2^(s - m)               four lanes per row (tcgen05.ld 16x256b), rounded to bf16 into the columns of S
//   O[128 x 128] += P . V       8 x tcgen05.mma, P from TMEM, V MN-major as TMA stored it
// A stream's chain is S, softmax, PV, S, ...; while one stream is in its softmax the tensor cores work for the other.
//
// The batch is ragged and its lengths are on the device, so the work is divided there: all items of the batch in a row, an item as long
// as the keys it sees plus kItemCost, are cut into equal shares, a CTA each (chunk_shares.h).  An item that is cut is written as partial
// sums to the workspace and merged by a second kernel; a CTA has at most two cuts.  That balances a prompt's triangle of items, single
// tokens over long caches and any mixture of the two without a case of its own.
//
// Bound by, and measured (32 query and 8 KV heads; the faster and the slower of the machines it was timed on): a prompt of 8,192 tokens
// takes 495 to 584 us for 0.55 TFLOP, 0.94 to 1.1 PFLOP/s or 57 to 68 % of a large library product, the tensor pipe active for 52 % of
// the time: a unit of two tiles takes 3900 cycles where its MMAs take 2048, the rest being what passes a unit from S to the softmax, to
// PV and on (issue()).  2,048 tokens behind 30,001 (64 heads): 2.0 to 2.2 ms for 2.08 TFLOP, 0.95 to 1.0 PFLOP/s.  16 single tokens over
// 4K to 16K keys: 727 MB in 126 to 145 us, 77 to 88 % of a copy's rate.  One token over 4K keys of 2 heads: 19 us, of which 5 are the
// merging launch and the rest a chain of cold steps (batch, division, tensor maps, page, tile, softmax).
//
// All waits are on mbarriers and bounded; one that gives up sets the status word, the CTA drains its copies and MMAs, frees TMEM and
// returns.
#include <cuda.h>
#include <cuda_bf16.h>

#include <stddef.h>

#include <algorithm>

#include "attn_common.cuh"
#include "chunk_shares.h"
#include "sv_host.h"
#include "sv_ptx.cuh"

namespace {

using namespace svk;

constexpr int kSoftmax = 16;                  // warps of the softmax, eight for either stream
constexpr int kThreads = (kSoftmax + 4) * 32;
constexpr int kUnit = kChunkUnit;             // keys of a unit
constexpr int kHalf = 16384;                 // [128 rows][64 bf16]: half of a Q, K or V tile
constexpr int kTileBytes = 2 * kHalf;
constexpr int kStages = 5;                   // ring of K and V tiles, in turn
constexpr int kOffQ = kStages * kTileBytes;
constexpr int kOffMisc = kOffQ + 2 * kTileBytes;
constexpr int kSmemBytes = 1024 + kOffMisc + 2048;
static_assert(kSmemBytes <= 232448, "shared memory budget");
constexpr int kRegsMany = 104, kRegsFew = 64;
static_assert((4 * kRegsMany + kRegsFew) * 128 <= 96 * kThreads, "registers of the launch");
constexpr float kLag = 8.f;                  // what the maximum may exceed the reference by (log2)

enum Bar {
    kFull = 0,                   // [kStages] a K or V tile has landed
    kEmpty = kFull + kStages,    // [kStages] the MMAs are through with it
    kQFull = kEmpty + kStages,   // the item's Q has landed
    kQFree,                      // all S of the item are through
    kS,                          // [2] S of the stream's unit is in TMEM
    kP0 = kS + 2,                // [2] P of the first 64 keys is
    kP1 = kP0 + 2,               // [2] ... of the others
    kO = kP1 + 2,                // [2] the stream's last PV of the item is through
    kX = kO + 2,                 // (one tile) the second stream's sums are there
    kXFree,                      // ... and have been taken
    kDone,                       // all MMAs are through
    kItem,                       // [2] the next item is in shared memory (items take the two places in turn)
    kItemTaken = kItem + 2,      // [2] ... and has been read by all roles
    kNumBars = kItemTaken + 2
};
constexpr int kReaders = kSoftmax + 2;   // warps that read the items
enum ItemWord { kSeq, kHead, kRow0, kTokens, kPos0, kKvEnd, kU0, kU1, kUnits, kParts };   // of a ChunkItem
static_assert(sizeof(ChunkItem) == 10 * 4 && offsetof(ChunkItem, units) == kUnits * 4 && offsetof(ChunkItem, kv_end) == kKvEnd * 4, "");
__device__ __forceinline__ int arrivals(int bar)
{
    if (bar >= kItemTaken) return kReaders;
    return (bar >= kP0 && bar < kO) || bar == kX || bar == kXFree ? kSoftmax / 2 : 1;   // (one lane of each warp of a stream)
}

struct Params {
    ChunkBatch batch;
    const int32_t *block_table;
    __nv_bfloat16 *out;
    float *lse;
    float *ws_o;      // [2 * gridDim.x][slot_rows][128]: of a CTA, the share of an item that began before and of one that goes on behind
    float2 *ws_ml;    // [2 * gridDim.x][slot_rows]
    int4 *cuts;       // [gridDim.x] the cut item that begins in a CTA's share: first row, tokens, KV head and (in the upper half) how many of
                      // the tokens see no key, parts (0: none)
    int32_t *status;
    int Hq, Hkv, G, TT, B, NBmax, n_pages, slot_rows;
    float scale_log2;
};

constexpr int kFound = kThreads / 32;
// The share of this CTA, found by all of its threads together; scratch: kFound + 2 words of shared memory.  False: none.
__device__ bool begin_walk(const Params &p, ChunkWalk &walk, long long *scratch)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    long long mine = 0, first = 0;
#pragma unroll 1
    for (int i = tid; i < p.batch.S; i += kThreads) {
        walk.load(i);
        mine += walk.per_head();
        if (i == tid) first = mine;
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, d);
    if (lane == 0) scratch[warp] = mine;
    __syncthreads();
    long long total = 0;
#pragma unroll 1
    for (int w = 0; w < kThreads / 32; ++w) total += scratch[w];
    if (!walk.divide(total * p.batch.Hkv, gridDim.x, blockIdx.x)) return false;
    long long ahead = 0;   // the sequence that the share begins in, by sums over the ones before
#pragma unroll 1
    for (int base = 0; base < p.batch.S && ahead <= walk.lo; base += kThreads) {
        const int i = base + tid;
        long long cost = first;
        if (base) {
            cost = 0;
            if (i < p.batch.S) walk.load(i), cost = walk.per_head();
        }
        cost *= p.batch.Hkv;
        long long upto = cost;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const long long o = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += o;
        }
        __syncthreads();
        if (lane == 31) scratch[warp] = upto;
        __syncthreads();
        upto += ahead;
#pragma unroll 1
        for (int w = 0; w < kThreads / 32; ++w) {
            if (w < warp) upto += scratch[w];
            ahead += scratch[w];
        }
        if (i < p.batch.S && cost > 0 && upto - cost <= walk.lo && walk.lo < upto) scratch[kFound] = i, scratch[kFound + 1] = upto - cost;
        __syncthreads();
    }
    walk.enter((int)scratch[kFound], scratch[kFound + 1]);
    return true;
}

__device__ __forceinline__ void load_box_3d(uint32_t dst, const void *map, int x, int y, int z, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
                 "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void load_box_4d(uint32_t dst, const void *map, int x, int y, int z, int w, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
                 "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar)
                 : "memory");
}

__device__ __forceinline__ void store_zero(uint32_t at) { asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at), "r"(0) : "memory"); }
__device__ __forceinline__ void store_pair(uint32_t at, float a, float b) { asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(at), "f"(a), "f"(b) : "memory"); }
__device__ __forceinline__ float2 load_pair(uint32_t at)
{
    float2 v;
    asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(at) : "memory");
    return v;
}

// What the warps of a CTA share, by its address in shared memory: barriers, and whether one of their waits gave up.
struct Shared {
    uint32_t at;
    static constexpr uint32_t kAbort = 384, kTmem = 388, kScratch = 400, kExchange = 576, kItems = 1600;
    __device__ uint32_t bar(int i) const { return at + i * 8; }
    __device__ static int load(uint32_t a)
    {
        int v;
        asm volatile("ld.volatile.shared.b32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
        return v;
    }
    __device__ static void store(uint32_t a, int v) { asm volatile("st.volatile.shared.b32 [%0], %1;" ::"r"(a), "r"(v) : "memory"); }
    __device__ void give_up(int32_t *status, int bit) const
    {
        store(at + kAbort, 1);
        if (status) atomicOr(status, bit);
    }
    // As few instructions as it takes: the code of a hand-over is cold when it is reached (the softmax has run through the instruction
    // caches meanwhile), and is fetched line by line.  With the waits unrolled four by four the kernel had 158 KB of code, and every step
    // of a hand-over took 400 cycles.
    __device__ static bool poll(uint32_t bar, uint32_t parity)   // 2^13 times
    {
        uint32_t ok;
        asm volatile(
            "{\n\t.reg .pred p, q;\n\t.reg .u32 n;\n\t"
            "mov.u32 n, 8192;\n"
            "POLL%=:\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
            "@p bra DONE%=;\n\t"
            "add.u32 n, n, -1;\n\t"
            "setp.ne.u32 q, n, 0;\n\t"
            "@q bra POLL%=;\n"
            "DONE%=:\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(bar), "r"(parity)
            : "memory");
        return ok != 0;
    }
    __device__ bool wait(int i, uint32_t parity, int32_t *status, int bit, int rounds = 64) const
    {
#pragma unroll 1
        for (int n = 0; n < rounds; ++n) {   // (looks at the flag between polls of a limited number)
            if (poll(bar(i), parity)) return true;
            if (load(at + kAbort)) return false;
        }
        give_up(status, bit);
        return false;
    }
    // the same for a converged warp: true if every lane has seen the phase
    __device__ bool warp_wait(int i, uint32_t parity, int32_t *status, int bit) const { return __all_sync(0xffffffffu, wait(i, parity, status, bit)); }
    // The same without the suspension that try_wait may take, for the issuing warp alone (for all warps, their polls get into one
    // another's way).
    __device__ bool spin_wait(int i, uint32_t parity, int32_t *status, int bit) const
    {
        const uint32_t b = bar(i);
#pragma unroll 1
        for (int n = 1; n < 1 << 22; ++n) {
            if (__all_sync(0xffffffffu, mbar_test(b, parity))) return true;
            if ((n & 8191) == 0 && __any_sync(0xffffffffu, load(at + kAbort))) return false;
        }
        give_up(status, bit);
        return false;
    }
    // words of an item (ChunkItem)
    __device__ int item(int n, int word) const { return load(at + kItems + (n & 1) * (uint32_t)sizeof(ChunkItem) + word * 4); }
};
static_assert(kNumBars * 8 <= Shared::kAbort && Shared::kScratch + (kFound + 2) * 8 <= Shared::kExchange && Shared::kExchange + 128 * 8 <= Shared::kItems &&
                  Shared::kItems + 2 * sizeof(ChunkItem) <= 2048,
              "");

// ---------------------------------------------------------------------- warp 18: the items, two ahead of the roles that read them
// (A walk of their own in every role cost the softmax its registers: spills of 17 loads a unit, two thirds of them from L2, were most of
// the time of a prompt of 8K.)
__device__ __forceinline__ void hand_out(ChunkWalk &walk, const Shared &sh, ChunkItem *items, int32_t *status)
{
#pragma unroll 1
    for (int n = 0;; ++n) {
        if (n > 1 && !__all_sync(0xffffffffu, sh.wait(kItemTaken + (n & 1), ((n >> 1) - 1) & 1, status, 64, 1 << 13))) return;   // (as long as an item)
        ChunkItem it;
        const bool more = walk.next(it);
        if (!more) it.units = -1;
        if ((threadIdx.x & 31) == 0) {
            items[n & 1] = it;
            mbar_arrive(sh.bar(kItem + (n & 1)));
        }
        __syncwarp();
        if (!more) return;
    }
}
// The item of this number is there, for a whole warp, until it says that it is through with it; false: there are no more, or a wait gave
// up.
__device__ __forceinline__ bool take(const Shared &sh, int n, int32_t *status)
{
    return sh.warp_wait(kItem + (n & 1), (n >> 1) & 1, status, 64) && sh.item(n, kUnits) >= 0;
}
__device__ __forceinline__ void taken(const Shared &sh, int n)
{
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(sh.bar(kItemTaken + (n & 1)));
}

// ---------------------------------------------------------------------- warp 16: copies
__device__ __forceinline__ void produce(const Params &p, const Shared &sh, uint32_t smem0, const CUtensorMap &tm_q, const CUtensorMap &tm_k,
                                        const CUtensorMap &tm_v)
{
    const int lane = threadIdx.x & 31;
    const int per_unit = kUnit / p.B;   // pages of a unit
    int slot = 0, items = 0;            // ring slots and items so far
    bool dead = false, clamped = false;
    const auto wait = [&](int bar, uint32_t parity, int bit) { return sh.warp_wait(bar, parity, p.status, bit); };
    for (int n = 0; !dead && take(sh, n, p.status); ++n) {
        const struct { int s, h, row0, tokens, kv_end, u0, u1, units; } it = {sh.item(n, kSeq), sh.item(n, kHead), sh.item(n, kRow0), sh.item(n, kTokens),
                                                                         sh.item(n, kKvEnd), sh.item(n, kU0), sh.item(n, kU1), sh.item(n, kUnits)};
        taken(sh, n);
        if (it.units == 0) continue;
        const int *pages = p.block_table + (size_t)it.s * p.NBmax;
        const int last_page = (it.kv_end - 1) / p.B;
        // Q: both halves of one or two tiles, as soon as the S of the item before are through
        if (items > 0 && !wait(kQFree, (items - 1) & 1, 1)) break;
        const int n_tiles = it.tokens > p.TT ? 2 : 1;
        if (elect_one()) {
            mbar_arrive_expect_tx(sh.bar(kQFull), (uint32_t)(n_tiles * 2 * p.G * p.TT * 128));
#pragma unroll 1
            for (int i = 0; i < 2 * n_tiles; ++i)
                load_box_4d(smem0 + kOffQ + (i >> 1) * kTileBytes + (i & 1) * kHalf, &tm_q, 0, it.h * p.G, it.row0 + (i >> 1) * p.TT, i & 1, sh.bar(kQFull));
        }
        __syncwarp();
        ++items;
        int known = 0, batch0 = -1;   // a page number a lane, 32 pages from batch0 on
        for (int u = it.u0; u < it.u1 && !dead; ++u) {
            const int first = u * per_unit;
            if (batch0 < 0 || first >= batch0 + 32) {   // (32 is a multiple of per_unit)
                batch0 = first;
                known = first + lane <= last_page ? __ldg(pages + first + lane) : 0;
                if ((unsigned)known >= (unsigned)p.n_pages) clamped = true, known = known < 0 ? 0 : p.n_pages - 1;
            }
            // rows of the pools, seen as [pages * Hkv * B][128], where the two halves of the unit begin
            const int keys = min(kUnit, it.kv_end - u * kUnit);
            const int page0 = __shfl_sync(0xffffffffu, known, first - batch0);
            const int page1 = __shfl_sync(0xffffffffu, known, (first - batch0 + 1) & 31);
            const int y0 = (page0 * p.Hkv + it.h) * p.B, y1 = per_unit == 2 ? (page1 * p.Hkv + it.h) * p.B : y0 + 64;
            const int halves = keys > 64 ? 2 : 1;
#pragma unroll 1
            for (int v = 0; v < 2; ++v, ++slot) {
                const int stage = slot % kStages, turn = slot / kStages;
                if (turn > 0 && !wait(kEmpty + stage, (turn - 1) & 1, 2)) {
                    dead = true;
                    break;
                }
                if (elect_one()) {
                    const uint32_t dst = smem0 + stage * kTileBytes, full = sh.bar(kFull + stage);
                    mbar_arrive_expect_tx(full, halves * kHalf);
                    for (int i = 0; i < halves; ++i) {
                        const int y = i ? y1 : y0;
                        if (v) {   // V: [64 keys] of both halves of the dims
                            load_box_3d(dst + i * kHalf, &tm_v, 0, y, 0, full);
                        } else {   // K: either half of the dims, [128 keys]
                            load_box_3d(dst + i * (kHalf / 2), &tm_k, 0, y, 0, full);
                            load_box_3d(dst + kHalf + i * (kHalf / 2), &tm_k, 0, y, 1, full);
                        }
                    }
                }
                __syncwarp();
            }
        }
    }
    if (clamped && p.status) atomicOr(p.status, kStatusIndex);
    // Copies in flight write to this CTA's memory: it stays until they have arrived (all of them have, unless somebody gave up).
#pragma unroll 1
    for (int stage = 0; stage < kStages; ++stage) {
        const int n = slot > stage ? (slot - stage + kStages - 1) / kStages : 0;   // copies requested into the stage
        if (n > 0 && !__all_sync(0xffffffffu, mbar_wait_bounded(sh.bar(kFull + stage), (n - 1) & 1)) && p.status) atomicOr(p.status, 1);
    }
    if (items > 0 && !__all_sync(0xffffffffu, mbar_wait_bounded(sh.bar(kQFull), (items - 1) & 1)) && p.status) atomicOr(p.status, 1);
}

// ---------------------------------------------------------------------- warp 17: all MMAs, of the two streams in turn
// The turns keep the streams half a unit apart, one in its softmax while the tensor cores work for the other; issued by a warp each, the
// streams fall into step and wait for the tensor cores together (4750 cycles a unit of a prompt).  A wait takes 250 to 300 cycles here even
// when there is nothing to wait for, so the lanes wait for different barriers at once: the stage of V, that of the next unit's K and the
// first half of P, then the rest of P, behind which PV and the next S go out together (a wait after the other, the warp itself was what a
// unit took: 4200 cycles).
__device__ __forceinline__ void issue(const Params &p, const Shared &sh, uint32_t smem0, uint32_t tmem)
{
    constexpr uint32_t idesc_s = umma_idesc_bf16(128, kUnit, false), idesc_pv = umma_idesc_bf16(128, 128, true);
    const uint64_t dq = umma_desc_sw128(smem0 + kOffQ, 16, 1024), dk = umma_desc_sw128(smem0, 16, 1024);
    const uint64_t dv = umma_desc_sw128(smem0, kHalf / 2, 1024);
    // Of every three lanes the second waits for stages of V and the third for stages of K: the ring stage and its parity of what a lane
    // waits for next.
    const int lane = threadIdx.x & 31, part = lane % 3;
    int stage = 0;
    uint32_t turn = 0;
    const auto wait = [&](int bar, uint32_t parity, bool for_stage, int bit) {
        return sh.spin_wait(for_stage ? kFull + stage : bar, for_stage ? turn : parity, p.status, bit);
    };
    const auto skip = [&](int slots) {   // (fewer than kStages)
        stage += slots;
        if (stage >= kStages) stage -= kStages, turn ^= 1;
    };
    // (the warp's own stages of V and K, as descriptors and barriers)
    int stage_v = 1, stage_k = 0;
    const auto next = [](int &at) { at += at >= kStages - 2 ? 2 - kStages : 2; };
    const auto issue_s = [&](int g, uint64_t dq_g) {
        const uint64_t dk_u = dk + (uint64_t)(stage_k * (kTileBytes >> 4));
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
            constexpr int kStep[8] = {0, 2, 4, 6, kHalf >> 4, (kHalf >> 4) + 2, (kHalf >> 4) + 4, (kHalf >> 4) + 6};
            tc_mma_bf16(tmem + g * 128, dq_g + kStep[ks], dk_u + kStep[ks], idesc_s, ks > 0);
        }
        tc_commit(sh.bar(kS + g));
    };
    if (part == 1) skip(1);
    uint32_t of_p = 0, of_q = 0; // parities: of the streams' next P, of the next Q
    bool dead = false;
#pragma unroll 1
    for (int n = 0; !dead && take(sh, n, p.status); ++n) {
        const int n_units = sh.item(n, kU1) - sh.item(n, kU0);
        const bool two = sh.item(n, kTokens) > p.TT, none = sh.item(n, kUnits) == 0;
        taken(sh, n);
        if (none) continue;
        const uint64_t dq_1 = dq + (uint64_t)(two ? kTileBytes >> 4 : 0);
        const int ahead = two ? 1 : 2;   // units from a stream's unit to its next one
        // S of the streams' first units
        dead = !wait(kQFull, of_q, part == 2, 4);
        if (part == 2) skip(2);
        if (!dead && !two && n_units > 1) {
            dead = !wait(kQFull, of_q, part == 2, 4);
            if (part == 2) skip(2);
        }
        if (dead) break;
        of_q ^= 1;
        tc_fence_after_sync();
        if (elect_one()) issue_s(0, dq);
        if (!two) {
            if (elect_one()) tc_commit(sh.bar(kEmpty + stage_k));
            next(stage_k);
        }
        if (two || n_units > 1) {
            if (elect_one()) issue_s(1, dq_1), tc_commit(sh.bar(kEmpty + stage_k));
            next(stage_k);
        }
        if (n_units <= ahead && elect_one()) tc_commit(sh.bar(kQFree));
        __syncwarp();
        int left = n_units;   // units whose PV is to come
#pragma unroll 1
        for (int g = 0; left > 0; g ^= 1) {   // PV of a stream's unit and S of its next
            const bool more = left > ahead, second = two && g, first_reader = two && !g;   // (of two tiles the second stream is the last reader, and the
                                                                                          // first one has seen the stages)
            const uint64_t dv_u = dv + (uint64_t)(stage_v * (kTileBytes >> 4));
            const uint32_t t_o = tmem + 256 + g * 128, t_p = tmem + g * 128, starts = n_units - left >= ahead;
            dead = !wait(kP0 + g, of_p >> g & 1, !second && (part == 1 || (part == 2 && more && two)), 8);
            if (dead) break;
            tc_fence_after_sync();
            if (elect_one()) {
#pragma unroll
                for (int m = 0; m < 4; ++m) tc_mma_bf16_ta(t_o, t_p + m * 8, dv_u + (uint64_t)(m * 2048 >> 4), idesc_pv, m ? 1u : starts);
            }
            __syncwarp();
            dead = !sh.spin_wait(kP1 + g, of_p >> g & 1, p.status, 8);
            if (dead) break;
            tc_fence_after_sync();
            if (elect_one()) {
#pragma unroll
                for (int m = 0; m < 4; ++m) tc_mma_bf16_ta(t_o, t_p + (4 + m) * 8, dv_u + (uint64_t)((kHalf + m * 2048) >> 4), idesc_pv, 1);
                if (two && more) issue_s(g, g ? dq_1 : dq);
                if (!more) tc_commit(sh.bar(kO + g));
                if (!first_reader) tc_commit(sh.bar(kEmpty + stage_v));
            }
            __syncwarp();
            if (!two && more) {   // (one tile: bound by the loads, V goes back before the next K is waited for)
                dead = !wait(kP1 + g, of_p >> g & 1, part == 2, 8);
                if (dead) break;
                tc_fence_after_sync();
                if (elect_one()) issue_s(g, dq);
                __syncwarp();
            }
            if (more && !first_reader && elect_one()) {
                tc_commit(sh.bar(kEmpty + stage_k));
                if (left == ahead + 1) tc_commit(sh.bar(kQFree));
            }
            __syncwarp();
            of_p ^= 1u << g;
            if (!second && (part == 1 || (part == 2 && more))) skip(2);
            if (!first_reader) {
                next(stage_v);
                if (more) next(stage_k);
                --left;
            }
        }
    }
    if (elect_one()) tc_commit(sh.bar(kDone));
    __syncwarp();
}

// ---------------------------------------------------------------------- warps 0-7 and 8-15: the softmax of stream g
// P of two rows of 8 scores each, from x (four words of the fragment of tcgen05.ld 16x256b for either eight keys): rounded to one word a
// row and eight keys, the unrounded ones added to the sums.  (P is bf16 because the matrix instruction takes A of V's type; l is the sum
// of what P was before, so that a row's weights are off by the rounding of each, 2^-8 at most, and not by that of the sum.)
__device__ __forceinline__ void exponentials(const uint32_t *x, uint32_t *w, unsigned long long scale2, const unsigned long long (&ref2)[2],
                                             unsigned long long (&sum2)[2])
{
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float a, b;
        f2_unpack(f2_fma(f2_pack(__uint_as_float(x[2 * h]), __uint_as_float(x[2 * h + 1])), scale2, ref2[h]), a, b);
        a = fast_exp2(a), b = fast_exp2(b);
        sum2[h] = f2_add(sum2[h], f2_pack(a, b));
        w[h] = pack_bf16(a, b);
    }
}
template <class T>
__device__ __forceinline__ T over_row(T v, T (*op)(T, T))   // over the four lanes that share a row
{
    v = op(v, __shfl_xor_sync(0xffffffffu, v, 1));
    return op(v, __shfl_xor_sync(0xffffffffu, v, 2));
}
__device__ __forceinline__ float larger(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ float sum_of(float a, float b) { return a + b; }
// Word i of lane q of every four lanes becomes word q of lane i.
__device__ __forceinline__ void transpose_4(uint32_t (&w)[4], int q)
{
    const bool odd = q & 1, high = q & 2;
    uint32_t a = __shfl_xor_sync(0xffffffffu, odd ? w[0] : w[1], 1), b = __shfl_xor_sync(0xffffffffu, odd ? w[2] : w[3], 1);
    if (odd) w[0] = a, w[2] = b;
    else w[1] = a, w[3] = b;
    a = __shfl_xor_sync(0xffffffffu, high ? w[0] : w[2], 2), b = __shfl_xor_sync(0xffffffffu, high ? w[1] : w[3], 2);
    if (high) w[0] = a, w[1] = b;
    else w[2] = a, w[3] = b;
}

// The eight warps of a stream: a lane quarter has two, for 16 rows each; a thread has rows i and i + 8 of these and every fourth pair of
// keys.
__device__ __forceinline__ void softmax(const Params &p, const Shared sh, uint32_t smem0, uint32_t tmem, int g)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, q = lane & 3;
    const int r0 = (warp & 3) * 32 + (warp >> 2 & 1) * 16 + (lane >> 2);   // first of the thread's rows of the tile
    const uint32_t t_lane = tmem + ((uint32_t)((warp & 3) * 32 + (warp >> 2 & 1) * 16) << 16), t_s = t_lane + g * 128, t_o = t_lane + 256 + g * 128;
    uint32_t phases = 0;   // parities of what this warp has waited for
    constexpr uint32_t kOfS = 1, kOfO = 2, kOfX = 4;
    const auto wait = [&](int bar, uint32_t of, int bit) {
        const bool ok = sh.warp_wait(bar, (phases & of) != 0, p.status, bit);
        phases ^= of;
        return ok;
    };
    const auto arrive = [&](int bar) {
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(sh.bar(bar));
    };
    int v_slot = 1;   // ring slot of the V of the item's first unit
    for (int n = 0; take(sh, n, p.status); ++n) {
        const bool two = sh.item(n, kTokens) > p.TT;
        const int n_units = sh.item(n, kU1) - sh.item(n, kU0), step = two ? 1 : 2, begin = two ? 0 : g;
        // keys counted from the share's first: behind the last one that any row sees, that every row of the tile sees, and these rows
        const int begins = sh.item(n, kU0) * kUnit, kv_end = sh.item(n, kKvEnd) - begins;
        const int pos0 = sh.item(n, kPos0) + (two ? g * p.TT : 0) - begins;
        const int all_see = min(pos0 + 1, kv_end);
        int sees[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) sees[h] = min(pos0 + (r0 + 8 * h) / p.G + 1, kv_end) - 2 * q;   // (less the thread's first key)
        float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
        for (int j = begin; j < n_units; j += step) {
            if (!wait(kS + g, kOfS, 16)) return;
            tc_fence_after_sync();
            uint32_t x[64];   // word 4 i + 2 h + e: row h, key 8 i + 2 q + e
            tmem_ld_16x256b_x16(t_s, x);
            tmem_ld_wait();
            if ((j + 1) * kUnit > all_see) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int seen = sees[h] - j * kUnit;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        if (8 * i >= seen) x[4 * i + 2 * h] = 0xff800000u;
                        if (8 * i + 1 >= seen) x[4 * i + 2 * h + 1] = 0xff800000u;
                    }
                }
            }
            float top[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float mx[2];
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    mx[c] = fmaxf(__uint_as_float(x[32 * c + 2 * h]), __uint_as_float(x[32 * c + 2 * h + 1]));
#pragma unroll
                    for (int i = 1; i < 8; ++i) mx[c] = max3f(mx[c], __uint_as_float(x[32 * c + 4 * i + 2 * h]), __uint_as_float(x[32 * c + 4 * i + 2 * h + 1]));
                }
                top[h] = over_row(fmaxf(mx[0], mx[1]), larger) * p.scale_log2;
            }
            // Each row goes by its own: a warp's other rows may be nobody's, of whatever the queries' tile holds there.
            if (__any_sync(0xffffffffu, top[0] > m[0] + kLag || top[1] > m[1] + kLag)) {
                float c[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const bool move = top[h] > m[h] + kLag;
                    c[h] = move ? fast_exp2(m[h] - top[h]) : 1.f;
                    if (move) m[h] = top[h];
                    l[h] *= c[h];
                }
                if (j > begin) {   // (S of this unit was issued behind the PV of the one before: O is at rest)
#pragma unroll 1
                    for (int o0 = 0; o0 < 128; o0 += 32) {
                        uint32_t o[16];
                        tmem_ld_16x256b_x4(t_o + o0, o);
                        tmem_ld_wait();
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * c[i >> 1 & 1]);
                        tmem_st_16x256b_x4(t_o + o0, o);
                    }
                    tmem_st_wait();
                }
            }
            // V rows behind the last key are another tile's or nobody's: zero, so that 0 * V is 0
            if ((j + 1) * kUnit > kv_end) {
                const int slot = v_slot + 2 * j, stage = slot % kStages;
                if (!sh.warp_wait(kFull + stage, (slot / kStages) & 1, p.status, 16)) return;
#pragma unroll 1
                for (int i = (kv_end - j * kUnit) * 16 + (int)(threadIdx.x & 255); i < kUnit * 16; i += 256) {
                    const int row = i >> 4, c = i & 15;
                    store_zero(smem0 + stage * kTileBytes + (row >> 6) * kHalf + (c >> 3) * (kHalf / 2) + swz128(row & 63, c & 7));
                }
                fence_proxy_async();
            }
            const unsigned long long scale2 = f2_pack(p.scale_log2, p.scale_log2);
            unsigned long long ref2[2], sum2[2] = {0ull, 0ull};
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float use = m[h] == -INFINITY ? 0.f : -m[h];
                ref2[h] = f2_pack(use, use);
            }
            const auto quarter = [&](int c) {
                uint32_t w[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) exponentials(x + 16 * c + 4 * i, w + 2 * i, scale2, ref2, sum2);
                tmem_st_16x128b_x4(t_s + c * 16, w);
            };
            quarter(0);
            quarter(1);
            tmem_st_wait();
            arrive(kP0 + g);
            quarter(2);
            quarter(3);
            tmem_st_wait();
            arrive(kP1 + g);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float a, b;
                f2_unpack(sum2[h], a, b);
                l[h] += a + b;
            }
        }
        v_slot += 2 * n_units;
        const bool had = begin < n_units, both = !two && n_units > 1;
        if (had) {
            if (!wait(kO + g, kOfO, 16)) return;
            tc_fence_after_sync();
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) l[h] = over_row(l[h], sum_of);
        // the rows: of two tiles each stream's own; of one tile those of both streams, added by the first
        if (both && g) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (q == 0) store_pair(sh.at + Shared::kExchange + (r0 + 8 * h) * 8, m[h], l[h]);
            arrive(kX);
            if (!wait(kXFree, kOfX, 32)) return;
            tc_fence_after_sync();
        }
        if (two || !g) {
            float w0[2] = {1.f, 1.f}, w1[2] = {0.f, 0.f};
            if (both) {
                if (!wait(kX, kOfX, 32)) return;
                tc_fence_after_sync();
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float2 o = load_pair(sh.at + Shared::kExchange + (r0 + 8 * h) * 8);
                    const float most = fmaxf(m[h], o.x), use = most == -INFINITY ? 0.f : most;
                    w0[h] = fast_exp2(m[h] - use), w1[h] = fast_exp2(o.x - use);
                    l[h] = l[h] * w0[h] + o.y * w1[h], m[h] = most;
                }
            }
            const int tokens = sh.item(n, kTokens), u0 = sh.item(n, kU0);
            const bool whole = u0 == 0 && sh.item(n, kU1) == sh.item(n, kUnits);
            bool real[2], blind[2];   // (blind: no key; a row that sees keys keeps what their scores made of it, a NaN too)
            size_t row[2], part[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = r0 + 8 * h, token = (two ? g * p.TT : 0) + r / p.G;
                real[h] = r < p.G * p.TT && token < tokens;
                row[h] = (size_t)(sh.item(n, kRow0) + token) * p.Hq + sh.item(n, kHead) * p.G + r % p.G;
                part[h] = ((size_t)blockIdx.x * 2 + (u0 == 0)) * p.slot_rows + (two ? g * 128 : 0) + r;
                blind[h] = sees[h] + 2 * q <= 0;
                const float inv = !whole ? 1.f : 1.f / l[h];
                w0[h] *= inv, w1[h] *= inv;
            }
#pragma unroll 1
            for (int o0 = 0; o0 < 128; o0 += 32) {
                float o[16];   // of O as of S: word 4 i + 2 h + e is row h, dim o0 + 8 i + 2 q + e
#pragma unroll
                for (int i = 0; i < 16; ++i) o[i] = 0.f;
                if (had) {
                    uint32_t x[16];
                    tmem_ld_16x256b_x4(t_o + o0, x);
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[i] = __uint_as_float(x[i]) * w0[i >> 1 & 1];
                }
                if (both) {
                    uint32_t x[16];
                    tmem_ld_16x256b_x4(t_o + 128 + o0, x);
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[i] += __uint_as_float(x[i]) * w1[i >> 1 & 1];
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (whole) {   // 16 bytes a lane, 64 consecutive ones a row
                        uint32_t w[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) w[i] = blind[h] ? 0u : pack_bf16(o[4 * i + 2 * h], o[4 * i + 2 * h + 1]);
                        transpose_4(w, q);
                        if (real[h]) *reinterpret_cast<uint4 *>(p.out + row[h] * 128 + o0 + 8 * q) = make_uint4(w[0], w[1], w[2], w[3]);
                    } else if (real[h]) {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            *reinterpret_cast<float2 *>(p.ws_o + part[h] * 128 + o0 + 8 * i + 2 * q) = make_float2(o[4 * i + 2 * h], o[4 * i + 2 * h + 1]);
                    }
                }
            }
            if (both) arrive(kXFree);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (q || !real[h]) continue;
                if (!whole) p.ws_ml[part[h]] = make_float2(m[h], l[h]);
                else if (p.lse) p.lse[row[h]] = blind[h] ? -INFINITY : (m[h] + log2f(l[h])) * 0.69314718055994531f;
            }
            const int parts = sh.item(n, kParts);
            if (threadIdx.x == 0 && parts) p.cuts[blockIdx.x] = make_int4(sh.item(n, kRow0), tokens, sh.item(n, kHead) | min(max(-sh.item(n, kPos0), 0), tokens) << 16, parts);
        }
        tc_fence_before_sync();
        taken(sh, n);
    }
}

__global__ void __launch_bounds__(kThreads, 1)
    chunk_attn_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                      const __grid_constant__ Params p)
{
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem0 = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t *misc = smem_raw + (smem0 - smem_u32(smem_raw)) + kOffMisc;
    const Shared sh{smem0 + kOffMisc};
    const int tid = threadIdx.x, warp = tid >> 5;

    if (tid == 0) {
#pragma unroll 1
        for (int i = 0; i < kNumBars; ++i) mbar_init(sh.bar(i), arrivals(i));
        mbar_fence_init();
        Shared::store(sh.at + Shared::kAbort, 0);
    }
    if (warp == kSoftmax && (tid & 31) == 0) tma_prefetch_desc(&tm_q), tma_prefetch_desc(&tm_k), tma_prefetch_desc(&tm_v);
    if (warp == kSoftmax + 1) tmem_alloc(sh.at + Shared::kTmem, 512);
    grid_dependency_wait();
    if (tid == 0) p.cuts[blockIdx.x] = make_int4(0, 0, 0, 0);
    ChunkWalk walk(p.batch);
    const bool some = begin_walk(p, walk, reinterpret_cast<long long *>(misc + Shared::kScratch));
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = Shared::load(sh.at + Shared::kTmem);
    if (some) {
        if (warp >= kSoftmax) {
            reg_dealloc<kRegsFew>();
            if (warp == kSoftmax) produce(p, sh, smem0, tm_q, tm_k, tm_v);
            else if (warp == kSoftmax + 1) issue(p, sh, smem0, tmem);
            else if (warp == kSoftmax + 2) hand_out(walk, sh, reinterpret_cast<ChunkItem *>(misc + Shared::kItems), p.status);
        } else {
            reg_alloc<kRegsMany>();
            softmax(p, sh, smem0, tmem, warp >> 3);
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (warp == kSoftmax + 1) {
        // (MMAs that nobody waited for, when a wait gave up)
        if (some && !__all_sync(0xffffffffu, mbar_wait_bounded(sh.bar(kDone), 0)) && p.status) atomicOr(p.status, 4);
        __syncwarp();
        tmem_dealloc(tmem, 512);
    }
    grid_launch_dependents();
}

// A cut item: the partial sums of its shares, which are numbered from the CTA that it begins in.  A warp per row, four dims a lane, four
// shares on their way at once.  Bound by latency: the 148 places where an item may begin, each with all the rows that a partial has room
// for, are more CTAs than there is work for, and most leave after a look at their cut (with four rows a warp one behind the other 1.4 us
// more for a batch of 1,582 tokens, most of them in three chunks).  Launched when the attention's CTAs are through: with the trigger at
// their beginning the calls take 0.5 to 1 us longer, since the merging CTAs then wait beside them.
constexpr int kMergeRows = 8;   // rows of a CTA
__global__ void __launch_bounds__(kMergeRows * 32) chunk_merge_kernel(const __grid_constant__ Params p)
{
    grid_dependency_wait();
    const int cta = blockIdx.x, lane = threadIdx.x & 31;
    const int4 cut = p.cuts[cta];
    if (cut.w == 0) return;
    const bool two = cut.y > p.TT;
    const int at = blockIdx.y * kMergeRows + (int)(threadIdx.x >> 5);
    const int r = at & 127, token = (two ? (at >> 7) * p.TT : 0) + r / p.G;
    if (at >= p.slot_rows || r >= p.G * p.TT || token >= cut.y || (!two && at >= 128)) return;
    SplitSum sum;
    constexpr int U = 4;
    for (int base = 0; base < cut.w; base += U) {
        float2 ml[U];
        float4 o[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const size_t part = ((size_t)(cta + base + k) * 2 + (base + k == 0)) * p.slot_rows + at;
            const bool in = base + k < cut.w;
            ml[k] = in ? __ldcg(p.ws_ml + part) : make_float2(-INFINITY, 0.f);
            o[k] = in ? __ldcg(reinterpret_cast<const float4 *>(p.ws_o + part * 128) + lane) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
        sum.add(ml, o);
    }
    const bool blind = token < (int)((unsigned)cut.z >> 16);
    const size_t row = (size_t)(cut.x + token) * p.Hq + (cut.z & 0xffff) * p.G + r % p.G;
    reinterpret_cast<uint2 *>(p.out + row * 128)[lane] = blind ? make_uint2(0u, 0u) : sum.out();
    if (p.lse && lane == 0) p.lse[row] = blind ? -INFINITY : sum.lse();
}

// Rows of a partial: the rows of the batch where these are one tile at most.
int slot_rows(const sv_geom *g, int32_t n_tokens)
{
    const int64_t rows = (int64_t)(g->n_q_heads / g->n_kv_heads) * n_tokens;
    return rows <= 128 ? (int)std::max<int64_t>(rows, 1) : 256;
}

}  // namespace

extern "C" size_t sv_chunk_workspace_bytes(const sv_geom *geom, int32_t n_tokens)
{
    if (svh::check_ragged(geom, n_tokens) != SV_OK) return 0;
    return (size_t)svh::sm_count() * (sizeof(int4) + 2 * (size_t)slot_rows(geom, n_tokens) * 130 * sizeof(float));
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
    if (!(softmax_scale >= 0.f && softmax_scale < INFINITY)) return SV_ERR_SHAPE;
    if (!svh::aligned(q, 16) || !svh::aligned(out, 16) || !svh::aligned(workspace, 16)) return SV_ERR_ALIGN;
    if (workspace_bytes < sv_chunk_workspace_bytes(geom, n_tokens)) return SV_ERR_WORKSPACE;
    if (!workspace) return SV_ERR_NULL;
    if (n_tokens == 0) return SV_OK;
    const int ctas = svh::sm_count();
    Params p = {};
    p.Hq = geom->n_q_heads, p.Hkv = geom->n_kv_heads, p.B = geom->block_size, p.NBmax = geom->max_blocks;
    p.G = p.Hq / p.Hkv, p.TT = 128 / p.G;
    p.batch = {q_start, kv->seq_lens, geom->n_seq, n_tokens, p.Hkv, p.TT, (long long)p.NBmax * p.B};
    p.n_pages = kv->n_pages, p.slot_rows = slot_rows(geom, n_tokens);
    p.block_table = kv->block_table;
    p.out = static_cast<__nv_bfloat16 *>(out), p.lse = lse, p.status = status_word;
    p.cuts = static_cast<int4 *>(workspace);
    p.ws_o = reinterpret_cast<float *>(p.cuts + ctas);
    p.ws_ml = reinterpret_cast<float2 *>(p.ws_o + (size_t)2 * ctas * p.slot_rows * 128);
    p.scale_log2 = (softmax_scale == 0.f ? 0.08838834764831845f : softmax_scale) * 1.4426950408889634f;
    CUtensorMap tm_q, tm_k, tm_v;
    const int64_t pool_rows = (int64_t)p.n_pages * p.Hkv * p.B;
    if (!rows_tensor_map(q, n_tokens, p.Hq, p.G, p.TT, &tm_q) || !half_rows_tensor_map(kv->k_pool, pool_rows, 1, &tm_k) ||
        !half_rows_tensor_map(kv->v_pool, pool_rows, 2, &tm_v))
        return SV_ERR_CUDA;
    static svh::OncePerDevice once;
    if (once.run([] { return cudaFuncSetAttribute(chunk_attn_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes); }) != cudaSuccess) {
        (void)cudaGetLastError();
        return SV_ERR_CUDA;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmemBytes;
    cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[1];
    svh::pdl_attribute(attr);
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, chunk_attn_kernel, tm_q, tm_k, tm_v, p) != cudaSuccess) return SV_ERR_CUDA;
    cfg.gridDim = dim3(ctas, (p.slot_rows + kMergeRows - 1) / kMergeRows);
    cfg.blockDim = dim3(kMergeRows * 32);
    cfg.dynamicSmemBytes = 0;
    return cudaLaunchKernelEx(&cfg, chunk_merge_kernel, p) == cudaSuccess ? svh::launch_status() : SV_ERR_CUDA;
}
