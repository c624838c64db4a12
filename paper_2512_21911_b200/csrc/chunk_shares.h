// How sv_chunk_attn divides a ragged batch among its CTAs (plain C++: the same arithmetic runs in the kernel and in its test).
//
// An item is up to 2 * TT tokens of a (sequence, KV head) and costs the keys it sees -- twice where it is two row tiles, whose streams
// both take every unit -- plus kItemCost.  The items of the batch, by sequence, KV head and place, lie one behind the other on a line,
// which is cut into equal shares.  Where an item is cut follows from the share's bounds alone, so neighbours agree without talking to one
// another.  Costs are whole numbers with closed sums: no table is needed.
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define SV_HD __host__ __device__ __forceinline__
#else
#define SV_HD inline
#endif

namespace svk {

constexpr int kChunkUnit = 128;   // keys of a unit, the grain of a cut
// A unit of two tiles takes 3900 cycles, of one tile 1900 (a prompt of 8K; single tokens whose keys are in L2), an item's beginning and end
// 5000, and more where they wait for nothing else (512 against 320: a ragged batch 104.7 -> 100.6 us, the prompt 515 -> 512).
constexpr int kItemCost = 512;    // keys (of one tile) that the beginning and the end of an item cost as much as
constexpr int kLeastShare = 256;  // ... of the shortest share worth a CTA; a unit of two tiles, so that no share inside an item is empty

struct ChunkBatch {
    const int32_t *q_start, *seq_lens;
    int S, N, Hkv, TT;
    long long cap;   // keys that the block table has room for
};

// A CTA's share of an item.
struct ChunkItem {
    int s, h, row0, tokens;   // sequence, KV head, first row of q, tokens of both tiles
    int pos0, kv_end;         // position of the first token; keys seen by any row
    int u0, u1, units;        // units of the share and of the whole item
    int parts;                // where the item is cut and begins here: its shares
    SV_HD bool whole() const { return u0 == 0 && u1 == units; }
};

// The items of a share, in order.
struct ChunkWalk {
    const ChunkBatch &b;
    long long total, lo, hi, at;   // on the line; `at`: where the next item begins
    int shares, mine;
    int s, h, t, n, row, prefix, tiles;   // next item: sequence (its tokens, first row, tokens cached before, items per head), KV head, number

    SV_HD explicit ChunkWalk(const ChunkBatch &b) : b(b) {}
    SV_HD static long long least(long long x, long long y) { return x < y ? x : y; }
    SV_HD int start(int i) const
    {
        const int x = b.q_start[i];
        return x < 0 ? 0 : x > b.N ? b.N : x;
    }
    SV_HD void load(int i)
    {
        s = i, row = start(i), n = start(i + 1) - row;
        if (n < 0) n = 0;
        prefix = b.seq_lens[i] - n, tiles = (n + 2 * b.TT - 1) / (2 * b.TT);
    }
    SV_HD long long seen_before() const { return prefix < 0 ? 0 : least(prefix, b.cap); }
    // cost of a key of item i of a KV head, of the items before it (two tiles each), of itself, of all of them
    SV_HD int weight(int i) const { return n - i * 2 * b.TT > b.TT ? 2 : 1; }
    SV_HD long long before(long long i) const { return i * (2 * seen_before() + kItemCost) + 2 * b.TT * i * (i + 1); }
    SV_HD long long cost(int i) const { return weight(i) * (seen_before() + least(n, (i + 1) * 2ll * b.TT)) + kItemCost; }
    SV_HD long long per_head() const { return n ? before(tiles - 1) + cost(tiles - 1) : 0; }
    SV_HD long long bound(int share) const { return total * share / shares; }

    // Of a line of this length among `ctas`: the share of number `cta`, if it has one.
    SV_HD bool divide(long long all, int ctas, int cta)
    {
        total = all, mine = cta;
        shares = (int)least(ctas, all / kLeastShare);
        if (shares < 1) shares = 1;
        if (all == 0 || cta >= shares) return false;
        lo = bound(cta), hi = bound(cta + 1);
        return true;
    }
    // The share begins in sequence i, whose items begin at `begin`.
    SV_HD void enter(int i, long long begin)
    {
        load(i);
        const long long one = per_head();
        h = (int)((lo - begin) / one);
        at = begin + h * one;
        int a = 0, z = tiles - 1;
        while (a < z) {
            const int mid = (a + z + 1) / 2;
            if (at + before(mid) <= lo) a = mid;
            else z = mid - 1;
        }
        t = a, at += before(a);
    }
    // the unit at x behind the beginning of an item of this cost
    SV_HD static int unit_at(long long x, long long cost, int weight, int units)
    {
        return x >= cost ? units : x <= kItemCost ? 0 : (int)least(units, (x - kItemCost) / (weight * kChunkUnit));
    }
    SV_HD bool next(ChunkItem &it)
    {
        while (s < b.S && at < hi) {
            const long long c = cost(t), x0 = lo - at, x1 = hi - at;
            const int t0 = t * 2 * b.TT, w = weight(t);
            it.s = s, it.h = h, it.row0 = row + t0, it.tokens = (int)least(2 * b.TT, n - t0), it.pos0 = prefix + t0;
            const long long end = least((long long)it.pos0 + it.tokens, b.cap);
            it.kv_end = end < 0 ? 0 : (int)end;
            it.units = (it.kv_end + kChunkUnit - 1) / kChunkUnit;
            it.u0 = unit_at(x0, c, w, it.units), it.u1 = unit_at(x1, c, w, it.units);
            it.parts = 0;
            if (it.u0 == 0 && it.u1 > 0 && it.u1 < it.units) {
                it.parts = 1;
                for (int share = mine + 1, u = it.u1; u < it.units; ++share, ++it.parts) u = unit_at(bound(share + 1) - at, c, w, it.units);
            }
            const bool take = it.u1 > it.u0 || (it.units == 0 && x0 <= 0);
            at += c;
            if (++t == tiles) {
                t = 0;
                if (++h == b.Hkv) {
                    h = 0;
                    do {
                        if (++s < b.S) load(s);
                    } while (s < b.S && n == 0);
                }
            }
            if (take) return true;
        }
        return false;
    }
};

}  // namespace svk
