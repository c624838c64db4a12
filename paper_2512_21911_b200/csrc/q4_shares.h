// How the attention over a 4-bit cache divides a batch among its workers (plain C++: the same arithmetic runs in the kernel and in its
// test).
//
// An entry is a (sequence, KV head); it has `tiles` items, tiles of query rows, of which item i costs a + b (i + 1): with b = 0 the rows of
// a draft, which all see the same keys, else those of a chunk, of which each tile sees `b / den` keys more than the one before.  An item
// has `units` of 128 keys and costs, in keys times den, what they are and kItemCost.  The items of all entries lie one behind the other on
// a line, which is cut into equal shares.  Where an item is cut follows from the share's bounds alone, so neighbours agree without talking
// to one another.
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define SVQ_HD __host__ __device__ __forceinline__
#else
#define SVQ_HD inline
#endif

namespace svq {

constexpr int kUnit = 128;        // keys of a unit, the grain of a cut
constexpr int kMostBlocks = 1 << 25;   // blocks that a table of less than 2^31 tokens may have, and a list that names none twice
constexpr int kItemCost = 128;    // keys that the beginning and the end of an item cost as much as

struct Entry {
    long long a, b;
    int tiles;
    SVQ_HD long long before(long long i) const { return i * a + b * (i * (i + 1) / 2); }   // cost of the items ahead of item i
    SVQ_HD long long cost(long long i) const { return a + b * (i + 1); }
    SVQ_HD long long all() const { return before(tiles); }
    // the item that x falls in
    SVQ_HD int item_at(long long x) const
    {
        int lo = 0, hi = tiles - 1;
        if (b == 0) return a > 0 && x / a < hi ? (int)(x / a) : hi;
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if (before(mid) <= x) lo = mid;
            else hi = mid - 1;
        }
        return lo;
    }
};

// `shares` equal parts of a line; a part is never shorter than a unit.
struct Line {
    long long total;
    int shares;
    SVQ_HD Line(long long all, int workers, int den, int least) : total(all), shares(workers)
    {
        const long long most = all / ((long long)least * den + 1);
        if (most < shares) shares = most < 1 ? 1 : (int)most;
    }
    SVQ_HD long long bound(int i) const { return total * i / shares; }
    // the first share that ends at x or behind it
    SVQ_HD int share_to(long long x) const { return (int)((x * shares + total - 1) / total) - 1; }
};

// The part of an item that lies between lo and hi of the line, the item beginning at `at`.
struct Part {
    int u0, u1;    // units
    int parts;     // where the item is cut and this is its first part: how many there are
    bool mine;     // there is something to do
};
SVQ_HD int unit_at(long long x, long long cost, int units, int den)
{
    if (x >= cost) return units;
    const long long first = (long long)kItemCost * den;
    if (x <= first) return 0;
    const long long u = (x - first) / ((long long)kUnit * den);
    return u < units ? (int)u : units;
}
SVQ_HD Part part_of(const Line &line, int share, long long at, long long cost, int units, int den)
{
    const long long x0 = line.bound(share) - at, x1 = line.bound(share + 1) - at;
    Part p;
    p.u0 = x0 <= 0 ? 0 : unit_at(x0, cost, units, den);
    p.u1 = x1 <= 0 ? 0 : unit_at(x1, cost, units, den);
    p.mine = p.u1 > p.u0 || (units == 0 && x0 <= 0 && x1 > 0);
    p.parts = 0;
    if (p.u0 == 0 && p.u1 > 0 && p.u1 < units) {
        const long long whole = ((long long)kItemCost + (long long)kUnit * units) * den;
        p.parts = line.share_to(at + (whole < cost ? whole : cost)) - share + 1;
    }
    return p;
}

}  // namespace svq
