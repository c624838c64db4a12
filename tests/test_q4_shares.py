"""How the attention over a 4-bit cache divides a batch among its workers (q4_shares.h, the arithmetic the kernels run, compiled for the
host): every unit of every item is in exactly one share, the shares of a cut item are neighbours and none of them is empty, a worker writes
at most one partial of an item that began before and one of an item that goes on, and the shares are even."""
import ctypes
import os
import random
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2512_21911_b200", "csrc")
SOURCE = r'''
#include "q4_shares.h"
using namespace svq;
extern "C" int item_cost() { return kItemCost; }
// entries: a, b, tiles; units of their items one after the other.  out: entry, item, u0, u1, parts
extern "C" int parts_of(const long long *entries, const int *units, int n, int den, int workers, int share, int *out, int room)
{
    long long total = 0;
    for (int e = 0; e < n; ++e) total += Entry{entries[3 * e], entries[3 * e + 1], (int)entries[3 * e + 2]}.all();
    const Line line(total, workers, den, kUnit);
    if (share >= line.shares || total == 0) return -1;
    const long long lo = line.bound(share), hi = line.bound(share + 1);
    int found = 0;
    long long at = 0;
    for (int e = 0; e < n; ++e) {
        const Entry x{entries[3 * e], entries[3 * e + 1], (int)entries[3 * e + 2]};
        if (at < hi && at + x.all() > lo && x.tiles) {
            int t = at >= lo ? 0 : x.item_at(lo - at);
            for (long long i_at = at + x.before(t); t < x.tiles && i_at < hi; i_at += x.cost(t), ++t) {
                const Part p = part_of(line, share, i_at, x.cost(t), units[t], den);
                if (p.mine && found < room) {
                    const int v[5] = {e, t, p.u0, p.u1, p.parts};
                    for (int i = 0; i < 5; ++i) out[5 * found + i] = v[i];
                    ++found;
                }
            }
        }
        at += x.all();
        units += x.tiles;
    }
    return found;
}
'''


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("shares")
    src, so = d / "shares.cpp", d / "shares.so"
    src.write_text(SOURCE)
    subprocess.run(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, str(src), "-o", str(so)], check=True)
    lib = ctypes.CDLL(str(so))
    lib.parts_of.argtypes = [ctypes.c_void_p] * 2 + [ctypes.c_int] * 4 + [ctypes.c_void_p, ctypes.c_int]
    return lib


def _drafts(slabs, tiles, cost):
    """Entries whose items all see the same keys: units of the cached slabs and one of the draft."""
    units = [(n + 1) // 2 + 1 for n in slabs]
    return [(cost + 128 * u, 0, tiles) for u in units], [[u] * tiles for u in units], 1


def _chunks(lens, new, Hkv, G, N, cap, cost):
    """Entries whose item i sees the keys up to the last of its rows."""
    entries, units = [], []
    for L, n in zip(lens, new):
        tiles = -(-n * G // N)
        for _ in range(Hkv):
            entries.append((G * (min(max(L - n, 0), cap) + cost), N, tiles))
            ends = [L - n + (min(n * G, (i + 1) * N) - 1) // G + 1 for i in range(tiles)]
            units.append([-(-min(max(e, 0), min(max(L, 0), cap)) // 128) for e in ends])
    return entries, units, G


def _check(lib, entries, units, den, workers):
    flat = np.array([x for e in entries for x in e], np.int64)
    u = np.array([x for item in units for x in item] + [0], np.int32)
    buf = np.zeros((len(u) + 2, 5), np.int32)   # (what a share may have at most)
    parts, work = {}, []
    for share in range(workers):
        n = lib.parts_of(flat.ctypes.data, u.ctypes.data, len(entries), den, workers, share, buf.ctypes.data, len(buf))
        if n < 0:
            continue
        work.append(0)
        before = behind = 0
        for e, t, u0, u1, count in buf[:n].tolist():
            parts.setdefault((e, t), []).append((share, u0, u1, count))
            before += u0 > 0
            behind += u0 == 0 and u1 < units[e][t]
            work[-1] += u1 - u0
        assert before <= 1 and behind <= 1
    assert set(parts) == {(e, t) for e, x in enumerate(entries) for t in range(x[2])}
    for (e, t), got in parts.items():
        at = 0
        for i, (share, u0, u1, count) in enumerate(got):
            assert u0 == at and (u1 > u0 or units[e][t] == 0) and share == got[0][0] + i
            assert count == (len(got) if i == 0 and len(got) > 1 else 0)
            at = u1
        assert at == units[e][t]
    return work


@pytest.mark.parametrize("workers", [1, 7, 296, 592])
def test_every_unit_is_in_one_part(lib, workers):
    cost = lib.item_cost()
    for slabs, tiles in (([64] * 8, 1), ([0], 1), ([0, 1, 2, 3], 5), ([2048] * 32, 1), ([1] * 1000, 2), ([5, 0, 700], 8)):
        _check(lib, *_drafts(slabs, tiles, cost), workers)
    for lens, new, Hkv, G, N in (([4096], [1], 2, 4, 16), ([8192], [8192], 8, 4, 64), ([10, 0, 300, 7000], [10, 0, 0, 3], 4, 7, 64),
                                 ([-5, 3, 400], [3, 10, 2], 2, 128, 64), ([1000, 90000], [500, 1], 2, 4, 64), ([4, 4], [4, 4], 3, 5, 32)):
        for cap in (1 << 20, 640):
            _check(lib, *_chunks(lens, new, Hkv, G, N, cap, cost), workers)


def test_drawn_batches(lib):
    rng, cost = random.Random(0), lib.item_cost()
    for _ in range(60):
        S = rng.randint(1, 40)
        workers = rng.choice([592, 296, 64, 3])
        _check(lib, *_drafts([rng.choice([0, 1, rng.randint(2, 40), rng.randint(40, 900)]) for _ in range(S)], rng.randint(1, 4), cost), workers)
        new = [rng.choice([0, 1, 1, rng.randint(1, 100), rng.randint(1, 2000)]) for _ in range(S)]
        lens = [n + rng.choice([0, rng.randint(0, 300), rng.randint(0, 20000), -3]) for n in new]
        _check(lib, *_chunks(lens, new, rng.randint(1, 8), rng.choice([1, 3, 4, 7, 8, 32, 128]), rng.choice([16, 32, 64]), rng.choice([1 << 20, 4096]), cost),
               workers)


def test_shares_are_even(lib):
    """No worker has more than the line's length / workers, but for a unit at either end."""
    cost = lib.item_cost()
    for slabs, tiles in (([512] * 8, 1), ([100, 2000, 7, 900] * 8, 2)):
        entries, units, den = _drafts(slabs, tiles, cost)
        assert max(_check(lib, entries, units, den, 592)) <= sum(a * t for a, _, t in entries) / 592 / 128 + 2
