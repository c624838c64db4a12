"""How sv_chunk_attn divides a ragged batch among CTAs (chunk_shares.h, the arithmetic the kernel runs, compiled for the host): every unit
of every item is in exactly one share, the shares of a cut item are neighbours and none of them is empty, a CTA writes at most one partial
of an item that began before and one of an item that goes on, and the shares are even."""
import ctypes
import os
import random
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2512_21911_b200", "csrc")
SOURCE = r'''
#include "chunk_shares.h"
using namespace svk;
extern "C" int item_cost() { return kItemCost; }
extern "C" int shares_of(const int32_t *q_start, const int32_t *lens, int S, int N, int Hkv, int TT, long long cap, int ctas, int cta, int32_t *out, int room)
{
    const ChunkBatch b{q_start, lens, S, N, Hkv, TT, cap};
    ChunkWalk w(b);
    long long total = 0;
    for (int i = 0; i < S; ++i) w.load(i), total += w.per_head() * Hkv;
    if (!w.divide(total, ctas, cta)) return 0;
    long long ahead = 0;
    for (int i = 0; i < S; ++i) {
        w.load(i);
        const long long cost = w.per_head() * Hkv;
        if (cost > 0 && ahead <= w.lo && w.lo < ahead + cost) {
            w.enter(i, ahead);
            break;
        }
        ahead += cost;
    }
    int n = 0;
    for (ChunkItem it; n < room && w.next(it); ++n) {
        const int v[10] = {it.s, it.h, it.row0, it.tokens, it.pos0, it.kv_end, it.u0, it.u1, it.units, it.parts};
        for (int i = 0; i < 10; ++i) out[n * 10 + i] = v[i];
    }
    return n;
}
'''


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("shares")
    src, so = d / "shares.cpp", d / "shares.so"
    src.write_text(SOURCE)
    subprocess.run(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, str(src), "-o", str(so)], check=True)
    lib = ctypes.CDLL(str(so))
    lib.shares_of.argtypes = [ctypes.c_void_p] * 2 + [ctypes.c_int] * 4 + [ctypes.c_longlong] + [ctypes.c_int] * 2 + [ctypes.c_void_p, ctypes.c_int]
    return lib


def _check(lib, lens, new, Hkv, G, cap, ctas):
    S, TT = len(lens), 128 // G
    start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    lens = np.array(lens, np.int32)
    buf = np.zeros((1 << 16, 10), np.int32)
    covered, first_of, work = {}, {}, []
    for cta in range(ctas):
        n = lib.shares_of(start.ctypes.data, lens.ctypes.data, S, int(start[-1]), Hkv, TT, cap, ctas, cta, buf.ctypes.data, len(buf))
        begun = going = 0
        work.append(0)
        for s, h, row0, tokens, pos0, kv_end, u0, u1, units, parts in buf[:n].tolist():
            key = (s, h, row0)
            covered.setdefault(key, []).append((cta, u0, u1, units, parts, tokens))
            assert start[s] <= row0 and row0 + tokens <= start[s + 1] and 0 < tokens <= 2 * TT and 0 <= h < Hkv
            assert pos0 == lens[s] - new[s] + row0 - start[s] and kv_end == max(0, min(pos0 + tokens, cap)) and units == -(-kv_end // 128)
            assert 0 <= u0 <= u1 <= units and (u0 < u1 or units == 0)
            begun += u0 > 0
            going += u0 == 0 and u1 < units
            # on the line a whole item is less than 128 keys shorter than its units; a cut lies less than a unit behind its place on the line,
            # so that a share that begins at a cut has that unit too (and, where it ends with the item, both)
            work[-1] += (2 if tokens > TT else 1) * max(0, (u1 - u0) * 128 - (256 if u0 > 0 and u1 == units else 128))
        assert begun <= 1 and going <= 1
    # every token of every head, every unit once
    for s in range(S):
        for h in range(Hkv):
            rows = sorted(k[2] for k in covered if k[:2] == (s, h))
            assert rows == list(range(start[s], start[s + 1], 2 * TT))
    for key, shares in covered.items():
        units = shares[0][3]
        at = 0
        for i, (cta, u0, u1, _, parts, _) in enumerate(shares):
            assert u0 == at and cta == shares[0][0] + i
            assert parts == (len(shares) if i == 0 and len(shares) > 1 else 0)
            at = u1
        assert at == units
    return work


@pytest.mark.parametrize("lens,new,Hkv,G,cap", [
    ([4096], [1], 2, 4, 1 << 20), ([1], [1], 1, 1, 64), ([8192], [8192], 8, 4, 1 << 20), ([32049], [2048], 8, 8, 1 << 20),
    ([5000] * 16, [1] * 16, 8, 4, 1 << 20), ([10, 0, 300, 7000], [10, 0, 0, 3], 4, 7, 1 << 20), ([-5, 3, 400], [3, 10, 2], 2, 128, 1 << 20),
    ([1000, 90000], [500, 1], 2, 4, 640), ([0, 0], [4, 4], 3, 5, 64)])
@pytest.mark.parametrize("ctas", [1, 7, 148])
def test_every_unit_is_in_one_share(lib, lens, new, Hkv, G, cap, ctas):
    _check(lib, lens, new, Hkv, G, cap, ctas)


def test_drawn_batches(lib):
    rng = random.Random(0)
    for _ in range(60):
        S = rng.randint(1, 40)
        new = [rng.choice([0, 1, 1, rng.randint(1, 100), rng.randint(1, 2000)]) for _ in range(S)]
        lens = [n + rng.choice([0, rng.randint(0, 300), rng.randint(0, 20000), -3]) for n in new]
        _check(lib, lens, new, rng.randint(1, 8), rng.choice([1, 2, 3, 4, 7, 8, 32, 128]), rng.choice([1 << 20, 4096]), rng.choice([148, 64, 3]))


def test_shares_are_even(lib):
    """No CTA has more than the line's length / CTAs, but for the rounding to units that _check has taken off."""
    item_cost = lib.item_cost()
    for lens, new, Hkv, G in (([8192], [8192], 8, 4), ([9000, 300, 16000, 5], [1, 1, 1, 1], 8, 4), ([3000, 5000, 100], [700, 1, 100], 4, 7)):
        TT = 128 // G
        line = Hkv * sum((2 if n - t > TT else 1) * (L - n + min(n, t + 2 * TT)) + item_cost for L, n in zip(lens, new) for t in range(0, n, 2 * TT))
        assert max(_check(lib, lens, new, Hkv, G, 1 << 20, 148)) <= line / 148 + 1
