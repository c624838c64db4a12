"""sv_kv_evict's kernel on the host (simt.h): its threads in several orders, with what nobody wrote in shared memory chosen.  What it does
to the cache is the same in all of them: nothing is read that another thread has yet to write, or that nobody wrote."""
import ctypes
import os
import re
import subprocess

import numpy as np
import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2512_21911_b200", "csrc")
ORDERS = dict(upper_first=0, lower_first=1, one_by_one=2, backwards=3, drawn=4)
DRIVER = r'''
template <int B>
static int evict(const Params &p, int S, int order, int poison, uint8_t *left)
{
    for (int s = 0; s < S; ++s)
        for (int h = 0; h < p.Hkv; ++h) {
            simt::Cluster c;
            c.ctas = kCluster, c.threads = kThreads, c.order = (simt::Order)order, c.seed = 12345;
            const size_t bytes = sizeof(Shared) + ((p.NBmax * B + kCluster - 1) / kCluster + 3) / 4 * 16;
            c.shared.assign(kCluster, std::vector<uint8_t>(bytes, (uint8_t)poison));
            simt::g_block = {0, (unsigned)h, (unsigned)s};
            c.body = [&] { kv_evict_kernel<B>(p); };
            if (!simt::run(c)) return 1;
            if (left) for (const auto &x : c.shared) memcpy(left, x.data(), sizeof(Shared)), left += sizeof(Shared);
        }
    return 0;
}
}  // namespace
extern "C" int shared_bytes() { return sizeof(Shared); }
extern "C" int evict(int B, int S, int Hkv, int NBmax, int n_pages, int n_sink, int n_recent, void *k, void *v, const int *table, const int *lens,
                     const int *budget, const float *w, float *w_out, float *reps, int *lens_out, int *status, int order, int poison, uint8_t *left)
{
    Params p = {};
    p.k_pool = (uint4 *)k, p.v_pool = (uint4 *)v, p.block_table = table, p.seq_lens = lens, p.budget = budget, p.weights = w, p.weights_out = w_out;
    p.reps = reps, p.seq_lens_out = lens_out, p.status = status, p.Hkv = Hkv, p.NBmax = NBmax, p.n_pages = n_pages, p.n_sink = n_sink, p.n_recent = n_recent;
    return B == 64 ? evict<64>(p, S, order, poison, left) : evict<128>(p, S, order, poison, left);
}
'''


def _replace(text, old, new):
    assert text.count(old) == 1, old
    return text.replace(old, new)


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("evict")
    read = lambda name: open(os.path.join(CSRC, name)).read()
    text = read("kv_evict.cu")
    text = text[:text.index("}  // namespace\n\nextern")]
    text = _replace(text, "extern __shared__ __align__(16) uint32_t keys[];", "uint32_t *keys = simt::shared<uint32_t>(sizeof(Shared));")
    text = _replace(text, "__shared__ Shared sh;", "Shared &sh = *simt::shared<Shared>();")
    text = re.sub(r'#include (<cuda_bf16.h>|"attn_common.cuh"|"sv_host.h"|"sv_ptx.cuh")\n', "", text)
    core = _replace(read("evict_core.cuh"), "#include <cooperative_groups.h>", "")
    (d / "evict_core.cuh").write_text(core)
    (d / "order_key.h").write_text(read("order_key.h"))
    (d / "evict.cpp").write_text('#include "simt.h"\n' + text + DRIVER)
    so = d / "evict.so"
    subprocess.run(["g++", "-O1", "-std=c++17", "-w", "-shared", "-fPIC", "-fno-strict-aliasing", "-I", HERE, str(d / "evict.cpp"), "-o", str(so)], check=True)
    lib = ctypes.CDLL(str(so))
    p, i = ctypes.c_void_p, ctypes.c_int
    lib.evict.argtypes = [i] * 7 + [p] * 10 + [i, i, p]
    return lib


def _case(L, n, B, seed=0):
    """One sequence and head: pools of small whole numbers, whose sums are exact."""
    rng, NB = np.random.default_rng(seed), -(-L // B) + 1
    rows = lambda: (rng.integers(-8, 8, (NB + 1, 1, B, 128)).astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)
    return dict(k=rows(), v=rows(), table=rng.permutation(NB + 1)[:NB].astype(np.int32), w=rng.random(NB * B).astype(np.float32), L=L, n=n, B=B, NB=NB)


def _kept(t, sink, recent):
    w = t["w"][:t["L"]].astype(np.float64)
    w[:sink] = w[t["L"] - recent:] = np.inf
    return np.sort(np.argsort(-w, kind="stable")[:t["n"]])


def _run(lib, t, sink, recent, reps, order, poison=0, left=None):
    k, v, w = t["k"].copy(), t["v"].copy(), t["w"].copy()
    ints = lambda x: np.array([x], np.int32)
    lens, budget, lens_out, status = ints(t["L"]), ints(t["n"]), ints(-7), ints(0)
    means = np.full((t["NB"], 128), 99.0, np.float32)
    at = lambda x: None if x is None else x.ctypes.data
    assert lib.evict(t["B"], 1, 1, t["NB"], t["NB"] + 1, sink, recent, at(k), at(v), at(t["table"]), at(lens), at(budget), at(w), at(w),
                     at(means) if reps else None, at(lens_out), at(status), ORDERS[order], poison, at(left)) == 0
    assert int(lens_out[0]) == t["n"] and int(status[0]) == 0
    return k, v, w, means


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("reps", [False, True])
@pytest.mark.parametrize("L,n,B", [(5000, 4500, 64), (4700, 2100, 128), (300, 200, 64)])
def test_every_order_of_the_threads_gives_the_same(lib, order, reps, L, n, B):
    t = _case(L, n, B)
    kept, i = _kept(t, 4, 64), np.arange(n)
    k, v, w, means = _run(lib, t, 4, 64, reps, order)
    rows = lambda pool, at: pool[t["table"][at // B], 0, at % B]
    assert np.array_equal(rows(k, i), rows(t["k"], kept)) and np.array_equal(rows(v, i), rows(t["v"], kept))
    assert np.array_equal(w[:n], t["w"][kept]) and (w[n:L] == 0).all() and np.array_equal(w[L:], t["w"][L:])
    if reps:
        held = (rows(k, i).astype(np.uint32) << 16).view(np.float32)
        want = np.stack([held[b * B:(b + 1) * B].sum(0) / np.float32(min(B, n - b * B)) for b in range(-(-n // B))])
        assert np.array_equal(means[:len(want)], want) and (means[len(want):] == 99.0).all()


@pytest.mark.parametrize("reps", [False, True])
@pytest.mark.parametrize("L,n,sink,recent", [(300, 200, 4, 64), (300, 0, 0, 0), (2500, 2300, 0, 0), (9, 1, 0, 0)])
def test_nothing_is_read_that_nobody_wrote(lib, reps, L, n, sink, recent):
    """What shared memory holds in the end is what it held in the beginning, or does not depend on it."""
    t, left = _case(L, n, 64), [np.zeros((8, lib.shared_bytes()), np.uint8) for _ in range(2)]
    a, b = (_run(lib, t, sink, recent, reps, "drawn", poison, x) for poison, x in zip((0, 0xff), left))
    assert all(np.array_equal(x, y) for x, y in zip(a, b))
    same = left[0] == left[1]
    assert (same | ((left[0] == 0) & (left[1] == 0xff))).all()


def _ranks(w):
    """The order that sv.h states, as numbers: zeros are equal, a NaN goes by its bits, the one of GPU arithmetic stands below zero."""
    bits = w.view(np.uint32)
    rank = np.nan_to_num(w).astype(np.float64)
    rank = np.where(np.isinf(w), np.where(bits >> 31, -1e200, 1e200), rank)
    rank = np.where(np.isnan(w), np.where(bits >> 31, -1e300, 1e300) * (1 + (bits & 0x7fffff) / 2.0 ** 23), rank)
    return np.where(bits == 0x7fffffff, -1e-300, rank)


ODD = [0x00000000, 0x80000000, 0x7fc00000, 0xffc00000, 0x7fffffff, 0xffffffff, 0x7f800000, 0xff800000, 0x00000001, 0x80000001, 0x3f800000, 0xbf800000,
       0x7f800001]


@pytest.mark.parametrize("values", [ODD, ODD[:2], ODD[:2] + ODD[4:5], ODD[4:5] + ODD[9:10]])
@pytest.mark.parametrize("n", [250, 60, 7])
def test_order_of_odd_weights(lib, values, n):
    t = _case(300, n, 64)
    t["w"][:300] = np.random.default_rng(1).choice(np.array(values, np.uint32), 300).view(np.float32)
    kept = np.sort(np.argsort(-_ranks(t["w"][:300]), kind="stable")[:n])
    k, v, w, _ = _run(lib, t, 0, 0, False, "drawn")
    rows = lambda pool, at: pool[t["table"][at // 64], 0, at % 64]
    assert np.array_equal(w[:n].view(np.uint32), t["w"][kept].view(np.uint32))
    assert np.array_equal(rows(k, np.arange(n)), rows(t["k"], kept)) and np.array_equal(rows(v, np.arange(n)), rows(t["v"], kept))
