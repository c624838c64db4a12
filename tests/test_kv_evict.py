"""sv_kv_evict against sorting on the host: which tokens stay, where they go, their weights, the lengths and representatives.  Everything is
a copy, and the representatives are those of sv_block_reps: compared bit for bit."""
import numpy as np
import pytest
import torch


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _inputs(lens, Hkv, B, budget, seed=0, weights=None):
    rng, S = np.random.default_rng(seed), len(lens)
    NB = max(1, max(-(-n // B) for n in lens)) + 2
    pool = lambda: torch.from_numpy(rng.integers(-2 ** 15, 2 ** 15, (S * NB + 3, Hkv, B, 128)).astype(np.int16)).cuda().view(torch.bfloat16).nan_to_num_(1.0, 2.0, 3.0)
    w = np.exp(2 * rng.normal(size=(S, Hkv, NB * B))).astype(np.float32) if weights is None else weights(rng, (S, Hkv, NB * B)).astype(np.float32)
    return dict(k=pool(), v=pool(), table=torch.from_numpy(rng.permutation(S * NB + 3)[:S * NB].astype(np.int32).reshape(S, NB)).cuda(), lens=_ints(lens),
                w=torch.from_numpy(w).cuda(), budget=_ints(budget), lens_out=_ints([-7] * S), status=_ints([0]),
                reps=torch.from_numpy(rng.normal(size=(S, Hkv, NB, 128)).astype(np.float32)).cuda(), dims=(S, Hkv, B, NB))


def _order(w):
    """The order that sv.h states, as whole numbers."""
    b = w.view(np.uint32).astype(np.int64)
    key = np.where(b >> 31, 0xffffffff - b, b + 0x80000000)
    return np.where(key == 0xffffffff, 0x7fffffff, key)


def _expected(t, sink, recent):
    """What everything is afterwards."""
    S, Hkv, B, NB = t["dims"]
    bits = lambda x: x.view(torch.int16).cpu().numpy().copy()
    k, v, w, table = bits(t["k"]), bits(t["v"]), t["w"].cpu().numpy(), t["table"].cpu().numpy()
    w_out, lens, kept_of = np.full(w.shape, -3.0, np.float32), [], {}
    for s in range(S):
        held = int(t["lens"][s])
        L = min(max(held, 0), NB * B)
        n = min(L, max(int(t["budget"][s]), min(L, sink + recent)))
        lens.append(n if n < L else held)
        for h in range(Hkv):
            key = _order(w[s, h, :L])
            key[:sink] = 1 << 40
            key[max(0, L - recent):] = 1 << 40
            kept = np.sort(np.argsort(-key, kind="stable")[:n])
            w_out[s, h, :L] = 0
            w_out[s, h, :n] = w[s, h, kept]
            at = np.arange(n)
            for pool in (k, v):
                pool[table[s, at // B], h, at % B] = pool[table[s, kept // B], h, kept % B]
            kept_of[s, h] = kept
    return k, v, w_out, lens, kept_of


def _run(sv, t, sink, recent, reps=True, in_place=False):
    S, Hkv, B, NB = t["dims"]
    geom = sv.make_geom(S, 2 * Hkv, Hkv, 128, B, NB, 1)
    out = t["w"] if in_place else torch.full_like(t["w"], -3.0)
    sv.sv_kv_evict(geom, t["k"], t["v"], t["table"], t["lens"], t["w"], t["budget"], sink, recent, t["lens_out"], out, reps=t["reps"] if reps else None,
                   status_word=t["status"])
    return out


def _check(sv, t, sink, recent, in_place=False, reps=True):
    S, Hkv, B, NB = t["dims"]
    k, v, w_out, lens, _ = _expected(t, sink, recent)
    reps_before, lens_before = t["reps"].clone(), t["lens"].tolist()
    out = _run(sv, t, sink, recent, reps, in_place)
    assert int(t["status"]) == 0 and t["lens_out"].tolist() == lens
    assert np.array_equal(t["k"].view(torch.int16).cpu().numpy(), k) and np.array_equal(t["v"].view(torch.int16).cpu().numpy(), v)
    got, held = out.cpu().numpy(), np.arange(NB * B) < np.minimum(np.maximum(np.array(lens_before), 0), NB * B)[:, None, None]
    held = np.broadcast_to(held, got.shape)
    assert np.array_equal(got[held].view(np.int32), w_out[held].view(np.int32)) and (in_place or (got[~held] == -3.0).all())
    want = torch.zeros_like(t["reps"])
    geom = sv.make_geom(S, 2 * Hkv, Hkv, 128, B, NB, 1)
    sv.sv_block_reps(geom, sv.make_kv(t["k"], t["v"], t["table"], t["lens_out"]), want)
    for s in range(S):
        shrank = reps and lens[s] < lens_before[s]
        n = -(-lens[s] // B) if shrank else 0
        bits = lambda x: x.view(torch.int32)   # (a mean may be a NaN)
        assert torch.equal(bits(t["reps"])[s, :, :n], bits(want)[s, :, :n]) and torch.equal(t["reps"][s, :, n:], reps_before[s, :, n:])


CASES = [([1], 1, 64, [1], 0, 0), ([1], 1, 64, [0], 0, 0), ([100, 64, 65, 3], 2, 64, [50, 63, 64, 1], 4, 10), ([1000, 300, 0], 3, 128, [300, 299, 5], 0, 1),
         ([5000], 2, 64, [77], 17, 40), ([4097, 4096], 2, 128, [4096, 4095], 1, 1), ([700, 800], 2, 64, [10, 1000], 0, 0), ([3000], 1, 64, [10], 300, 500),
         ([100, 100], 2, 64, [-5, 20], 60, 60), ([20000, 9000], 2, 64, [2500, 8999], 4, 64), ([1025], 1, 128, [1], 0, 0)]


@pytest.mark.gpu
@pytest.mark.parametrize("lens,Hkv,B,budget,sink,recent", CASES)
@pytest.mark.parametrize("in_place", [False, True])
def test_evict(lens, Hkv, B, budget, sink, recent, in_place):
    import paper_2512_21911_b200 as sv
    _check(sv, _inputs(lens, Hkv, B, budget), sink, recent, in_place)


@pytest.mark.gpu
@pytest.mark.parametrize("weights", [
    lambda r, s: np.zeros(s), lambda r, s: r.integers(0, 3, s), lambda r, s: -np.abs(r.normal(size=s)), lambda r, s: r.normal(size=s) * 1e-42,
    lambda r, s: np.where(r.random(s) < 0.3, np.nan, r.normal(size=s)), lambda r, s: np.where(r.random(s) < 0.3, np.inf, np.where(r.random(s) < 0.5, -np.inf, -0.0)),
    lambda r, s: 1.0 + r.integers(0, 40, s) * 2.0 ** -23, lambda r, s: np.full(s, np.nan)])
def test_weights_that_are_equal_or_odd(weights):
    """Equal ones, neighbours, negative and subnormal ones, NaN and infinities: the order is that of the numbers' keys, ties the earlier."""
    import paper_2512_21911_b200 as sv
    _check(sv, _inputs([3000, 517, 64], 2, 64, [1000, 100, 63], weights=weights), 3, 70)


@pytest.mark.gpu
def test_without_representatives_and_the_longest_table():
    import paper_2512_21911_b200 as sv
    _check(sv, _inputs([700], 2, 64, [300]), 4, 64, reps=False)
    t = _inputs([900], 1, 64, [400])
    S, Hkv, B, NB = t["dims"]
    wide = 6144                                # 393,216 tokens
    t["table"] = torch.cat([t["table"], torch.full((1, wide - NB), -1, dtype=torch.int32, device="cuda")], 1)
    t["w"] = torch.cat([t["w"], torch.zeros((1, 1, (wide - NB) * B), device="cuda")], 2)
    t["reps"] = torch.cat([t["reps"], torch.zeros((1, 1, wide - NB, 128), device="cuda")], 2)
    t["dims"] = (1, 1, 64, wide)
    _check(sv, t, 4, 64)


@pytest.mark.gpu
def test_a_long_sequence_fills_the_shared_memory():
    """393,216 tokens: every key of a CTA's slice has its place, and the runs of its warps all their words."""
    import paper_2512_21911_b200 as sv
    rng = np.random.default_rng(0)
    L, B = 393216, 128
    t = dict(k=torch.randn((L // B, 1, B, 128), device="cuda").bfloat16(), v=torch.randn((L // B, 1, B, 128), device="cuda").bfloat16(),
             table=torch.from_numpy(rng.permutation(L // B).astype(np.int32)[None]).cuda(), lens=_ints([L]), budget=_ints([100001]), lens_out=_ints([0]),
             status=_ints([0]), w=torch.rand((1, 1, L), device="cuda"), reps=torch.zeros((1, 1, L // B, 128), device="cuda"), dims=(1, 1, B, L // B))
    _check(sv, t, 4, 64)


@pytest.mark.gpu
def test_rows_without_a_page_are_left_out():
    import paper_2512_21911_b200 as sv
    t = _inputs([600], 1, 64, [200])
    t["table"][0, 2], t["table"][0, 7] = -1, t["k"].shape[0]
    used = {int(x) for i, x in enumerate(t["table"][0, :4].tolist()) if i != 2}
    before = t["k"].view(torch.int16).clone()
    _run(sv, t, 4, 64)
    assert int(t["status"]) == sv.SV_STATUS_INDEX and t["lens_out"].tolist() == [200]
    for page in set(range(before.shape[0])) - used:
        assert torch.equal(t["k"].view(torch.int16)[page], before[page])


@pytest.mark.gpu
def test_captured_and_on_another_stream():
    import paper_2512_21911_b200 as sv
    a, b = (_inputs([3000, 500], 2, 64, [700, 600]) for _ in range(2))
    wa = _run(sv, a, 4, 64)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        wb = _run(sv, b, 4, 64)
    graph.replay()
    torch.cuda.synchronize()
    same = lambda x, y: torch.equal(x.view(torch.int16), y.view(torch.int16))
    assert same(a["k"], b["k"]) and same(a["v"], b["v"]) and torch.equal(wa[:, :, :500], wb[:, :, :500]) and same(a["reps"], b["reps"])


def test_peers_are_reached_behind_the_barrier():
    """A CTA may reach a peer's shared memory only once the peer runs, and leaves when no peer reaches its own any more."""
    import os
    import re
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2512_21911_b200", "csrc")
    core, kernel = (re.sub(r"//[^\n]*", "", open(os.path.join(csrc, f)).read()) for f in ("evict_core.cuh", "kv_evict.cu"))
    first = core.index("keep_heaviest(")
    assert "map_shared_rank" not in core[:first] and core.index("cluster.sync()", first) < core.index("map_shared_rank", first)
    body = kernel[kernel.index("kv_evict_kernel("):]
    assert "map_shared_rank" not in body
    assert body.index("keep_heaviest(") < body.index("source_of(") < body.rindex("cluster.sync()")
