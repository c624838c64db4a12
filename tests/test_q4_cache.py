"""sv_rope_append_q4, sv_kv_append_q4, sv_kv_read_q4: rows into a 4-bit cache and back, against the plain form of tests/q4_reference.py.

Coding is defined step by step in fp32 and rotated keys are those of sv_rope_append, so the bytes of a cache are compared bit for bit;
what is not a new token's keeps the bytes it had.  Representatives are sums of at most 128 values in fp32 in another order than the
reference's 64 bits: off by at most 128 2^-24 of the mean of the absolute values."""
import numpy as np
import pytest
import torch

from q4_reference import SLAB, bf16, get, put

CASES = [  # before, new, Hq, Hkv, B, rot, interleaved, fused
    ([0], [1], 4, 2, 64, 128, False, True),
    ([63], [2], 4, 2, 64, 128, True, False),
    ([0, 5, 64, 127, 40], [130, 0, 1, 66, 24], 8, 2, 64, 64, False, True),
    ([31, 100, 128, 0], [33, 28, 129, 1], 7, 1, 128, 32, True, True),
    ([200, 0, 64], [1, 300, 64], 6, 3, 128, 0, False, False),
    ([0], [1100], 4, 1, 64, 128, False, True)]


def _batch(sv, before, new, Hq, Hkv, B, rot, fused, seed=0, spare=1):
    """Inputs of a ragged batch, the pool filled with other bytes so that every stray write shows."""
    S, N = len(before), sum(new)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    NB = max(-(-(b + n) // B) for b, n in zip(before, new)) + spare
    table = torch.from_numpy(np.random.default_rng(seed).permutation(S * NB).astype(np.int32).reshape(S, NB)).cuda()
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    t = dict(pool=torch.randint(0, 120, (S * NB, Hkv, B // 64, SLAB), generator=gen, device="cuda", dtype=torch.uint8), table=table, lens=ints(before),
             start=ints(np.concatenate([[0], np.cumsum(new)]).tolist()), lens_out=ints([-7] * S), status=ints([0]),
             q_out=torch.full((N, Hq, 128), float("nan"), dtype=torch.bfloat16, device="cuda"),
             reps=torch.randn((S, Hkv, NB, 128), generator=gen, device="cuda"), geom=sv.make_geom(S, Hq, Hkv, 128, B, NB, 1))
    if fused:
        t["q"], t["k"], t["v"] = normal(N, Hq + 2 * Hkv, 128).split([Hq, Hkv, Hkv], dim=1)
    else:
        t["q"], t["k"], t["v"] = normal(N, Hq, 128), normal(N, Hkv, 128), normal(N, Hkv, 128)
    t["rope"] = None
    if rot:
        angle = torch.arange(max(b + n for b, n in zip(before, new)), dtype=torch.float64, device="cuda")[:, None] * \
            10000.0 ** (-torch.arange(rot // 2, device="cuda") / (rot // 2))
        t["rope"] = torch.cat([angle.cos(), angle.sin()], 1).float()
    return t


def _host(x):
    return x.double().cpu().numpy()


def _expected(t, before, new, B, k):
    """The pool with the batch's tokens, and the representatives: [S][Hkv][NB][128] and how far they may be off."""
    pool, table, v = t["pool"].cpu().numpy().copy(), t["table"].cpu().numpy(), _host(t["v"])
    reps, tol = _host(t["reps"]), np.zeros(t["reps"].shape)
    row = 0
    for s, (b, n) in enumerate(zip(before, new)):
        for i in range(n):
            page, r = table[s, (b + i) // B], (b + i) % B
            for h in range(pool.shape[1]):
                put(pool[page, h, r // 64], r % 64, k[row + i, h], v[row + i, h])
        row += n
        for j in range(b // B, -(-(b + n) // B) if n else 0):
            m = min(B, b + n - j * B)
            for h in range(pool.shape[1]):
                held = np.concatenate([get(x)[0] for x in pool[table[s, j], h]])[:m]
                reps[s, h, j], tol[s, h, j] = held.mean(0), 128 * 2.0 ** -24 * np.abs(held).mean(0)
    return pool, reps, tol


def _append(sv, t, interleaved=False, **over):
    a = {**t, **over}
    sv.sv_rope_append_q4(a["geom"], a["pool"], a["table"], a["lens"], a["q"], a["k"], a["v"], a["start"], a["q_out"], a["lens_out"], rope=a["rope"],
                         interleaved=interleaved, reps=a["reps"], status_word=a["status"])


def _rotated(sv, t, Hkv, B, interleaved):
    """Rotated keys and queries as sv_rope_append makes them, by way of a bfloat16 cache."""
    S, NB = t["table"].shape
    pools = [torch.zeros((S * NB, Hkv, B, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    q, lens = torch.empty_like(t["q_out"]), torch.empty_like(t["lens"])
    sv.sv_rope_append(t["geom"], *pools, t["table"], t["lens"], t["q"], t["k"], t["v"], t["start"], q, lens, rope=t["rope"], interleaved=interleaved)
    start, before, table = (x.tolist() for x in (t["start"], t["lens"], t["table"]))
    k = torch.cat([pools[0][table[s][(before[s] + i) // B], :, (before[s] + i) % B][None] for s in range(S) for i in range(start[s + 1] - start[s])])
    return _host(k), q


@pytest.mark.gpu
@pytest.mark.parametrize("before,new,Hq,Hkv,B,rot,interleaved,fused", CASES)
def test_append(before, new, Hq, Hkv, B, rot, interleaved, fused):
    import paper_2512_21911_b200 as sv
    t = _batch(sv, before, new, Hq, Hkv, B, rot, fused)
    k, q = _rotated(sv, t, Hkv, B, interleaved)
    pool, reps, tol = _expected(t, before, new, B, k)
    _append(sv, t, interleaved)
    assert np.array_equal(t["pool"].cpu().numpy(), pool)
    assert torch.equal(t["q_out"], q) and t["lens_out"].tolist() == [b + n for b, n in zip(before, new)] and int(t["status"]) == 0
    assert (np.abs(_host(t["reps"]) - reps) <= tol).all()


@pytest.mark.gpu
@pytest.mark.parametrize("before,new,Hq,Hkv,B,rot,interleaved,fused", CASES)
def test_read(before, new, Hq, Hkv, B, rot, interleaved, fused):
    import paper_2512_21911_b200 as sv
    t = _batch(sv, before, new, Hq, Hkv, B, 0, fused)
    _append(sv, t)
    kv = sv.make_kv_q4(t["pool"], t["table"], t["lens_out"])
    pool, table = t["pool"].cpu().numpy(), t["table"].tolist()
    # the new tokens, and three rows that nobody's sequence has
    N = sum(new)
    k, v = (torch.full((N + 3, Hkv, 128), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    sv.sv_kv_read_q4(t["geom"], kv, t["lens"], t["start"], k, v, status_word=t["status"])
    assert int(t["status"]) == 0
    row = 0
    for s, (b, n) in enumerate(zip(before, new)):
        for i in range(n):
            for h in range(Hkv):
                held = get(pool[table[s][(b + i) // B], h, (b + i) % B // 64])
                assert np.array_equal(_host(k[row, h]), held[0][(b + i) % 64]) and np.array_equal(_host(v[row, h]), held[1][(b + i) % 64])
            row += 1
    assert (k[N:] == 7.0).all() and (v[N:] == 7.0).all()


@pytest.mark.gpu
def test_read_of_positions_that_are_not_there():
    import paper_2512_21911_b200 as sv
    t = _batch(sv, [70, 10], [0, 3], 4, 2, 64, 0, False)
    _append(sv, t)
    kv = sv.make_kv_q4(t["pool"], t["table"], t["lens_out"])
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    k, v = (torch.full((90, 2, 128), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    sv.sv_kv_read_q4(t["geom"], kv, ints([-3, 11]), ints([0, 85, 89]), k, v, status_word=t["status"])
    assert int(t["status"]) == sv.SV_STATUS_INDEX
    for x in (k, v):
        assert (x[:3] == 0).all() and (x[73:85] == 0).all() and (x[87:89] == 0).all() and (x[89] == 7.0).all()
        assert x[3:73].float().abs().amax((1, 2)).min() > 0 and x[85:87].float().abs().amax((1, 2)).min() > 0


@pytest.mark.gpu
@pytest.mark.parametrize("B,before,kept", [(64, [0, 60, 64, 200], [3, 5, 0, 1]), (128, [127, 5, 64, 128], [64, 1, 64, 2])])
def test_commit(B, before, kept):
    import paper_2512_21911_b200 as sv
    S, T, Hkv = 4, 64, 2
    t = _batch(sv, before, kept, 4, Hkv, B, 0, False)
    gen = torch.Generator(device="cuda").manual_seed(3)
    dk, dv = (torch.empty((S, T, Hkv, 128), dtype=torch.bfloat16, device="cuda").normal_(generator=gen) for _ in range(2))
    idx = torch.full((S, T), -1, dtype=torch.int32)
    for s in range(S):
        idx[s, :kept[s]] = torch.randperm(T, generator=torch.Generator().manual_seed(s))[:kept[s]]
    rows = [(s, int(j)) for s in range(S) for j in idx[s, :kept[s]]]
    t["v"] = torch.stack([dv[s, j] for s, j in rows])
    pool, reps, tol = _expected(t, before, kept, B, _host(torch.stack([dk[s, j] for s, j in rows])))
    geom = sv.make_geom(S, 4, Hkv, 128, B, t["table"].shape[1], T)
    sv.sv_kv_append_q4(geom, t["pool"], t["table"], t["lens"], dk, dv, idx.cuda(), torch.tensor(kept, dtype=torch.int32, device="cuda"), t["lens_out"],
                       reps=t["reps"])
    assert np.array_equal(t["pool"].cpu().numpy(), pool) and t["lens_out"].tolist() == [b + n for b, n in zip(before, kept)]
    assert (np.abs(_host(t["reps"]) - reps) <= tol).all()


@pytest.mark.gpu
def test_values_that_are_hard_to_code():
    """Groups without a spread, of two neighbours, of the largest and smallest numbers, of subnormal ones, with a NaN or an infinity."""
    import paper_2512_21911_b200 as sv
    t = _batch(sv, [7], [12], 2, 1, 64, 0, False)
    k = torch.zeros((12, 1, 128))
    k[1] = 3.0
    k[2, 0, :5] = 1.0078125
    k[3] = torch.linspace(-1e38, 1e38, 128)
    k[4] = torch.linspace(-1e-38, 1e-38, 128)
    k[5, 0, 127] = 9.2e-41
    k[6, 0, 3] = float("nan")
    k[7, 0, 70] = float("inf")
    k[8, 0, 70] = -float("inf")
    k[9] = torch.linspace(0, 1e-20, 128) + 1000.0
    k[10, 0, ::2] = -0.0
    k[11] = torch.linspace(100.0, 101.0, 128)
    t["k"], t["v"] = k.cuda().bfloat16(), k.flip(2).cuda().bfloat16()
    t["reps"] = None
    pool = t["pool"].cpu().numpy().copy()
    for i in range(12):
        put(pool[int(t["table"][0, 0]), 0, 0], 7 + i, _host(t["k"])[i, 0], _host(t["v"])[i, 0])
    _append(sv, t)
    got = [get(x[int(t["table"][0, 0]), 0, 0]) for x in (t["pool"].cpu().numpy(), pool)]
    for a, b in zip(*got):
        assert np.array_equal(a[7:19], b[7:19], equal_nan=True)
    assert np.isnan(got[0][0][13, :64]).all() and not np.isnan(got[0][0][13, 64:]).any()


@pytest.mark.gpu
@pytest.mark.parametrize("factor", [1.0, 3.0, 0.40625, 2.0 ** -99, 2.0 ** -112, 2.0 ** 104, 1.9921875])
def test_values_in_the_middle_of_two_codes(factor):
    """Quarters of a step: every fourth value lies in the middle between two codes, and goes to the even one, as do their neighbours in bfloat16
    to theirs.  (With a factor of few bits the scale stays exact.)"""
    import paper_2512_21911_b200 as sv
    t = _batch(sv, [0], [8], 2, 1, 64, 0, False)
    quarters = torch.arange(64).double() / 4    # 0 .. 15.75
    quarters[61:] = 15.0
    k = torch.zeros((8, 1, 128), dtype=torch.float64)
    for i in range(8):
        x = (quarters if i % 2 else quarters - 7.0) * factor
        k[i, 0] = torch.cat([x, x.roll(5)])
    t["k"] = k.cuda().bfloat16()
    bits = t["k"].view(torch.int16).clone()
    bits[2:4] += (torch.arange(128, device="cuda") % 64 % 3 == 1) * (torch.arange(128, device="cuda") % 64 > 0)     # a step away from the middle
    bits[4:6] -= (torch.arange(128, device="cuda") % 64 % 4 == 2).short()
    t["k"] = bits.view(torch.bfloat16)
    t["v"], t["reps"] = t["k"].flip(2), None
    pool = t["pool"].cpu().numpy().copy()
    for i in range(8):
        put(pool[int(t["table"][0, 0]), 0, 0], i, _host(t["k"])[i, 0], _host(t["v"])[i, 0])
    _append(sv, t)
    assert np.array_equal(t["pool"].cpu().numpy(), pool)


@pytest.mark.gpu
def test_tokens_without_room_are_dropped():
    import paper_2512_21911_b200 as sv
    t = _batch(sv, [60, 100, -4], [10, 200, 5], 4, 2, 64, 0, False, spare=0)
    t["table"][0, 1] = -1                       # sequence 0: no page behind the first
    NB = t["table"].shape[1]
    before = t["pool"].clone()
    _append(sv, t)
    assert t["lens_out"].tolist() == [64, 300, -4] and int(t["status"]) == sv.SV_STATUS_INDEX
    touched = {int(t["table"][0, 0])} | {int(p) for p in t["table"][1, 1:NB]}
    for page in set(range(before.shape[0])) - touched:
        assert torch.equal(t["pool"][page], before[page])


@pytest.mark.gpu
def test_captured_and_on_another_stream():
    import paper_2512_21911_b200 as sv
    a, b = (_batch(sv, [10, 64], [70, 1], 8, 2, 64, 128, True) for _ in range(2))
    _append(sv, a)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        _append(sv, b)
    graph.replay()
    torch.cuda.synchronize()
    for name in ("pool", "q_out", "reps", "lens_out"):
        assert torch.equal(a[name], b[name]), name
