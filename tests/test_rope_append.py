"""sv_rope_append: rotated queries and keys of ragged batches of new tokens, the cache they are written to, the new lengths and the
representatives, against the formula in 64 bits; what the call refuses.

A rotated value y = a cos - b sin is two products and a sum, rounded to fp32 one by one, and one rounding to bf16: bit for bit what
separate fp32 operations give, and within 2^-8 |y| (half a unit of the last of 8 significant bits) + 2^-22 (|a| + |b|) of the formula in 64
bits.  Everything that is not rotated is a copy, and the representatives are those of sv_block_reps, bit for bit."""
import ctypes

import numpy as np
import pytest
import torch


def _batch(sv, before, new, Hq, Hkv, B, rot, interleaved, fused, seed=0, spare=1, rope_rows=None):
    """Inputs of a ragged batch, the pools filled with other values so that every stray write shows."""
    S, N = len(before), sum(new)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    NB = max(-(-(b + n) // B) for b, n in zip(before, new)) + spare
    table = np.random.default_rng(seed).permutation(S * NB).astype(np.int32).reshape(S, NB)
    t = dict(k_pool=normal(S * NB, Hkv, B, 128), v_pool=normal(S * NB, Hkv, B, 128), table=torch.from_numpy(table).cuda(),
             lens=torch.tensor(before, dtype=torch.int32, device="cuda"),
             start=torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device="cuda"))
    if fused:
        t["q"], t["k"], t["v"] = normal(N, Hq + 2 * Hkv, 128).split([Hq, Hkv, Hkv], dim=1)
    else:
        t["q"], t["k"], t["v"] = normal(N, Hq, 128), normal(N, Hkv, 128), normal(N, Hkv, 128)
    rows = rope_rows or max(b + n for b, n in zip(before, new))
    if rot:
        angle = torch.arange(rows, dtype=torch.float64, device="cuda")[:, None] * 10000.0 ** (-torch.arange(rot // 2, device="cuda") / (rot // 2))
        t["rope"] = torch.cat([angle.cos(), angle.sin()], 1).float()
    else:
        t["rope"] = None
    t["q_out"] = torch.full((N, Hq, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    t["lens_out"] = torch.full((S,), -7, dtype=torch.int32, device="cuda")
    t["reps"] = torch.randn((S, Hkv, NB, 128), generator=gen, device="cuda")
    t["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    t["geom"] = sv.make_geom(S, Hq, Hkv, 128, B, NB, 1)
    t["interleaved"] = interleaved
    return t


def _call(sv, t, **over):
    a = {**t, **over}
    sv.sv_rope_append(a["geom"], a["k_pool"], a["v_pool"], a["table"], a["lens"], a["q"], a["k"], a["v"], a["start"], a["q_out"], a["lens_out"],
                      rope=a["rope"], interleaved=a["interleaved"], reps=a["reps"], status_word=a["status"])


def _turned(x, rope, positions, interleaved):
    """Rotated rows in 64 bits and how far a right result may be off."""
    x = x.double()
    if rope is None:
        return x, torch.zeros_like(x)
    half = rope.shape[1] // 2
    c, s = (rope[positions][:, None, i * half:(i + 1) * half].double() for i in (0, 1))
    lo, hi = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    a, b, y, tol = x[..., lo], x[..., hi], x.clone(), torch.zeros_like(x)
    y[..., lo], y[..., hi] = a * c - b * s, b * c + a * s
    tol[..., lo] = tol[..., hi] = 2.0 ** -22 * (a.abs() + b.abs())
    tol[..., lo] += 2.0 ** -8 * y[..., lo].abs()
    tol[..., hi] += 2.0 ** -8 * y[..., hi].abs()
    return y, tol


def _turned_32(x, rope, positions, interleaved):
    """The same in fp32, an operation at a time, rounded to bf16."""
    y = x.clone()
    if rope is None:
        return y
    half = rope.shape[1] // 2
    c, s = (rope[positions][:, None, i * half:(i + 1) * half] for i in (0, 1))
    lo, hi = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    a, b = x[..., lo].float(), x[..., hi].float()
    y[..., lo], y[..., hi] = (a * c - b * s).to(torch.bfloat16), (b * c + a * s).to(torch.bfloat16)
    return y


def _is_turned(got, x, rope, positions, interleaved):
    want, tol = _turned(x, rope, positions, interleaved)
    off = (got.double() - want).abs()
    assert bool((off <= tol).all()), float((off - tol).max())
    assert torch.equal(got, _turned_32(x, rope, positions, interleaved))


def _check(sv, t, before, new, kept=None):
    """Runs the call and compares everything; kept: tokens of each sequence that the table has room for."""
    kept = new if kept is None else kept
    B, Hkv = t["geom"].block_size, t["geom"].n_kv_heads
    k0, v0, reps0 = t["k_pool"].clone(), t["v_pool"].clone(), t["reps"].clone()
    q_in = None if t["q"] is None else t["q"].clone()
    _call(sv, t)
    at = 0
    fresh = torch.zeros(k0.shape[:3], dtype=torch.bool, device="cuda").transpose(1, 2).contiguous()      # [page][slot][head]
    for s, (b, n) in enumerate(zip(before, new)):
        rows = slice(at, at + n)
        pos = torch.arange(b, b + n, device="cuda")
        row = pos if t["rope"] is None else pos.clamp(max=t["rope"].shape[0] - 1)
        if q_in is not None:
            _is_turned(t["q_out"][rows], q_in[rows], t["rope"], row, t["interleaved"])
        m = kept[s]
        if m:
            page, slot = t["table"][s].long()[pos[:m] // B], pos[:m] % B
            _is_turned(t["k_pool"][page, :, slot], t["k"][rows][:m], t["rope"], row[:m], t["interleaved"])
            assert torch.equal(t["v_pool"][page, :, slot], t["v"][rows][:m])
            fresh[page, slot] = True
        assert int(t["lens_out"][s]) == b + m
        at += n
    old = ~fresh.transpose(1, 2)
    assert torch.equal(t["k_pool"][old], k0[old]) and torch.equal(t["v_pool"][old], v0[old])
    # representatives: those of a full rebuild where a block grew, untouched elsewhere
    rebuilt = torch.zeros_like(reps0)
    lens = torch.tensor([b + m for b, m in zip(before, kept)], dtype=torch.int32, device="cuda")
    sv.sv_block_reps(t["geom"], sv.make_kv(t["k_pool"], t["v_pool"], t["table"], lens), rebuilt)
    for s, (b, m) in enumerate(zip(before, kept)):
        lo, hi = b // B, -(-(b + m) // B) if m else b // B
        assert torch.equal(t["reps"][s, :, lo:hi], rebuilt[s, :, lo:hi])
        assert torch.equal(t["reps"][s, :, :lo], reps0[s, :, :lo]) and torch.equal(t["reps"][s, :, hi:], reps0[s, :, hi:])


@pytest.mark.gpu
@pytest.mark.parametrize("B", [64, 128])
@pytest.mark.parametrize("rot,interleaved", [(128, False), (128, True), (64, False), (64, True), (16, False), (112, False), (48, True), (0, False)])
def test_ragged_batches(B, rot, interleaved):
    import paper_2512_21911_b200 as sv
    before = [0, 0, 1, B - 1, B, B + 1, 2 * B - 1, 5, 3 * B - 7, 17]
    new = [1, 0, 2 * B + 3, 1, 1, B, 2, 0, 7, 3 * B]
    for Hq, Hkv, fused in ((8, 2, True), (7, 1, False), (3, 3, True)):
        t = _batch(sv, before, new, Hq, Hkv, B, rot, interleaved, fused, seed=B + rot + Hq)
        _check(sv, t, before, new)
        assert int(t["status"]) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("rot,interleaved", [(128, False), (64, True)])
@pytest.mark.parametrize("last", [1, 2, 9])
def test_on_either_side_of_the_size_that_changes_the_tiles(last, rot, interleaved):
    """1,024 tokens and a few more, of sequences that begin inside a tile of tokens; odd numbers of heads."""
    import paper_2512_21911_b200 as sv
    before, new = [10, 0, 64, 3, 700], [501, 5, 1, 516, last]
    for Hq, Hkv in ((1, 1), (5, 1), (33, 3)):
        t = _batch(sv, before, new, Hq, Hkv, 64, rot, interleaved, True, seed=last + Hq)
        _check(sv, t, before, new)


@pytest.mark.gpu
def test_many_sequences_of_one_token():
    """More sequences than a CTA has threads, lengths at and around the ends of blocks, some of them empty."""
    import paper_2512_21911_b200 as sv
    before = [(37 * i) % 200 for i in range(700)]
    new = [0 if i % 13 == 5 else 1 for i in range(700)]
    t = _batch(sv, before, new, 4, 2, 64, 128, False, True)
    _check(sv, t, before, new)


@pytest.mark.gpu
def test_a_long_prompt_in_chunks_equals_one_call():
    import paper_2512_21911_b200 as sv
    n, B = 1000, 64
    t = _batch(sv, [0], [n], 8, 2, B, 128, False, True)
    one = {k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in t.items()}
    _call(sv, one)
    at = 0
    for m in (1, 62, 1, 64, 65, 300, 507):
        lens = torch.tensor([at], dtype=torch.int32, device="cuda")
        start = torch.tensor([0, m], dtype=torch.int32, device="cuda")
        rows = slice(at, at + m)
        _call(sv, t, lens=lens, start=start, q=t["q"][rows], k=t["k"][rows], v=t["v"][rows], q_out=t["q_out"][rows])
        at += m
        assert int(t["lens_out"]) == at
    for name in ("k_pool", "v_pool", "q_out", "reps"):
        assert torch.equal(t[name], one[name]), name


@pytest.mark.gpu
def test_what_the_table_has_no_room_for_is_dropped():
    import paper_2512_21911_b200 as sv
    B = 64
    before, new = [60, 60, 0, 10, 250], [200, 200, 130, 5, 30]
    t = _batch(sv, before, new, 4, 2, B, 64, False, False, spare=0)                  # five blocks a sequence
    t["table"][0, 2] = -1                                                           # the table ends behind two blocks
    t["table"][1, 0] = t["geom"].n_seq * t["geom"].max_blocks + 5                    # not a page of the pool: nothing fits
    t["table"][2, 1] = -1
    t["table"][2, 2] = -1
    before.append(2 * B), new.append(0)
    _check(sv, {**t, "geom": t["geom"]}, before[:5], new[:5], kept=[2 * B - 60, 0, B, 5, 30])


@pytest.mark.gpu
def test_positions_beyond_the_rotation_table():
    import paper_2512_21911_b200 as sv
    before, new = [90, 3], [20, 4]
    t = _batch(sv, before, new, 4, 2, 64, 128, False, False, rope_rows=100)
    _check(sv, t, before, new)
    assert int(t["status"]) == sv.SV_STATUS_INDEX


@pytest.mark.gpu
def test_without_queries_in_place_and_on_another_stream():
    import paper_2512_21911_b200 as sv
    before, new = [33, 70], [40, 1]
    t = _batch(sv, before, new, 8, 2, 64, 128, False, False)
    plain = {k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in t.items()}
    _call(sv, plain)
    cache_only = {**{k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in t.items()}, "q": None, "q_out": None}
    _call(sv, cache_only)
    assert torch.equal(cache_only["k_pool"], plain["k_pool"]) and torch.equal(cache_only["reps"], plain["reps"])
    here = {k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in t.items()}
    here["q_out"] = here["q"]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _call(sv, here)
    side.synchronize()
    assert torch.equal(here["q"], plain["q_out"]) and torch.equal(here["v_pool"], plain["v_pool"])


@pytest.mark.gpu
def test_captured_in_a_graph():
    import paper_2512_21911_b200 as sv
    before, new = [5, 64], [70, 2]
    t = _batch(sv, before, new, 8, 2, 64, 128, True, True)
    want = {k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in t.items()}
    _call(sv, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _call(sv, t)
    g.replay()
    torch.cuda.synchronize()
    for name in ("k_pool", "v_pool", "q_out", "reps", "lens_out"):
        assert torch.equal(t[name], want[name]), name


@pytest.mark.gpu
def test_tensors_that_do_not_fit_are_refused():
    import paper_2512_21911_b200 as sv
    t = _batch(sv, [3], [10], 8, 2, 64, 128, False, False)
    for over in (dict(k=t["k"].float()), dict(k=t["k"].cpu()), dict(k=t["k"][:, :1]), dict(q=t["q"].transpose(1, 2)), dict(rope=t["rope"].double()),
                 dict(k_pool=t["k_pool"].transpose(1, 2))):
        with pytest.raises(TypeError):
            _call(sv, t, **over)
    for over in (dict(v=t["v"][:9]), dict(q_out=t["q_out"][:9]), dict(start=t["start"][:1]), dict(lens=t["lens"][:0]), dict(reps=t["reps"][:, :, :1].contiguous()),
                 dict(q_out=None), dict(v_pool=t["v_pool"][:1])):
        with pytest.raises(ValueError):
            _call(sv, t, **over)
    with pytest.raises(sv.SvError):
        _call(sv, t, lens_out=t["lens"])
    with pytest.raises(sv.SvError):
        _call(sv, t, rope=t["rope"][:, :24].contiguous())
    wide = torch.zeros((10, 2, 256), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(TypeError):
        _call(sv, t, k=wide[..., :128])                      # the heads of a token are not contiguous
    odd = torch.zeros((10 * 260,), dtype=torch.bfloat16, device="cuda").as_strided((10, 2, 128), (260, 128, 1))
    with pytest.raises(sv.SvError):
        _call(sv, t, k=odd)                                  # tokens that do not start on 16 bytes


def test_refusals_without_a_device():
    import paper_2512_21911_b200.binding as b
    g = b.make_geom(2, 8, 2, 128, 64, 16, 1)
    call = lambda geom=g, kp=0x1000, pages=32, table=0x2000, lens=0x3000, q=0x4000, k=0x5000, v=0x6000, qs=1024, ks=256, vs=256, start=0x7000, n=10, \
        rope=0x8000, rows=100, rot=128, q_out=0x9000, lens_out=0xa000, reps=0xb000: \
        b._lib.sv_rope_append(ctypes.byref(geom), kp, 0xc000, pages, table, lens, q, k, v, qs, ks, vs, start, n, rope, rows, rot, 0, q_out, lens_out, reps, None, None)
    assert call(kp=None) == 1 and call(table=None) == 1 and call(k=None) == 1 and call(start=None) == 1 and call(lens_out=None) == 1
    assert call(q=None) == 1 and call(q_out=None) == 1
    assert call(pages=0) == 2 and call(n=-1) == 2 and call(lens_out=0x3000) == 2
    assert call(rot=0) == 2 and call(rot=24) == 2 and call(rot=144) == 2 and call(rows=0) == 2
    assert call(ks=128) == 2 and call(qs=1016) == 2 and call(q=0x9000, qs=1280) == 2
    assert call(ks=260) == 3 and call(kp=0x1040) == 3 and call(k=0x5008) == 3 and call(rope=0x8004) == 3
    assert call(geom=b.make_geom(2, 8, 3, 128, 64, 16, 1)) == 2 and call(geom=b.make_geom(2, 8, 2, 64, 64, 16, 1)) == 6
    assert call(geom=b.make_geom(2, 8, 2, 128, 32, 16, 1)) == 6
