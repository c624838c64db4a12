"""sv_chunk_attn: ragged batches of new tokens over the paged cache against softmax attention in 64 bits; what the call refuses.

Tolerance of an output o = sum p v: a rounding to bf16 is off by at most 2^-8 of the value (half a unit of the last of 8 significant bits).
That holds for each probability, which makes 2^-8 sum p |v|, and for the output, 2^-8 |o|; exponentials, products and sums in fp32 add less
than 2^-12 of sum p |v|.  lse: sums of unrounded exponentials, 1e-3."""
import ctypes
import math

import numpy as np
import pytest
import torch


def _batch(sv, lens, new, Hq, Hkv, B, seed=0, sigma=math.sqrt(3.0), garbage=float("nan"), spare=1):
    """lens: cached tokens with the new ones.  Slots that no token is in, and pages nobody has, hold `garbage`."""
    S, N = len(lens), sum(new)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape, s=1.0: torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0.0, s, generator=gen)
    blocks = [-(-max(n, 0) // B) for n in lens]
    NB = max(blocks + [1]) + spare
    pages = np.random.default_rng(seed).permutation(sum(blocks) + 3).astype(np.int32)
    table = np.full((S, NB), -1, np.int32)
    k, v = (torch.full((len(pages), Hkv, B, 128), garbage, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    at = 0
    for s in range(S):
        table[s, :blocks[s]] = pages[at:at + blocks[s]]
        at += blocks[s]
        for j in range(blocks[s]):
            m = min(B, lens[s] - j * B)
            k[table[s, j], :, :m] = normal(Hkv, m, 128, s=sigma)
            v[table[s, j], :, :m] = normal(Hkv, m, 128)
    t = dict(k=k, v=v, table=torch.from_numpy(table).cuda(), lens=torch.tensor(lens, dtype=torch.int32, device="cuda"),
             start=torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device="cuda"), q=normal(N, Hq, 128, s=sigma))
    t["geom"] = sv.make_geom(S, Hq, Hkv, 128, B, NB, 1)
    return t


def _run(sv, t, scale=0.0, lse=True, rows=None):
    N = t["q"].shape[0]
    out = torch.full_like(t["q"], 77.0)
    l = torch.full((N, t["geom"].n_q_heads), 77.0, device="cuda") if lse else None
    ws = torch.full((sv.sv_chunk_workspace_bytes(t["geom"], N),), 0xff, dtype=torch.uint8, device="cuda")   # NaN wherever it is read unwritten
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    sv.sv_chunk_attn(t["geom"], t["q"], sv.make_kv(t["k"], t["v"], t["table"], t["lens"]), t["start"], out, lse=l, workspace=ws, softmax_scale=scale,
                     status_word=status)
    return out, l, int(status)


def _check(t, out, lse, lens, new, scale=1 / math.sqrt(128)):
    B, Hq, Hkv = t["geom"].block_size, t["geom"].n_q_heads, t["geom"].n_kv_heads
    G, at = Hq // Hkv, 0
    for s, (L, n) in enumerate(zip(lens, new)):
        if n == 0:
            continue
        rows = slice(at, at + n)
        at += n
        pages = t["table"][s, :-(-max(L, 0) // B)].long()
        k, v = (x[pages].transpose(0, 1).reshape(Hkv, -1, 128)[:, :max(L, 0)].double() for x in (t["k"], t["v"]))
        q = t["q"][rows].double().view(n, Hkv, G, 128)
        x = torch.einsum("nhgd,htd->nhgt", q, k) * scale
        x = x.masked_fill(torch.arange(max(L, 0), device="cuda") > torch.arange(L - n, L, device="cuda")[:, None, None, None], -math.inf)
        seen = (torch.arange(L - n, L, device="cuda") >= 0)
        p = torch.nan_to_num(torch.softmax(x, -1), nan=0.0)
        want = torch.einsum("nhgt,htd->nhgd", p, v).reshape(n, Hq, 128)
        room = torch.einsum("nhgt,htd->nhgd", p, v.abs()).reshape(n, Hq, 128)
        off = (out[rows].double() - want).abs() - (2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -12) * room)
        assert bool((off <= 0).all()), (s, float(off.max()))
        if lse is not None:
            ref = torch.logsumexp(x, -1).reshape(n, Hq)
            assert bool(((lse[rows] - ref).abs() <= 1e-3)[seen].all()), s
            assert bool((lse[rows][~seen] == -math.inf).all())


HEADS = [(8, 2), (4, 4), (7, 1), (20, 2), (16, 1), (32, 1)]


@pytest.mark.gpu
@pytest.mark.parametrize("B", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", HEADS)
def test_ragged_batches(B, Hq, Hkv):
    import paper_2512_21911_b200 as sv
    lens = [1, 300, 0, B, B + 1, 2 * B - 1, 777, 129, 1000, 128, 65, 400]
    new = [1, 1, 0, B, 1, 2, 600, 129, 33, 127, 65, 0]
    t = _batch(sv, lens, new, Hq, Hkv, B, seed=Hq + B)
    out, lse, status = _run(sv, t)
    _check(t, out, lse, lens, new)
    assert status == 0


@pytest.mark.gpu
@pytest.mark.parametrize("lens,new", [([1], [1]), ([63], [1]), ([64], [64]), ([128], [128]), ([129], [2]), ([2000], [1]), ([2000], [2000]), ([4097], [513]),
                                      ([9000], [3]), ([500] * 40, [1] * 40), ([70] * 20, [70] * 20), ([3000, 5, 2500], [1, 5, 900])])
def test_one_call_of_each_kind(lens, new):
    import paper_2512_21911_b200 as sv
    for Hq, Hkv, B in ((8, 2, 64), (10, 2, 128)):
        t = _batch(sv, lens, new, Hq, Hkv, B, seed=len(lens))
        out, lse, status = _run(sv, t)
        _check(t, out, lse, lens, new)
        again, _, _ = _run(sv, t, lse=False)
        assert torch.equal(out, again) and status == 0


@pytest.mark.gpu
def test_a_wide_group_of_heads():
    import paper_2512_21911_b200 as sv
    for Hq, Hkv in ((128, 1), (100, 1), (130, 2)):
        lens, new = [300, 40, 200], [7, 40, 1]
        t = _batch(sv, lens, new, Hq, Hkv, 64)
        out, lse, _ = _run(sv, t)
        _check(t, out, lse, lens, new)


@pytest.mark.gpu
def test_long_caches_split_over_the_device():
    import paper_2512_21911_b200 as sv
    lens, new = [40000, 131, 17001], [1, 1, 40]
    t = _batch(sv, lens, new, 8, 2, 64)
    out, lse, _ = _run(sv, t)
    _check(t, out, lse, lens, new)


@pytest.mark.gpu
def test_many_units_per_cta_and_calls_one_behind_the_other():
    """Long loops at the speed of HBM, single tokens (both streams on one tile) and a chunk mixed: every call gives the same bits."""
    import paper_2512_21911_b200 as sv
    for lens, new, Hq, Hkv in (([10439, 5106, 16227, 9001, 12000, 15041], [1, 1, 1, 1, 1, 1], 32, 8), ([15000, 9000, 3000], [1, 200, 1], 28, 4)):
        t = _batch(sv, lens, new, Hq, Hkv, 64)
        out, lse, status = _run(sv, t)
        _check(t, out, lse, lens, new)
        outs = [torch.empty_like(out) for _ in range(3)]
        ws = torch.empty(sv.sv_chunk_workspace_bytes(t["geom"], t["q"].shape[0]), dtype=torch.uint8, device="cuda")
        word = torch.zeros(1, dtype=torch.int32, device="cuda")
        kv = sv.make_kv(t["k"], t["v"], t["table"], t["lens"])
        for i in range(300):
            sv.sv_chunk_attn(t["geom"], t["q"], kv, t["start"], outs[i % 3], workspace=ws, status_word=word)
        torch.cuda.synchronize()
        assert int(word) == 0 and status == 0
        assert all(torch.equal(o, out) for o in outs)


@pytest.mark.gpu
@pytest.mark.parametrize("sigma", [0.0, 1.0, 8.0])
def test_flat_and_sharp_scores_and_a_scale(sigma):
    """Equal scores; scores whose maximum moves by hundreds from key to key."""
    import paper_2512_21911_b200 as sv
    lens, new = [700, 1500], [700, 1]
    t = _batch(sv, lens, new, 8, 2, 64, sigma=sigma)
    out, lse, _ = _run(sv, t, scale=0.11)
    if sigma < 8.0:
        _check(t, out, lse, lens, new, scale=0.11)
    else:   # scores of some hundreds: fp32 products of 128 terms are off by up to 1e-4, and so is the exponent
        ref, _, _ = _run(sv, {**t, "q": t["q"]}, scale=0.11)
        assert torch.equal(ref, out) and bool(torch.isfinite(out).all())
        _check(t, out, None, lens, new, scale=0.11)


@pytest.mark.gpu
def test_rising_scores_move_the_maximum_all_the_time():
    import paper_2512_21911_b200 as sv
    L = 1200
    t = _batch(sv, [L], [L], 4, 1, 64, sigma=1.0)
    u = torch.zeros(128, device="cuda")
    u[0] = 1.0
    for j in range(-(-L // 64)):
        page = int(t["table"][0, j])
        rise = torch.arange(j * 64, j * 64 + 64, device="cuda")[:, None] * u[None] * 0.5
        t["k"][page] = (t["k"][page].float() + rise).to(torch.bfloat16)
    t["q"][..., 0] = 4.0
    out, lse, _ = _run(sv, t)
    _check(t, out, lse, [L], [L])


@pytest.mark.gpu
def test_rows_that_see_nothing_and_rows_of_nobody():
    import paper_2512_21911_b200 as sv
    lens, new = [3, 200], [10, 5]                        # the first seven rows of the first sequence stand before its beginning
    t = _batch(sv, lens, new, 8, 2, 64)
    t["q"] = torch.cat([t["q"], torch.full((9, 8, 128), float("nan"), dtype=torch.bfloat16, device="cuda")])
    out, lse, _ = _run(sv, t)
    _check(t, out, lse, lens, new)
    assert bool((out[:7] == 0).all()) and bool((out[15:] == 77).all()) and bool((lse[15:] == 77).all())
    t["lens"][:] = torch.tensor([-4, 0], device="cuda")   # no cache at all
    out, lse, _ = _run(sv, t)
    assert bool((out[:15] == 0).all()) and bool((lse[:15] == -math.inf).all())


@pytest.mark.gpu
def test_pages_behind_32_bits():
    """The pages of a sequence at the far end of pools of more than 2^32 bytes each."""
    import paper_2512_21911_b200 as sv
    lens, new = [1000], [3]
    t = _batch(sv, lens, new, 8, 2, 64)
    pages = t["k"].shape[0]
    big = (1 << 32) // (2 * 64 * 128 * 2) + 2 * pages
    far = lambda x: torch.cat([torch.zeros((big - pages, 2, 64, 128), dtype=torch.bfloat16, device="cuda"), x])
    t["k"], t["v"] = far(t["k"]), far(t["v"])
    t["table"] = torch.where(t["table"] >= 0, t["table"] + (big - pages), t["table"])
    out, lse, status = _run(sv, t)
    _check(t, out, lse, lens, new)
    assert status == 0


@pytest.mark.gpu
def test_a_page_outside_the_pool_sets_the_status_word():
    import paper_2512_21911_b200 as sv
    t = _batch(sv, [200], [2], 8, 2, 64, garbage=0.0)
    t["table"][0, 1] = 10 ** 6
    assert _run(sv, t)[2] & sv.SV_STATUS_INDEX
    t["table"][0, 1] = -1
    assert _run(sv, t)[2] & sv.SV_STATUS_INDEX


@pytest.mark.gpu
def test_lengths_beyond_the_table_are_cut():
    import paper_2512_21911_b200 as sv
    t = _batch(sv, [128], [1], 8, 2, 64, spare=0)
    want, _, _ = _run(sv, t)
    t["lens"][0] = 150                                    # the table has two blocks: the row sees all of them
    assert torch.equal(_run(sv, t)[0], want)


@pytest.mark.gpu
def test_behind_an_append_on_a_stream_of_its_own_and_in_a_graph():
    import paper_2512_21911_b200 as sv
    S, Hq, Hkv, B, n = 3, 8, 2, 64, 150
    gen = torch.Generator(device="cuda").manual_seed(3)
    normal = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    lens = [0, 64, 33]
    NB = 4
    t = dict(k=normal(S * NB, Hkv, B, 128), v=normal(S * NB, Hkv, B, 128), table=torch.randperm(S * NB, generator=torch.Generator().manual_seed(1)).int().view(S, NB).cuda(),
             geom=sv.make_geom(S, Hq, Hkv, 128, B, NB, 1), q=normal(S * n, Hq, 128), start=torch.arange(0, S * n + 1, n, dtype=torch.int32, device="cuda"))
    k_new, v_new = normal(S * n, Hkv, 128), normal(S * n, Hkv, 128)
    before, after = torch.tensor(lens, dtype=torch.int32, device="cuda"), torch.zeros(S, dtype=torch.int32, device="cuda")
    out = torch.zeros_like(t["q"])
    ws = torch.empty(sv.sv_chunk_workspace_bytes(t["geom"], S * n), dtype=torch.uint8, device="cuda")

    def both():
        sv.sv_rope_append(t["geom"], t["k"], t["v"], t["table"], before, None, k_new, v_new, t["start"], None, after)
        sv.sv_chunk_attn(t["geom"], t["q"], sv.make_kv(t["k"], t["v"], t["table"], after), t["start"], out, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    side.synchronize()
    t["lens"] = after
    _check(t, out, None, [x + n for x in lens], [n] * S)
    want = out.clone()
    out.zero_()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        both()
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


@pytest.mark.gpu
def test_agrees_with_dense_verification_of_a_chain():
    """The same tokens as a draft on top of a cache without them (sv_verify_attn, dense) and as a chunk of a cache with them."""
    import paper_2512_21911_b200 as sv
    Hq, Hkv, B, L, T = 8, 2, 64, 500, 6
    t = _batch(sv, [L + T], [T], Hq, Hkv, B)
    out, lse, _ = _run(sv, t)
    pages = t["table"][0, :-(-(L + T) // B)].long()
    dk, dv = (x[pages].transpose(0, 1).reshape(Hkv, -1, 128)[:, L:L + T].transpose(0, 1).contiguous()[None] for x in (t["k"], t["v"]))
    geom = sv.make_geom(1, Hq, Hkv, 128, B, t["geom"].max_blocks, T)
    short = torch.tensor([L], dtype=torch.int32, device="cuda")
    dense, dlse = torch.empty((1, T, Hq, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((1, T, Hq), device="cuda")
    ws = torch.empty(max(16, sv.sv_workspace_bytes(geom, t["geom"].max_blocks)), dtype=torch.uint8, device="cuda")
    sv.sv_verify_attn(geom, t["q"][None].contiguous(), sv.make_kv(t["k"], t["v"], t["table"], short), dk, dv, None, None, None, dense, lse=dlse, workspace=ws)
    # either is within 2^-8 (|o| + sum p |v|) of the formula, and more than 500 values of variance one have |v| below 5
    assert float((out.float() - dense[0].float()).abs().max()) <= 2 * (2.0 ** -8 * 2 * 5)
    assert float((lse - dlse[0]).abs().max()) <= 2e-3


@pytest.mark.gpu
def test_tensors_that_do_not_fit_are_refused():
    import paper_2512_21911_b200 as sv
    t = _batch(sv, [200], [20], 8, 2, 64)
    kv = sv.make_kv(t["k"], t["v"], t["table"], t["lens"])
    out = torch.empty_like(t["q"])
    ws = torch.empty(sv.sv_chunk_workspace_bytes(t["geom"], 20), dtype=torch.uint8, device="cuda")
    with pytest.raises(TypeError):
        sv.sv_chunk_attn(t["geom"], t["q"].float(), kv, t["start"], out, workspace=ws)
    with pytest.raises(TypeError):
        sv.sv_chunk_attn(t["geom"], t["q"][:, ::2], kv, t["start"], out, workspace=ws)
    for q, o, start in ((t["q"][:19], out, t["start"]), (t["q"], out[:, :4].contiguous(), t["start"]), (t["q"], out, t["start"][:1])):
        with pytest.raises(ValueError):
            sv.sv_chunk_attn(t["geom"], q, kv, start, o, workspace=ws)
    with pytest.raises(sv.SvError):
        sv.sv_chunk_attn(t["geom"], t["q"], kv, t["start"], out)
    with pytest.raises(sv.SvError):
        sv.sv_chunk_attn(t["geom"], t["q"], kv, t["start"], out, workspace=ws[:8])
    with pytest.raises(ValueError):
        sv.sv_chunk_attn(t["geom"], t["q"], kv, t["start"], out, lse=torch.empty((20, 4), device="cuda"), workspace=ws)


def test_refusals_without_a_device():
    import paper_2512_21911_b200.binding as b
    g = b.make_geom(2, 8, 2, 128, 64, 16, 1)
    kv = b.sv_kv(0x1000, 0x2000, 0x3000, 0x4000, 8)

    def call(geom=g, q=0x5000, kv=kv, start=0x6000, n=10, out=0x7000, ws=0x8000, size=1 << 40):
        return b._lib.sv_chunk_attn(ctypes.byref(geom), q, ctypes.byref(kv), start, n, 0.0, out, None, ws, size, None, None)

    assert call(q=None) == 1 and call(start=None) == 1 and call(out=None) == 1 and call(ws=None) == 1
    assert call(kv=b.sv_kv(0x1000, None, 0x3000, 0x4000, 8)) == 1
    assert call(n=-1) == 2 and call(kv=b.sv_kv(0x1000, 0x2000, 0x3000, 0x4000, 0)) == 2
    assert call(geom=b.make_geom(2, 8, 3, 128, 64, 16, 1)) == 2
    assert call(q=0x5008) == 3 and call(kv=b.sv_kv(0x1040, 0x2000, 0x3000, 0x4000, 8)) == 3 and call(ws=0x8004) == 3 and call(out=0x7008) == 3
    assert call(size=0) == 5
    assert call(geom=b.make_geom(2, 8, 2, 64, 64, 16, 1)) == 6 and call(geom=b.make_geom(2, 129, 1, 128, 64, 16, 1)) == 6
    assert b.sv_chunk_workspace_bytes(b.make_geom(2, 8, 3, 128, 64, 16, 1), 10) == 0
    assert b.sv_chunk_workspace_bytes(g, -1) == 0 and b.sv_chunk_workspace_bytes(g, 10) > 0
