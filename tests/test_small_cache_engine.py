"""SparseVerifier with a cache in 4 bits, and with tokens evicted by attention weight: the engine's steps are the calls of sv.h on its
buffers, bit for bit; what is left after an eviction is what verification and prefill go over; the example runs both ways."""
import math
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HQ, HKV, B, L, T = 8, 2, 64, 3, 4


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _normal(gen, *shape):
    return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)


def _verifier(S, blocks, four_bits, keep, anchors=None):
    import paper_2512_21911_b200 as sv
    table = torch.randperm(S * blocks, generator=torch.Generator().manual_seed(5)).int().view(S, blocks).cuda()
    v = sv.SparseVerifier(n_seq=S, n_q_heads=HQ, n_kv_heads=HKV, head_dim=128, block_size=B, max_blocks=blocks, n_draft=T, n_layers=L, block_table=table,
                          seq_lens=_ints([0] * S), budget_blocks=_ints([keep] * S), max_sel=keep, anchors=anchors)
    if four_bits:
        pools = [torch.full((S * blocks, HKV, B // 64, sv.SV_Q4_SLAB_BYTES), 0x7f, dtype=torch.uint8, device="cuda") for _ in range(L)]
        for l in range(L):
            v.set_layer_kv_q4(l, pools[l])
    else:
        pools = [torch.full((L, S * blocks, HKV, B, 128), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        v.set_kv_stack(*pools)
    return v, pools


def _rope(n):
    angle = torch.arange(n, device="cuda")[:, None] * 10000.0 ** (-torch.arange(64, device="cuda") / 64)
    return torch.cat([angle.cos(), angle.sin()], 1)


def _prefill(v, gen, lens, rope):
    start = _ints([sum(lens[:s]) for s in range(len(lens) + 1)])
    outs = []
    for l in range(L):
        q, k, val = _normal(gen, sum(lens), HQ + 2 * HKV, 128).split([HQ, HKV, HKV], dim=1)
        outs.append(torch.empty((sum(lens), HQ, 128), dtype=torch.bfloat16, device="cuda"))
        v.prefill_layer(l, q, k, val, start, outs[-1], rope=rope)
    v.end_prefill()
    return outs


@pytest.mark.gpu
def test_steps_over_a_cache_in_4_bits():
    import paper_2512_21911_b200 as sv
    lens, blocks, keep = [700, 130], 13, 4
    gen = torch.Generator(device="cuda").manual_seed(0)
    v, pools = _verifier(2, blocks, True, keep, anchors=[True, False, True])
    _prefill(v, gen, lens, _rope(800))
    assert v.seq_lens.tolist() == lens
    # the same tokens through the calls, on buffers of their own
    geom, kv = v.geom, [sv.make_kv_q4(p, v.block_table, v.seq_lens) for p in pools]
    q, out = _normal(gen, L, 2, T, HQ, 128), torch.empty((L, 2, T, HQ, 128), dtype=torch.bfloat16, device="cuda")
    dk, dv = _normal(gen, L, 2, T, HKV, 128), _normal(gen, L, 2, T, HKV, 128)
    v.verify_step(q, dk, dv, out, refresh_tail=True)
    idx, cnt = torch.zeros((2, HKV, keep), dtype=torch.int32, device="cuda"), torch.zeros((2, HKV), dtype=torch.int32, device="cuda")
    ws, want = torch.empty_like(v._q4_workspace), torch.empty_like(q[0])
    for l in range(L):
        if l != 1:
            sv.sv_select_blocks(geom, q[l], v.reps[l], v.seq_lens, v.budget, v.n_sink, v.n_local, idx, cnt)
        sv.sv_verify_attn_q4(geom, q[l], kv[l], dk[l], dv[l], None, idx, cnt, want, workspace=ws)
        assert torch.equal(out[l], want)
    v.dense_step(q, dk, dv, out)
    sv.sv_verify_attn_q4(geom, q[2], kv[2], dk[2], dv[2], None, None, None, want, workspace=ws)
    assert torch.equal(out[2], want)
    path, n_path = _ints([[0, 2, -1, -1], [0, 1, 2, 3]]), _ints([2, 4])
    copies, lens_out = [p.clone() for p in pools], torch.empty_like(v.seq_lens)
    reps = v.reps.clone()
    for l in range(L):
        sv.sv_kv_append_q4(geom, copies[l], v.block_table, v.seq_lens, dk[l], dv[l], path, n_path, lens_out, reps=reps[l])
    v.commit(dk, dv, path, n_path)
    assert v.seq_lens.tolist() == [702, 134] == lens_out.tolist()
    assert all(torch.equal(a, b) for a, b in zip(pools, copies)) and torch.equal(v.reps, reps)
    v.check_status()


@pytest.mark.gpu
def test_a_step_over_a_cache_in_4_bits_is_captured():
    lens, gen = [300, 64], torch.Generator(device="cuda").manual_seed(1)
    v, _ = _verifier(2, 7, True, 3)
    _prefill(v, gen, lens, _rope(400))
    q, dk, dv = _normal(gen, L, 2, T, HQ, 128), _normal(gen, L, 2, T, HKV, 128), _normal(gen, L, 2, T, HKV, 128)
    out, again = (torch.zeros((L, 2, T, HQ, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        v.verify_step(q, dk, dv, out)
    graph.replay()
    v.verify_step(q, dk, dv, again)
    assert torch.equal(out, again)


def _dense(v, pools, l, q, dk, dv, s, h):
    """Attention of a sequence's draft in 64 bits over what the engine's cache holds now, and sum w |v|."""
    n = int(v.seq_lens[s])
    pages = v.block_table[s, :-(-n // B)].long()
    k, val = (torch.cat([p[l][pages, h].reshape(-1, 128)[:n], d[l, s, :, h]]).double() for p, d in ((pools[0], dk), (pools[1], dv)))
    G = HQ // HKV
    w = (q[l, s, :, h * G:(h + 1) * G].double() @ k.T / math.sqrt(128)).clone()
    hidden = torch.ones((T, T), dtype=torch.bool, device="cuda").triu(1)
    w[:, :, n:] = w[:, :, n:].masked_fill(hidden[:, None], -math.inf)
    p = torch.softmax(w, -1)
    return p @ val, p @ val.abs()


@pytest.mark.gpu
def test_weights_and_eviction():
    """Which tokens stay follows from the weights (sv_kv_evict has its own tests); verification afterwards is attention over those, positions go
    on counting, and a prompt that follows is rotated for them."""
    import paper_2512_21911_b200 as sv
    lens, blocks, gen = [700, 130], 13, torch.Generator(device="cuda").manual_seed(2)
    rope = _rope(900)
    v, pools = _verifier(2, blocks, False, blocks)
    _prefill(v, gen, lens, rope)
    q, dk, dv = _normal(gen, L, 2, T, HQ, 128), _normal(gen, L, 2, T, HKV, 128), _normal(gen, L, 2, T, HKV, 128)
    out = torch.empty((L, 2, T, HQ, 128), dtype=torch.bfloat16, device="cuda")
    path, n_path = _ints([[0, 1, -1, -1], [0, 1, 2, 3]]), _ints([2, 4])
    for l in range(L):
        lse = torch.empty((2, T, HQ), device="cuda")
        v.verify_layer(l, q[l], dk[l], dv[l], out[l], lse=lse)
        v.weigh_layer(l, q[l], lse, path, n_path)
    for s, n in enumerate(n_path.tolist()):       # the cache's part of the accepted rows' softmax: below one a row and query head, not by much
        total = torch.stack([w[s, :, :lens[s]].sum(-1) for w in v.weights])
        assert bool(((total < n * HQ // HKV) & (total > 0.5 * n * HQ // HKV)).all())
    heavy = v.weights[1][0, 1, :700].argmax()
    row = pools[0][1][v.block_table[0, int(heavy) // B].long(), 1, int(heavy) % B].clone()
    v.evict(_ints([300, 300]), n_sink=4, n_recent=32)
    assert v.seq_lens.tolist() == [300, 130] and v.positions().tolist() == lens
    at = int(v.weights[1][0, 1].argmax())
    assert torch.equal(pools[0][1][v.block_table[0, at // B].long(), 1, at % B], row) and at <= int(heavy)
    for l in range(L):
        v.verify_layer(l, q[l], dk[l], dv[l], out[l])
        for s in range(2):
            for h in range(HKV):
                want, A = _dense(v, pools, l, q, dk, dv, s, h)
                got = out[l, s, :, h * (HQ // HKV):(h + 1) * (HQ // HKV)].double()
                assert bool(((got - want).abs() <= 2.0 ** -8 * (A + want.abs()) + 2.0 ** -12 * A).all())
    # 40 more tokens: placed behind the 300 that are left, rotated for 700 ..
    start, parts = _ints([0, 40, 40]), _normal(gen, 40, HQ + 2 * HKV, 128)
    qn, kn, vn = parts.split([HQ, HKV, HKV], dim=1)
    v.prefill_layer(0, qn, kn, vn, start, torch.empty((40, HQ, 128), dtype=torch.bfloat16, device="cuda"), rope=rope)
    c, s = rope[700:740].chunk(2, 1)
    a, b = kn.float().chunk(2, -1)
    want = torch.cat([a * c[:, None] - b * s[:, None], b * c[:, None] + a * s[:, None]], -1).bfloat16()
    got = torch.stack([pools[0][0][v.block_table[0, p // B].long(), :, p % B] for p in range(300, 340)])
    assert torch.equal(got, want)
    v.check_status()


@pytest.mark.gpu
def test_rope_append_at_is_rope_append_at_other_positions():
    import paper_2512_21911_b200 as sv
    gen = torch.Generator(device="cuda").manual_seed(4)
    geom, table = sv.make_geom(2, 4, 2, 128, 64, 5, 1), _ints([[3, 1, 0, 2, 4], [9, 8, 7, 6, 5]])
    q, k, v = _normal(gen, 70, 8, 128).split([4, 2, 2], dim=1)
    start, rope = _ints([0, 69, 70]), _rope(400)
    res = []
    for lens, positions in (([100, 200], None), ([20, 40], _ints([100, 200])), ([20, 40], _ints([370, -3]))):
        pools, q_out, lens_out, status = [torch.zeros((10, 2, 64, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)], torch.empty((70, 4, 128), dtype=torch.bfloat16, device="cuda"), _ints([0, 0]), _ints([0])
        sv.sv_rope_append_at(geom, *pools, table, _ints(lens), positions, q, k, v, start, q_out, lens_out, rope=rope, status_word=status)
        assert lens_out.tolist() == [lens[0] + 69, lens[1] + 1]
        rows = [pools[0][table[s, (lens[s] + i) // 64].long(), :, (lens[s] + i) % 64] for s, n in ((0, 69), (1, 1)) for i in range(n)]
        res.append((q_out, torch.stack(rows), int(status)))
    assert torch.equal(res[0][0], res[1][0]) and torch.equal(res[0][1], res[1][1]) and res[0][2] == res[1][2] == 0
    assert res[2][2] == sv.SV_STATUS_INDEX                     # positions outside the table take its nearest row


@pytest.mark.gpu
@pytest.mark.parametrize("how", [dict(four_bits=True), dict(most=300)])
def test_the_example(how):
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import generate as example
    texts, kept, verifier = example.generate([list(range(500)), list(range(40))], new=12, layers=2, **how)
    assert all(len(t) >= 12 and all(0 <= x < example.VOCAB for x in t) for t in texts) and kept >= 1.0
    if "most" in how:
        assert verifier.seq_lens.max() <= 300 + example.DRAFT and verifier.positions()[0] >= 500 + 11


@pytest.mark.gpu
def test_layers_of_both_kinds():
    """Layer 1 in 4 bits between two of bfloat16: what the layers give alone."""
    import paper_2512_21911_b200 as sv
    lens, blocks, keep = [700, 130], 13, 4
    res = []
    for kinds in ([0, 0, 0], [1, 1, 1], [0, 1, 0]):
        gen = torch.Generator(device="cuda").manual_seed(6)
        v, _ = _verifier(2, blocks, True, keep, anchors=[True, False, True])
        v.kv_q4, v._grown_kv_q4 = [None] * L, [None] * L
        for l, kind in enumerate(kinds):
            if kind:
                v.set_layer_kv_q4(l, torch.zeros((2 * blocks, HKV, 1, sv.SV_Q4_SLAB_BYTES), dtype=torch.uint8, device="cuda"))
            else:
                v.set_layer_kv(l, *(torch.zeros((2 * blocks, HKV, B, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)))
        outs = _prefill(v, gen, lens, _rope(800))
        q, dk, dv = _normal(gen, L, 2, T, HQ, 128), _normal(gen, L, 2, T, HKV, 128), _normal(gen, L, 2, T, HKV, 128)
        out = torch.empty((L, 2, T, HQ, 128), dtype=torch.bfloat16, device="cuda")
        v.verify_step(q, dk, dv, out)
        v.commit(dk, dv, _ints([[0, 2, -1, -1], [0, 1, 2, 3]]), _ints([2, 4]))
        again = torch.empty_like(out)
        v.verify_step(q, dk, dv, again, refresh_tail=True)
        res.append([torch.stack(outs), out, again, v.reps])
        assert v.seq_lens.tolist() == [702, 134]
    bf16, q4, both = res
    assert all(torch.equal(b[l], (a, c)[l % 2][l]) for a, c, b in zip(bf16[:1] + bf16[3:], q4[:1] + q4[3:], both[:1] + both[3:]) for l in range(L))
    for i in (1, 2):                            # layer 1 reuses the list of layer 0, whose representatives differ between the two alone
        assert torch.equal(both[i][0], bf16[i][0]) and torch.equal(both[i][2], bf16[i][2])


@pytest.mark.gpu
def test_weights_over_replays():
    """The first call makes the buffer and is not captured; a captured one adds to it at every replay."""
    lens, gen = [300, 64], torch.Generator(device="cuda").manual_seed(7)
    v, _ = _verifier(2, 7, False, 3)
    _prefill(v, gen, lens, _rope(400))
    q, dk, dv = _normal(gen, 2, T, HQ, 128), _normal(gen, 2, T, HKV, 128), _normal(gen, 2, T, HKV, 128)
    out, lse = torch.empty_like(q), torch.empty((2, T, HQ), device="cuda")
    v.verify_layer(0, q, dk, dv, out, lse=lse)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(RuntimeError):
            v.weigh_layer(0, q, lse)
        v.verify_layer(0, q, dk, dv, out, lse=lse)
    v.weigh_layer(0, q, lse)
    once = v.weights[0].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        v.verify_layer(0, q, dk, dv, out, lse=lse)
        v.weigh_layer(0, q, lse)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(v.weights[0], (once + once) + once)


@pytest.mark.gpu
def test_what_the_engine_refuses():
    v, _ = _verifier(1, 3, True, 2)
    with pytest.raises(TypeError):
        v.evict(_ints([10]))
    with pytest.raises(TypeError):
        v.weigh_layer(0, None, None)
    w, pools = _verifier(1, 3, False, 2)
    with pytest.raises(AssertionError):
        w.set_layer_kv_q4(0, torch.zeros((3, HKV, 1, 9216), dtype=torch.uint8, device="cuda"))
