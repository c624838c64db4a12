"""SparseVerifier.prefill_layer and end_prefill where a serving loop can go wrong: tokens that the block table has no pages for, captured
graphs beside larger batches, a turn of the loop without new tokens."""
import gc
import weakref

import pytest
import torch

pytestmark = pytest.mark.gpu
HQ, HKV, B, L = 8, 2, 64, 2


def _verifier(S, blocks, draft=4):
    from paper_2512_21911_b200.engine import SparseVerifier
    table = torch.randperm(S * blocks, generator=torch.Generator().manual_seed(5)).int().view(S, blocks).cuda()
    v = SparseVerifier(n_seq=S, n_q_heads=HQ, n_kv_heads=HKV, head_dim=128, block_size=B, max_blocks=blocks, n_draft=draft, n_layers=L, block_table=table,
                       seq_lens=torch.zeros(S, dtype=torch.int32, device="cuda"), budget_blocks=torch.full((S,), blocks, dtype=torch.int32, device="cuda"),
                       max_sel=blocks)
    v.set_kv_stack(*[torch.zeros((L, S * blocks, HKV, B, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)])
    return v


class _Batch:
    """New tokens of the sequences, n[s] of sequence s, the same in all layers."""

    def __init__(self, n, seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda heads: torch.empty((sum(n), heads, 128), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
        self.q, self.k, self.v = normal(HQ), normal(HKV), normal(HKV)
        self.start = torch.tensor([sum(n[:s]) for s in range(len(n) + 1)], dtype=torch.int32, device="cuda")
        self.out = [torch.zeros_like(self.q) for _ in range(L)]

    def run(self, v):
        for l in range(L):
            v.prefill_layer(l, self.q, self.k, self.v, self.start, self.out[l])


def test_tokens_without_pages_are_reported():
    import paper_2512_21911_b200 as sv
    for break_table in (False, True):
        v = _verifier(2, 3)
        _Batch([100, 150], 1).run(v)
        v.end_prefill()
        v.check_status()
        if break_table:
            v.block_table[1, 2] = -1                 # 150 tokens end in the block of this entry's page: 42 more would fit if it had one
        _Batch([5, 30 if break_table else 60], 2).run(v)
        v.end_prefill()
        with pytest.raises(sv.SvError):
            v.check_status()
        assert int(v.status) == sv.SV_STATUS_INDEX and v.seq_lens.tolist() == [105, 150 if break_table else 192]


@pytest.mark.parametrize("length,new,bad", [(0, 193, True), (0, 192, False), (192, 1, True), (192, 0, False), (191, 1, False), (200, 0, False), (-3, 2, True), (-3, 0, False)])
def test_the_status_of_an_append(length, new, bad):
    import paper_2512_21911_b200 as sv
    b = _Batch([new], 3)
    pool = torch.zeros((3, HKV, B, 128), dtype=torch.bfloat16, device="cuda")
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    out, status = ints(0), ints(0)
    sv.sv_rope_append(sv.make_geom(1, HQ, HKV, 128, B, 3, 1), pool, pool.clone(), ints(0, 1, 2).view(1, 3), ints(length), b.q, b.k, b.v, b.start,
                      torch.empty_like(b.q), out, status_word=status)
    assert int(status) == (sv.SV_STATUS_INDEX if bad else 0)
    assert int(out) == (length if length < 0 else max(length, min(length + new, 192)))


def test_a_buffer_that_was_used_stays_when_larger_batches_follow():
    """What a captured graph has the address of; together the buffers stay below twice the largest."""
    v = _verifier(1, 40)
    used, sizes = [], []
    for n in (1, 5, 6, 100, 20, 101, 300, 301):
        _Batch([n], n).run(v)
        used += [weakref.ref(v._turned), weakref.ref(v._chunk_workspace)]
        sizes.append(v._turned.shape[0])
    gc.collect()
    assert all(r() is not None for r in used)
    assert len({r().data_ptr() for r in used[1::2]}) == 1
    assert sum(set(sizes)) <= 2 * sizes[-1] and sizes[-1] <= 2 * 301


def test_the_workspace_does_for_every_batch():
    import paper_2512_21911_b200 as sv
    for Hq, Hkv in ((8, 2), (1, 1), (128, 1), (7, 1), (64, 64)):
        g = sv.make_geom(3, Hq, Hkv, 128, B, 40, 1)
        assert all(sv.sv_chunk_workspace_bytes(g, n) <= sv.sv_chunk_workspace_bytes(g, 129) for n in (1, 2, 31, 127, 128, 129, 130, 5000, 30000))


@pytest.mark.parametrize("first", [True, False])
def test_a_captured_batch_beside_a_larger_one(first):
    """A graph of a decoding batch, which may be the engine's first call; a larger batch runs, memory that was given back is taken and filled, the graph runs again."""
    v, w = _verifier(2, 20), _verifier(2, 20)
    prompt, small, large = _Batch([70, 200], 1), _Batch([1, 3], 2), _Batch([300, 500], 3)
    for x in (v, w):
        prompt.run(x)
        x.end_prefill()
    v._turned = v._chunk_workspace = None
    if not first:
        _Batch([4, 0], 4).run(v)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        small.run(v)
        v.end_prefill()
    large.run(v)
    v.end_prefill()
    taken = [torch.full((n,), 0x7f7f, dtype=torch.int16, device="cuda") for n in (512, 4096, 1 << 15, 1 << 20, 1 << 24)]
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    got = [o.clone() for o in small.out]
    assert all(bool((t == 0x7f7f).all()) for t in taken)
    large.run(w)
    w.end_prefill()
    small.run(w)
    w.end_prefill()
    assert all(torch.equal(a, b) for a, b in zip(got, small.out)) and v.seq_lens.tolist() == w.seq_lens.tolist() == [371, 703]
    for x in (v, w):
        x.check_status()


def test_the_end_of_a_prefill_that_was_not_there():
    v = _verifier(2, 20)
    v.seq_lens.copy_(torch.tensor([7, 0], dtype=torch.int32))
    v.end_prefill()
    assert v.seq_lens.tolist() == [7, 0]
    _Batch([100, 30], 1).run(v)
    v.end_prefill()
    assert v.seq_lens.tolist() == [107, 30]
    v.end_prefill()
    assert v.seq_lens.tolist() == [107, 30]
    gen = torch.Generator(device="cuda").manual_seed(2)
    draft_k, draft_v = (torch.empty((L, 2, 4, HKV, 128), dtype=torch.bfloat16, device="cuda").normal_(generator=gen) for _ in range(2))
    v.commit(draft_k, draft_v, torch.arange(4, dtype=torch.int32, device="cuda").repeat(2, 1), torch.tensor([3, 1], dtype=torch.int32, device="cuda"))
    assert v.seq_lens.tolist() == [110, 31]
    v.end_prefill()
    assert v.seq_lens.tolist() == [110, 31]
    v.seq_lens.copy_(torch.tensor([0, 31], dtype=torch.int32))     # the first place goes to another request
    v.end_prefill()
    assert v.seq_lens.tolist() == [0, 31]
    _Batch([2, 0], 3).run(v)
    v.end_prefill()
    assert v.seq_lens.tolist() == [2, 31]


@pytest.mark.parametrize("end_inside", [False, True])
def test_layers_in_a_graph_and_the_end_in_it_or_behind_it(end_inside):
    v = _verifier(2, 20)
    b = _Batch([3, 1], 1)
    b.run(v)
    v.end_prefill()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.run(v)
        if end_inside:
            v.end_prefill()
    for i in range(2, 5):
        graph.replay()
        if not end_inside:
            v.end_prefill()
        assert v.seq_lens.tolist() == [3 * i, i]
    v.check_status()
