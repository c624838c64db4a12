"""SparseVerifier.prefill_layer and end_prefill where a serving loop can go wrong: tokens that the block table has no pages for, captured
graphs beside larger batches, a turn of the loop without new tokens."""
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
