"""launches_per_step and kernels_per_step of stacks with 4-bit layers against the kernels that a capture of the calls holds."""
import pytest
import torch

from test_launch_counts import _kernels

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kinds", [[1, 1, 1], [0, 1, 0], [1, 0, 1]])
@pytest.mark.parametrize("S,Hq,Hkv,T,NB,keep", [(1, 8, 2, 4, 40, 16), (2, 8, 2, 40, 40, 24), (1, 32, 8, 20, 400, 300), (19, 32, 8, 5, 20, 15),
                                                (2, 8, 2, 40, 9000, 8), (20, 64, 8, 16, 18, 16), (1, 1, 1, 64, 2, 2), (1, 2, 1, 64, 2, 2)])
def test_launches_are_counted_as_they_are_made(kinds, S, Hq, Hkv, T, NB, keep):
    import paper_2512_21911_b200 as sv
    L, pages = len(kinds), S * min(NB, 30)
    lens = torch.full((S,), min(NB, 30) * 64 - 9, dtype=torch.int32, device="cuda")
    table = torch.zeros((S, NB), dtype=torch.int32, device="cuda")
    table[:, :30] = torch.arange(pages, dtype=torch.int32, device="cuda").view(S, -1)
    eng = sv.SparseVerifier(n_seq=S, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=128, block_size=64, max_blocks=NB, n_draft=T, n_layers=L, block_table=table,
                            seq_lens=lens, max_sel=keep, budget_blocks=torch.full_like(lens, keep), anchors=[True, False, True])
    rows = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")
    for l, kind in enumerate(kinds):
        if kind:
            eng.set_layer_kv_q4(l, torch.zeros((pages, Hkv, 1, sv.SV_Q4_SLAB_BYTES), dtype=torch.uint8, device="cuda"))
        else:
            eng.set_layer_kv(l, rows(pages, Hkv, 64, 128), rows(pages, Hkv, 64, 128))
    q, dk, dv, out = (rows(S, T, h, 128) for h in (Hq, Hkv, Hkv, Hq))
    step = lambda: [eng.verify_layer(l, q, dk, dv, out, behind_own_layer=l > 0) for l in range(L)]
    assert _kernels(step) == eng.launches_per_step() <= eng.kernels_per_step()

    def with_tail():
        eng._refresh_tail(eng._anchor_flags())
        step()
    assert _kernels(with_tail) == eng.launches_per_step(refresh_tail=True) <= eng.kernels_per_step(refresh_tail=True)
    dense = lambda: [eng.dense_layer(l, q, dk, dv, out) for l in range(L)]
    assert _kernels(dense) <= eng.kernels_per_step(dense=True) and _kernels(lambda: eng.dense_layer(kinds.index(1), q, dk, dv, out)) == eng._q4_launches(True)
    eng.check_status()
