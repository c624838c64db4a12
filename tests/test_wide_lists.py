"""Block lists whose rows are longer than 2^24 entries: a list is found by the length of the rows, whatever that is."""
import pytest
import torch

from test_q4_attn import SIGMA, _cache, _drafts, _ints, _verify

pytestmark = pytest.mark.gpu
WIDE = (1 << 24) + 64


def _lists():
    """The same lists in rows of eight and in long ones, whose other entries are zero."""
    narrow = _ints([[[0, 2, 3, 5, 0, 0, 0, 0], [1, 2, 4, 0, 0, 0, 0, 0]]])
    wide = torch.zeros((1, 2, WIDE), dtype=torch.int32, device="cuda")
    wide[:, :, :8] = narrow
    return narrow, wide, _ints([[4, 3]])


@pytest.mark.parametrize("T", [3, 40])
def test_verify(T):
    import paper_2512_21911_b200 as sv
    c = _cache([500], 2, 64)
    q, dk, dv, _ = _drafts(1, T, 8, 2, 0, False)
    narrow, wide, cnt = _lists()
    want, lse_want, _ = _verify(sv, c, q, dk, dv, None, (narrow, cnt), True)
    out, lse, status = _verify(sv, c, q, dk, dv, None, (wide, cnt), True)
    assert status == 0 and torch.equal(out, want) and torch.equal(lse, lse_want)


def test_weights():
    import paper_2512_21911_b200 as sv
    gen = torch.Generator(device="cuda").manual_seed(0)
    pool, q = (torch.empty(s, dtype=torch.bfloat16, device="cuda").normal_(0.0, SIGMA, generator=gen) for s in ((8, 2, 64, 128), (1, 3, 8, 128)))
    geom, table, lens = sv.make_geom(1, 8, 2, 128, 64, 8, 3), _ints([[7, 1, 0, 2, 4, 5, 3, 6]]), _ints([500])
    lse, got = torch.full((1, 3, 8), 9.0, device="cuda"), []
    narrow, wide, cnt = _lists()
    for idx in (narrow, wide):
        w = torch.zeros((1, 2, 512), device="cuda")
        sv.sv_attn_weights(geom, q, sv.make_kv(pool, None, table, lens), lse, w, w, sel_idx=idx, sel_cnt=cnt)
        got.append(w)
    assert torch.equal(*got) and int((got[0] > 0).sum()) > 300
