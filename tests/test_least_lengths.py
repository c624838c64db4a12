"""Chunks of sequences whose lengths are negative, down to the least number there is: every row is at a position below zero and sees nothing."""
import numpy as np
import pytest
import torch

from test_chunk_shares import lib  # noqa: F401


@pytest.mark.parametrize("length", [-1, -1000, -2 ** 31 + 5, -2 ** 31])
@pytest.mark.parametrize("new,G", [(3, 4), (700, 4), (2, 1)])
def test_division(lib, length, new, G):  # noqa: F811
    start, lens, buf, rows = np.array([0, new, new + 5], np.int32), np.array([length, 300], np.int32), np.zeros((1024, 10), np.int32), set()
    for cta in range(8):
        n = lib.shares_of(start.ctypes.data, lens.ctypes.data, 2, new + 5, 2, 128 // G, 640, 8, cta, buf.ctypes.data, len(buf))
        for s, h, row0, tokens, pos0, kv_end, u0, u1, units, parts in buf[:n].tolist():
            if s == 0:
                assert pos0 + tokens <= 0 and kv_end == units == u0 == u1 == parts == 0
                rows |= {(h, row0 + i) for i in range(tokens)}
    assert rows == {(h, i) for h in range(2) for i in range(new)}


@pytest.mark.gpu
@pytest.mark.parametrize("length", [-1, -1000, -2 ** 31 + 5, -2 ** 31])
@pytest.mark.parametrize("new,little", [(3, False), (90, False), (90, True)])
def test_rows_below_zero(length, new, little):
    """Over a 4-bit cache, decoded first or not, and with as many rows over a bfloat16 one; the other sequence has what it has alone."""
    import paper_2512_21911_b200 as sv
    from test_q4_attn import SIGMA, _cache, _chunk, _ints
    c = _cache([0, 300], 2, 64, seed=3)
    q = torch.empty((new + 40, 8, 128), dtype=torch.bfloat16, device="cuda").normal_(0.0, SIGMA, generator=torch.Generator(device="cuda").manual_seed(0))
    want, lse_want, _ = _chunk(sv, c, q, [new, 40], little)
    c["lens"] = _ints([length, 300])
    out, lse, status = _chunk(sv, c, q, [new, 40], little)
    assert status == 0 and (out[:new] == 0).all() and torch.isneginf(lse[:new]).all()
    assert torch.equal(out[new:], want[new:]) and torch.equal(lse[new:], lse_want[new:])
    geom, pools = sv.make_geom(2, 8, 2, 128, 64, c["NB"], 1), [torch.zeros((c["pool"].shape[0], 2, 64, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    ws = torch.empty(sv.sv_chunk_workspace_bytes(geom, new + 40), dtype=torch.uint8, device="cuda")
    sv.sv_chunk_attn(geom, q, sv.make_kv(*pools, c["table"], c["lens"]), _ints([0, new, new + 40]), out.fill_(7.0), lse=lse.fill_(7.0), workspace=ws)
    assert (out == 0).all() and torch.isneginf(lse[:new]).all() and torch.isfinite(lse[new:]).all()
