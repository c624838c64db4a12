"""sv_attn_weights against the sum of exponentials in 64 bits.

A score is off by at most 128 2^-24 sum |q k| scale, some 1e-4 here at the most and 1e-5 as a rule; the exponent's rounding to fp32 (up to
60) by 60 2^-24 = 4e-6; the sum of n terms of one sign by n 2^-24.  So a weight is off by at most 2e-4 of what is added to it, and by 2^-24 of
itself."""
import math

import numpy as np
import pytest
import torch

SIGMA = math.sqrt(3.0)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _inputs(lens, Hq, Hkv, B, T, keep=0, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    S, NB = len(lens), max(1, max(-(-n // B) for n in lens)) + 1
    t = dict(k=torch.empty((S * NB, Hkv, B, 128), dtype=torch.bfloat16, device="cuda").normal_(0.0, SIGMA, generator=gen), lens=_ints(lens),
             table=torch.from_numpy(rng.permutation(S * NB).astype(np.int32).reshape(S, NB)).cuda(),
             q=torch.empty((S, T, Hq, 128), dtype=torch.bfloat16, device="cuda").normal_(0.0, SIGMA, generator=gen),
             lse=torch.rand((S, T, Hq), generator=gen, device="cuda") * 4 + 6, w=torch.rand((S, Hkv, NB * B), generator=gen, device="cuda"),
             idx=None, cnt=None, path=None, n_path=None, dims=(lens, Hq, Hkv, B, T, NB))
    for s, n in enumerate(lens):               # what no sequence holds is NaN
        if n % B:
            t["k"][int(t["table"][s, n // B]), :, n % B:] = float("nan")
    if keep:
        idx, cnt = np.full((S, Hkv, keep), 10 ** 6, np.int32), np.zeros((S, Hkv), np.int32)
        for s, n in enumerate(lens):
            for h in range(Hkv):
                cnt[s, h] = min(-(-n // B), keep if h else keep // 2)
                idx[s, h, :cnt[s, h]] = np.sort(rng.permutation(-(-n // B))[:cnt[s, h]])
        t["idx"], t["cnt"] = torch.from_numpy(idx).cuda(), torch.from_numpy(cnt).cuda()
    return t


def _run(sv, t, out=None):
    lens, Hq, Hkv, B, T, NB = t["dims"]
    geom, status = sv.make_geom(len(lens), Hq, Hkv, 128, B, NB, T), _ints([0])
    kv = sv.make_kv(t["k"], None, t["table"], t["lens"])
    out = torch.full_like(t["w"], -3.0) if out is None else out
    sv.sv_attn_weights(geom, t["q"], kv, t["lse"], t["w"], out, sel_idx=t["idx"], sel_cnt=t["cnt"], path=t["path"], n_path=t["n_path"], status_word=status)
    return out, int(status)


def _exact(t):
    lens, Hq, Hkv, B, T, NB = t["dims"]
    G, added = Hq // Hkv, torch.zeros(t["w"].shape, dtype=torch.float64, device="cuda")
    for s, n in enumerate(lens):
        rows = list(range(T)) if t["path"] is None else t["path"][s, :int(t["n_path"][s])].tolist()
        for h in range(Hkv):
            tok = torch.arange(n, device="cuda")
            if t["idx"] is not None:
                kept = t["idx"][s, h, :int(t["cnt"][s, h])].long()
                tok = (kept[:, None] * B + torch.arange(B, device="cuda")).reshape(-1)
                tok = tok[tok < n]
            k = t["k"][t["table"][s].long(), h].reshape(-1, 128)[tok].double()
            for i in rows:
                w = t["q"][s, i, h * G:(h + 1) * G].double() @ k.T / math.sqrt(128) - t["lse"][s, i, h * G:(h + 1) * G].double()[:, None]
                added[s, h, tok] += torch.exp(w).sum(0)
    return added


def _close(t, got):
    added, held = _exact(t), torch.arange(t["w"].shape[-1], device="cuda") < t["lens"][:, None, None]
    held = held.expand_as(got)
    assert (got[~held] == -3.0).all()
    want = t["w"].double() + added
    assert bool(((got.double() - want).abs()[held] <= (2e-4 * added + 2.0 ** -24 * want)[held]).all())


CASES = [([1], 1, 1, 64, 1, 0), ([0, 5], 4, 2, 64, 3, 0), ([63, 64, 65, 129, 400], 8, 2, 64, 1, 0), ([700, 2000], 14, 2, 128, 5, 0), ([333], 32, 8, 64, 8, 0),
         ([1000, 77], 128, 1, 64, 1, 0), ([500], 64, 2, 128, 16, 0), ([300, 900], 16, 16, 64, 2, 0), ([3000, 60, 1], 8, 2, 64, 4, 6), ([5000, 640], 28, 4, 128, 60, 9),
         ([0, 200], 8, 2, 64, 2, 3), ([30000], 8, 2, 64, 1, 0)]


@pytest.mark.gpu
@pytest.mark.parametrize("lens,Hq,Hkv,B,T,keep", CASES)
def test_weights(lens, Hq, Hkv, B, T, keep):
    import paper_2512_21911_b200 as sv
    t = _inputs(lens, Hq, Hkv, B, T, keep)
    out, status = _run(sv, t)
    assert status == 0
    _close(t, out)
    again, _ = _run(sv, t)
    assert torch.equal(out, again)
    held = torch.arange(out.shape[-1], device="cuda") < t["lens"][:, None, None]
    same = t["w"].clone()                       # in place
    t["w"] = same
    got, _ = _run(sv, t, out=same)
    assert torch.equal(got[held.expand_as(got)], out[held.expand_as(out)])


@pytest.mark.gpu
def test_the_rows_that_were_accepted():
    import paper_2512_21911_b200 as sv
    t = _inputs([500, 900, 64], 20, 4, 64, 7, 5)
    t["path"] = _ints([[0, 3, 6, -1, -1, -1, -1], [0, 1, 2, 3, 4, 5, 6], [-1] * 7])
    t["n_path"] = _ints([3, 7, 0])
    out, status = _run(sv, t)
    assert status == 0
    _close(t, out)
    assert torch.equal(out[2, :, :64], t["w"][2, :, :64])


@pytest.mark.gpu
def test_rows_without_a_denominator_and_bad_indices():
    import paper_2512_21911_b200 as sv
    t = _inputs([200], 4, 1, 64, 2)
    t["lse"][0, 0, 1] = -math.inf               # a row that saw nothing gives nothing
    out, _ = _run(sv, t)
    t["lse"][0, 0, 1] = math.inf
    assert torch.equal(out, _run(sv, t)[0])
    t["lse"][0, 1, 0] = float("nan")
    assert torch.isnan(_run(sv, t)[0][0, 0, :200]).all()
    t = _inputs([200], 4, 1, 64, 2)
    t["path"], t["n_path"] = _ints([[0, 9]]), _ints([2])
    assert _run(sv, t)[1] == sv.SV_STATUS_INDEX
    t = _inputs([200], 4, 1, 64, 2, 2)
    t["idx"][0, 0, 0] = -1
    t["cnt"][0, 0] = 1
    assert _run(sv, t)[1] == sv.SV_STATUS_INDEX
    t["idx"][0, 0, 0] = -(2 ** 31)              # (what is kept as it was begins behind an index that is clamped too)
    out, status = _run(sv, t)
    assert status == sv.SV_STATUS_INDEX and bool((out[0, 0, 64:200] == t["w"][0, 0, 64:200]).all())
    t["cnt"][0, 0] = -1
    out, status = _run(sv, t)
    assert status == sv.SV_STATUS_NO_LIST and torch.equal(out[0, 0, :200], t["w"][0, 0, :200])


@pytest.mark.gpu
@pytest.mark.parametrize("odd", [float("nan"), float("inf"), -float("inf")])
def test_a_key_that_is_not_finite_concerns_rows_that_count(odd):
    """Of three rows (the tile has room for 16) one has no denominator: without it, or with no row at all, an odd key gets nothing."""
    import paper_2512_21911_b200 as sv
    t = _inputs([200], 3, 1, 64, 1)
    t["k"][int(t["table"][0, 1]), 0, 7] = odd   # token 71
    t["lse"].fill_(-math.inf)
    out, _ = _run(sv, t)
    assert torch.equal(out[0, 0, :200], t["w"][0, 0, :200])
    t = _inputs([200], 3, 1, 64, 1)
    t["q"].abs_()
    want, _ = _run(sv, t)
    t["k"][int(t["table"][0, 1]), 0, 7] = odd
    out, _ = _run(sv, t)
    got, others = float(out[0, 0, 71]), torch.arange(200, device="cuda") != 71
    assert torch.equal(out[0, 0, :200][others], want[0, 0, :200][others])
    assert got == float(t["w"][0, 0, 71]) if odd == -math.inf else got == math.inf if odd == math.inf else math.isnan(got)


@pytest.mark.gpu
def test_weights_of_a_verification_sum_to_one():
    """With the lse of sv_verify_attn over the same blocks, a row's weights and those of its own draft tokens are a softmax."""
    import paper_2512_21911_b200 as sv
    lens, Hq, Hkv, B, T = [900, 333], 8, 2, 64, 3
    t = _inputs(lens, Hq, Hkv, B, T)
    NB = t["dims"][-1]
    geom = sv.make_geom(2, Hq, Hkv, 128, B, NB, T)
    gen = torch.Generator(device="cuda").manual_seed(9)
    dk, dv = (torch.empty((2, T, Hkv, 128), dtype=torch.bfloat16, device="cuda").normal_(generator=gen) for _ in range(2))
    kv = sv.make_kv(t["k"], torch.zeros_like(t["k"]), t["table"], t["lens"])
    ws = torch.empty(max(16, sv.sv_workspace_bytes(geom, NB)), dtype=torch.uint8, device="cuda")
    sv.sv_verify_attn(geom, t["q"], kv, dk, dv, None, None, None, torch.empty_like(t["q"]), lse=t["lse"], workspace=ws)
    t["w"].zero_()
    out, _ = _run(sv, t)
    own = torch.zeros((2, Hkv), dtype=torch.float64, device="cuda")
    for i in range(T):
        for j in range(i + 1):
            w = (t["q"][:, i].double().view(2, Hkv, -1, 128) * dk[:, j].double()[:, :, None]).sum(-1) / math.sqrt(128)
            own += torch.exp(w - t["lse"][:, i].double().view(2, Hkv, -1)).sum(-1)
    held = torch.arange(out.shape[-1], device="cuda") < t["lens"][:, None, None]
    total = (out.double() * held).sum(-1) + own
    assert bool(((total - T * Hq // Hkv).abs() <= 1e-3 * T * Hq // Hkv + 1e-3).all())
