"""sv_chunk_attn on numbers that are not finite: what a row sees shows in its output and its lse, what it does not see leaves it alone.

The pattern of NaNs is that of softmax attention in 64 bits; where that is finite the output is within 2^-8 |o| + (2^-8 + 2^-12) sum p |v| (its
rounding, that of the probabilities, fp32)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), math.inf


def _case(lens, new, Hq=8, Hkv=2, B=64, seed=0):
    import paper_2512_21911_b200 as sv
    S, N = len(lens), sum(new)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    NB = max(-(-n // B) for n in lens)
    return dict(q=normal(N, Hq, 128), k=normal(S, NB, Hkv, B, 128), v=normal(S, NB, Hkv, B, 128), lens=lens, new=new, geom=sv.make_geom(S, Hq, Hkv, 128, B, NB, 1))


def _run(t):
    import paper_2512_21911_b200 as sv
    S, NB = t["k"].shape[:2]
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    start = [sum(t["new"][:s]) for s in range(S + 1)]
    out, lse = torch.full_like(t["q"], 77.0), torch.full(t["q"].shape[:2], 77.0, device="cuda")
    ws = torch.empty(sv.sv_chunk_workspace_bytes(t["geom"], len(out)), dtype=torch.uint8, device="cuda")
    status, table, lens = ints([0]), ints(range(S * NB)).view(S, NB), ints(t["lens"])     # (a kv holds addresses: its tensors have to stay)
    kv = sv.make_kv(t["k"].view(S * NB, *t["k"].shape[2:]), t["v"].view(S * NB, *t["v"].shape[2:]), table, lens)
    sv.sv_chunk_attn(t["geom"], t["q"], kv, ints(start), out, lse=lse, workspace=ws, status_word=status)
    assert int(status) == 0
    return out, lse


def _check(t):
    out, lse = _run(t)
    at, (Hq, Hkv) = 0, (t["geom"].n_q_heads, t["geom"].n_kv_heads)
    nans = 0
    for s, (L, n) in enumerate(zip(t["lens"], t["new"])):
        k, v = (x[s].transpose(0, 1).flatten(1, 2)[:, :L].double() for x in (t["k"], t["v"]))
        for i in range(n):
            seen = L - n + i + 1
            x = torch.einsum("hgd,htd->hgt", t["q"][at + i].double().view(Hkv, Hq // Hkv, 128), k[:, :seen]) / math.sqrt(128)
            p = torch.softmax(x, -1)
            want, room = (torch.einsum("hgt,htd->hgd", p, w).view(Hq, 128) for w in (v[:, :seen], v[:, :seen].abs()))
            got = out[at + i].double()
            assert torch.equal(got.isnan(), want.isnan()), (s, i)
            fine = want.isfinite()
            assert bool(((got - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -12) * room)[fine].all())
            ref = torch.logsumexp(x, -1).view(Hq)
            # (of an infinite score the sum is infinite: inf or NaN; of scores that are all -infinity its logarithm is -infinity)
            known = ref.isfinite()
            assert bool(((lse[at + i].double() - ref).abs() <= 1e-3)[known].all()) and not bool(lse[at + i][~known].isfinite().any())
            assert bool((lse[at + i][ref == -INF] == -INF).all())
            nans += int(want.isnan().sum())
        at += n
    return nans


def _slot(t, s, position):
    return s, position // t["k"].shape[3], slice(None), position % t["k"].shape[3]


@pytest.mark.parametrize("value", [NAN, INF])
@pytest.mark.parametrize("lens,new,at", [([1], [1], 0), ([200], [200], 70), ([300], [300], 129), ([70, 300, 64], [70, 40, 1], 280), ([20000], [1], 3),
                                         ([20000], [1], 13000), ([20000], [40], 19990)])
def test_a_key_that_is_seen(lens, new, at, value):
    """Whole items of one and two tiles; items cut into many shares; rows on both sides of the key."""
    t = _case(lens, new, seed=at)
    t["k"][_slot(t, len(lens) // 2, at)][:, 5] = value     # (of an infinity times a query of either sign half of the rows have a NaN)
    assert _check(t) > 0


@pytest.mark.parametrize("lens,new", [([5], [5]), ([300], [300]), ([20000], [1])])
def test_a_query(lens, new):
    t = _case(lens, new)
    t["q"][len(t["q"]) // 2, 3, 77] = NAN
    assert _check(t) == 128


@pytest.mark.parametrize("lens,new", [([1], [1]), ([500], [1]), ([20000], [1]), ([70, 900], [1, 1])])
def test_a_value(lens, new):
    t = _case(lens, new)
    t["v"][_slot(t, len(lens) - 1, lens[-1] // 2)][:, 9] = NAN
    assert _check(t) == 8


def test_keys_behind_a_row_and_slots_that_nobody_has():
    t = _case([100, 200], [100, 50])
    for s, L in enumerate(t["lens"]):
        k, v = (x[s].transpose(0, 1).flatten(1, 2) for x in (t["k"].clone(), t["v"].clone()))
        k[:, L:], v[:, L:] = NAN, NAN
        for x, y in ((t["k"], k), (t["v"], v)):
            x[s] = y.unflatten(1, x.shape[1:2] + x.shape[3:4]).transpose(0, 1)
    t["k"][_slot(t, 0, 99)] = NAN                          # the last token's key: no other row sees it
    assert _check(t) == 8 * 128


@pytest.mark.parametrize("lens,new", [([1], [1]), ([30], [5]), ([20000], [1]), ([20000], [30])])
def test_rows_whose_scores_are_all_minus_infinity(lens, new):
    """They see keys, so that softmax has nothing to say (0 / 0); rows that stand before the beginning see none and stay zero."""
    t = _case(lens, new)
    t["q"][:] = 1.0
    t["k"][..., 0] = -INF
    out, lse = _run(t)
    assert bool(out.isnan().all()) and bool((lse == -INF).all())
    assert _check(t) == 128 * 8 * new[0]


def test_rows_before_the_beginning():
    """Next to rows that see a NaN, in a whole item and in one that is cut."""
    for L, n, Hq, Hkv in ((3, 10, 8, 2), (3000, 3020, 64, 1)):
        t = _case([L], [n], Hq, Hkv)
        t["k"][0, 0, :, 0] = NAN
        out, lse = _run(t)
        assert bool((out[:n - L] == 0).all()) and bool((lse[:n - L] == -INF).all())
        assert bool(out[n - L:].isnan().all()) and bool(lse[n - L:].isnan().all())
