"""sv_sample: the kept entries, their distribution and the token drawn, against the rule in 64 bits; what the call refuses.

Tolerances: an exponential and the sums that go with it are good to 2^-20 of themselves, so a probability is within 1e-5 of itself.
Which entries stay is decided by comparisons: the parameters of the cases lie in the middle of what decides the same (half a token's mass
away from either side), so the sets have to be equal.  A token is right if the sums on either side of it enclose u to 1e-6 of the whole."""
import ctypes
import math

import numpy as np
import pytest
import torch


def _rule(x, temperature=None, k=None, top_p=None, min_p=None):
    """The distribution of a row in 64 bits (numpy), and the entries in order with what is ahead of them, of the first k."""
    x = np.asarray(x, np.float64)
    x = np.where(np.isnan(x), -np.inf, x)
    there = x > -np.inf
    p = np.zeros(len(x))
    if not there.any():
        return p, None
    T = 1.0 if temperature is None else temperature
    order = np.lexsort((np.arange(len(x)), -x))
    order = order[:there.sum()]
    if not T > 0:
        p[order[0]] = 1
        return p, None
    with np.errstate(invalid="ignore"):
        e = np.where(x == x[order[0]], 1.0, np.exp((x - x[order[0]]) / T))
    if k is not None and k > 0:
        order = order[:k]
    ahead = np.concatenate([[0], np.cumsum(e[order])])
    whole = ahead[-1]
    n = len(order)
    if top_p is not None and top_p < 1:
        n = max(1, int((ahead[:-1] < top_p * whole).sum()))
    keep = order[:n]
    if min_p is not None and min_p > 0:
        keep = keep[(e[keep] >= min_p) | (np.arange(len(keep)) == 0)]
    p[keep] = e[keep] / e[keep].sum()
    return p, ahead / whole


def _middle(x, top_p, **kw):
    """The middle of the mass of the entry that top_p falls into."""
    _, ahead = _rule(x, **kw)
    i = min(np.searchsorted(ahead, top_p, side="right") - 1, len(ahead) - 2)
    return float((ahead[i] + ahead[i + 1]) / 2)


def _sample(logits, u, probs=True, **kw):
    import paper_2512_21911_b200 as sv
    R = logits.numel() // logits.shape[-1]
    tokens = torch.full((R,), -9, dtype=torch.int32, device="cuda")
    p = torch.full((R, logits.shape[-1]), 7.0, device="cuda") if probs else None
    dev = lambda a, t: None if a is None else torch.as_tensor(a, dtype=t, device="cuda")
    sv.sv_sample(logits, dev(u, torch.float32), tokens, probs=p, temperature=dev(kw.get("temperature"), torch.float32), top_k=dev(kw.get("k"), torch.int32),
                 top_p=dev(kw.get("top_p"), torch.float32), min_p=dev(kw.get("min_p"), torch.float32))
    return tokens.cpu().numpy(), None if p is None else p.cpu().numpy().astype(np.float64)


def _check_rows(x, u, tokens, p, temperature=None, k=None, top_p=None, min_p=None):
    pick = lambda a, i: None if a is None else float(a[i])
    for i in range(len(x)):
        want, _ = _rule(x[i], pick(temperature, i), None if k is None else int(k[i]), pick(top_p, i), pick(min_p, i))
        if p is not None:
            far = np.abs(p[i] - want) > 1e-5 * want + 1e-30
            # entries whose exponential is below what fp32 holds are zero; nothing else may differ
            far &= ~((want < 1e-37) & (p[i] == 0))
            assert not far.any(), (i, np.nonzero(far)[0][:5], p[i][far][:5], want[far][:5])
        t = int(tokens[i])
        if not want.any():
            assert t == -1
            continue
        cum = np.cumsum(want)
        assert want[t] > 0
        assert cum[t] - want[t] <= u[i] + 1e-6 and cum[t] >= u[i] - 1e-6, (i, t, cum[t] - want[t], u[i], cum[t])


def _logits(R, V, seed=0, half=False, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((R, V + pad), generator=g, device="cuda") / 0.35
    return (x.bfloat16() if half else x)[:, :V]


SIZES = [1, 2, 31, 1000, 1023, 4096, 32003, 128256, 200001]


@pytest.mark.gpu
@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("V", SIZES)
def test_sizes_and_every_restriction(V, half):
    R = 9
    logits = _logits(R, V, V, half, pad=0 if V % 2 else 24)
    x = logits.float().cpu().numpy()
    g = np.random.default_rng(V)
    u = g.random(R).astype(np.float32)
    T = np.float32([1.0, 0.7, 0.0, 1.5, 1.0, 0.3, 1.0, 2.0, 1.0])
    k = np.int32([0, 50, 5, 1, 7, 300, -1, 2 * V, 20])
    top_p = [2.0, 0.9, 0.5, 0.9, 0.99, 0.8, 0.999, 0.3, 0.0]
    min_p = np.float32([0, 0, 0.3, 0, 0.021, 0, 0.0101, 0, 0])
    kk = lambda i: int(k[i]) if k[i] > 0 else None
    top_p = np.float32([a if a >= 1 or a == 0 or not T[i] > 0 else _middle(x[i], a, temperature=float(T[i]), k=kk(i)) for i, a in enumerate(top_p)])
    tokens, p = _sample(logits, u, temperature=T, k=k, top_p=top_p, min_p=min_p)
    _check_rows(x, u, tokens, p, T, k, top_p, min_p)
    for only in (dict(), dict(temperature=T), dict(k=k), dict(min_p=min_p), dict(temperature=T, k=k)):
        tokens, p = _sample(logits, u, **only)
        _check_rows(x, u, tokens, p, **only)
    assert np.array_equal(_sample(logits, u, probs=False, temperature=T, k=k, top_p=top_p, min_p=min_p)[0],
                          _sample(logits, u, temperature=T, k=k, top_p=top_p, min_p=min_p)[0])


@pytest.mark.gpu
def test_ties_go_to_the_lowest_index():
    V = 5000
    x = np.zeros((6, V), np.float32)
    x[1, ::7] = 2.0
    x[2] = np.repeat(np.arange(V // 10), 10)[::-1] / 40.0
    x[3, :] = -0.0
    x[3, 1::2] = 0.0                                       # two zeros of different sign are equal
    x[4] = np.random.default_rng(0).integers(0, 4, V)
    x[5, 4999] = 1.0
    k = np.int32([10, 3, 13, 11, 700, 4])
    logits = torch.from_numpy(x).cuda()
    for u in (0.0, 0.37, 0.999):
        us = np.full(6, u, np.float32)
        tokens, p = _sample(logits, us, k=k)
        _check_rows(x, us, tokens, p, k=k)
        assert np.array_equal(np.nonzero(p[0])[0], np.arange(10)) and np.array_equal(np.nonzero(p[3])[0], np.arange(11))
    # half of the mass of V equal entries: the first half of them (the goal is half an entry's mass off the sums)
    top_p = np.float32([(V / 2 - 0.5) / V] * 6)
    for i in (1, 2, 4, 5):
        top_p[i] = _middle(x[i], 0.5)
    tokens, p = _sample(logits, us, top_p=top_p)
    _check_rows(x, us, tokens, p, top_p=top_p)
    assert np.array_equal(np.nonzero(p[0])[0], np.arange(V // 2))
    both = np.float32([_middle(x[i], 0.6, k=int(k[i])) for i in range(6)])
    tokens, p = _sample(logits, us, k=k, top_p=both)
    _check_rows(x, us, tokens, p, k=k, top_p=both)


@pytest.mark.gpu
@pytest.mark.parametrize("V", [100, 128256])
def test_entries_that_are_not_there(V):
    g = np.random.default_rng(V)
    x = (g.standard_normal((9, V)) * 3).astype(np.float32)
    x[0] = -np.inf
    x[1] = np.nan
    x[2, g.random(V) < 0.9] = -np.inf                      # most of the vocabulary is masked
    x[3] = np.finfo(np.float32).min                        # masked with the type's lowest value, all but one, and all
    x[3, V // 2] = 1.0
    x[4] = np.finfo(np.float32).min
    x[5, [3, V - 1]] = np.inf
    x[6, ::2] = np.nan
    x[7] = -np.inf
    x[7, V - 1] = -5.0
    x[8, 1:] = -np.inf
    u = g.random(9).astype(np.float32)
    logits = torch.from_numpy(x).cuda()
    T = np.float32([1, 1, 0.5, 1, 2, 1, 0, 1, 0.8])
    tokens, p = _sample(logits, u, temperature=T)
    _check_rows(x, u, tokens, p, T)
    assert tokens[0] == tokens[1] == -1 and tokens[3] == V // 2 and tokens[7] == V - 1 and tokens[8] == 0
    k = np.full(9, 5, np.int32)
    tokens, p = _sample(logits, u, k=k, temperature=T)
    _check_rows(x, u, tokens, p, T, k)
    top_p = np.float32([0.5, 0.5] + [_middle(x[i], 0.7, temperature=float(T[i])) if T[i] > 0 else 0.5 for i in range(2, 9)])
    tokens, p = _sample(logits, u, top_p=top_p, temperature=T)
    _check_rows(x, u, tokens, p, T, top_p=top_p)
    odd = np.float32(["nan", -1, 1, 1, "nan", 1, 1, 1, 1])
    tokens, p = _sample(logits, u, temperature=odd, top_p=np.float32(["nan"] * 9), min_p=np.float32(["nan"] * 9))
    _check_rows(x, u, tokens, p, np.nan_to_num(odd))


@pytest.mark.gpu
def test_many_entries_of_nearly_the_same_logit():
    """Everything in one corner of the range: the search meets crowded bins at every step."""
    V = 100000
    g = np.random.default_rng(1)
    x = np.stack([1e-3 * g.random(V), 50 + np.float32(2.0 ** -17) * g.integers(0, 3, V), -30 + 1e-5 * g.standard_normal(V),
                  np.where(np.arange(V) < 10, 40.0, 1e-6 * g.random(V))]).astype(np.float32)
    u = np.float32([0.5, 0.25, 0.75, 0.99])
    logits = torch.from_numpy(x).cuda()
    for T in (1.0, 1e-4, 100.0):
        t = np.full(4, T, np.float32)
        k = np.int32([1234, 50000, 99999, 12])
        tokens, p = _sample(logits, u, temperature=t, k=k)
        _check_rows(x, u, tokens, p, t, k)
        top_p = np.float32([_middle(x[i], 0.5, temperature=float(t[i])) for i in range(4)])
        tokens, p = _sample(logits, u, temperature=t, top_p=top_p)
        want = [_rule(x[i], float(t[i]), None, float(top_p[i]))[0] for i in range(4)]
        for i in range(4):
            # 100000 entries of the same mass: half of one is 5e-6 of the whole, which top_p in fp32 holds, but exponentials in fp32 may
            # move the cut by a few entries
            assert abs(int((p[i] > 0).sum()) - int((want[i] > 0).sum())) <= 1e-5 * V
            assert abs(p[i].sum() - 1) <= 1e-5


@pytest.mark.gpu
@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("n", [1, 31, 32, 33, 255, 300, 512, 513, 767, 768, 769, 1500])
def test_the_boundary_lies_among_n_neighbours(n, half):
    """2,000 entries ahead, n of nearly or exactly the same logit, 5,000 behind; the boundary at the first, inside and at the last of the n."""
    V = 9000
    g = np.random.default_rng(n)
    places = np.stack([g.permutation(V) for _ in range(9)])
    x = np.full((9, V), -9.0, np.float32)
    step = np.float32(2.0 ** -20)
    for i in range(9):
        near = [np.arange(n) * step, np.zeros(n), (np.arange(n) % 3 == 0) * step][i // 3].astype(np.float32)
        x[i, places[i, :2000]] = g.uniform(-1, 2, 2000)
        x[i, places[i, 2000:2000 + n]] = np.float32(-3) + near
        x[i, places[i, 2000 + n:2000 + n + 5000]] = g.uniform(-8, -4, 5000)
    logits = torch.from_numpy(x).cuda()
    if half:
        logits = logits.bfloat16()
        x = logits.float().cpu().numpy()
    u = g.random(9).astype(np.float32)
    k = np.int32([2000 + m for m in (1, (n + 1) // 2, n)] * 3)
    tokens, p = _sample(logits, u, k=k)
    _check_rows(x, u, tokens, p, k=k)
    for kw in (dict(), dict(k=np.full(9, 2000 + n, np.int32))):
        _, ahead = zip(*[_rule(row, k=None if not kw else 2000 + n) for row in x])
        top_p = np.float32([(a[at - 1] + a[at]) / 2 for a, at in zip(ahead, k)])   # (entry number k is the last that begins below it)
        tokens, p = _sample(logits, u, top_p=top_p, **kw)
        _check_rows(x, u, tokens, p, top_p=top_p, **kw)


@pytest.mark.gpu
def test_tokens_follow_the_distribution_and_u_of_zero_and_one():
    V, R = 50, 4000
    logits = _logits(1, V, 3).expand(R, V).contiguous()
    u = (np.arange(R) + 0.5).astype(np.float32) / R
    tokens, p = _sample(logits, u, temperature=np.full(R, 1.0, np.float32))
    counts = np.bincount(tokens, minlength=V) / R
    assert np.abs(counts - p[0]).max() <= 1.5 / R
    tokens, p = _sample(logits[:4], np.float32([0.0, 1.0, -3.0, np.nan]))
    there = np.nonzero(p[0])[0]
    assert tokens[0] == there[0] and tokens[1] == there[-1] and tokens[2] == there[0] and tokens[3] == there[0]


@pytest.mark.gpu
def test_sequences_of_rows_share_their_parameters():
    import paper_2512_21911_b200 as sv
    S, T, V = 3, 4, 1000
    x = _logits(S * T, V, 5).view(S, T, V)
    temp, k = torch.tensor([0.5, 1.0, 0.0], device="cuda"), torch.tensor([3, 0, 5], dtype=torch.int32, device="cuda")
    u = torch.rand(S * T, device="cuda")
    tok, p = torch.zeros((S, T), dtype=torch.int32, device="cuda"), torch.zeros((S, T, V), device="cuda")
    sv.sv_sample(x, u, tok, probs=p, temperature=temp, top_k=k)
    flat = np.repeat(temp.cpu().numpy(), T), np.repeat(k.cpu().numpy(), T)
    t2, p2 = _sample(x.reshape(S * T, V), u.cpu().numpy(), temperature=flat[0], k=flat[1])
    assert np.array_equal(tok.cpu().numpy().ravel(), t2) and np.array_equal(p.cpu().numpy().reshape(S * T, V), p2.astype(np.float32))


@pytest.mark.gpu
def test_feeds_acceptance():
    """Target distributions equal to the draft's: every draft token is accepted."""
    import paper_2512_21911_b200 as sv
    S, T, V = 2, 5, 32000
    x = _logits(S * T, V, 6).view(S, T, V)
    p = torch.empty((S, T, V), device="cuda")
    tok = torch.empty((S, T), dtype=torch.int32, device="cuda")
    sv.sv_sample(x, torch.rand(S * T, device="cuda"), tok, probs=p, temperature=torch.tensor([0.8, 1.0], device="cuda"), top_p=torch.tensor([0.9, 0.8], device="cuda"))
    tokens = torch.cat([torch.zeros((S, 1), dtype=torch.int32, device="cuda"), tok[:, :-1]], 1).contiguous()   # row i + 1: drawn from row i
    path, n_path, nxt = (torch.empty(s, dtype=torch.int32, device="cuda") for s in ((S, T), (S,), (S,)))
    sv.sv_accept(p, p, tokens, None, torch.rand((S, T), device="cuda"), torch.rand(S, device="cuda"), path, n_path, nxt)
    assert n_path.tolist() == [T, T]


@pytest.mark.gpu
def test_on_another_stream_and_in_a_graph():
    import paper_2512_21911_b200 as sv
    x, u = _logits(20, 30000, 8), torch.rand(20, device="cuda")
    k = torch.full((20,), 40, dtype=torch.int32, device="cuda")
    want, got = (torch.zeros(20, dtype=torch.int32, device="cuda") for _ in range(2))
    sv.sv_sample(x, u, want, top_k=k)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        sv.sv_sample(x, u, got, top_k=k)
    side.synchronize()
    assert torch.equal(got, want)
    got.zero_()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sv.sv_sample(x, u, got, top_k=k)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, want)


@pytest.mark.gpu
def test_tensors_that_do_not_fit_are_refused():
    import paper_2512_21911_b200 as sv
    x, u, tok = _logits(4, 100), torch.rand(4, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    for bad in (x.double(), x.cpu(), x.t(), x[0], x.view(2, 2, 100).transpose(0, 1)):
        with pytest.raises(TypeError):
            sv.sv_sample(bad, u, tok)
    with pytest.raises(TypeError):
        sv.sv_sample(x, u, tok.long())
    for kw in (dict(u=u[:3]), dict(tokens=tok[:3]), dict(probs=torch.zeros((4, 99), device="cuda")), dict(top_p=u[:2]), dict(top_k=tok[:1])):
        with pytest.raises(ValueError):
            sv.sv_sample(**{**dict(logits=x, u=u, tokens=tok), **kw})
    with pytest.raises(sv.SvError):
        sv.sv_sample(x, None, tok)
    with pytest.raises(sv.SvError):
        sv.sv_sample(x, u, None)


def test_refusals_without_a_device():
    import paper_2512_21911_b200.binding as b

    def call(rows=4, V=1000, x=0x1000, half=0, stride=1000, per=1, u=0x2000, tokens=0x3000, probs=0x4000):
        return b._lib.sv_sample(rows, V, x, half, stride, per, None, None, None, None, u, tokens, probs, None)

    assert call(x=None) == 1 and call(u=None) == 1 and call(tokens=None, probs=None) == 1
    assert call(rows=-1) == 2 and call(V=0) == 2 and call(stride=999) == 2 and call(per=0) == 2 and call(per=3) == 2
    assert call(V=(1 << 20) + 1, stride=1 << 21) == 6
    assert call(x=0x1002) == 3 and call(probs=0x4002) == 3 and call(x=0x1001, half=1) == 3
    assert call(rows=0) == 0
