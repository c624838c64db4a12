"""sv_sample where an entry stays or goes by little: goals next to an edge between two entries, limits of the parameters, the largest
vocabularies."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def _draw(x, u=None, **parameters):
    """Tokens and distributions of rows x (a CUDA tensor), parameters one a row."""
    import paper_2512_21911_b200 as sv
    R, V = x.shape
    tokens, probs = torch.full((R,), -9, dtype=torch.int32, device="cuda"), torch.full((R, V), 7.0, device="cuda")
    types = dict(top_k=torch.int32)
    sv.sv_sample(x, torch.full((R,), 0.5, device="cuda") if u is None else u, tokens, probs=probs,
                 **{k: torch.as_tensor(v, dtype=types.get(k, torch.float32), device="cuda") for k, v in parameters.items()})
    return tokens, probs


def test_the_rate_keeps_more_bits_than_a_float():
    """Half of the mass in one entry, half in 2^17 of them 16 to 18 powers of two below, and temperatures whose log2 e / T is half a unit of
    its last place away from a float.  A rate rounded to a float is off by up to 2^-24, which changes the 2^17 by 17 ln 2 2^-24 = 7e-7 of
    themselves and the sums between them by a quarter of that, 1.8e-7 of the whole.  Exponentials good to 2^-22 change the sums by 6e-8 at
    most (all of them off the same way); the other roundings are a hundred thousand independent ones.  So goals from 9e-8 on beside an edge
    between entries have to fall on the right side of it."""
    rng = np.random.default_rng(0)
    rate = lambda T: math.log2(math.e) / float(T)
    off = lambda T: float(np.float32(rate(T))) / rate(T) - 1
    Ts = [T for T in rng.uniform(0.5, 1.5, 4000).astype(np.float32) if abs(off(T)) > 0.85 * 2.0 ** -24]
    Ts = [T for T in Ts if off(T) > 0][:8] + [T for T in Ts if off(T) < 0][:8]
    assert len(Ts) == 16
    rows, top_p, want = [], [], []
    for T in Ts:
        x = np.concatenate([[0.0], -(16 + 2 * rng.random(1 << 17)) * math.log(2) * float(T)]).astype(np.float32)
        order = np.argsort(-x, kind="stable")
        edge = np.cumsum(np.exp(x[order].astype(np.float64) / float(T)))
        edge /= edge[-1]
        for side in (-1, 1):
            p = np.float32(edge + side * 1.05e-7)     # a float next to every edge, the first of them that is as near as wanted
            far = side * (p.astype(np.float64) - edge)
            n = int(np.nonzero((far >= 0.9e-7) & (far <= 1.2e-7) & (edge > 0.6) & (edge < 0.9))[0][0])
            keep = order[:n + 1 + (side > 0)]         # the entries that begin below the goal
            rows.append(x), top_p.append(p[n]), want.append(np.sort(keep))
    logits = torch.from_numpy(np.stack(rows)).cuda()
    _, probs = _draw(logits, temperature=np.repeat(np.float32(Ts), 2), top_p=np.float32(top_p))
    kept = (probs > 0).cpu().numpy()
    wrong = [(i, int(kept[i].sum()) - len(w)) for i, w in enumerate(want) if not np.array_equal(np.nonzero(kept[i])[0], w)]
    assert not wrong, wrong


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("V", [5, 1000, 128256])
def test_min_p_around_one_and_tied_maxima(V, half):
    """Above 1 the first entry alone stays, with or without other restrictions; at 1 all that equal the largest."""
    gen = torch.Generator(device="cuda").manual_seed(V)
    x = torch.randn((6, V), generator=gen, device="cuda")
    tied = [V // 3, V // 2 + 1, V - 1]
    x[:, tied] = 9.0
    if half:
        x = x.bfloat16()
    min_p = [1.5, math.inf, float(np.nextafter(np.float32(1), np.float32(2))), 1.0, float(np.nextafter(np.float32(1), np.float32(0))), 1.5]
    kept = [tied[:1]] * 3 + [tied] * 2 + [tied[:1]]
    for more in (dict(), dict(temperature=[0.3] * 5 + [0.0]), dict(top_k=[3, 3, 0, 7, 50, 2]), dict(top_p=[0.999999] * 6), dict(temperature=[4.0] * 6, top_p=[2.0] * 6, top_k=[0] * 6)):
        tokens, probs = _draw(x, min_p=min_p, **more)
        for i, want in enumerate(kept):
            assert probs[i].nonzero().flatten().tolist() == want, (i, more)
            assert bool((probs[i, want] - 1 / len(want)).abs().max() <= 1e-6) and int(tokens[i]) == want[(len(want) - 1) // 2]


def _tiny(rng, n):
    """Numbers below the smallest normal one, of either sign, and zeros."""
    return (rng.integers(-3, 4, n) * np.float32(2.0 ** -130)).astype(np.float32)


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("V", [40, 5000, 50000])
def test_logits_below_the_smallest_normal_number_are_zeros(V, half):
    """So that all of them are equal, and the first ones stay; as the largest entries of a row and among others."""
    rng = np.random.default_rng(V)
    x = np.full((4, V), -3.0, np.float32)
    x[0] = _tiny(rng, V)
    x[1, ::3] = _tiny(rng, len(x[1, ::3]))
    x[2, ::2] = _tiny(rng, len(x[2, ::2]))
    x[2, :3] = 1.0
    x[3] = _tiny(rng, V)
    x[3, V // 2] = np.float32(2.0 ** -120)                 # larger than all, and e is 1 as theirs
    ahead = [np.arange(V), np.arange(0, V, 3), np.concatenate([np.arange(3), np.arange(4, V, 2)]), np.concatenate([[V // 2], np.delete(np.arange(V), V // 2)])]
    logits = torch.from_numpy(x).cuda()
    if half:
        logits = logits.bfloat16()
        assert bool((logits.float().abs().cpu() > 0).numpy()[x != 0].all())
    for k in (1, 5, 11):
        tokens, probs = _draw(logits, top_k=[k] * 4, u=torch.zeros(4, device="cuda"))
        for i in range(4):
            want = np.sort(ahead[i][:k])
            assert probs[i].nonzero().flatten().tolist() == want.tolist(), (k, i)
            assert abs(float(probs[i].double().sum()) - 1) <= 1e-5 and int(tokens[i]) == want[0]
    tokens, probs = _draw(logits, temperature=[0.0] * 4)
    assert tokens.tolist() == [0, 0, 0, V // 2] and probs.count_nonzero(1).tolist() == [1] * 4
    n = [V // 2, len(ahead[1]) // 2]
    top_p = [(n[0] - 0.5) / V, (n[1] - 0.5) / (len(ahead[1]) + (V - len(ahead[1])) * math.exp(-3))]
    _, probs = _draw(logits[:2], top_p=top_p)
    for i in range(2):
        assert probs[i].nonzero().flatten().tolist() == ahead[i][:n[i]].tolist()


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("V", [217089, 262145, 300001, 350208, 393215, 393216])
def test_the_largest_vocabularies(V, half):
    """Parts of 14 to 24 grains of 2,048 entries: up to 192 KB of a row's fp32 entries in a CTA's shared memory, and the limit itself."""
    rng = np.random.default_rng(V)
    gen = torch.Generator(device="cuda").manual_seed(V)
    x = torch.randn((5, V), generator=gen, device="cuda") * 3
    x[:, V - 1] = 14.0                                     # the largest by far is the last entry
    if half:
        x = x.bfloat16()
    rows = x.double().cpu().numpy()
    order = np.argsort(-rows, axis=1, kind="stable")
    e = np.exp(rows - rows.max(1, keepdims=True))
    ranked = np.take_along_axis(e, order, 1)
    whole = np.cumsum(ranked, 1)
    n = [1, 40, 2000, 100000, V - 1]

    def check(probs, tokens, counts, u):
        for i, m in enumerate(counts):
            want = np.zeros(V)
            want[order[i, :m]] = ranked[i, :m] / whole[i, m - 1]
            got = probs[i].double().cpu().numpy()
            assert (np.abs(got - want) <= 1e-5 * want).all(), i
            upto = np.cumsum(want)
            t = int(tokens[i])
            assert want[t] > 0 and upto[t] - want[t] <= u[i] + 1e-6 and upto[t] >= u[i] - 1e-6

    u = rng.random(5).astype(np.float32)
    draw = lambda **kw: _draw(x, u=torch.from_numpy(u).cuda(), **kw)
    for parameters, counts in ((dict(), [V] * 5), (dict(top_k=n), n),
                               (dict(top_p=[(whole[i, m - 1] - ranked[i, m - 1] / 2) / whole[i, -1] for i, m in enumerate([1, 40, 2000, 9000, 3])]), [1, 40, 2000, 9000, 3])):
        tokens, probs = draw(**parameters)
        check(probs, tokens, counts, u)


def test_a_larger_vocabulary_is_refused():
    import paper_2512_21911_b200 as sv
    x = torch.zeros((1, 393217), device="cuda")
    with pytest.raises(sv.SvError):
        sv.sv_sample(x, torch.zeros(1, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"))
