"""sv_verify_attn_q4 and sv_chunk_attn_q4 against softmax attention in 64 bits over the values that the cache's codes stand for.

With weights w of the softmax and A = sum w |v|: the rounding of a weight to bf16 is off by 2^-8 of it, that of the output by 2^-8 of it.
Scores are sums of 128 products of bf16 numbers in fp32, off by at most 128 2^-24 sum |q k| scale (some 1e-4 here); that and the
exponentials' 2^-22 count twice, in the weight and in the sum.  So |out - exact| <= 2^-8 (A + |exact|) + 5e-4 A, and lse is off by 3e-4."""
import math

import numpy as np
import pytest
import torch

from q4_reference import SLAB, get

SIGMA = math.sqrt(3.0)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _cache(lens, Hkv, B, seed=0, spare=1, junk=0x7f):
    """Random codes and sensible scales; what no sequence holds has `junk` in every byte (scales that are NaN).  Keys and values of every
    sequence in 64 bits as well."""
    rng = np.random.default_rng(seed)
    S, NB = len(lens), max(1, max(-(-max(n, 0) // B) for n in lens)) + spare
    pool = np.full((S * NB, Hkv, B // 64, SLAB), junk, np.uint8)
    table = rng.permutation(S * NB).astype(np.int32).reshape(S, NB)
    to_bits = lambda x: (np.asarray(x, np.float32).view(np.uint32) >> 16).astype(np.uint16)
    keys, values = [], []
    for s, n in enumerate(lens):
        k, v = np.zeros((Hkv, max(n, 0), 128)), np.zeros((Hkv, max(n, 0), 128))
        for j in range(-(-max(n, 0) // 64)):
            for h in range(Hkv):
                slab = pool[table[s, j * 64 // B], h, j * 64 % B // 64]
                m = min(64, n - j * 64)
                full = rng.integers(0, 256, 8192).astype(np.uint8)
                # a token's codes: of the keys whole bytes, of the values one nibble of a word
                slab[:4096].reshape(4, 64, 16)[:, :m] = full[:4096].reshape(4, 64, 16)[:, :m]
                slab[4096:8192] = full[4096:]
                d = rng.uniform(6.0, 10.0, (64, 2)) * SIGMA / 1.7
                sc = np.stack([to_bits(d), to_bits(-1.5 * d + rng.normal(size=(64, 2)))], -1)               # [token][group][D, M]
                slab[8192:8704].reshape(64, 8)[:m] = sc.view(np.uint8).reshape(64, 8)[:m]
                d = rng.uniform(3.0, 6.0, (2, 1, 64))
                sc = np.concatenate([to_bits(d), to_bits(-1.5 * d)], 1)                                     # [group][D, M][token]
                slab[8704:].reshape(4, 64, 2)[:, :m] = sc.view(np.uint8).reshape(4, 64, 2)[:, :m]
                kk, vv = get(slab)
                k[h, j * 64:j * 64 + m], v[h, j * 64:j * 64 + m] = kk[:m], vv[:m]
        keys.append(torch.from_numpy(k).cuda())
        values.append(torch.from_numpy(v).cuda())
    return dict(pool=torch.from_numpy(pool).cuda(), table=torch.from_numpy(table).cuda(), lens=_ints(lens), k=keys, v=values, NB=NB, B=B, Hkv=Hkv)


def _softmax(w, v):
    """Output, denominator and A of rows of scores w over values v."""
    lse = torch.logsumexp(w, -1)
    p = torch.exp(w - lse[:, None])
    return p @ v, lse, p @ v.abs()


def _close(out, lse, want, lse_want, A):
    out, lse = out.double(), lse.double()
    assert torch.isfinite(out).all()
    assert bool(((out - want).abs() <= 2.0 ** -8 * (A + want.abs()) + 5e-4 * A).all())
    assert bool(((lse - lse_want).abs() <= 3e-4).all())


def _drafts(S, T, Hq, Hkv, seed, tree):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda h, sigma: torch.empty((S, T, h, 128), dtype=torch.bfloat16, device="cuda").normal_(0.0, sigma, generator=gen)
    parent = None
    if tree:
        rng = np.random.default_rng(seed)
        parent = _ints([[-1] + [int(rng.integers(max(0, i - 9), i)) for i in range(1, T)] for _ in range(S)])
    return normal(Hq, SIGMA), normal(Hkv, SIGMA), normal(Hkv, 1.0), parent


def _exact_verify(c, q, dk, dv, parent, lists):
    S, T, Hq = q.shape[:3]
    G = Hq // c["Hkv"]
    out, lse, A = (torch.zeros(s, dtype=torch.float64, device="cuda") for s in (q.shape, q.shape[:3], q.shape))
    for s in range(S):
        sees = torch.eye(T, dtype=torch.bool, device="cuda") if parent is not None else torch.ones((T, T), dtype=torch.bool, device="cuda").tril()
        if parent is not None:
            for i in range(1, T):
                sees[i] |= sees[int(parent[s, i])]
        n = c["k"][s].shape[1]
        for h in range(c["Hkv"]):
            t = torch.arange(n, device="cuda")
            if lists is not None:
                kept = lists[0][s, h, :max(0, int(lists[1][s, h]))].long()
                t = (kept[:, None] * c["B"] + torch.arange(c["B"], device="cuda")).reshape(-1)
                t = t[t < n]
            k, v = torch.cat([c["k"][s][h, t], dk[s, :, h].double()]), torch.cat([c["v"][s][h, t], dv[s, :, h].double()])
            w = (q[s, :, h * G:(h + 1) * G].double() @ k.T / math.sqrt(128)).clone()
            w[:, :, len(t):] = w[:, :, len(t):].masked_fill(~sees[:, None], -math.inf)
            o, l, a = _softmax(w.reshape(T * G, -1), v)
            out[s, :, h * G:(h + 1) * G], lse[s, :, h * G:(h + 1) * G], A[s, :, h * G:(h + 1) * G] = o.view(T, G, 128), l.view(T, G), a.view(T, G, 128)
    return out, lse, A


def _lists(c, keep, seed, shuffled=False):
    rng = np.random.default_rng(seed)
    S, Hkv = len(c["k"]), c["Hkv"]
    idx, cnt = np.full((S, Hkv, keep), 10 ** 6, np.int32), np.zeros((S, Hkv), np.int32)
    for s in range(S):
        blocks = -(-c["k"][s].shape[1] // c["B"])
        for h in range(Hkv):
            cnt[s, h] = min(blocks, int(rng.integers(0, keep + 1)) if h else keep)
            got = rng.permutation(blocks)[:cnt[s, h]]
            idx[s, h, :cnt[s, h]] = got if shuffled else np.sort(got)
    return torch.from_numpy(idx).cuda(), torch.from_numpy(cnt).cuda()


def _scratch(sv, geom, little):
    """Workspace for the geometry; or as much as any call takes, which leaves no room for a decoded cache."""
    size = sv.sv_workspace_bytes_q4(sv.make_geom(1, 1, 1, 128, 64, 1, 1) if little else geom)
    return torch.full((size,), 0xff, dtype=torch.uint8, device="cuda")


def _verify(sv, c, q, dk, dv, parent, lists, little=False, **over):
    S, T, Hq = q.shape[:3]
    geom = sv.make_geom(S, Hq, c["Hkv"], 128, c["B"], c["NB"], T)
    kv = sv.make_kv_q4(c["pool"], c["table"], c["lens"])
    ws = _scratch(sv, geom, little)
    out, lse = torch.full_like(q, float("nan")), torch.full((S, T, Hq), float("nan"), device="cuda")
    status = _ints([0])
    sv.sv_verify_attn_q4(geom, q, kv, dk, dv, parent, *(lists or (None, None)), out, lse=lse, workspace=ws, status_word=status, **over)
    return out, lse, int(status)


@pytest.mark.gpu
@pytest.mark.parametrize("lens,Hq,Hkv,B,T,tree,keep", [
    ([1], 1, 1, 64, 1, False, 0), ([0], 4, 2, 64, 1, False, 0), ([63, 64, 65, 127, 128, 129], 8, 2, 64, 1, False, 0), ([5, 0, 700, 191], 8, 2, 128, 3, False, 0),
    ([1000, 64], 14, 2, 64, 5, True, 0), ([333, 2100], 32, 2, 128, 1, False, 0), ([640], 16, 16, 64, 2, False, 0), ([300, 257], 128, 1, 64, 1, False, 0),
    ([900], 64, 1, 64, 2, False, 0), ([1500, 20], 28, 4, 64, 60, True, 0), ([400], 40, 8, 128, 64, True, 0), ([90, 3000, 1], 8, 2, 64, 4, True, 5),
    ([6000, 700, 128], 32, 8, 128, 8, False, 7), ([9000], 8, 2, 64, 1, False, 40), ([20000, 3, 9000], 8, 4, 64, 1, False, 0)])
def test_verify(lens, Hq, Hkv, B, T, tree, keep):
    import paper_2512_21911_b200 as sv
    c = _cache(lens, Hkv, B, seed=len(lens) + T)
    q, dk, dv, parent = _drafts(len(lens), T, Hq, Hkv, T, tree)
    lists = _lists(c, keep, 1) if keep else None
    exact = _exact_verify(c, q, dk, dv, parent, lists)
    for little in (False, True):
        out, lse, status = _verify(sv, c, q, dk, dv, parent, lists, little)
        assert status == 0
        _close(out, lse, *exact)


@pytest.mark.gpu
def test_lists_in_any_order_and_marked_ones():
    import paper_2512_21911_b200 as sv
    c = _cache([1000, 500, 100], 2, 64)
    q, dk, dv, _ = _drafts(3, 2, 8, 2, 0, False)
    lists = _lists(c, 9, 3, shuffled=True)
    out, lse, status = _verify(sv, c, q, dk, dv, None, lists)
    assert status == 0
    _close(out, lse, *_exact_verify(c, q, dk, dv, None, lists))
    lists[1][1, 0] = -1                        # a list that selection marked: the draft alone, and the status says so
    out, lse, status = _verify(sv, c, q, dk, dv, None, lists)
    assert status == sv.SV_STATUS_NO_LIST
    _close(out, lse, *_exact_verify(c, q, dk, dv, None, lists))


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 20])
def test_indices_outside_their_tables_are_clamped(T):
    import paper_2512_21911_b200 as sv
    c = _cache([300], 1, 64, junk=0)
    q, dk, dv, _ = _drafts(1, T, 4, 1, 0, False)
    for bad in (-5, c["NB"], 1 << 30):
        out, _, status = _verify(sv, c, q, dk, dv, None, (_ints([[[0, bad]]]), _ints([[2]])))
        assert status == sv.SV_STATUS_INDEX and torch.isfinite(out.float()).all()
    c["table"][0, 1] = c["pool"].shape[0]
    assert _verify(sv, c, q, dk, dv, None, None)[2] == sv.SV_STATUS_INDEX
    c["lens"][0] = 10 ** 9                     # a length beyond the table is cut to it
    c["table"][0, 1] = 0
    assert torch.isfinite(_verify(sv, c, q, dk, dv, None, None)[0].float()).all()


@pytest.mark.gpu
@pytest.mark.parametrize("T", [2, 40])
def test_nan_and_infinite_scores_show(T):
    import paper_2512_21911_b200 as sv
    c = _cache([200, 200], 1, 64)
    q, dk, dv, _ = _drafts(2, T, 2, 1, 0, False)
    clean, _, _ = _verify(sv, c, q, dk, dv, None, None)
    q[0, 0, 1, 5] = float("nan")
    q[1, 1, 0, 5] = float("inf")
    out, _, status = _verify(sv, c, q, dk, dv, None, None)
    bad = torch.isnan(out.float()).all(-1)
    assert status == 0 and bad.nonzero().tolist() == [[0, 0, 1], [1, 1, 0]]
    assert torch.equal(out[~bad], clean[~bad])


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [0.0, 1e-9, 3.0])
def test_scale(scale):
    """All tokens alike, and the likeliest alone: sums of products are then off by 128 2^-24 of a sum of absolute values of 600 * scale, 1.4e-2
    in all.  A weight below 2^-126 of the largest is zero in fp32: of 703 tokens with values up to 10 that is 703 * 10 * 2^-126 < 1e-34."""
    import paper_2512_21911_b200 as sv
    c = _cache([700], 2, 64)
    q, dk, dv, _ = _drafts(1, 3, 8, 2, 0, False)
    out, _, _ = _verify(sv, c, q, dk, dv, None, None, softmax_scale=scale)
    s = scale * math.sqrt(128) if scale else 1.0
    want, _, A = _exact_verify(c, q.double() * s, dk, dv, None, None)
    assert bool(((out.double() - want).abs() <= 2.0 ** -8 * (A + want.abs()) + (3e-2 if scale > 1 else 5e-4) * A + 1e-34).all())


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    """A pool of 4.5 GB, its last pages in use."""
    import paper_2512_21911_b200 as sv
    c = _cache([500, 70], 8, 64)
    n = (1 << 32) // (8 * SLAB) + 100
    big = torch.empty((n, 8, 1, SLAB), dtype=torch.uint8, device="cuda")
    used = c["pool"].shape[0]
    big[n - used:].copy_(c["pool"])
    q, dk, dv, _ = _drafts(2, 3, 16, 8, 0, False)
    want = _verify(sv, c, q, dk, dv, None, None)
    c["pool"], c["table"] = big, c["table"] + (n - used)
    got = _verify(sv, c, q, dk, dv, None, None)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


# ------------------------------------------------------------------------------------------------ ragged batches


def _chunk(sv, c, q, new, little=False, **over):
    S, Hq = len(new), q.shape[1]
    geom = sv.make_geom(S, Hq, c["Hkv"], 128, c["B"], c["NB"], 1)
    kv = sv.make_kv_q4(c["pool"], c["table"], c["lens"])
    ws = _scratch(sv, geom, little)
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    status = _ints([0])
    start = _ints(np.concatenate([[0], np.cumsum(new)]).tolist())
    sv.sv_chunk_attn_q4(geom, q, kv, start, out, lse=lse, workspace=ws, status_word=status, **over)
    return out, lse, int(status)


def _exact_chunk(c, q, lens, new):
    out, lse, A = (torch.zeros(s, dtype=torch.float64, device="cuda") for s in (q.shape, q.shape[:2], q.shape))
    G, row = q.shape[1] // c["Hkv"], 0
    for s, (L, n) in enumerate(zip(lens, new)):
        for h in range(c["Hkv"]):
            if n == 0:
                continue
            w = (q[row:row + n, h * G:(h + 1) * G].double().reshape(n * G, 128) @ c["k"][s][h].T / math.sqrt(128)).clone()
            last = torch.arange(L - n, L, device="cuda").repeat_interleave(G)
            w[torch.arange(w.shape[1], device="cuda") > last[:, None]] = -math.inf
            o, l, a = _softmax(w, c["v"][s][h])
            seen = last >= 0
            o, a = (torch.where(seen[:, None], x, 0.0) for x in (o, a))
            out[row:row + n, h * G:(h + 1) * G], A[row:row + n, h * G:(h + 1) * G] = o.view(n, G, 128), a.view(n, G, 128)
            lse[row:row + n, h * G:(h + 1) * G] = l.view(n, G)
        row += n
    return out, lse, A


@pytest.mark.gpu
@pytest.mark.parametrize("lens,new,Hq,Hkv,B", [
    ([1], [1], 4, 1, 64), ([300], [300], 8, 2, 64), ([500, 64, 0, 129, 1000], [1, 64, 0, 2, 1], 8, 2, 64), ([700, 900], [200, 33], 14, 2, 128),
    ([40, 3], [40, 3], 128, 1, 64), ([2000], [77], 16, 16, 128), ([3, 260, 90], [5, 4, 100], 6, 2, 64), ([5000, 100], [1, 1], 32, 8, 64),
    ([64, 128, 192], [64, 128, 192], 5, 1, 64)])
def test_chunk(lens, new, Hq, Hkv, B):
    """Also rows at positions below zero (more new tokens than the cache has), and rows behind the last sequence, which stay."""
    import paper_2512_21911_b200 as sv
    c = _cache(lens, Hkv, B, seed=7)
    gen = torch.Generator(device="cuda").manual_seed(2)
    N = sum(new)
    q = torch.empty((N + 2, Hq, 128), dtype=torch.bfloat16, device="cuda").normal_(0.0, SIGMA, generator=gen)
    want, lse_want, A = _exact_chunk(c, q[:N], lens, new)
    blind = torch.isinf(lse_want)
    for little in (False, True):
        out, lse, status = _chunk(sv, c, q, new, little)
        assert status == 0 and (out[N:] == 7.0).all() and (lse[N:] == 7.0).all()
        out, lse = out[:N], lse[:N]
        assert torch.equal(torch.isneginf(lse), blind) and (out[blind] == 0).all()
        _close(out, lse.masked_fill(blind, 0.0), want, lse_want.masked_fill(blind, 0.0), A)


@pytest.mark.gpu
def test_chunk_is_the_verification_of_its_tokens():
    """A chain of drafts that the cache holds already, as sv_rope_append_q4 leaves it, is a chunk: bit for bit the same weights but for the
    draft's own keys, so the two agree where there is one token whose own key is the cache's."""
    import paper_2512_21911_b200 as sv
    lens = [400, 77]
    c = _cache(lens, 2, 64)
    q, _, _, _ = _drafts(2, 1, 8, 2, 0, False)
    own = lambda x: torch.stack([x[s][:, n - 1] for s, n in enumerate(lens)])[:, None].bfloat16()
    dk, dv = own(c["k"]), own(c["v"])
    a, la, _ = _chunk(sv, c, q.view(2, 8, 128), [1, 1])
    c["lens"] = _ints([n - 1 for n in lens])
    b, lb, _ = _verify(sv, c, q, dk, dv, None, None)
    tol = 2.0 ** -6 * torch.maximum(a.float().abs(), torch.tensor(1.0, device="cuda"))
    assert bool(((a.view_as(b).float() - b.float()).abs() <= tol).all()) and bool(((la.view_as(lb) - lb).abs() <= 3e-4).all())


@pytest.mark.gpu
def test_nothing_to_do():
    import paper_2512_21911_b200 as sv
    c = _cache([100, 7], 2, 64)
    out, lse, status = _chunk(sv, c, torch.zeros((3, 8, 128), dtype=torch.bfloat16, device="cuda"), [0, 0])
    assert status == 0 and (out == 7.0).all() and (lse == 7.0).all()
    _chunk(sv, c, torch.zeros((0, 8, 128), dtype=torch.bfloat16, device="cuda"), [0, 0])


@pytest.mark.gpu
def test_captured_repeated_and_side_by_side():
    """A graph that is replayed, calls on two streams with workspaces of their own, and the same call again give the same bits."""
    import paper_2512_21911_b200 as sv
    c = _cache([3000, 64, 700, 1], 2, 64)
    q, dk, dv, _ = _drafts(4, 5, 8, 2, 0, False)
    geom = sv.make_geom(4, 8, 2, 128, 64, c["NB"], 5)
    kv = sv.make_kv_q4(c["pool"], c["table"], c["lens"])
    want, _, _ = _verify(sv, c, q, dk, dv, None, None)
    streams = [torch.cuda.Stream() for _ in range(2)]
    ws = [torch.empty(sv.sv_workspace_bytes_q4(geom), dtype=torch.uint8, device="cuda") for _ in range(2)]
    outs = [torch.empty_like(q) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, w, o in zip(streams, ws, outs):
            sv.sv_verify_attn_q4(geom, q, kv, dk, dv, None, None, None, o, workspace=w, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want) and torch.equal(outs[1], want)
    graph, out = torch.cuda.CUDAGraph(), torch.zeros_like(q)
    with torch.cuda.graph(graph):
        sv.sv_verify_attn_q4(geom, q, kv, dk, dv, None, None, None, out, workspace=ws[0])
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    c["lens"].copy_(_ints([10, 64, 3000, 0]))            # a replay goes by the lengths of its time (the table has room for 3,000 tokens)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out[1], want[1])
