"""SparseVerifier around a verification: prompts in chunks through prefill_layer / end_prefill, the representatives ready for selection,
draw and its distributions for accept; and the example that runs them together.

Tolerance of an attention output o = sum p v: 2^-8 |o| for its rounding, 2^-8 sum p |v| for that of the probabilities, 2^-12 sum p |v| for
everything in fp32."""
import math
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HQ, HKV, B, L = 8, 2, 64, 3


def _verifier(S, blocks, draft=4, keep=None):
    from paper_2512_21911_b200.engine import SparseVerifier
    table = torch.randperm(S * blocks, generator=torch.Generator().manual_seed(5)).int().view(S, blocks).cuda()
    keep = keep or blocks
    v = SparseVerifier(n_seq=S, n_q_heads=HQ, n_kv_heads=HKV, head_dim=128, block_size=B, max_blocks=blocks, n_draft=draft, n_layers=L, block_table=table,
                       seq_lens=torch.zeros(S, dtype=torch.int32, device="cuda"), budget_blocks=torch.full((S,), keep, dtype=torch.int32, device="cuda"), max_sel=keep)
    pools = [torch.full((L, S * blocks, HKV, B, 128), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    v.set_kv_stack(*pools)
    return v, pools


def _tokens(lens, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [[torch.empty((n, HQ + 2 * HKV, 128), dtype=torch.bfloat16, device="cuda").normal_(generator=g) for n in lens] for _ in range(L)]


def _rope(n):
    angle = torch.arange(n, device="cuda")[:, None] * 10000.0 ** (-torch.arange(64, device="cuda") / 64)
    return torch.cat([angle.cos(), angle.sin()], 1)


def _prefill(v, tokens, cuts, rope):
    """Sequence s's tokens cut at cuts[s]; outputs of every layer and sequence, put together."""
    S, outs = len(tokens[0]), [[[] for _ in tokens[0]] for _ in range(L)]
    for i in range(len(cuts[0]) - 1):
        parts = [slice(c[i], c[i + 1]) for c in cuts]
        sizes = [p.stop - p.start for p in parts]
        start = torch.tensor([sum(sizes[:s]) for s in range(S + 1)], dtype=torch.int32, device="cuda")
        for l in range(L):
            q, k, val = torch.cat([tokens[l][s][parts[s]] for s in range(S)]).split([HQ, HKV, HKV], dim=1)
            out = torch.empty((sum(sizes), HQ, 128), dtype=torch.bfloat16, device="cuda")
            v.prefill_layer(l, q, k, val, start, out, rope=rope)
            for s, o in enumerate(out.split(sizes)):
                outs[l][s].append(o)
        v.end_prefill()
    return [[torch.cat(o) for o in per] for per in outs]


def test_prompts_in_chunks():
    lens, blocks = [500, 129, 1], 9
    tokens, rope = _tokens(lens), _rope(600)
    one, pools_1 = _verifier(3, blocks)
    want = _prefill(one, tokens, [[0, n] for n in lens], rope)
    many, pools_2 = _verifier(3, blocks)
    got = _prefill(many, tokens, [[0, 200, 201, 500], [0, 0, 128, 129], [0, 1, 1, 1]], rope)
    assert many.seq_lens.tolist() == one.seq_lens.tolist() == lens
    for a, b in zip(pools_1, pools_2):
        assert torch.equal(torch.nan_to_num(a, nan=7.0), torch.nan_to_num(b, nan=7.0))
    assert torch.equal(one.reps, many.reps)
    rebuilt = torch.zeros_like(one.reps)
    one.reps, kept = rebuilt, one.reps
    for l in range(L):
        one.build_reps(l)
    assert torch.equal(rebuilt, kept)
    half = rope.shape[1] // 2
    for l in range(L):
        for s, n in enumerate(lens):
            x = tokens[l][s]
            turn = lambda y: torch.cat([y[..., :half] * rope[:n, None, :half] - y[..., half:] * rope[:n, None, half:],
                                        y[..., half:] * rope[:n, None, :half] + y[..., :half] * rope[:n, None, half:]], -1).to(torch.bfloat16).double()
            q, k, val = turn(x[:, :HQ].float()), turn(x[:, HQ:HQ + HKV].float()), x[:, HQ + HKV:].double()
            score = torch.einsum("nhgd,thd->nhgt", q.view(n, HKV, HQ // HKV, 128), k) / math.sqrt(128)
            p = torch.softmax(score.masked_fill(torch.ones(n, n, device="cuda").triu(1).bool()[:, None, None], -math.inf), -1)
            exact, room = (torch.einsum("nhgt,thd->nhgd", p, w).reshape(n, HQ, 128) for w in (val, val.abs()))
            for o in (want[l][s], got[l][s]):
                assert bool(((o.double() - exact).abs() <= 2.0 ** -8 * exact.abs() + (2.0 ** -8 + 2.0 ** -12) * room).all())
    one.check_status()
    many.check_status()


def test_verification_follows_a_prompt():
    """Selection and sparse attention on the representatives that the prompt left, against those of a full rebuild."""
    lens, blocks = [900, 333], 16
    v, _ = _verifier(2, blocks, keep=6)
    _prefill(v, _tokens(lens), [[0, 400, 900], [0, 200, 333]], _rope(1000))
    g = torch.Generator(device="cuda").manual_seed(9)
    normal = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    q, dk, dv = normal(L, 2, 4, HQ, 128), normal(L, 2, 4, HKV, 128), normal(L, 2, 4, HKV, 128)
    out, again = torch.zeros_like(q), torch.zeros_like(q)
    v.verify_step(q, dk, dv, out)
    for l in range(L):
        v.build_reps(l)
    v.verify_step(q, dk, dv, again)
    assert torch.equal(out, again) and bool(torch.isfinite(out).all())
    v.check_status()


def test_draw_makes_what_accept_takes():
    v, _ = _verifier(2, 4)
    g = torch.Generator(device="cuda").manual_seed(2)
    logits = torch.randn((2, 4, 1024), generator=g, device="cuda") * 3
    u = torch.rand(8, generator=g, device="cuda")
    p, t = v.draw(logits, u, top_k=torch.tensor([7, 1], dtype=torch.int32, device="cuda"))
    assert p.shape == logits.shape and t.shape == (2, 4) and torch.equal((p > 0).sum(-1).cpu(), torch.tensor([[7] * 4, [1] * 4]))
    assert torch.equal(t[1].long(), logits[1].argmax(-1)) and bool((p.gather(-1, t[..., None].long()) > 0).all())
    none, t2 = v.draw(logits.view(8, 1024), u, distributions=False)
    assert none is None and t2.shape == (8,)
    path, n_path, _ = v.accept(p, p, torch.cat([t[:, :1], t[:, :-1]], 1).contiguous(), torch.rand((2, 4), device="cuda"), torch.rand(2, device="cuda"))
    assert n_path.tolist() == [4, 4] and path.shape == (2, 4)


def test_the_example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import generate as example
    rng = torch.Generator().manual_seed(1)
    prompts = [torch.randint(0, example.VOCAB, (n,), generator=rng).tolist() for n in (700, 65, 3)]
    texts, kept, verifier = example.generate(prompts, new=12, layers=2, chunk=256)
    assert all(len(t) >= 12 and all(0 <= x < example.VOCAB for x in t) for t in texts) and 1.0 <= kept <= example.DRAFT
    # the cache holds the prompt and all tokens but the last one drawn
    assert verifier.seq_lens.tolist() == [len(p) + len(t) - 1 for p, t in zip(prompts, texts)]
    again, _, _ = example.generate(prompts, new=12, layers=2, chunk=100)
    assert all(a[0] == t[0] for a, t in zip(again, texts))     # (the prompt's chunks change nothing but roundings)
