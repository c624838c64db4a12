"""examples/generate.py: the cache and the rotary table have room for the sequence that keeps most, however unevenly the steps' tokens are
kept; the loop ends when the slowest sequence has what was asked for."""
import os
import random
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def _positions(prompts, new, draft, kept):
    """The loop's lengths alone: the last position that any step or commit touches; kept(step, s): tokens of a step."""
    cached, texts, last, step = list(prompts), [1] * len(prompts), max(prompts) - 1, 0
    while min(texts) < new:
        last = max(last, max(cached) + draft - 1)
        for s in range(len(prompts)):
            n = kept(step, s)
            cached[s] += n
            texts[s] += n
        step += 1
    return last


@pytest.mark.parametrize("new", [0, 1, 2, 3, 12, 32, 200])
def test_room_for_every_way_of_keeping(new):
    import generate as example
    D = example.DRAFT
    rng = random.Random(new)
    for prompts in ([3000, 700], [1], [64, 64, 64], [5, 900]):
        room = example.most_tokens([[0] * n for n in prompts], new)
        longest = prompts.index(max(prompts))
        for kept in (lambda i, s: D if s == longest else 1, lambda i, s: 1, lambda i, s: D, lambda i, s: rng.randint(1, D), lambda i, s: rng.choice([1, D])):
            assert _positions(prompts, new, D, kept) < room
        if new > 1 and len(prompts) > 1:
            assert _positions(prompts, new, D, lambda i, s: D if s == longest else 1) == room - 1     # and no more than that


@pytest.mark.gpu
def test_one_sequence_keeps_everything_and_another_one_token(monkeypatch):
    import generate as example
    import paper_2512_21911_b200 as sv

    def accept(self, p_target, p_draft, tokens, u_accept, u_next):
        S, T = tokens.shape
        path = torch.arange(T, dtype=torch.int32, device="cuda").repeat(S, 1)
        return path, torch.tensor([T] + [1] * (S - 1), dtype=torch.int32, device="cuda"), tokens[:, 0].contiguous()

    monkeypatch.setattr(sv.SparseVerifier, "accept", accept)
    prompts, new = [list(range(100)), list(range(30))], 20
    texts, _, verifier = example.generate(prompts, new=new, layers=1)
    assert [len(t) for t in texts] == [1 + (new - 1) * example.DRAFT, new]
    assert verifier.seq_lens.tolist() == [100 + (new - 1) * example.DRAFT, 30 + new - 1]
    assert verifier.seq_lens.max() <= verifier.geom.max_blocks * example.BLOCK
