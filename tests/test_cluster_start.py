"""A CTA may reach a peer's shared memory only once the peer runs.  Nothing starts the CTAs of a cluster in the same instant, so every kernel
that writes to or reads from its peers arrives at the cluster's barrier and waits for it first.  Read from the sources: the order of the
two in each kernel's body.  (A late CTA shows on no machine on demand, and where it does its peers' writes are lost.)"""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2512_21911_b200", "csrc")
ARRIVE = r"cluster_arrive\(\)|barrier\.cluster\.arrive|cluster\.sync\(\)"
WAIT = r"cluster_wait\(\)|barrier\.cluster\.wait|cluster\.sync\(\)"
REACH = r"map_shared_rank\(|cluster_map_shared\(|st_async_cluster|bulk_copy_cluster\("


def _without_comments(text):
    return re.sub(r"//[^\n]*|/\*.*?\*/", "", text, flags=re.S)


def _body(text, at):
    """From the brace that opens behind `at` to the one that closes it."""
    begin = text.index("{", at)
    depth = 0
    for i in range(begin, len(text)):
        depth += (text[i] == "{") - (text[i] == "}")
        if depth == 0:
            return text[begin:i + 1]
    raise AssertionError("no end")


def _reaching(text):
    """What reaches a peer: the primitives, and this file's functions in whose bodies they are."""
    pattern, names = REACH, set()
    while True:
        found = {m[1] for m in re.finditer(r"__device__[^;{}()]*?(\w+)\([^;{}]*\)\s*(?=\{)", text) if re.search(pattern, _body(text, m.start()))}
        if found <= names:
            return pattern
        names |= found
        pattern = "|".join([REACH] + [rf"\b{n}\(" for n in sorted(names)])


@pytest.mark.parametrize("file,kernel", [("sample.cu", "sample_kernel"), ("accept.cu", "accept_kernel"), ("select_blocks.cu", "select_kernel")])
def test_peers_are_reached_behind_the_barrier(file, kernel):
    with open(os.path.join(CSRC, file)) as f:
        text = _without_comments(f.read())
    pattern = _reaching(text)
    body = _body(text, text.index(kernel + "("))
    arrive, wait, reach = (re.search(p, body) for p in (ARRIVE, WAIT, pattern))
    assert arrive and wait and reach
    assert arrive.start() <= wait.start() < reach.start(), body[reach.start():reach.start() + 60]


def test_every_file_that_reaches_peers_is_looked_at():
    """verify_attn_tc.cu waits in several places, by role; its copies to peers all stand behind the wait of the merging threads."""
    found = {f for f in os.listdir(CSRC) if f.endswith(".cu") and re.search(REACH, _without_comments(open(os.path.join(CSRC, f)).read()))}
    assert found == {"sample.cu", "accept.cu", "select_blocks.cu", "verify_attn_tc.cu"}
    text = _without_comments(open(os.path.join(CSRC, "verify_attn_tc.cu")).read())
    last_role = text.index("have_mine = k > 0 && !dead")
    assert re.search(REACH, text).start() > re.search(WAIT, text[last_role:]).start() + last_role


@pytest.mark.gpu
@pytest.mark.parametrize("half", [False, True])
def test_short_rows_call_behind_call(half):
    """Parts of 2,048 entries, whose load hides little of what lies between the starts of a cluster's CTAs; every call gives the same bits."""
    import torch

    import paper_2512_21911_b200 as sv
    gen = torch.Generator(device="cuda").manual_seed(4)
    for R, V in ((1, 4097), (7, 16384), (18, 9001)):
        x = torch.randn((R, V), generator=gen, device="cuda") * 3
        x[:, V - 1] = 20.0 + torch.arange(R, device="cuda")   # the maximum, in the last CTA's part
        x = x.bfloat16() if half else x
        u, temperature = torch.rand(R, generator=gen, device="cuda"), torch.full((R,), 9.0, device="cuda")
        tokens, probs = torch.empty((200, R), dtype=torch.int32, device="cuda"), [torch.empty((R, V), device="cuda") for _ in range(2)]
        want = torch.softmax(x.double() / 9.0, -1)
        for i in range(200):
            sv.sv_sample(x, u, tokens[i], probs=probs[i > 0], temperature=temperature)
        assert torch.equal(probs[0], probs[1]) and bool((tokens == tokens[0]).all())
        assert bool(((probs[1].double() - want).abs() <= 1e-5 * want).all())
