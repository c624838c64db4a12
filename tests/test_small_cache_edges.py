"""SparseVerifier with 4-bit caches and evictions: what it refuses, and what the calls around them say."""
import pytest
import torch


def _bare(n_layers, **attributes):
    """A verifier without a device: what a refusal looks at."""
    import paper_2512_21911_b200 as sv
    v = object.__new__(sv.SparseVerifier)
    v.n_layers, v.kv, v.kv_q4, v._pools, v._grown_kv = n_layers, [None] * n_layers, [None] * n_layers, [None] * n_layers, [None] * n_layers
    v.__dict__.update(attributes)
    return v


def test_a_layer_with_a_4_bit_pool_takes_no_others():
    """Either way of giving it bfloat16 pools, before anything of the verifier has changed."""
    pool, kv = (torch.zeros(1),), object()
    v = _bare(2, kv_q4=[None, kv], _pools=[None, pool])
    with pytest.raises(AssertionError, match="4-bit"):
        v.set_layer_kv(1, torch.zeros(1), torch.zeros(1))
    with pytest.raises(AssertionError, match="4-bit"):
        v.set_kv_stack(torch.zeros((2, 1)), torch.zeros((2, 1)))
    assert v._pools == [None, pool] and v.kv == [None, None] and v.kv_q4 == [None, kv]


def test_representatives_of_a_4_bit_layer_are_not_rebuilt():
    v = _bare(2, kv_q4=[None, object()], geom=None, reps=[None, None])
    with pytest.raises(TypeError, match="build_reps: .*4-bit"):
        v.build_reps(1)


@pytest.mark.gpu
def test_the_example_evicts_from_the_sequences_that_are_too_long():
    import os
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import generate as example
    lens = [500, 260]
    _, _, verifier = example.generate([list(range(n)) for n in lens], new=4, layers=1, most=300)
    assert int(verifier.evicted[0]) >= 200 and int(verifier.evicted[1]) == 0
    assert 260 < int(verifier.seq_lens[1]) <= 300 and verifier.seq_lens.tolist() == (verifier.positions() - verifier.evicted).tolist()


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["sv_rope_append", "sv_rope_append_at", "sv_rope_append_q4"])
def test_an_append_that_does_not_fit_is_named(name):
    import paper_2512_21911_b200 as sv
    rows, ints = (lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")), (lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda"))
    geom, pools = sv.make_geom(2, 4, 2, 128, 64, 5, 1), [rows(10, 2, 64, 128), rows(10, 2, 64, 128)]
    if name == "sv_rope_append_q4":
        pools = [torch.zeros((10, 2, 1, sv.SV_Q4_SLAB_BYTES), dtype=torch.uint8, device="cuda")]
    lens = [ints(3)] + ([None] if name == "sv_rope_append_at" else [])      # lengths of three sequences for two
    with pytest.raises(Exception, match=name + r"\b"):
        getattr(sv, name)(geom, *pools, ints(2, 5), *lens, None, rows(1, 2, 128), rows(1, 2, 128), ints(3), None, ints(2))


@pytest.mark.gpu
@pytest.mark.parametrize("weighed", [0, 1, 3])
def test_an_eviction_that_is_refused_in_a_capture_leaves_nothing_in_it(weighed):
    """The first evict, whichever layers have weights already: a replay of what was captured around it changes no cache."""
    from test_small_cache_engine import HQ, L, T, _ints, _normal, _prefill, _rope, _verifier
    gen = torch.Generator(device="cuda").manual_seed(0)
    v, pools = _verifier(2, 7, False, 3)
    _prefill(v, gen, [300, 64], _rope(400))
    q, lse, count = _normal(gen, 2, T, HQ, 128), torch.full((2, T, HQ), 9.0, device="cuda"), torch.zeros(1, device="cuda")
    for l in range(weighed):
        v.weigh_layer(l, q, lse, dense=True)
    before, budget = [p.view(torch.int16).clone() for p in pools], _ints([100, 100])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(RuntimeError):
            v.evict(budget)
        count += 1
    graph.replay()
    torch.cuda.synchronize()
    assert float(count) == 1.0 and all(torch.equal(p.view(torch.int16), b) for p, b in zip(pools, before))
    assert v.evicted is None and v.seq_lens.tolist() == [300, 64] and [w is None for w in v.weights] == [l >= weighed for l in range(L)]
    v.evict(budget)
    assert v.seq_lens.tolist() == [100, 64] and v.positions().tolist() == [300, 64]


def test_positions_are_the_callers_own():
    """A step forward in place does not change the lengths of the cache, whether tokens were evicted or not."""
    for evicted in (None, torch.tensor([5, 0], dtype=torch.int32)):
        v = _bare(1, seq_lens=torch.tensor([3, 7], dtype=torch.int32), evicted=evicted)
        p = v.positions()
        p += 1
        assert v.seq_lens.tolist() == [3, 7] and p.tolist() == ([4, 8] if evicted is None else [9, 8])
