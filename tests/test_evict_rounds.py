"""sv_kv_evict over several rounds of moves (more than 2,048 tokens that stay), with and without representatives, against the host as in
test_kv_evict.py."""
import pytest

from test_kv_evict import _check, _inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens,Hkv,B,budget", [
    ([20000, 9000], 2, 64, [2500, 8999]), ([20000, 9000], 2, 128, [2500, 8999]), ([16384, 16385, 4100], 3, 128, [16383, 16384, 2049]),
    ([32768], 8, 64, [8192]), ([6145], 1, 64, [6144])])
@pytest.mark.parametrize("reps", [False, True])
@pytest.mark.parametrize("in_place", [False, True])
def test_several_rounds(lens, Hkv, B, budget, reps, in_place):
    import paper_2512_21911_b200 as sv
    _check(sv, _inputs(lens, Hkv, B, budget), 4, 64, in_place, reps)


def test_zeros_of_both_signs_are_equal(monkeypatch):
    import numpy as np

    import paper_2512_21911_b200 as sv
    import test_kv_evict
    order = test_kv_evict._order
    monkeypatch.setattr(test_kv_evict, "_order", lambda w: order(np.where(w == 0, np.float32(0), w)))
    zeros = lambda r, s: np.where(r.random(s) < 0.5, 0.0, np.where(r.random(s) < 0.9, -0.0, -1.0))
    _check(sv, _inputs([3000, 517], 2, 64, [1000, 100], weights=zeros), 3, 70)
