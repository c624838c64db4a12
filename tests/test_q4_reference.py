"""The plain form of the 4-bit cache that the GPU tests go by: what is put is what is got, and no value is off by more than the format
allows."""
import numpy as np
import pytest

from q4_reference import SLAB, bf16, code, get, put, value


def test_put_and_get():
    rng = np.random.default_rng(0)
    slab = rng.integers(0, 256, SLAB).astype(np.uint8)
    rows = bf16(rng.normal(size=(64, 2, 128)))
    for t in rng.permutation(64):
        put(slab, t, rows[t, 0], rows[t, 1])
    k, v = get(slab)
    assert np.array_equal(k, value(*code(rows[:, 0]))) and np.array_equal(v, value(*code(rows[:, 1])))


def test_a_token_changes_nothing_else():
    rng = np.random.default_rng(1)
    slab = rng.integers(0, 120, SLAB).astype(np.uint8)   # (no scale is a NaN)
    k0, v0 = get(slab)
    put(slab, 37, bf16(rng.normal(size=128)), bf16(rng.normal(size=128)))
    k1, v1 = get(slab)
    others = np.arange(64) != 37
    assert np.array_equal(k0[others], k1[others]) and np.array_equal(v0[others], v1[others])


@pytest.mark.parametrize("size", [1e-20, 1.0, 1e20])
def test_how_far_values_are_off(size):
    """Half a step of D / 16 between codes; at the ends D's and M's rounding: D is off by 2^-8 D, so that 15 steps reach 15 / 16 2^-8 D less
    or more, M by 2^-8 |M|; and the rounding of the value."""
    x = bf16(np.random.default_rng(2).normal(size=(200, 128)) * size)
    c, d, m = code(x)
    wide = lambda a: np.repeat(a, 64, -1)
    tol = wide(d) / 32 + 2.0 ** -8 * (wide(d) + np.abs(wide(m)) + np.abs(x))
    assert (np.abs(value(c, d, m) - x) <= tol).all() and c.min() == 0 and c.max() == 15


def test_groups_without_a_spread_and_with_a_nan():
    x = np.full((3, 128), 2.5)
    x[1, 3], x[2, 100] = np.nan, np.inf
    got = value(*code(x))
    assert (got[0] == 2.5).all() and np.isnan(got[1, :64]).all() and (got[1, 64:] == 2.5).all() and np.isnan(got[2, 64:]).all()
