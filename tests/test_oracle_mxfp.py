"""Pins of the 64-bit forms that the operators on tables held in 4 bits and the draws are tested against: by hand and by other means."""
import itertools

import numpy as np
import pytest

import mxfp_util as mu


def test_levels_and_ties_by_hand():
    x = np.zeros((1, 32))
    x[0, :20] = [7.9, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.75, 0.2, 0.3, 0.74, 1.3, 5.1, 6.0, -5.0, 4.9, -0.0, 4.0]
    codes, scales = mu.quantise(x)
    assert scales.tolist() == [[127]]
    v = mu.values(codes, scales, 32)[0, :20].tolist()
    assert v == [6, 0, 1, 1, 2, 2, 4, 4, 0, -1, 0, 0.5, 0.5, 1.5, 6, 6, -4, 4, 0, 4]
    assert codes[0, 0] == 7 and codes[0, 1] == 2 | 2 << 4    # even column in the low half


def test_values_of_levels_come_back():
    g = np.random.default_rng(0)
    codes = g.integers(0, 256, (50, 32), dtype=np.uint8)
    codes[:, ::16] = 0x67                                    # every block holds a 6: its scale is its own
    scales = g.integers(3, 250, (50, 2), dtype=np.uint8)
    again, s = mu.quantise(mu.values(codes, scales, 64))
    assert np.array_equal(again, codes) and np.array_equal(s, scales)


def test_no_level_is_nearer():
    g = np.random.default_rng(1)
    x = g.standard_normal((20, 45)) * 10
    v = mu.values(*mu.quantise(x), 45)
    pad = np.zeros((20, 64))
    pad[:, :45] = x
    unit = np.repeat(np.exp2(np.floor(np.log2(np.abs(pad).reshape(20, 2, 32).max(2))) - 2), 32, axis=1)[:, :45]
    least = np.min(np.abs(np.abs(x)[:, :, None] - unit[:, :, None] * mu.LEVELS), axis=2)
    assert np.array_equal(np.abs(x - v), least)


@pytest.mark.parametrize("temperature,top_k,top_p,min_p", itertools.product((0.5, 1.0), (0, 3), (1.0, 0.6), (0.0, 0.3)))
def test_kept_rows_one_by_one(temperature, top_k, top_p, min_p):
    s = np.array([0.5, 2.0, 2.0, -np.inf, 1.0, np.nan, 0.5, 1.75])
    order = [1, 2, 7, 4, 0, 6]
    weights = {j: np.exp((s[j] - 2.0) / temperature) for j in order}
    first = order[:top_k] if top_k else order
    total, before, want = sum(weights[j] for j in first), 0.0, []
    for j in first:
        if before < top_p * total and weights[j] >= min_p:
            want.append(j)
        before += weights[j]
    ids, w = mu.kept_rows(s, None, temperature, top_k, top_p, min_p)
    assert ids.tolist() == sorted(want)
    assert np.allclose(w.astype(float), [weights[j] for j in sorted(want)], rtol=1e-14, atol=0)


def test_draws_split_the_unit_interval():
    s = np.log(np.array([1.0, 2.0, 4.0, 1.0]))
    ids, lp, kept = mu.draws(s, None, 1.0, 0, 1.0, 0.0, [0.0, 0.124, 0.126, 0.374, 0.376, 0.874, 0.876, 0.999, 1.0])
    assert ids.tolist() == [0, 0, 1, 1, 2, 2, 3, 3, 3] and kept == 4
    assert np.allclose(lp[[0, 2, 4, 6]], np.log([0.125, 0.25, 0.5, 0.125]), rtol=0, atol=1e-15)
    assert mu.draws(s, np.zeros(4, dtype=bool), 1.0, 0, 1.0, 0.0, [0.5])[0].tolist() == [-1]
    assert mu.draws(s, None, 0.0, 0, 1.0, 0.0, [0.9])[0].tolist() == [2]
