"""The oracle of tokens next to certain against the one it refines and against exact fractions."""
from fractions import Fraction

import numpy as np

from oracle import ends_ref as R


def test_apart_is_the_same_probability():
    rng = np.random.default_rng(1)
    z, tokens = rng.normal(size=(7, 11)) * 2, [0, 10, 3, -1, 11, 5, 5]
    logp, _, p = R.logprob(z, tokens, 0.7)
    alone, rest, q = R.logprob_apart(z, tokens, 0.7)
    there = np.array([0 <= t < 11 for t in tokens])
    assert np.allclose(alone, logp, rtol=1e-13, atol=1e-14) and np.allclose(q, p, rtol=1e-13, atol=1e-15) and np.allclose(q.sum(1), there)
    assert np.allclose(rest[there], 1 - p[there, np.array(tokens)[there]]) and not rest[~there].any()


def test_apart_of_what_is_next_to_certain():
    """Others of 2^-60 and 2^-61: 1 - p = o / (1 + o), logp = -o + o^2 / 2 to 1e-36."""
    ln2 = np.log(2.0)
    logp, rest, p = R.logprob_apart(np.array([[-60 * ln2, 0.0, -61 * ln2]]), [1], 1.0)
    o = Fraction(3, 2 ** 61)
    assert abs(rest[0] / float(o / (1 + o)) - 1) < 1e-13 and abs(logp[0] / -float(o - o * o / 2) - 1) < 1e-13 and p[0, 1] == 1.0
    assert np.allclose(p[0, [0, 2]], [2.0 ** -60, 2.0 ** -61], rtol=1e-13, atol=0)
