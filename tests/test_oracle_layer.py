"""The oracle of the layer operators: its gradients against central differences, its generator against the published vectors, its masks
against the definition pair by pair."""
import os

import numpy as np
import pytest

from oracle import layer_ref as R

HERE = os.path.dirname(os.path.abspath(__file__))


def _difference(f, x, h=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        y = x.copy()
        y[i] += h
        up = f(y)
        y[i] -= 2 * h
        g[i] = (up - f(y)) / (2 * h)
    return g


@pytest.mark.parametrize("softcap,slope,causal,docs", [(0.0, 0.0, True, False), (2.0, 0.0, False, False), (1.5, 0.3, True, True), (0.0, 0.5, False, True)])
def test_attention_gradients_against_differences(softcap, slope, causal, docs):
    rng = np.random.default_rng(3)
    n, m, d = 4, 6, 3
    q, k, v, g = rng.standard_normal((n, d)), rng.standard_normal((m, d)), rng.standard_normal((m, d)), rng.standard_normal((n, d))
    doc = dict(q_doc=[0, 0, -1, 1], k_doc=[0, 0, 0, 1, -1, 1]) if docs else {}
    see, far = R.visible(n, m, causal=causal, **doc)
    loss = lambda a, b, c: float(np.sum(g * R.attention_head(a, b, c, see, far, 0.7, softcap, slope)["out"]))   # noqa: E731
    r = R.attention_head(q, k, v, see, far, 0.7, softcap, slope, g)
    # central differences of a smooth function of order 1 with step 1e-6: error about 1e-16 / 1e-6 + 1e-12
    for name, x, f in (("dq", q, lambda x: loss(x, k, v)), ("dk", k, lambda x: loss(q, x, v)), ("dv", v, lambda x: loss(q, k, x))):
        np.testing.assert_allclose(r[name], _difference(f, x), atol=2e-8)


@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("interleaved,rot", [(True, 4), (False, 4), (False, 6), (True, 0)])
def test_norm_rope_gradients_against_differences(norm, interleaved, rot):
    rng = np.random.default_rng(4)
    x, g, w = rng.standard_normal((2, 2, 2, 6)), rng.standard_normal((2, 2, 2, 6)), rng.standard_normal(6)
    pos, f = np.array([[0, 3], [7, 100000]]), 1.0 / (1.0 + np.arange(rot // 2))
    run = lambda a, b: float(np.sum(g * R.norm_rope(a, pos, f, b, norm, interleaved, 1.3, 1e-6)))   # noqa: E731
    dx, dw = R.norm_rope_grad(g, x, pos, f, w, norm, interleaved, 1.3, 1e-6)
    np.testing.assert_allclose(dx, _difference(lambda a: run(a, w), x), atol=2e-8)
    if norm:
        np.testing.assert_allclose(dw, _difference(lambda b: run(x, b), w), atol=2e-8)


def test_rotation_of_pairs_and_of_nothing():
    x = np.arange(1.0, 9.0).reshape(1, 1, 1, 8)
    quarter = [np.pi / 2]
    np.testing.assert_allclose(R._turn(x, np.array([[1]]), quarter, True, 1.0, 1.0)[0, 0, 0], [-2, 1, 3, 4, 5, 6, 7, 8], atol=1e-12)
    half = [np.pi / 2, 0.0]
    np.testing.assert_allclose(R._turn(x, np.array([[1]]), half, False, 1.0, 1.0)[0, 0, 0], [-3, 2, 1, 4, 5, 6, 7, 8], atol=1e-12)
    np.testing.assert_array_equal(R._turn(x, np.array([[0]]), half, False, 1.0, 1.0), x)


def test_generator_against_the_published_vectors():
    lines = [l.split() for l in open(os.path.join(HERE, "golden", "philox4x32_10_kat.txt")) if l.strip() and not l.startswith("#")]
    assert lines
    for words in lines:
        v = [int(x, 16) for x in words if all(c in "0123456789abcdefxABCDEF" for c in x)][-10:]
        out = [int(x) for x in R.philox4x32_10([np.array([c]) for c in v[:4]], v[4:6])]
        assert out == v[6:]


def test_dropout_rate_and_its_parts():
    kept, factor = R.dropout_kept(0, 200000, 0.25, 12345, 6)
    assert factor == 65536.0 / 49152
    assert abs(kept.mean() - 0.75) < 5 * np.sqrt(0.25 * 0.75 / 200000)      # five standard deviations
    part, _ = R.dropout_kept(1001, 777, 0.25, 12345, 6)
    np.testing.assert_array_equal(part, kept[1001:1778])
    assert not np.array_equal(kept, R.dropout_kept(0, 200000, 0.25, 12345, 7)[0])


def test_visible_pair_by_pair():
    n, m, keys, prefix = 3, 7, 5, 4
    see, far = R.visible(n, m, causal=True, prefix=prefix, keys=keys)
    for i in range(n):
        for j in range(m):
            at = i + keys - n
            assert see[i, j] == (j < keys and (j <= at or j < prefix)) and far[i, j] == abs(at - j)
