"""The oracle of the operators at the ends of a model: gradients against differences, and values that are known without it."""
import numpy as np
import pytest

from oracle import ends_ref as R


def _differences(f, x, step=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        keep = x[i]
        x[i] = keep + step
        up = f()
        x[i] = keep - step
        g[i] = (up - f()) / (2 * step)
        x[i] = keep
    return g


def test_embedding_gradient():
    rng = np.random.default_rng(0)
    table, tokens, d = rng.normal(size=(5, 3)), np.array([4, 1, -1, 1, 9, 1]), rng.normal(size=(6, 3))
    g, size, count = R.embedding_gradient(d, tokens, 5, 1.5)
    assert np.allclose(g, _differences(lambda: (R.embedding(tokens, table, 1.5) * d).sum(), table), atol=1e-8)
    assert count.tolist() == [0, 3, 0, 0, 1] and np.all(size >= np.abs(g) - 1e-12)
    assert np.all(R.embedding(tokens, table, 1.5)[[2, 4]] == 0)


@pytest.mark.parametrize("center", [True, False])
def test_layer_norm_gradient(center):
    rng = np.random.default_rng(1)
    h, w, b, dy = rng.normal(size=(4, 7)), rng.normal(size=7), rng.normal(size=7), rng.normal(size=(4, 7))
    f = lambda: (R.layer_norm(h, w, b, center, 0.1)[0] * dy).sum()   # noqa: E731
    for got, x in zip(R.layer_norm_gradient(dy, h, w, center, 0.1), (h, w, b)):
        assert np.allclose(got, _differences(f, x), atol=1e-7)


def test_logprob_and_gradient():
    rng = np.random.default_rng(2)
    z, tokens, d = rng.normal(size=(4, 6)), np.array([0, 5, -1, 3]), rng.normal(size=4)
    logp, lse, p = R.logprob(z, tokens, 0.7)
    assert np.allclose(p.sum(1), [1, 1, 0, 1]) and logp[2] == lse[2] == 0
    assert np.allclose(R.logprob_gradient(d, p, tokens, 0.7), _differences(lambda: (R.logprob(z, tokens, 0.7)[0] * d).sum(), z), atol=1e-8)
    z[0] = -np.inf
    z[1, :5] = -np.inf
    logp, lse, p = R.logprob(z, tokens, 0.7)
    assert logp[0] == -np.inf and np.all(p[0] == 0) and logp[1] == 0 and p[1, 5] == 1


@pytest.mark.parametrize("old,kl", [(False, 0.0), (True, 0.0), (True, 0.3), (False, 0.3)])
def test_policy_rows(old, kl):
    rng = np.random.default_rng(3)
    logp, A, w = rng.normal(size=30) - 2, rng.normal(size=30), rng.uniform(size=30)
    given = dict(advantages=A, old=logp + 0.3 * rng.normal(size=30) if old else None, ref=logp + rng.normal(size=30), weights=w, low=0.2, high=0.4, kl=kl)
    there = rng.uniform(size=30) < 0.8
    l, d, dd = R.policy_rows(logp, there, **given)
    x = logp.copy()
    assert np.allclose(d, _differences(lambda: R.policy_rows(x, there, **given)[0].sum(), x), atol=1e-7)
    second = _differences(lambda: R.policy_rows(x, there, **given)[1].sum(), x)
    assert np.all(np.abs(second) <= dd + 1e-6)
    if old:
        assert np.any((d == 0) & there) == (kl == 0.0)        # some ratios are cut off


def test_policy_row_values():
    one = np.ones(1, dtype=bool)
    z = np.zeros(1)
    assert R.policy_rows(np.log([0.25]), one)[0][0] == pytest.approx(np.log(4))                                        # cross entropy
    assert R.policy_rows(np.log([1.5]), one, advantages=np.array([2.0]), old=z)[0][0] == pytest.approx(-2.4)            # held at 1.2
    assert R.policy_rows(np.log([1.5]), one, advantages=np.array([-2.0]), old=z)[0][0] == pytest.approx(3.0)            # the worse one counts
    assert R.policy_rows(np.log([0.5]), one, advantages=np.array([-2.0]), old=z)[0][0] == pytest.approx(1.6)            # held at 0.8
    assert R.policy_rows(z, one, advantages=z, old=z, ref=np.log([2.0]), kl=1.0)[0][0] == pytest.approx(1 - np.log(2))
