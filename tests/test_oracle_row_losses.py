"""The 64-bit losses on rows of logits: their gradients against differences of
the losses, and the cases whose value is known."""

import math

import numpy as np
import pytest

from oracle import row_losses_oracle as O

STEP = 1e-5


def problem(seed, T=14, V=7):
    r = np.random.default_rng(seed)
    x = r.standard_normal((T, V)) * 2
    y = r.integers(0, V, T)
    y[[1, 6]] = -1
    return r, x, y


def differences(f, x):
    """d f / d x by central differences: error about STEP^2 |f'''| + 1e-16 |f| / STEP."""
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        at = x[i]
        x[i] = at + STEP
        up = f(x)
        x[i] = at - STEP
        g[i] = (up - f(x)) / (2 * STEP)
        x[i] = at
    return g


OFF = [1, 4, 6, 6, 13]           # two pairs, an empty sequence, rows before and behind


@pytest.mark.parametrize("kind", ["sigmoid", "hinge", "squared"])
@pytest.mark.parametrize("average,smoothing,margin,tau", [(False, 0.0, 0.0, 1.0), (True, 0.1, 0.3, 0.7)])
def test_preference_gradient(kind, average, smoothing, margin, tau):
    r, x, y = problem(3)
    ref = r.standard_normal((2, 2))
    kw = dict(beta=0.3, kind=kind, margin=margin, smoothing=smoothing, average=average, scale=1.7, tau=tau)
    _, _, coef = O.preference(x, y, OFF, ref, **kw)
    got = O.logits_gradient(x, y, coef, tau)
    np.testing.assert_allclose(got, differences(lambda v: O.preference(v, y, OFF, ref, **kw)[0], x.copy()), atol=2e-8)


@pytest.mark.parametrize("reduction", ["tokens", "sequences", "sum"])
@pytest.mark.parametrize("kl,tau", [(0.0, 1.0), (0.2, 1.4)])
def test_policy_gradient(reduction, kl, tau):
    r, x, y = problem(4)
    logp = O.rows(x, y, tau)[0]
    old, ref, adv = (logp + 0.3 * r.standard_normal(14), logp + 0.5 * r.standard_normal(14), r.standard_normal(14))
    kw = dict(clip=(0.2, 0.3), kl=kl, off=OFF, reduction=reduction, scale=0.9, tau=tau)
    _, terms, _, coef = O.policy(x, y, old, adv, ref, **kw)
    assert terms[2] > 0
    got = O.logits_gradient(x, y, coef, tau)
    np.testing.assert_allclose(got, differences(lambda v: O.policy(v, y, old, adv, ref, **kw)[0], x.copy()), atol=2e-8)


def test_balance_gradient_and_even_load():
    r, x, _ = problem(5, 9, 6)
    mask = np.ones(9, np.uint8)
    mask[4] = 0
    loss, counts, choice, g = O.balance(x, 2, mask, alpha=0.5)
    assert counts.sum() == 16 and (choice[4] == -1).all()
    fixed = lambda v: O.balance(v, 2, mask, choice, alpha=0.5)[0]
    assert fixed(x) == loss
    np.testing.assert_allclose(g, differences(fixed, x.copy()), atol=2e-9)
    # equal loads: alpha, whatever the probabilities
    even = np.arange(8, dtype=np.int32).reshape(8, 1) % 4
    loss, _, _, g = O.balance(r.standard_normal((8, 4)), 1, choice=even, alpha=0.25)
    assert loss == pytest.approx(0.25, rel=1e-14) and np.abs(g).max() < 1e-16


def test_known_values():
    x = np.zeros((2, 8))
    logp, m, L, p = O.rows(x, np.array([3, -1]))
    assert logp[0] == pytest.approx(-math.log(8)) and logp[1] == 0 and (p[1] == 0).all()
    # equal scores: the sigmoid loss is log 2
    loss, scores, _ = O.preference(x, np.array([0, 5]), [0, 1, 2])
    assert loss == pytest.approx(math.log(2)) and scores[0, 0] == scores[0, 1]
    # ratio 1: minus the mean advantage
    loss, terms, lp, coef = O.policy(x, np.array([0, 5]), [logp[0]] * 2, [2.0, 1.0])
    assert loss == pytest.approx(-1.5) and terms[2] == 0 and coef.tolist() == pytest.approx([-1.0, -0.5])
