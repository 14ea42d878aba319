"""CPU pins of the fp64 oracle of the policy and preference losses and of
gradient clipping: worked values, central differences, invariances."""
import math

import numpy as np
import pytest

import oracle
from oracle.objective_oracle import HINGE, MEAN_SEQS, MEAN_TOKENS, SIGMOID, SQUARE, SUM


def _tokens(seed, T=23):
    g = np.random.default_rng(seed)
    nll = g.exponential(1.0, T)
    return nll, nll + 0.3 * g.standard_normal(T), nll + 0.3 * g.standard_normal(T), g.integers(0, 2, T)


def test_policy_worked():
    """Two tokens by hand: rho = 2 with A = 1 is clipped at 1.5; rho = 1 with A = -1 is not."""
    ln2 = math.log(2.0)
    loss, w, kl, share = oracle.policy_loss([0.0, 1.0], [ln2, 1.0], None, [1.0, -1.0], None, [0, 1, 2], 0.5, 0.5,
                                            0.0, 1.0, SUM)
    assert loss == pytest.approx(-1.5 + 1.0) and kl == 0.0 and share == 0.5
    assert list(w) == [0.0, -1.0]
    # the mean over tokens, with e = nll - ref = ln 2: exp(e) - 1 - e = 1 - ln 2
    loss, w, kl, _ = oracle.policy_loss([ln2], [ln2], [0.0], [3.0], None, [0, 1], 0.2, 0.2, 0.1, 2.0, MEAN_TOKENS)
    assert loss == pytest.approx(2 * (-3.0 + 0.1 * (1 - ln2))) and kl == pytest.approx(1 - ln2)
    assert w[0] == pytest.approx(2 * (3.0 + 0.1))


@pytest.mark.parametrize("reduction", [SUM, MEAN_TOKENS, MEAN_SEQS])
def test_policy_differences(reduction):
    nll, old, ref, mask = _tokens(1)
    off = [0, 4, 4, 15, 23]
    adv = np.array([1.3, 5.0, -0.7, 0.4])
    args = (old, ref, adv, mask, off, 0.2, 0.3, 0.05, 1.7, reduction)
    _, w, _, _ = oracle.policy_loss(nll, *args)
    for i in range(len(nll)):
        h = 1e-6
        up, down = nll.copy(), nll.copy()
        up[i] += h
        down[i] -= h
        d = (oracle.policy_loss(up, *args)[0] - oracle.policy_loss(down, *args)[0]) / (2 * h)
        assert d == pytest.approx(w[i], abs=2e-8)


def test_policy_mean_of_sequences_counts_empty_ones():
    loss, _, _, _ = oracle.policy_loss([1.0, 1.0], [1.0, 1.0], None, [2.0, 7.0], [1, 1], [0, 2, 2], 0.2, 0.2, 0.0,
                                       1.0, MEAN_SEQS)
    assert loss == pytest.approx(-1.0)


@pytest.mark.parametrize("kind,smoothing", [(SIGMOID, 0.0), (SIGMOID, 0.2), (HINGE, 0.0), (SQUARE, 0.0)])
@pytest.mark.parametrize("mean_tokens", [False, True])
def test_pref_differences(kind, smoothing, mean_tokens):
    nll, _, ref, mask = _tokens(2)
    args = (ref, mask, [0, 5, 9, 9, 23], kind, mean_tokens, 0.4, 0.1, smoothing, 0.9)
    _, w, _ = oracle.pref_loss(nll, *args)
    for i in range(len(nll)):
        h = 1e-6
        up, down = nll.copy(), nll.copy()
        up[i] += h
        down[i] -= h
        d = (oracle.pref_loss(up, *args)[0] - oracle.pref_loss(down, *args)[0]) / (2 * h)
        assert d == pytest.approx(w[i], abs=2e-8)


def test_pref_worked():
    """R = (1, -1), beta = 0.5: m = 1 for the sigmoid, the square's distance is 1 - 1/2 over beta."""
    args = ([1.0, 0.0], None, [0, 1, 2])
    loss, w, r = oracle.pref_loss([0.0, 1.0], *args, SIGMOID, False, 0.5, 0.0, 0.0, 1.0)
    assert list(r) == [0.5, -0.5] and loss == pytest.approx(math.log(1 + math.exp(-1.0)))
    assert w[0] == pytest.approx(0.5 / (1 + math.e)) and w[1] == -w[0]
    assert oracle.pref_loss([0.0, 1.0], *args, SQUARE, False, 0.5, 0.0, 0.0, 1.0)[0] == pytest.approx(1.0)
    # swapping the answers of every pair changes the sign of the derivative of an unsmoothed hinge below 1
    a = oracle.pref_loss([0.0, 0.5], *args, HINGE, False, 0.1, 0.0, 0.0, 1.0)
    assert a[1][0] == pytest.approx(0.1) and a[1][1] == pytest.approx(-0.1)


def test_clip():
    norm, coef, (a, b) = oracle.clip_grads([np.array([3.0]), np.array([[0.0], [4.0]])], 1.0)
    assert norm == 5.0 and coef == 0.2 and a[0] == pytest.approx(0.6) and b[1, 0] == pytest.approx(0.8)
    assert oracle.clip_grads([np.array([3.0])], 3.0)[1] == 1.0
    assert oracle.clip_grads([np.array([math.inf])], 3.0)[1] == 1.0
    assert oracle.clip_grads([np.zeros(3)], 0.0)[:2] == (0.0, 1.0)
