"""The oracle of log probabilities, their gradient, the loss against a teacher and rows in 4 bits, pinned by definitions written another
way: differences, closed forms, rational arithmetic."""
import math

import numpy as np
import pytest

from oracle import answers_oracle as ao


def _scores(seed, B, V, masked=0.0):
    rng = np.random.default_rng(seed)
    X = 2.0 * rng.standard_normal((B, V))
    X[rng.random((B, V)) < masked] = -np.inf
    return rng, X


def _differences(f, X, h=1e-6):
    d = np.zeros_like(X)
    for i in np.ndindex(*X.shape):
        if np.isfinite(X[i]):
            up, down = X.copy(), X.copy()
            up[i] += h
            down[i] -= h
            d[i] = (f(up) - f(down)) / (2 * h)
    return d


@pytest.mark.parametrize("T", [1.0, 0.7, 3.0])
@pytest.mark.parametrize("masked", [0.0, 0.4])
def test_gradient_of_log_probabilities_is_their_derivative(T, masked):
    rng, X = _scores(3, 4, 11, masked)
    X[:, :3] = rng.standard_normal((4, 3))
    labels = np.array([[0, 1, -1], [2, 2, 0], [1, 11, 0], [-5, 99, -1]])
    g, h = rng.standard_normal((4, 3)), rng.standard_normal(4)

    def f(x):
        r = ao.label_logprobs(x, labels, T)
        return (r["logp"] * g).sum() + (r["entropy"] * h).sum()
    # central differences with h = 1e-6: h^2 of a third derivative of order 1 / T^3, and 2^-52 |f| / h = 1e-9
    assert np.abs(ao.label_logprobs_grad(X, labels, g, T, h) - _differences(f, X)).max() < 1e-7


@pytest.mark.parametrize("T", [1.0, 2.0])
@pytest.mark.parametrize("tail", [False, True])
def test_gradient_of_the_loss_is_its_derivative(T, tail):
    rng, X = _scores(5, 5, 9, 0.2)
    labels = np.array([[0, 3, 8], [1, 1, 4], [2, -1, 9], [-1, -1, -1], [5, 6, 7]])
    X[np.arange(5)[:, None], np.clip(labels, 0, 8)] = rng.standard_normal((5, 3))
    teacher = np.log(rng.dirichlet(np.ones(4), size=5)[:, :3])
    weight = np.array([1.0, 0.5, 2.0, 1.0, -1.0])
    loss, dX, _ = ao.distill(X, labels, teacher, T, tail, weight)
    d = _differences(lambda x: ao.distill(x, labels, teacher, T, tail, weight)[0].sum(), X)
    assert loss[3] == 0 and (dX[3] == 0).all() and np.abs(dX - d).max() < 1e-7


def test_loss_against_the_whole_distribution_is_the_divergence():
    rng, X = _scores(7, 3, 6)
    t = np.log(rng.dirichlet(np.ones(6), size=3))
    labels = np.tile(np.arange(6), (3, 1))
    want = (np.exp(t) * (t - np.stack([ao.log_softmax(x, 1.0) for x in X]))).sum(1)
    for tail in (False, True):
        loss, dX, _ = ao.distill(X, labels, t, 1.0, tail)
        assert np.abs(loss - want).max() < 1e-12
        assert np.abs(dX - (np.exp([ao.log_softmax(x, 1.0) for x in X]) - np.exp(t))).max() < 1e-12
    assert abs(ao.distill(t, labels, t, 1.0, True)[0]).max() < 1e-12


def test_log_probabilities_entropy_and_top():
    X = np.array([[0.0, 1.0, 1.0, -np.inf, 0.5], [-np.inf] * 5, [-3e38] * 5, [np.nan, 1, 2, 3, 4]])
    r = ao.label_logprobs(X, np.array([[1, 3], [0, -1], [4, 5], [1, 2]]), 1.0, 3)
    s = 1 + 2 * math.e + math.sqrt(math.e)
    assert abs(r["logp"][0, 0] - (1 - math.log(s))) < 1e-14 and r["logp"][0, 1] == -np.inf
    assert r["top"].tolist() == [[1, 2, 4], [-1, -1, -1], [0, 1, 2], [4, 3, 2]]
    assert r["logp"][1].tolist() == [-np.inf, 0.0] and r["entropy"][1] == 0 and (r["norm"][1] == -np.inf).all()
    assert abs(r["logp"][2, 0] + math.log(5)) < 1e-14 and abs(r["entropy"][2] - math.log(5)) < 1e-14
    assert np.isnan(r["logp"][3]).all() and np.isnan(r["entropy"][3]) and np.isnan(r["norm"][3, 1])


def test_codes_are_the_nearest_in_rational_arithmetic():
    rng = np.random.default_rng(1)
    x = np.concatenate([np.arange(-63, 64) / 8.0, rng.uniform(-8, 8, 300), np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]) * (1 + 2.0 ** -23),
                        np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]) * (1 - 2.0 ** -24)])
    x = np.concatenate([x, np.zeros(-x.size % 31)])
    X = np.concatenate([x.reshape(-1, 31), np.full((x.size // 31, 1), 7.5)], 1)      # every block's scale is 1
    codes, scale = ao.microscale_rows(X)
    assert (scale[:, 0] == 127).all() and (codes[:, 32:] == 0).all() and (scale[:, 1:] == 0).all()
    for i in np.ndindex(*X.shape):
        assert codes[i] % 8 == ao.code_of(float(X[i])) % 8, X[i]
    assert np.allclose(ao.values(codes, scale)[:, :32], np.sign(X) * np.array(ao.GRID)[codes[:, :32] % 8])


def test_scales():
    for m, e in ((1.0, -2), (7.9, 0), (8.0, 1), (0.49, -4), (2.0 ** -126, -127), (2.0 ** -140, -127), (2.0 ** 127, 125)):
        assert ao.scale_byte(m) == e + 127
    assert ao.scale_byte(0.0) == 0 and ao.scale_byte(math.inf) == 255


@pytest.mark.parametrize("T", [1.0, 2.0])
@pytest.mark.parametrize("tail", [False, True])
def test_a_label_listed_several_times_is_one_label(tail, T):
    """Loss and gradient are those of the list in which every label stands once, with the sum of its probabilities."""
    rng, X = _scores(9, 4, 12)
    labels = np.array([[3, 3, 3, 3, 3], [0, 7, 0, 7, 11], [5, -1, 5, 12, 2], [1, 2, 3, 4, 1]])
    q = rng.dirichlet(np.ones(6), size=4)[:, :5]
    once, merged = np.full((4, 5), -1), np.zeros((4, 5))
    for b in range(4):
        for j, v in enumerate(dict.fromkeys(v for v in labels[b].tolist() if 0 <= v < 12)):
            once[b, j], merged[b, j] = v, np.log(q[b][labels[b] == v].sum())
    a, b = ao.distill(X, labels, np.log(q), T, tail), ao.distill(X, once, merged, T, tail)
    assert np.abs(a[0] - b[0]).max() < 1e-13 and np.abs(a[1] - b[1]).max() < 1e-13
    if not tail:                                           # the student has nothing but the label: no divergence
        X[0], X[0, 3] = -np.inf, 1.0
        assert abs(ao.distill(X, labels, np.log(q), T)[0][0]) < 1e-13
