"""Pins of the oracle of the dense 8-bit scores, the check of drafted labels and dropout (CPU)."""
import math

import numpy as np
import pytest
import torch

from oracle import astra_oracle as orc
from oracle import serving_oracle as so


def test_integers_are_the_nearest_with_halves_to_even_in_rational_arithmetic():
    rng = np.random.default_rng(3)
    X = torch.tensor(rng.normal(size=(20, 48)), dtype=torch.float32).double().numpy()
    X[0] = np.float32(rng.integers(-254, 255, size=48)) * np.float32(2.0 ** -9)          # many halves: m = 254 / 512
    X[0, 0] = 254 * 2.0 ** -9
    X[1] = torch.tensor(rng.normal(size=48)).to(torch.bfloat16).double().numpy()
    X[1, 3] = np.abs(X[1]).max() / 2                                                      # 63.5 exactly
    X[2] = 0.0
    X[3, 5] = np.inf
    X[4, 5] = np.nan
    Q, scale = so.quantize_rows(X)
    for i in list(range(2)) + list(range(5, 20)):
        m = np.abs(X[i]).max()
        assert [so.quantize_element(x, m) for x in X[i]] == Q[i].tolist()
        assert scale[i] == np.float32(np.float32(m) / np.float32(127))
        assert np.abs(Q[i]).max() == 127
    assert not Q[2:5].any() and scale[2] == 0.0 and np.isnan(scale[3:5]).all()


def test_rows_are_padded_to_16_and_scores_of_their_values_come_back():
    rng = np.random.default_rng(4)
    Z, W = rng.normal(size=(5, 24)).astype(np.float32).astype(np.float64), rng.normal(size=(9, 24)).astype(np.float32).astype(np.float64)
    P, a = so.quantize_rows(Z)
    Q, s = so.quantize_rows(W)
    assert P.shape == (5, 32) and not P[:, 24:].any()
    got = so.scores_quantized(P, a, Q, s)
    want = torch.tensor(P.astype(np.int64)[:, None, :] * Q.astype(np.int64)[None, :, :]).sum(2).double().numpy() * np.outer(a.astype(np.float64), s.astype(np.float64))
    assert np.allclose(got, want, rtol=1e-15, atol=0)
    # half a step per element on either side
    bound = 0.5 * (np.outer(a, np.abs(W).sum(1)) + np.outer(np.abs(Z).sum(1), s)) + 0.25 * 24 * np.outer(a, s)
    assert (np.abs(got - Z @ W.T) <= bound * 1.000001).all()


def _grid(n):
    return (np.arange(n) + 0.5) / n


def test_kept_labels_are_distributed_as_the_target():
    """Every draft and a grid of both random numbers, small rational probabilities: the first label's law is the target's, exactly."""
    p = np.array([1, 6, 0, 5, 4]) / 16
    q = np.array([4, 2, 3, 6, 1]) / 16
    target = np.stack([p, np.full(5, 0.2)])
    mass = np.zeros(5)
    for x in range(5):
        for u0 in _grid(48):                              # thresholds p/q are multiples of 1/48 here
            for u1 in _grid(49):                          # the left-over weights are 4 and 3 of 7
                t, a = so.verify_drafts(np.array([[x]]), target[None], q[None, None], np.array([[u0, u1]]))
                mass[t[0, 0]] += q[x] / 48 / 49
                assert a[0] == (1 if u0 * q[x] < p[x] else 0)
    assert np.abs(mass - p).max() < 1e-12


def test_looked_up_drafts_keep_the_target_too():
    p = np.array([1, 6, 0, 5, 4]) / 16
    target = np.stack([p, np.full(5, 0.2)])
    for x in range(5):
        mass = np.zeros(5)
        left = round(16 * (1 - p[x]))                     # the weights without x are sixteenths that add up to this many
        for u0 in _grid(16):
            for u1 in _grid(left):
                t, _ = so.verify_drafts(np.array([[x]]), target[None], None, np.array([[u0, u1]]))
                mass[t[0, 0]] += 1 / 16 / left
        assert np.abs(mass - p).max() < 1e-12


def test_padding_ends_the_drafts_and_empty_rows_give_none():
    V = 6
    target = np.zeros((3, 3, V))
    target[0, :, 2] = 1.0
    target[1, 0, 4] = 1.0                                 # row 1: no drafts at all
    u = np.zeros((3, 3))
    tokens, accepted = so.verify_drafts(np.array([[2, V], [-1, 2], [1, 1]]), target, np.full((3, 2, V), 1 / V), u)
    assert tokens.tolist() == [[2, 2, -1], [4, -1, -1], [-1, -1, -1]] and accepted.tolist() == [1, 0, 0]


def test_nothing_left_above_the_draft_falls_back_to_the_target():
    p = np.array([0.25, 0.0, 0.5, 0.0])
    q = np.array([0.25, 0.25, 0.5, 0.0])
    tokens, accepted = so.verify_drafts(np.array([[1]]), np.stack([p, p])[None], q[None, None], np.array([[0.5, 0.9]]))
    assert accepted.tolist() == [0] and tokens.tolist() == [[2, -1]]


def test_weights_that_are_no_probabilities_count_as_zero():
    p = np.array([np.nan, -1.0, np.inf, 0.5, 0.25])
    for u, want in ((0.0, 3), (0.6, 3), (0.7, 4), (1.0, 4), (2.0, 4)):
        assert so.verify_drafts(np.zeros((1, 0), dtype=np.int32), p[None, None], None, np.array([[u]]))[0].tolist() == [[want]]


def test_dropout_words_are_the_samplers_mixer_with_a_key_of_their_own():
    seed, i, g = 12345678901234567, 3, 2
    word = orc.draw_u64(seed ^ so.K_DROPOUT, i, g)
    keep = so.dropout_kept(i + 1, 4 * g + 4, 0.3, seed)
    least = so.dropout_least(0.3)
    assert [(int(word) >> (16 * e)) % 65536 >= least for e in range(4)] == keep[i, 4 * g:].tolist()
    assert (so.dropout_kept(2, 9, 0.3, seed, row0=2) == so.dropout_kept(4, 9, 0.3, seed)[2:]).all()


@pytest.mark.parametrize("rate", [0.0, 0.1, 0.5, 0.9])
def test_dropout_rate_and_mean(rate):
    keep = so.dropout_kept(200, 250, rate, 99)
    drop = so.dropout_least(rate) / 65536
    assert abs(drop - rate) <= 1 / 131072 + 1e-7
    sd = math.sqrt(drop * (1 - drop) / keep.size)
    assert abs((1 - keep.mean()) - drop) <= 5 * sd
    for e in range(4):                                    # each of a word's fields on its own
        assert abs((1 - keep[:, e::4].mean()) - drop) <= 5 * sd * 2.01
    X = np.ones((200, 250))
    assert abs(so.dropout(X, rate, 99).mean() - 1) <= 5 * sd / (1 - drop)
