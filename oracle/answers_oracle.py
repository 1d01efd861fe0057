"""Oracle of the operators by which scores are answered with and learnt from, in numpy float64, written from their definitions: rows in
4-bit floating point and scores from them, log probabilities of labels with entropy and top labels, their gradient, and the loss
against a teacher's top labels with its gradient."""
from __future__ import annotations

import math
from fractions import Fraction

import numpy as np

GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)            # the value of a code's low three bits


# ---------------------------------------------------------------------------------------------------------------
# rows in 4 bits
# ---------------------------------------------------------------------------------------------------------------
def code_of(x: float) -> int:
    """The code nearest to |x|, in rational arithmetic; of two equally near ones the even."""
    a = abs(Fraction(x))
    best = min(range(8), key=lambda k: (abs(a - Fraction(GRID[k])), k % 2))
    return best + (8 if math.copysign(1.0, x) < 0 else 0)


def scale_byte(m: float) -> int:
    """Of a block whose largest magnitude is m."""
    if not math.isfinite(m):
        return 255
    if m == 0:
        return 0
    return max(0, math.frexp(m)[1] - 1 - 2 + 127)


def microscale_rows(X: np.ndarray):
    """X float64 [N, d] holding fp32 or bf16 values -> (codes uint8 [N, pitch], one to an element, scale uint8 [N, pitch / 32])."""
    N, d = X.shape
    pitch = (d + 127) // 128 * 128
    Y = np.zeros((N, pitch))
    Y[:, :d] = X
    Y = Y.reshape(N, pitch // 32, 32)
    edge = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    up = np.array([False, True, False, True, False, True, False])          # half way: to the even code
    codes = np.zeros(Y.shape, dtype=np.uint8)
    scale = np.zeros(Y.shape[:2], dtype=np.uint8)
    for i in range(N):
        for b in range(Y.shape[1]):
            m = np.abs(Y[i, b]).max() if np.isfinite(Y[i, b]).all() else math.inf
            scale[i, b] = s = scale_byte(float(m))
            if s == 255:
                continue
            v = np.ldexp(Y[i, b], 127 - int(s))
            a = np.abs(v)[:, None]
            codes[i, b] = (np.where(up, a >= edge, a > edge).sum(1) + 8 * np.signbit(v)).astype(np.uint8)
    return codes.reshape(N, pitch), scale


def packed(codes: np.ndarray) -> np.ndarray:
    return (codes[:, ::2] | (codes[:, 1::2] << 4)).astype(np.uint8)


def values(codes: np.ndarray, scale: np.ndarray) -> np.ndarray:
    """float64 [N, pitch]; a block with scale 255 is not a number"""
    grid = np.array(GRID + tuple(-g for g in GRID))
    v = grid[codes].reshape(codes.shape[0], -1, 32)
    e = scale.astype(np.int64)[:, :, None] - 127
    return np.where(scale[:, :, None] == 255, np.nan, np.ldexp(v, e)).reshape(codes.shape)


# ---------------------------------------------------------------------------------------------------------------
# log probabilities
# ---------------------------------------------------------------------------------------------------------------
def log_softmax(x: np.ndarray, T: float) -> np.ndarray:
    """Of one row; all -inf where no label is there, not a number where one is, or is +inf."""
    m = np.max(x) if not np.isnan(x).any() else np.nan
    if m == -np.inf:
        return np.full_like(x, -np.inf)
    with np.errstate(invalid="ignore", over="ignore", under="ignore"):
        y = (x - m) / T
        return y - np.log(np.exp(y).sum())


def label_logprobs(X, labels, T=1.0, top=0):
    """X float64 [B, V], labels int [B, n] -> dict of float64 arrays, and top int32 [B, top]."""
    B, V = X.shape
    n = labels.shape[1]
    out = {"logp": np.zeros((B, n)), "entropy": np.zeros(B), "norm": np.zeros((B, 2)), "top": np.full((B, top), -1, dtype=np.int32),
           "top_logp": np.full((B, top), -np.inf)}
    for b in range(B):
        lp = log_softmax(X[b], T)
        with np.errstate(invalid="ignore", over="ignore", under="ignore"):
            p = np.exp(lp)
            out["entropy"][b] = -(p * np.where(p > 0, lp, 0.0)).sum() if not np.isnan(lp).any() else np.nan
            real = X[b][~np.isnan(X[b])]
            m = real.max() if real.size else -np.inf
            total = np.exp((X[b] - m) / T).sum() if m > -np.inf else (np.nan if np.isnan(X[b]).any() else 0.0)
            out["norm"][b] = m, np.log(total) if total > 0 else (np.nan if np.isnan(total) else -np.inf)
        for j in range(n):
            if 0 <= labels[b, j] < V:
                out["logp"][b, j] = lp[labels[b, j]]
        order = sorted((v for v in range(V) if X[b, v] > -np.inf), key=lambda v: (-X[b, v], v))[:top]
        for r, v in enumerate(order):
            out["top"][b, r] = v
            out["top_logp"][b, r] = lp[v]
    return out


def label_logprobs_grad(X, labels, dlogp, T=1.0, dentropy=None):
    B, V = X.shape
    dX = np.zeros((B, V))
    for b in range(B):
        lp = log_softmax(X[b], T)
        if (lp == -np.inf).all():
            continue
        p = np.exp(lp)
        H = -(p * np.where(p > 0, lp, 0.0)).sum()
        there = [(int(v), dlogp[b, j]) for j, v in enumerate(labels[b]) if 0 <= v < V]
        inner = sum(g for _, g in there)
        if dentropy is not None:
            inner = inner + dentropy[b] * (np.where(p > 0, lp, 0.0) + H)
        dX[b] = -p * inner
        for v, g in there:
            dX[b, v] += g
    return dX / T


# ---------------------------------------------------------------------------------------------------------------
# a teacher's top labels
# ---------------------------------------------------------------------------------------------------------------
def distill(X, labels, teacher, T=1.0, tail=False, weight=None):
    """(loss float64 [B], gradient float64 [B, V], parts: dict of arrays that bounds are formed from)."""
    B, V = X.shape
    K = labels.shape[1]
    loss, dX = np.zeros(B), np.zeros((B, V))
    parts = {"p_r": np.zeros(B), "q_r": np.zeros(B), "mass": np.zeros(B), "logp": np.zeros((B, V)), "q": np.zeros((B, V)),
             "listed": np.zeros((B, V), dtype=bool)}
    for b in range(B):
        w = 1.0 if weight is None else float(weight[b])
        at = [k for k in range(K) if 0 <= labels[b, k] < V]
        if w == 0 or not at or (not tail and (teacher[b, at] == -np.inf).all()):
            continue
        t = teacher[b, at]
        with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
            q = np.exp(t) if tail else np.exp(t - t.max()) / np.exp(t - t.max()).sum()
            lp = log_softmax(X[b], T)
            p = np.exp(lp)
            ids = labels[b, at].astype(np.int64)
            listed = np.zeros(V, dtype=bool)
            listed[ids] = True
            target = np.zeros(V)
            np.add.at(target, ids, q)
            lq = t if tail else t - t.max() - np.log(np.exp(t - t.max()).sum())
            # (a label that is listed several times has the sum of its probabilities)
            merged = {v: (target[v], np.logaddexp.reduce(lq[ids == v])) for v in ids.tolist()}
            value = sum(qv * (l - lp[v]) for v, (qv, l) in merged.items() if qv != 0)
            p_r = q_r = 0.0
            if tail:
                rest = X[b][~listed]
                rest = rest[rest > -np.inf] if not np.isnan(rest).any() else rest
                if rest.size:
                    q_r = max(0.0, 1.0 - q.sum()) if not np.isnan(q.sum()) else np.nan
                    top = lp[~listed][lp[~listed] > -np.inf].max() if (lp[~listed] > -np.inf).any() else -np.inf
                    log_r = np.log(np.exp(lp[~listed] - top).sum()) + top if top > -np.inf else -np.inf
                    p_r = np.exp(log_r)
                    if q_r != 0:
                        value = value + q_r * (np.log(q_r) - log_r)
                        target[~listed] = q_r * np.exp(lp[~listed] - log_r)
            mass = q.sum() + q_r if tail else 1.0
            loss[b] = w * T * T * value
            dX[b] = w * T * (mass * p - target)
            for name, v in (("p_r", p_r), ("q_r", q_r), ("mass", mass), ("logp", lp), ("q", target), ("listed", listed)):
                parts[name][b] = v
    return loss, dX, parts
