"""Oracle of the operators around the classifier's product, in numpy float64 and Python integers, written from their
definitions: rows in 8 bits, dense scores from them, the check of drafted labels, dropout from a counter-based generator."""
from __future__ import annotations

import math
from fractions import Fraction

import numpy as np

MASK = (1 << 64) - 1
K_ROW, K_WORD, K_DROPOUT = 0x9E3779B97F4A7C15, 0xD1B54A32D192ED03, 0x64726F706F757431


# ---------------------------------------------------------------------------------------------------------------
# rows in 8 bits
# ---------------------------------------------------------------------------------------------------------------
def quantize_rows(X: np.ndarray):
    """X float64 [N, d] holding fp32 or bf16 values -> (Q int8 [N, d rounded up to 16], scale float32 [N])."""
    N, d = X.shape
    Q = np.zeros((N, (d + 15) // 16 * 16), dtype=np.int8)
    scale = np.zeros(N, dtype=np.float32)
    for i in range(N):
        if not np.isfinite(X[i]).all():
            scale[i] = np.nan
            continue
        m = np.abs(X[i]).max()
        with np.errstate(under="ignore"):
            scale[i] = np.float32(m) / np.float32(127.0)
        if m > 0:
            Q[i, :d] = np.rint(X[i] * 127.0 / m)          # 127 x is exact in 64 bits, and no quotient but a half lies within 2^-40 of one
    return Q, scale


def quantize_element(x: float, m: float) -> int:
    """127 x / m to the nearest integer, halves to even, in rational arithmetic."""
    return int(round(Fraction(x) * 127 / Fraction(m)))


def scores_quantized(P, a, Q, scale) -> np.ndarray:
    """float64 [B, L]: integers P [B, pitch] with scales a, times Q [L, pitch] with scales scale."""
    s = P.astype(np.float64) @ Q.astype(np.float64).T      # whole numbers below 2^53
    with np.errstate(invalid="ignore"):
        return s * a.astype(np.float64)[:, None] * scale.astype(np.float64)[None, :]


# ---------------------------------------------------------------------------------------------------------------
# drafted labels
# ---------------------------------------------------------------------------------------------------------------
def _weights(w: np.ndarray) -> np.ndarray:
    with np.errstate(invalid="ignore"):
        return np.where((w > 0) & np.isfinite(w), w, 0.0)


def verify_drafts(drafts, target, draft_probs, u):
    """drafts int [B, n], target float64 [B, n+1, V], draft_probs float64 [B, n, V] or None, u float64 [B, n+1]."""
    B, n = drafts.shape
    V = target.shape[2]
    tokens = np.full((B, n + 1), -1, dtype=np.int32)
    accepted = np.zeros(B, dtype=np.int32)
    for b in range(B):
        a, w = 0, None
        while a < n and 0 <= drafts[b, a] < V:
            x = int(drafts[b, a])
            q = 1.0 if draft_probs is None else draft_probs[b, a, x]
            if not u[b, a] * q < target[b, a, x]:
                with np.errstate(invalid="ignore"):
                    w = target[b, a] - (draft_probs[b, a] if draft_probs is not None else 0.0)
                if draft_probs is None:
                    w = w.copy()
                    w[x] = 0.0
                w = _weights(w)
                break
            tokens[b, a] = x
            a += 1
        if w is None or not w.any():
            w = _weights(target[b, a])
        accepted[b] = a
        if w.any():
            run = np.cumsum(w)
            above = np.flatnonzero((run > u[b, n] * run[-1]) & (w > 0))
            tokens[b, a] = above[0] if above.size else np.flatnonzero(w)[-1]
    return tokens, accepted


# ---------------------------------------------------------------------------------------------------------------
# dropout
# ---------------------------------------------------------------------------------------------------------------
def _fmix(x: int) -> int:
    x ^= x >> 30
    x = x * 0xBF58476D1CE4E5B9 & MASK
    x ^= x >> 27
    x = x * 0x94D049BB133111EB & MASK
    return x ^ (x >> 31)


def dropout_least(rate: float) -> int:
    """Elements whose 16 random bits are below this are dropped."""
    return math.floor(float(np.float32(rate)) * 65536 + 0.5)


def dropout_kept(B: int, d: int, rate: float, seed: int, row0: int = 0) -> np.ndarray:
    """bool [B, d]"""
    least = dropout_least(rate)
    kept = np.zeros((B, d), dtype=bool)
    for i in range(B):
        row = _fmix(((seed ^ K_DROPOUT) ^ (K_ROW * (row0 + i + 1))) & MASK)
        for g in range((d + 3) // 4):
            word = _fmix((row + K_WORD * (g + 1)) & MASK)
            for j in range(4 * g, min(4 * g + 4, d)):
                kept[i, j] = (word >> (16 * (j % 4)) & 0xFFFF) >= least
    return kept


def dropout(X: np.ndarray, rate: float, seed: int, row0: int = 0) -> np.ndarray:
    """float64 [B, d]"""
    keep = dropout_kept(X.shape[0], X.shape[1], rate, seed, row0)
    return np.where(keep, X * (65536 / (65536 - dropout_least(rate))), 0.0)
