"""fp64 oracle of the token log probabilities, their entropy, alternatives and gradient -- TEST INFRASTRUCTURE ONLY.

Only `tests/` may import this module.  Plain numpy, float64, the definitions written out.

Readings (definitions of our own where the mathematics leaves a choice): a logit of minus infinity masks its token (probability 0, never an
alternative); a row that masks every token has log probability -inf everywhere, entropy 0 and no alternatives; a NaN
or plus infinity makes everything of its row NaN (alternatives: token -1); a token that is negative or not below V
stands for "none given": log probability 0, no gradient.
"""
from __future__ import annotations

from typing import Optional, Tuple

import numpy as np


def log_probabilities(z: np.ndarray) -> np.ndarray:
    """log softmax of the rows of z; rows of minus infinities stay so, rows with a NaN or plus infinity become NaN."""
    z = np.asarray(z, np.float64)
    m = z.max(axis=1, keepdims=True)
    with np.errstate(invalid="ignore", divide="ignore"):
        d = np.where(m == -np.inf, -np.inf, z - np.where(np.isfinite(m), m, 0.0))
        d = np.where(np.isnan(m) | (m == np.inf), np.nan, d)
        # the entry equal to the maximum is left out of the sum, so that log1p sees the others
        first = np.argmax(np.where(np.isnan(d), -np.inf, d), axis=1)
        e = np.exp(d)
        e[np.arange(len(z)), first] = np.where(np.isnan(m[:, 0]) | (m[:, 0] == np.inf), np.nan, 0.0)
        return np.where(m == -np.inf, -np.inf, d - np.log1p(e.sum(axis=1, keepdims=True)))


def score(z: np.ndarray, tokens: np.ndarray, k: int) -> Tuple[np.ndarray, np.ndarray, np.ndarray, np.ndarray]:
    """(logprob [M], entropy [M], alternative tokens [M,k], their log probabilities [M,k])."""
    lp = log_probabilities(z)
    M, V = lp.shape
    tokens = np.asarray(tokens, np.int64)
    given = (tokens >= 0) & (tokens < V)
    logprob = np.where(given, lp[np.arange(M), np.where(given, tokens, 0)], 0.0)
    with np.errstate(invalid="ignore"):
        entropy = -np.where(lp == -np.inf, 0.0, np.exp(lp) * lp).sum(axis=1)
    alt = np.full((M, k), -1, np.int64)
    alt_lp = np.full((M, k), -np.inf)
    for row in range(M):
        if np.isnan(lp[row]).any():
            alt_lp[row] = np.nan
            continue
        order = np.argsort(-np.asarray(z[row], np.float64), kind="stable")[:k]     # the lower index first on ties
        order = order[lp[row, order] > -np.inf]
        alt[row, :len(order)] = order
        alt_lp[row, :len(order)] = lp[row, order]
    return logprob, entropy, alt, alt_lp


def score_gradient(z: np.ndarray, tokens: np.ndarray, d_logprob: Optional[np.ndarray],
                   d_entropy: Optional[np.ndarray]) -> np.ndarray:
    """d / dz of sum_m d_logprob[m] log p(tokens[m]) + d_entropy[m] H[m]; zeros where both factors of a row are 0."""
    lp = log_probabilities(z)
    M, V = lp.shape
    tokens = np.asarray(tokens, np.int64)
    given = (tokens >= 0) & (tokens < V)
    g = np.where(given, 0.0 if d_logprob is None else d_logprob, 0.0)
    h = np.zeros(M) if d_entropy is None else np.asarray(d_entropy, np.float64)
    with np.errstate(invalid="ignore"):
        p = np.exp(lp)
        plogp = np.where(lp == -np.inf, 0.0, p * lp)
        H = -plogp.sum(axis=1, keepdims=True)
        dz = -g[:, None] * p - h[:, None] * (plogp + p * H)
    dz[np.nonzero(given)[0], tokens[given]] += g[given]
    dz[(g == 0) & (h == 0)] = 0.0
    return dz
