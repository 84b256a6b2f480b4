"""Oracle of truncated sampling and of a row's largest logits — test infrastructure only.

The tokens of a row are its finite logits, ordered descending, equal ones by ascending index.
Kept of that order is the prefix with rank < top_k, sum of exp((l - l_max) / T) before the token
< top_p times the sum over the first top_k, and l >= l_max + T ln(min_p).  The draw is the
Gumbel-max draw of :mod:`oracle.sampler` (same noise, same float32 scores) over the kept tokens.
Sums are float64.

Pins (tests/test_oracle_truncated.py): kept sets of hand-made distributions in closed form, each
condition alone and together, ties, empty rows; the draw equals oracle.sampler's where nothing is cut
and wherever that draw is kept; chi-square of draws against the renormalised distribution.
"""
from __future__ import annotations

import math

import numpy as np

from . import sampler


def order(logits: np.ndarray) -> np.ndarray:
    """Indices of the finite logits, descending, ties to the lowest index."""
    l = np.asarray(logits, dtype=np.float32)
    at = np.flatnonzero(np.isfinite(l))
    return at[np.argsort(-(l[at].astype(np.float64)), kind="stable")]


def top_logits(logits: np.ndarray, k: int, temperature: float = 1.0):
    """(float32 values [k], int32 indices [k], float64 log-sum-exp of l / T over the other finite logits)."""
    l = np.asarray(logits, dtype=np.float32)
    at = order(l)
    values = np.full(k, -np.inf, np.float32)
    indices = np.full(k, -1, np.int32)
    m = min(k, at.size)
    values[:m], indices[:m] = l[at[:m]], at[:m]
    others = l[at[m:]].astype(np.float64) / float(np.float32(temperature))
    rest = -math.inf
    if others.size:
        rest = others.max() + math.log(np.exp(others - others.max()).sum())
    return values, indices, rest


def kept_tokens(logits: np.ndarray, temperature: float, top_k: int = 0, top_p: float = 1.0,
                min_p: float = 0.0) -> np.ndarray:
    """The kept tokens' indices, in order."""
    l = np.asarray(logits, dtype=np.float32).astype(np.float64)
    T = float(np.float32(temperature))
    at = order(logits)
    if not at.size:
        return at
    if top_k > 0:
        at = at[:top_k]
    n = at.size
    if top_p < 1.0:
        w = np.exp((l[at] - l[at[0]]) / T)
        before = np.concatenate([[0.0], np.cumsum(w)])
        n = int(np.count_nonzero(before[:-1] < top_p * before[-1]))
    if min_p > 0.0:
        n = min(n, int(np.count_nonzero(l[at] >= l[at[0]] + T * math.log(min_p))))
    return at[:n]


def sample_row(logits: np.ndarray, seq_uid: int, step: int, temperature: float, seed: int, top_k: int = 0,
               top_p: float = 1.0, min_p: float = 0.0):
    """(token, float64 log-prob under the whole softmax(l / T)); (-1, nan) where nothing can be drawn."""
    l = np.asarray(logits, dtype=np.float32)
    kept = kept_tokens(l, temperature, top_k, top_p, min_p)
    only = np.full(l.shape, -np.inf, np.float32)
    only[kept] = l[kept]
    token, _ = sampler.sample_row(only, seq_uid, step, temperature, seed)
    if token < 0:
        return -1, math.nan
    T = float(np.float32(temperature))
    z = l[np.isfinite(l)].astype(np.float64)
    m = z.max()
    return token, (float(l[token]) - m) / T - math.log(np.exp((z - m) / T).sum())


def sample(logits: np.ndarray, seq_uid, step, temperature: float, seed: int, top_k: int = 0, top_p: float = 1.0,
           min_p: float = 0.0, row_of=None):
    """Every draw b from logits[row_of[b]] (or logits[b]): (int32 [n], float64 [n])."""
    seq_uid = np.asarray(seq_uid)
    step = np.broadcast_to(np.asarray(step), seq_uid.shape)
    got = [sample_row(logits[b if row_of is None else int(row_of[b])], int(seq_uid[b]), int(step[b]), temperature, seed,
                      top_k, top_p, min_p) for b in range(seq_uid.size)]
    return np.array([t for t, _ in got], np.int32), np.array([p for _, p in got], np.float64)
