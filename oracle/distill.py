"""Oracle of the distillation loss from a teacher's largest logits — test infrastructure only.

The KL term of the paper (Sec. 3.2, D_KL of the original model against the policy) over the outcomes
that a teacher's row is reduced to: its k tokens, and all other tokens as one outcome.
float64 throughout; every value an explicit sum over the row.

Pins (tests/test_oracle_distill.py): with every token listed it is oracle.policy.kl_rows; two-token
closed forms; zero at equality; grouping tokens never increases a KL divergence; the gradient against
central differences, its sum over the row, and torch's autograd.
"""
from __future__ import annotations

import dataclasses
import math

import numpy as np


@dataclasses.dataclass
class Row:
    loss: float
    grad: np.ndarray      # float64 [vocab]: dloss / ds
    p: np.ndarray         # the teacher's probabilities of its entries (0 for padding)
    p_rest: float
    q: np.ndarray         # the student's probabilities [vocab]
    q_rest: float


def _exp_sum(x: np.ndarray) -> tuple[float, float]:
    """(m, sum of exp(x - m)) with m the maximum; (0, 0) of nothing."""
    if not x.size or x.max() == -np.inf:
        return 0.0, 0.0
    m = x.max()
    return m, float(np.exp(x - m).sum())


def row(s: np.ndarray, values: np.ndarray, indices: np.ndarray, rest: float | None = None,
        temperature: float = 1.0) -> Row:
    T = float(np.float32(temperature))
    s = np.asarray(s, np.float64) / T
    V = s.size
    indices = np.asarray(indices, np.int64)
    known = (indices >= 0) & (indices < V)
    at = indices[known]
    t = np.where(known, np.asarray(values, np.float64) / T, -np.inf)
    outcomes = np.append(t, -np.inf if rest is None else float(rest))
    m, z = _exp_sum(outcomes)
    if z == 0.0:  # the row has no teacher
        return Row(0.0, np.zeros(V), np.zeros(t.size), 0.0, np.exp(s - s.max()), 0.0)
    if np.unique(at).size != at.size:
        nan = np.full(V, np.nan)
        return Row(math.nan, nan, nan, math.nan, nan, math.nan)
    lp = outcomes - m - math.log(z)
    p = np.exp(lp)
    if not np.isfinite(s).any() or np.isnan(s).any() or (s == np.inf).any():
        nan = np.full(V, np.nan)
        return Row(math.nan, nan, p[:-1], float(p[-1]), nan, math.nan)
    s = s - s.max()  # nothing depends on a shift, and the lowest float32 would swallow the logarithm
    lse = math.log(np.exp(s).sum())
    other = np.ones(V, bool)
    other[at] = False
    mr, zr = _exp_sum(s[other])
    lq_rest = mr + math.log(zr) - lse if zr else -math.inf
    lq = np.full(t.size, -np.inf)
    lq[known] = s[at] - lse
    loss = 0.0
    for a, b in zip(lp, np.append(lq, lq_rest)):
        if a > -np.inf:
            loss += math.exp(a) * (a - b) if b > -np.inf else math.inf
    q = np.exp(s - lse)
    share = np.exp(s - mr) / zr if zr else np.zeros(V)  # of the other tokens' mass
    grad = (math.exp(lq_rest) - float(p[-1])) * share
    grad[at] = q[at] - p[:-1][known]
    return Row(loss, grad / T, p[:-1], float(p[-1]), q, math.exp(lq_rest))
