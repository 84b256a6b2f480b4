"""The special rows of the distillation loss (masks, padding, NaN, repeated indices, teachers without mass, sure students)
in every variant of the kernels: rows cut into stretches, rows of one work-group, loss and gradient in one launch, and
gradients over the logits.  Bounds as in test_gpu_distill.py."""
import math

import numpy as np
import pytest
import torch

from oracle import distill
from paper_2505_17218_amd import engine

from gpu_util import dev_i32, require_gpu
from test_gpu_distill import _check_grad, _check_loss, _f32, _pair, _teacher

pytestmark = pytest.mark.gpu

K = 12
KINDS = ["plain", "padded", "past the vocabulary", "only a rest", "no teacher", "no mass", "no mass, repeated", "half masked",
         "empty", "first token masked", "teacher's tokens only", "lowest", "NaN at the end", "inf in the middle",
         "NaN at a token", "repeated at the start", "repeated at the end", "a stretch masked", "sure", "sure of others",
         "one other left", "NaN without weight"]


def _special(V, T, seed):
    """A row of every kind: student logits, the teacher's values, indices and rest, weights."""
    n = len(KINDS)
    t, s, rng = _pair(n, V, seed)
    v, i, rest = _teacher(t, K, T)
    w = (0.5 + rng.random(n)).astype(np.float32)
    for r, kind in enumerate(KINDS):
        at = i[r].copy()
        others = np.setdiff1d(np.arange(V), at)
        if kind == "padded":
            v[r, 5:], i[r, 5:] = -np.inf, -1
        elif kind == "past the vocabulary":
            v[r, 3], i[r, 3], i[r, 4] = np.nan, V, np.iinfo(np.int32).min
        elif kind == "only a rest":
            i[r] = -1
        elif kind == "no teacher":
            i[r], rest[r] = -1, -np.inf
        elif kind.startswith("no mass"):
            v[r], rest[r] = -np.inf, -np.inf
            if kind.endswith("repeated"):
                i[r] = 0
        elif kind == "half masked":
            s[r, rng.random(V) < 0.5] = -np.inf
            s[r, at] = 1.0
        elif kind == "empty":
            s[r] = -np.inf
        elif kind == "first token masked":
            s[r, at[0]] = -np.inf
        elif kind == "teacher's tokens only":
            s[r, others] = -np.inf
        elif kind == "lowest":
            s[r] = np.finfo(np.float32).min
        elif kind == "NaN at the end":
            s[r, others[-1]] = np.nan
        elif kind == "inf in the middle":
            s[r, others[V // 2]] = np.inf
        elif kind == "NaN at a token":
            s[r, at[K - 1]] = np.nan
        elif kind == "repeated at the start":
            i[r, 7] = i[r, 2] = 1
        elif kind == "repeated at the end":
            i[r, 11] = i[r, 10] = V - 1
        elif kind == "a stretch masked":
            s[r, V // 5:4 * V // 5] = -np.inf
            s[r, at] = 1.0
        elif kind == "sure":
            s[r, at] += np.float32(70)
        elif kind == "sure of others":
            s[r, at] -= np.float32(70)
        elif kind == "one other left":
            s[r, others] = -np.inf
            s[r, others[-1]] = 0.5
        elif kind == "NaN without weight":
            s[r, ::7], w[r] = np.nan, 0.0
    return s, v, i, rest, w


def _equal(a, b):
    """Same bits, NaN for NaN."""
    return torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(0.0, math.inf, -math.inf),
                                                             b.nan_to_num(0.0, math.inf, -math.inf))


def _check_all(s, v, i, rest, w, T, dtype, at):
    """Rows `at` of the special ones: both ways to the gradient, apart and in place; every kind against the oracle."""
    dev, vd, id_, wd = _f32(s[at]), _f32(v[at]), dev_i32(i[at]), _f32(w[at])
    rd = None if rest is None else _f32(rest[at])
    held = dev.clone()
    loss, norm = engine.distill_loss(dev, vd, id_, rd, T)
    grad = engine.distill_grad(dev, vd, id_, norm, rd, T, wd, dtype=dtype)
    both_loss, both = engine.distill_loss_grad(dev, vd, id_, rd, T, wd, dtype=dtype)
    assert _equal(dev, held)
    assert _equal(both_loss, torch.where(wd == 0, 0.0, loss)) and _equal(grad, both)
    if dtype == torch.float32:
        over = dev.clone()
        assert _equal(engine.distill_grad(over, vd, id_, norm, rd, T, wd, out=over), grad)
        over_loss, over = engine.distill_loss_grad(dev, vd, id_, rd, T, wd, out=dev)
        assert over.data_ptr() == dev.data_ptr() and _equal(over, grad) and _equal(over_loss, both_loss)
    seen = {}
    for r, kind in enumerate(at):
        if kind in seen:  # equal rows, equal bits
            assert _equal(grad[r], grad[seen[kind]]) and _equal(loss[r], loss[seen[kind]]), KINDS[kind]
            continue
        seen[kind] = r
        want = distill.row(s[kind], v[kind], i[kind], None if rest is None else rest[kind], T)
        what = (KINDS[kind], r, dev.shape, T, rest is None)
        _check_loss(loss[r].item(), want, what)
        _check_grad(grad[r].double().cpu().numpy(), want, T, float(w[kind]), dtype, what)


@pytest.mark.parametrize("with_rest", [True, False])
@pytest.mark.parametrize("T", [1.0, 0.6])
@pytest.mark.parametrize("rows, V, dtype", [
    (len(KINDS), 20001, torch.float32), (len(KINDS), 20001, torch.bfloat16),   # cut into four stretches
    (len(KINDS), 151936, torch.float32),                                       # into 37
    (len(KINDS), 2500, torch.float32),                                         # a work-group per row
    (600, 20001, torch.float32), (600, 20001, torch.bfloat16),                 # the same, the gradient cut
    (520, 40961, torch.float32), (513, 65537, torch.bfloat16),                 # one launch
    (513, 118787, torch.float32)])                                             # with a part that is read twice
def test_special_rows(rows, V, dtype, T, with_rest):
    require_gpu()
    s, v, i, rest, w = _special(V, T, 41)
    at = np.arange(rows) % len(KINDS)
    if rows > len(KINDS):
        at[3 * len(KINDS):-len(KINDS)] = 0  # mostly plain rows
    _check_all(s, v, i, rest if with_rest else None, w, T, dtype, at)


@pytest.mark.parametrize("kind", KINDS)
def test_special_rows_alone(kind):
    """A single row of more than 2^18 entries: 64 stretches for the loss, 146 for the gradient."""
    require_gpu()
    s, v, i, rest, w = _special(600_001, 1.0, 42)
    _check_all(s, v, i, rest, w, 1.0, torch.float32, np.array([KINDS.index(kind)]))
