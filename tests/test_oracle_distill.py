"""Pins of oracle/distill.py: closed forms, oracle.policy, differences and torch's autograd."""
import math

import numpy as np
import pytest
import torch

from oracle import distill, policy, truncated


def _pair(seed, V=37, scale=2.0):
    rng = np.random.default_rng(seed)
    t = (rng.standard_normal(V) * scale).astype(np.float32)
    return t, (t + rng.standard_normal(V)).astype(np.float32), rng


def test_every_token_listed_is_the_whole_kl():
    t, s, rng = _pair(0)
    at = rng.permutation(t.size)
    want, _ = policy.kl_rows(s[None], t[None])
    assert distill.row(s, t[at], at).loss == pytest.approx(float(want[0]), abs=1e-12)
    v, i, rest = truncated.top_logits(t, t.size)
    assert rest == -math.inf and distill.row(s, v, i, rest).loss == pytest.approx(float(want[0]), abs=1e-12)


def test_two_tokens_closed_form():
    # teacher 3/4 : 1/4, student 1/2 : 1/2, the second token only as the rest
    loss = distill.row(np.zeros(2), np.array([math.log(3.0)]), np.array([0]), 0.0)
    assert loss.loss == pytest.approx(0.75 * math.log(1.5) + 0.25 * math.log(0.5), abs=1e-12)
    np.testing.assert_allclose(loss.grad, [0.5 - 0.75, 0.5 - 0.25], atol=1e-12)
    # without a rest the first token is all the teacher has
    loss = distill.row(np.zeros(2), np.array([math.log(3.0)]), np.array([0]))
    assert loss.loss == pytest.approx(math.log(2.0)) and loss.grad.tolist() == pytest.approx([-0.5, 0.5])


@pytest.mark.parametrize("T", [1.0, 2.0, 0.5])
def test_zero_at_equality_and_below_the_whole_kl(T):
    t, s, _ = _pair(1)
    v, i, rest = truncated.top_logits(t, 7, T)
    same = distill.row(t, v, i, rest, T)
    assert abs(same.loss) < 1e-6 and np.abs(same.grad).max() < 1e-6
    whole = distill.row(s, t, np.arange(t.size), None, T).loss
    assert 0 < distill.row(s, v, i, rest, T).loss < whole + 1e-9


@pytest.mark.parametrize("T, with_rest", [(1.0, True), (1.0, False), (1.7, True), (0.6, False)])
def test_gradient_is_the_difference_quotient_and_autograds(T, with_rest):
    t, s, _ = _pair(2)
    v, i, rest = truncated.top_logits(t, 6, T)
    rest = rest if with_rest else None
    got = distill.row(s, v, i, rest, T)
    s64, h = s.astype(np.float64), 1e-5
    for j in range(s.size):
        d = np.zeros(s.size)
        d[j] = h
        diff = (distill.row(s64 + d, v, i, rest, T).loss - distill.row(s64 - d, v, i, rest, T).loss) / (2 * h)
        assert got.grad[j] == pytest.approx(diff, abs=1e-8)
    assert abs(got.grad.sum()) < 1e-12
    x = torch.tensor(s64, requires_grad=True)
    Tf = float(np.float32(T))
    lq = (x / Tf).log_softmax(0)
    tt = torch.tensor(np.append(v.astype(np.float64) / Tf, rest if with_rest else -math.inf))
    p = tt.softmax(0)
    loss = (p[:-1] * (p[:-1].log() - lq[torch.tensor(i, dtype=torch.int64)])).sum()
    if with_rest:
        mask = torch.ones(s.size, dtype=torch.bool)
        mask[torch.tensor(i, dtype=torch.int64)] = False
        loss = loss + p[-1] * (p[-1].log() - lq[mask].logsumexp(0))
    loss.backward()
    assert got.loss == pytest.approx(loss.item(), abs=1e-12)
    np.testing.assert_allclose(got.grad, x.grad.numpy(), atol=1e-12)


def test_padding_duplicates_and_empty_rows():
    t, s, _ = _pair(3)
    v, i, rest = truncated.top_logits(t, 5)
    padded = distill.row(s, np.append(v, [9.0, np.nan]), np.append(i, [-1, t.size]), rest)
    whole = distill.row(s, v, i, rest)
    # (seven terms are summed in another order than five: a few roundings of 2^-53)
    assert padded.loss == pytest.approx(whole.loss, abs=1e-14)
    np.testing.assert_allclose(padded.grad, whole.grad, atol=1e-14)
    assert math.isnan(distill.row(s, np.append(v, v[0]), np.append(i, i[0]), rest).loss)
    none = distill.row(s, np.array([1.0]), np.array([-1]))
    assert none.loss == 0.0 and not none.grad.any()
    dead = s.copy()
    dead[:] = -np.inf
    assert math.isnan(distill.row(dead, v, i, rest).loss)
    dead = s.copy()
    dead[i[0]] = -np.inf
    got = distill.row(dead, v, i, rest)
    assert got.loss == math.inf and got.grad[i[0]] == pytest.approx(-got.p[0])
