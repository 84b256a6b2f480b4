"""Pins of oracle/truncated.py: kept sets in closed form, draws against oracle.sampler and statistics."""
import math

import numpy as np
import pytest

from oracle import sampler, truncated

# probabilities 1/2, 1/4, 1/8, 1/16, 1/16 at scrambled places
P = np.array([1 / 16, 1 / 2, 1 / 16, 1 / 8, 1 / 4])
L = np.log(P).astype(np.float32)


@pytest.mark.parametrize("top_k, top_p, min_p, want", [
    (0, 1.0, 0.0, [1, 4, 3, 0, 2]), (1, 1.0, 0.0, [1]), (3, 1.0, 0.0, [1, 4, 3]), (9, 1.0, 0.0, [1, 4, 3, 0, 2]),
    (0, 0.3, 0.0, [1]), (0, 0.6, 0.0, [1, 4]), (0, 0.8, 0.0, [1, 4, 3]), (0, 0.9, 0.0, [1, 4, 3, 0]),
    (0, 0.99, 0.0, [1, 4, 3, 0, 2]), (0, 1e-9, 0.0, [1]),
    (0, 1.0, 0.4, [1, 4]), (0, 1.0, 0.2, [1, 4, 3]), (0, 1.0, 1.0, [1]),
    (2, 0.7, 0.0, [1, 4]),   # of 1/2 and 1/4 renormalised, 1/2 is 2/3 < 0.7
    (2, 0.6, 0.0, [1]), (3, 0.99, 0.4, [1, 4]),
])
def test_kept_closed_form(top_k, top_p, min_p, want):
    assert truncated.kept_tokens(L, 1.0, top_k, top_p, min_p).tolist() == want


def test_kept_at_a_temperature():
    # at T = 1/2 the probabilities are squared: 4/5.4.. of the mass is the first token's
    q = P ** 2 / (P ** 2).sum()
    assert q[1] < 0.75 and truncated.kept_tokens(L, 0.5, 0, 0.75).tolist() == [1, 4]
    assert truncated.kept_tokens(L, 0.5, 0, q[1] - 1e-6).tolist() == [1]
    assert truncated.kept_tokens(L, 0.5, 0, 1.0, 0.2).tolist() == [1, 4]  # (1/2)^2 >= 0.2 > (1/4)^2


def test_ties_and_borders():
    flat = np.zeros(8, np.float32)
    assert truncated.kept_tokens(flat, 1.0, 3).tolist() == [0, 1, 2]
    assert truncated.kept_tokens(flat, 1.0, 0, 0.5).tolist() == [0, 1, 2, 3]  # four of eight reach one half
    assert truncated.kept_tokens(flat, 1.0, 0, np.nextafter(0.5, 1.0)).tolist() == [0, 1, 2, 3, 4]
    assert truncated.kept_tokens(flat, 1.0, 0, 1.0, 1.0).tolist() == list(range(8))
    assert truncated.kept_tokens(np.array([-0.0, 0.0], np.float32), 1.0, 1).tolist() == [0]


def test_rows_without_entries():
    for bad in (-np.inf, np.inf, np.nan):
        l = np.full(6, bad, np.float32)
        assert truncated.kept_tokens(l, 1.0, 2, 0.5, 0.5).size == 0
        token, lp = truncated.sample_row(l, 0, 0, 1.0, 1, 2, 0.5)
        assert token == -1 and math.isnan(lp)
        l[4] = -3.0
        assert truncated.sample_row(l, 0, 0, 1.0, 1, 2, 0.5) == (4, 0.0)
    lowest = np.full(6, np.finfo(np.float32).min, np.float32)  # finite: a uniform row
    assert truncated.kept_tokens(lowest, 1.0, 0, 0.5).tolist() == [0, 1, 2]


def test_top_logits_closed_form():
    v, i, rest = truncated.top_logits(L, 2)
    assert i.tolist() == [1, 4] and v.tolist() == L[[1, 4]].tolist() and rest == pytest.approx(math.log(1 / 4))
    v, i, rest = truncated.top_logits(np.array([1.0, np.nan, -np.inf, np.inf], np.float32), 3)
    assert i.tolist() == [0, -1, -1] and v.tolist() == [1.0, -math.inf, -math.inf] and rest == -math.inf
    _, _, rest = truncated.top_logits(L, 1, 2.0)
    assert rest == pytest.approx(math.log(np.sqrt(P)[[0, 2, 3, 4]].sum()))


def test_draws_equal_the_untruncated_ones_where_kept():
    rng = np.random.default_rng(0)
    l = (rng.standard_normal((40, 301)) * 2).astype(np.float32)
    uid, step = np.arange(40), rng.integers(0, 99, 40)
    whole, lp = sampler.sample(l, uid, step, 0.8, 5)
    same, lp2 = truncated.sample(l, uid, step, 0.8, 5)
    assert np.array_equal(whole, same) and np.allclose(lp, lp2, atol=1e-12)
    cut, _ = truncated.sample(l, uid, step, 0.8, 5, 20, 0.9, 0.01)
    hits = 0
    for b in range(40):
        kept = truncated.kept_tokens(l[b], 0.8, 20, 0.9, 0.01)
        assert cut[b] in kept
        if whole[b] in kept:
            hits += 1
            assert cut[b] == whole[b]
    assert 0 < hits < 40


def test_frequencies_are_the_renormalised_distribution():
    n = 4000
    toks, _ = truncated.sample(np.broadcast_to(L, (n, 5)), np.arange(n), 3, 1.0, 11, 3, 0.99)
    count = np.bincount(toks, minlength=5)
    want = n * np.array([0, 4, 0, 1, 2]) / 7
    assert count[[0, 2]].sum() == 0
    chi = ((count - want)[[1, 3, 4]] ** 2 / want[[1, 3, 4]]).sum()
    assert chi < 13.8  # 2 degrees of freedom, p = 0.001
