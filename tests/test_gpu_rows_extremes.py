"""The operators on rows of logits at the ends of the float32 range: temperatures near the largest float32 over logits that
use the whole range, and weights that the temperature carries past it.

Bounds as in test_gpu_truncated.py and test_gpu_distill.py: they count roundings relative to an exponent's size, so they do
not depend on the scale of logits and temperature."""
import numpy as np
import pytest
import torch

from oracle import distill
from paper_2505_17218_amd import engine

from gpu_util import dev_i32, require_gpu
from test_gpu_distill import _check_grad, _check_loss, _f32, _pair, _teacher
from test_gpu_truncated import _check_sample, _check_top

pytestmark = pytest.mark.gpu

HIGH = np.finfo(np.float32).max


@pytest.mark.parametrize("rows, V", [(5, 3001), (4, 20001), (600, 9001)])
@pytest.mark.parametrize("T", [1e36, 4e36])
def test_top_p_next_to_the_largest_float(T, rows, V):
    """The largest logit rounds up to a whole number of octaves that lies past the float32 range: a reference there would
    leave every exponential 0.  Uncut rows, cut rows, and rows enough that none is cut."""
    require_gpu()
    assert round(float(HIGH) / T * 1.4426950408889634) * 0.6931471805599453 * T > float(HIGH)
    rng = np.random.default_rng([31, V])
    l = (HIGH - T * 2.0 * np.abs(rng.standard_normal((min(rows, 7), V)))).astype(np.float32)
    l[:, V // 3] = HIGH
    for top_p, min_p in ((0.9, 0.0), (0.3, 0.0), (0.95, 0.05), (1.0, 0.1)):
        _check_sample(l, T, 0, top_p, min_p, row_of=np.arange(rows) % l.shape[0])


def _wide(rows, V, seed):
    l = np.random.default_rng([seed, V]).uniform(-1, 1, (rows, V)).astype(np.float32) * np.float32(3.3e38)
    l[:, V // 2] = HIGH
    l[0, V // 5] = -HIGH
    l[-1, 1:] = -HIGH  # one token far above all others
    return l


@pytest.mark.parametrize("rows, V", [(5, 3001), (4, 20001), (600, 9001)])
@pytest.mark.parametrize("T", [1e37, 4e37, 1e38, 3.4e38])
def test_draws_over_the_whole_range(T, rows, V):
    """Differences of two logits are up to twice the largest float32, and still only a few T."""
    require_gpu()
    l = _wide(min(rows, 7), V, 32)
    for top_k, top_p, min_p in ((0, 0.9, 0.0), (0, 1.0, 0.0), (0, 0.95, 0.3), (0, 1.0, 0.2), (30, 0.9, 0.0), (700, 0.6, 0.0)):
        _check_sample(l, T, top_k, top_p, min_p, row_of=np.arange(rows) % l.shape[0])


@pytest.mark.parametrize("V", [3001, 20001])
@pytest.mark.parametrize("T", [1e37, 4e37, 1e38, 3.4e38])
def test_largest_logits_over_the_whole_range(T, V):
    require_gpu()
    l = _wide(5, V, 33)
    l[2, :V // 2] = -HIGH
    for k in (1, 50, 1000):
        _check_top(l, k, T)


@pytest.mark.parametrize("rows, V, k", [(5, 3001, 20), (4, 20001, 30), (520, 40961, 30)])
@pytest.mark.parametrize("T", [1e37, 4e37, 1e38, 3.4e38])
def test_distillation_over_the_whole_range(T, rows, V, k):
    require_gpu()
    few = min(rows, 5)
    t, s = _wide(few, V, 34), _wide(few, V, 35)
    v, i, rest = _teacher(t, k, T)
    w = np.full(few, T / 8, np.float32)
    at = np.arange(rows) % few
    dev, vd, id_, rd, wd = _f32(s[at]), _f32(v[at]), dev_i32(i[at]), _f32(rest[at]), _f32(w[at])
    loss, norm = engine.distill_loss(dev, vd, id_, rd, T)
    grad = engine.distill_grad(dev, vd, id_, norm, rd, T, wd)
    both_loss, both = engine.distill_loss_grad(dev, vd, id_, rd, T, wd)
    assert torch.equal(loss, both_loss) and torch.equal(grad, both)
    for r in [*range(few), rows - 1]:
        want = distill.row(s[at[r]], v[at[r]], i[at[r]], rest[at[r]], T)
        _check_loss(loss[r].item(), want, (r, V, T))
        _check_grad(grad[r].double().cpu().numpy(), want, T, float(w[at[r]]), torch.float32, (r, V, T))


@pytest.mark.parametrize("rows, V", [(4, 3001), (4, 20001), (520, 40961)])
@pytest.mark.parametrize("T, weight", [(1e-39, 6.0), (1e-38, 6000.0), (0.1, 3e38)])
def test_weights_over_the_temperature_past_the_float_range(T, weight, rows, V):
    """weight / T times a row's mass difference is above the largest float32: entries whose share is 0 (masked ones among
    them) have gradient 0, those in between what the product gives."""
    require_gpu()
    few = min(rows, 4)
    t, s, rng = _pair(few, V, 36)
    s[:, rng.random(V) < 0.3] = -np.inf
    v, i, _ = _teacher(t, 20, 1.0)
    s[1, np.flatnonzero(~np.isin(np.arange(V), i[1]))[V // 2]] = 30.0  # (not the teacher's)
    w = np.full(few, weight, np.float32)
    at = np.arange(rows) % few
    dev, vd, id_, wd = _f32(s[at]), _f32(v[at]), dev_i32(i[at]), _f32(w[at])
    _, norm = engine.distill_loss(dev, vd, id_, None, T)
    grad = engine.distill_grad(dev, vd, id_, norm, None, T, wd)
    _, both = engine.distill_loss_grad(dev, vd, id_, None, T, wd)
    assert torch.equal(grad, both)
    for r in [*range(few), rows - 1]:
        want = distill.row(s[at[r]], v[at[r]], i[at[r]], None, T)
        got = grad[r].double().cpu().numpy()
        with np.errstate(over="ignore"):
            past = np.isinf((want.grad * float(w[at[r]])).astype(np.float32))  # past the float32 range themselves
        assert past.any() or at[r] != 1
        np.testing.assert_array_equal(got[past], np.sign(want.grad[past]) * np.inf)
        want.grad[past] = got[past] = 0.0
        _check_grad(got, want, T, float(w[at[r]]), torch.float32, (r, V, T))


@pytest.mark.parametrize("rows, V", [(4, 3001), (4, 20001), (300, 9001)])
@pytest.mark.parametrize("T, low, high", [(1e-38, 4.0, 9.0), (1e-30, 1e9, 2e9), (0.5, 2e38, 3.3e38), (0.5, -3.3e38, -2e38)])
def test_ascending_rows_whose_quotients_overflow(T, low, high, rows, V):
    """Every score is infinite, so a draw takes the lowest index: down an ascending row one entry at a time, if each pass
    leaves out only what came before.  The largest logits are equal; rows cut, uncut and in two rounds."""
    require_gpu()
    rng = np.random.default_rng([37, V])
    l = np.sort(rng.uniform(low, high, (4, V)).astype(np.float32), axis=1)
    assert (np.abs(l.astype(np.float64) / T) > 2.0 ** 128).all()
    l[0, -5:] = l[0, -1]
    l[1, V // 3] = l[1, -1]
    l[2, ::7] = -np.inf
    for top_p, min_p in ((0.9, 0.0), (0.3, 0.0), (0.5, 0.1), (1.0, 0.2)):
        _check_sample(l, T, 0, top_p, min_p, row_of=np.arange(rows) % 4)
