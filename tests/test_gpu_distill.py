"""Distillation from a teacher's largest logits against oracle/distill.py.

Bounds.  The sum over the tokens that are not the teacher's has relative error d = 2.5e-6: terms y powers of two below
the reference are off by y ln 2 times two float32 roundings (difference, product with the two-part scale: 2^-24 each) and
a float32 exponential (2^-23), y averaging at most log2(vocab) < 18, and the row's float32 record of a sum adds 2^-24.
An error d of that sum moves ln q of a teacher's token by q_rest d and ln q_rest by (1 - q_rest) d, so the loss by
(q_rest - p_rest) d to first order and by d^2 beyond; float64 does the rest and the result is rounded to float32.
Gradients: q_rest and a token's share of it are each off by d at most (2 d), a teacher's q by q_rest d and, since the
row's normaliser is recorded in float32, by q 2^-24 (a difference q - p may be smaller than q by any factor, so this is no
rounding of the result); rounding to the gradient's type adds half a step, at float32 once more for the product with the
weight."""
import math

import numpy as np
import pytest
import torch

from oracle import distill, truncated
from paper_2505_17218_amd import engine

from gpu_util import dev_i32, require_gpu

pytestmark = pytest.mark.gpu

D = 2.5e-6
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def _pair(rows, V, seed, scale=2.5, noise=0.4):
    rng = np.random.default_rng([seed, rows, V])
    t = (rng.standard_normal((rows, V)) * scale).astype(np.float32)
    return t, (t + noise * rng.standard_normal((rows, V))).astype(np.float32), rng


def _teacher(t, k, T):
    got = [truncated.top_logits(r, k, T) for r in t]
    return (np.stack([g[0] for g in got]), np.stack([g[1] for g in got]),
            np.array([g[2] for g in got], np.float32))


def _f32(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda()


def _check_loss(got, want, what):
    what = (*what, want.loss, got)
    if math.isnan(want.loss) or math.isinf(want.loss):
        assert math.isnan(want.loss) == math.isnan(got) and math.isinf(want.loss) == math.isinf(got), what
    else:
        tol = (abs(want.q_rest - want.p_rest) + D) * D + 2.0 ** -24 * abs(want.loss) + 1e-12
        assert abs(got - want.loss) <= tol, (what, tol)


def _check_grad(got, want, T, w, dtype, what):
    if w == 0.0:
        assert not got.any(), what
        return
    if np.isnan(want.grad).any():
        assert np.isnan(got).all(), what
        return
    T = float(np.float32(T))
    g64 = want.grad * w
    share = np.where(want.q_rest > 0, want.q / max(want.q_rest, 1e-300), 0.0)
    tol = abs(w) / T * (abs(want.q_rest - want.p_rest) * 2 * D * share + want.q_rest * D * share + D * want.q_rest * want.q +
                        2.0 ** -24 * want.q)
    tol = tol + np.abs(g64) * (HALF[dtype] + 3 * 2.0 ** -24) + abs(w) / T * 1e-12 + 1.5e-38
    off = np.abs(got - g64)
    assert (off <= tol).all(), (what, int((off - tol).argmax()), off.max())


def _check(s, v, i, rest, T, weight=None, dtype=torch.float32, dev=None, out=None):
    rows, V = s.shape
    dev = _f32(s) if dev is None else dev
    vd, id_, rd, wd = _f32(v), dev_i32(i), _f32(rest), _f32(weight)
    loss, norm = engine.distill_loss(dev, vd, id_, rd, T)
    grad = engine.distill_grad(dev, vd, id_, norm, rd, T, wd, dtype=dtype)
    both_loss, both = engine.distill_loss_grad(dev, vd, id_, rd, T, wd, out=out, dtype=dtype)
    assert torch.equal(grad, both) or torch.equal(grad.isnan(), both.isnan())
    loss, both_loss = loss.cpu().numpy().astype(np.float64), both_loss.cpu().numpy().astype(np.float64)
    got = [grad.double().cpu().numpy(), both.double().cpu().numpy()]
    for r in range(rows):
        want = distill.row(s[r], v[r], i[r], None if rest is None else rest[r], T)
        w = 1.0 if weight is None else float(weight[r])
        _check_loss(loss[r], want, (r, s.shape, T))
        if w == 0.0:
            assert both_loss[r] == 0.0
        else:
            assert both_loss[r] == loss[r] or math.isnan(loss[r]) and math.isnan(both_loss[r])
        for g in got:
            _check_grad(g[r], want, T, w, dtype, (r, s.shape, T))
    return loss


@pytest.mark.parametrize("T", [1.0, 2.0, 0.7])
@pytest.mark.parametrize("with_rest", [True, False])
@pytest.mark.parametrize("V, k", [(2, 1), (5, 3), (1000, 64), (4097, 1024), (20001, 50), (300, 300)])
def test_loss_and_gradients(V, k, with_rest, T):
    require_gpu()
    t, s, rng = _pair(5, V, 1)
    v, i, rest = _teacher(t, k, T)
    w = rng.random(5).astype(np.float32)
    w[2] = 0.0
    for dtype in (torch.float32, torch.bfloat16):
        _check(s, v, i, rest if with_rest else None, T, w, dtype)
    _check(s, v, i, rest if with_rest else None, T)


@pytest.mark.parametrize("V", [1, 3, 4, 4095, 4096, 4100, 8191, 12289])
def test_sizes(V):
    require_gpu()
    t, s, _ = _pair(2, V, 2)
    v, i, rest = _teacher(t, min(V, 9), 1.0)
    _check(s, v, i, rest, 1.0)


@pytest.mark.parametrize("rows, V, k, dtype", [
    (513, 40960, 20, torch.float32), (520, 50257, 30, torch.float32), (513, 40959, 30, torch.float32),
    (513, 65536, 30, torch.bfloat16), (520, 65535, 30, torch.bfloat16),
    (513, 90112, 40, torch.float32), (513, 90115, 40, torch.bfloat16), (513, 118784, 1024, torch.bfloat16),
    (514, 118785, 300, torch.float32), (520, 151936, 64, torch.bfloat16), (520, 151933, 64, torch.float32),
    (513, (1 << 18) + 6, 64, torch.bfloat16), (1100, 8200, 64, torch.float32), (3000, 300, 20, torch.bfloat16)])
def test_many_rows(rows, V, k, dtype):
    """Enough rows that none is cut into stretches: the pair of calls and the single one give the same bits, apart, in
    place and in rows of weight 0; some rows against the oracle."""
    require_gpu()
    gen = torch.Generator(device="cuda").manual_seed(V)
    teacher = torch.randn(rows, V, device="cuda", generator=gen) * 2.5
    s = teacher + 0.4 * torch.randn(rows, V, device="cuda", generator=gen)
    w = torch.rand(rows, device="cuda", generator=gen)
    w[5] = 0.0
    v, i, rest = engine.top_logits(teacher, k, 0.8)
    del teacher
    loss, norm = engine.distill_loss(s, v, i, rest, 0.8)
    grad = engine.distill_grad(s, v, i, norm, rest, 0.8, w, dtype=dtype)
    both_loss, both = engine.distill_loss_grad(s, v, i, rest, 0.8, w, dtype=dtype)
    loss[5] = 0.0
    assert torch.equal(loss, both_loss) and torch.equal(grad, both)
    for r in (0, 5, 6, rows // 2, rows - 1):
        want = distill.row(s[r].cpu().numpy(), v[r].cpu().numpy(), i[r].cpu().numpy(), float(rest[r]), 0.8)
        if r != 5:
            _check_loss(loss[r].item(), want, (r, V))
        _check_grad(grad[r].double().cpu().numpy(), want, 0.8, float(w[r]), dtype, (r, V))
    if dtype == torch.float32:
        both_loss, both = engine.distill_loss_grad(s, v, i, rest, 0.8, w, out=s)
        assert torch.equal(loss, both_loss) and torch.equal(grad, both)


@pytest.mark.parametrize("rows, V, k", [(3, 151936, 64), (40, 50257, 20), (1, 151936, 1024), (1, 600_001, 100)])
def test_large(rows, V, k):
    require_gpu()
    t, s, rng = _pair(rows, V, 3)
    v, i, rest = _teacher(t, k, 1.0)
    _check(s, v, i, rest, 1.0, rng.random(rows).astype(np.float32))
    _check(s, v, i, None, 1.0, None, torch.bfloat16)


@pytest.mark.parametrize("T", [1e-30, 1e-3, 1e3, 1e30])
def test_small_and_large_temperatures(T):
    require_gpu()
    t, s, rng = _pair(3, 3001, 14)
    v, i, rest = _teacher(t, 20, T)
    w = rng.random(3).astype(np.float32)
    _check(s, v, i, rest, T, w)
    _check(s, v, i, None, T, w)


def test_a_gradient_of_zero_at_a_denormal_temperature():
    """1 / T is above the float32 range, the gradient of an equal student still 0."""
    require_gpu()
    t, _, _ = _pair(3, 3001, 15)
    v, i, _ = _teacher(t, 20, 1.0)
    vd, id_ = _f32(v), dev_i32(i)
    loss, norm = engine.distill_loss(_f32(t), vd, id_, None, 1e-39)
    grad = engine.distill_grad(_f32(t), vd, id_, norm, None, 1e-39)
    both_loss, both = engine.distill_loss_grad(_f32(t), vd, id_, None, 1e-39)
    for x in (loss, grad, both_loss, both):
        assert not x.any()


def test_sure_students():
    """The teacher's tokens hold all but 1e-30 of the student's mass, or the other tokens do: nothing cancels, and what is
    left of p_rest is spread over the others."""
    require_gpu()
    t, s, rng = _pair(4, 3000, 4)
    v, i, rest = _teacher(t, 10, 1.0)
    for gap in (70.0, -70.0, 400.0):
        sure = s.copy()
        np.put_along_axis(sure, i.astype(np.int64), np.take_along_axis(s, i.astype(np.int64), 1) + np.float32(gap), 1)
        _check(sure, v, i, rest, 1.0)
        _check(sure, v, i, None, 1.0)
    same = t.copy()
    loss = _check(same, v, i, rest, 1.0)
    assert (np.abs(loss) < 1e-9).all()


def test_masks_padding_and_empty_rows():
    require_gpu()
    V, k = 2500, 12
    t, s, rng = _pair(9, V, 5)
    v, i, rest = _teacher(t, k, 1.0)
    v[0, 5:], i[0, 5:] = -np.inf, -1       # fewer entries than k
    i[1, 3], v[1, 3] = V, np.nan           # an index past the vocabulary is padding, whatever its value
    i[2] = -1                              # only a rest
    i[3], rest[3] = -1, -np.inf            # no teacher
    s[4, rng.random(V) < 0.5] = -np.inf    # masked logits
    s[4, i[4]] = 1.0
    s[5] = -np.inf                         # a row that its mask leaves empty
    s[6, i[6, 0]] = -np.inf                # the teacher's first token is masked
    keep = np.zeros(V, bool)
    keep[i[7]] = True
    s[7, ~keep] = -np.inf                  # nothing but the teacher's tokens
    s[8] = np.finfo(np.float32).min        # finite: uniform
    _check(s, v, i, rest, 1.0)
    _check(s, v, i, None, 1.0, None, torch.bfloat16)
    w = np.ones(9, np.float32)
    w[[5, 6]] = 0.0                        # padded rows may hold anything
    s[5, 7] = np.nan
    _check(s, v, i, rest, 1.0, w)


def test_nan_inf_and_repeated_indices():
    require_gpu()
    V = 5000
    t, s, _ = _pair(6, V, 6)
    v, i, rest = _teacher(t, 8, 1.0)
    s[0, 4321], s[1, 17], s[2, i[2, 3]] = np.nan, np.inf, np.nan
    i[3, 5] = i[3, 0]
    i[4, 7] = i[4, 6]
    _check(s, v, i, rest, 1.0)


def test_in_place_strides_and_what_lies_past_a_row():
    require_gpu()
    V, k = 4099, 20
    t, s, rng = _pair(6, V, 7)
    v, i, rest = _teacher(t, k, 1.3)
    w = rng.random(6).astype(np.float32)
    wide = torch.full((6, V + 11), 77.0, device="cuda")
    dev = wide[:, 3:V + 3]
    dev.copy_(_f32(s))
    for dtype in (torch.float32, torch.bfloat16):
        room = torch.full((6, V + 7), -5.0, dtype=dtype, device="cuda")
        _check(s, v, i, rest, 1.3, w, dtype, dev, room[:, 1:V + 1])
        assert (room[:, 0] == -5).all() and (room[:, V + 1:] == -5).all()
    want_loss, want = engine.distill_loss_grad(dev, _f32(v), dev_i32(i), _f32(rest), 1.3, _f32(w))
    loss, got = engine.distill_loss_grad(dev, _f32(v), dev_i32(i), _f32(rest), 1.3, _f32(w), out=dev)
    assert got.data_ptr() == dev.data_ptr() and torch.equal(got, want) and torch.equal(loss, want_loss)
    assert (wide[:, :3] == 77).all() and (wide[:, V + 3:] == 77).all()
    dev.copy_(_f32(s))
    _, norm = engine.distill_loss(dev, _f32(v), dev_i32(i), _f32(rest), 1.3)
    assert torch.equal(engine.distill_grad(dev, _f32(v), dev_i32(i), norm, _f32(rest), 1.3, _f32(w), out=dev), want)


def test_gradient_is_the_difference_quotient_of_the_loss():
    """(loss(s + h) - loss(s - h)) / 2h along random directions: the losses are off by D (q_rest - p_rest) at most and the
    quotient by h^2 times the third derivative, below 1 for |direction| <= 1 at T = 1."""
    require_gpu()
    t, s, rng = _pair(8, 900, 8, scale=1.5)
    v, i, rest = _teacher(t, 30, 1.0)
    vd, id_, rd = _f32(v), dev_i32(i), _f32(rest)
    loss, grad = engine.distill_loss_grad(_f32(s), vd, id_, rd)
    h = 2.0 ** -6
    d = rng.choice([-1.0, 1.0], s.shape).astype(np.float32)
    up = engine.distill_loss(_f32(s + h * d), vd, id_, rd)[0].double()
    down = engine.distill_loss(_f32(s - h * d), vd, id_, rd)[0].double()
    along = (grad.double().cpu().numpy() * d).sum(1)
    quotient = ((up - down) / (2 * h)).cpu().numpy()
    # rounding of s +- h d to float32 moves each entry by 2^-22 at most, the loss by |gradient|_1 times that
    tol = h * h + (2 * D + 2.0 ** -21) / (2 * h) * 2
    assert (np.abs(along - quotient) <= tol).all(), (along, quotient)


def test_teacher_to_student_chain_other_stream_and_graph():
    """The operators together: a teacher's rows reduced to their largest entries, the student's loss and gradient against
    them, a gradient step on the logits, and a draw from the result; eager, on a side stream and as a replayed graph."""
    require_gpu()
    rows, V = 12, 20011
    t, s, _ = _pair(rows, V, 9)
    teacher, student = _f32(t), _f32(s)
    uid = dev_i32(np.arange(rows))
    w = torch.full((rows,), 1.0 / rows, device="cuda")

    def calls():
        v, i, rest = engine.top_logits(teacher, 50, 1.0)
        loss, grad = engine.distill_loss_grad(student, v, i, rest, 1.0, w)
        loss2, norm = engine.distill_loss(student, v, i, rest, 1.0)
        grad2 = engine.distill_grad(student, v, i, norm, rest, 1.0, w)
        moved = student - 5.0 * rows * grad
        after, _ = engine.distill_loss(moved, v, i, rest, 1.0)
        tok, lp = engine.sample_truncated(moved, uid, uid, 1.0, 3, 50, 0.9)
        return v, i, rest, loss, grad, loss2, grad2, after, tok, lp

    got = calls()
    assert torch.equal(got[3], got[5]) and torch.equal(got[4], got[6])
    for r in range(rows):
        want = distill.row(s[r], got[0][r].cpu().numpy(), got[1][r].cpu().numpy(), float(got[2][r]), 1.0)
        assert got[3][r].item() == pytest.approx(want.loss, abs=D, rel=1e-6)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = calls()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = calls()
    for seed in (10, 11, 12):
        t2, s2, _ = _pair(rows, V, seed)
        teacher.copy_(_f32(t2))
        student.copy_(_f32(s2))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(calls(), held))


def test_offsets_past_32_bits():
    require_gpu()
    V, ld, rows = 1501, 1 << 28, 6
    t, s, _ = _pair(rows, V, 13)
    v, i, rest = _teacher(t, 10, 1.0)
    flat = torch.zeros((rows - 1) * ld + V, dtype=torch.float32, device="cuda")
    dev = flat.as_strided((rows, V), (ld, 1))
    dev.copy_(_f32(s))
    out = torch.empty((rows - 1) * ld + V, dtype=torch.float32, device="cuda").as_strided((rows, V), (ld, 1))
    _check(s, v, i, rest, 1.0, dev=dev, out=out)
