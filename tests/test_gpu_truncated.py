"""dash_sample_truncated and dash_top_logits against oracle/truncated.py: tokens, indices and values exactly, sums
within the derived bounds.

Bound on a log of a sum of exponentials: an entry y powers of two below the reference is off by y ln 2 times three
float32 roundings (difference, scale, product: 2^-24 each) and one float32 exponential (2^-23); a row's mass-weighted y
is at most log2(vocab) < 18 here, so the log is off by less than 18 * 0.7 * 3 * 2^-24 + 2^-23 < 2.5e-6, to which the
float32 result adds half a step."""
import math

import numpy as np
import pytest
import torch

from oracle import truncated
from paper_2505_17218_amd import engine

from gpu_util import dev_i32, require_gpu

pytestmark = pytest.mark.gpu

LSE_TOL = 2.5e-6
HALF = 2.0 ** -24
LOWEST = float(np.finfo(np.float32).min)


def _close(got, want, what):
    got = np.asarray(got, np.float64)
    with np.errstate(over="ignore"):  # the output is float32: LOWEST / 0.3 = -1.13e39 is -inf in it
        want = np.where(np.isinf(np.asarray(want, np.float32)), np.asarray(want, np.float32), np.asarray(want, np.float64))
    fine = np.isfinite(want)
    np.testing.assert_array_equal(np.isfinite(got), fine, err_msg=what)
    np.testing.assert_array_equal(got[~fine], want[~fine], err_msg=what)
    off = np.abs(got[fine] - want[fine])
    assert (off <= LSE_TOL + 2 * HALF * np.abs(want[fine])).all(), (what, off.max())


def _rows(kind: str, rows: int, V: int, seed: int) -> np.ndarray:
    rng = np.random.default_rng([seed, rows, V])
    l = (rng.standard_normal((rows, V)) * 2.5).astype(np.float32)
    if kind == "peak":
        at = rng.integers(0, V, (rows, 12))
        np.put_along_axis(l, at, (10 + 6 * rng.random((rows, 12))).astype(np.float32), 1)
    elif kind == "ties":  # few distinct values: equal logits across every border
        l = np.round(l).astype(np.float32)
    elif kind == "equal":
        l[:] = 1.5
    elif kind == "up":
        l = np.sort(l, axis=1)
    elif kind == "down":
        l = np.sort(l, axis=1)[:, ::-1].copy()
    elif kind == "masked":
        l[rng.random(l.shape) < 0.97] = -np.inf
        l[:, rng.integers(0, V)] = np.nan
        l[:, rng.integers(0, V)] = np.inf
        l[0] = -np.inf                      # a row that its mask leaves empty
        if rows > 1:
            l[1] = np.nan
        if rows > 2:
            l[2] = -np.inf
            l[2, V // 2] = -7.0             # one token left
        if rows > 3:
            l[3] = LOWEST                   # finite: uniform over the type's lowest value
        if rows > 4:
            l[4, rng.random(V) < 0.9] = LOWEST
    elif kind == "far":  # differences past what a float32 exponential holds
        l = (rng.standard_normal((rows, V)) * 200).astype(np.float32)
        l[:, 0] = 3e38
        if rows > 1:
            l[1, 0], l[1, 1:] = -3e38, -3.2e38
    return l


def _check_top(l: np.ndarray, k: int, T: float, dev=None):
    v, i, rest = engine.top_logits(torch.from_numpy(l).cuda() if dev is None else dev, k, T)
    want = [truncated.top_logits(r, k, T) for r in l]
    np.testing.assert_array_equal(i.cpu().numpy(), np.stack([w[1] for w in want]))
    np.testing.assert_array_equal(v.cpu().numpy(), np.stack([w[0] for w in want]))
    _close(rest.cpu().numpy(), [w[2] for w in want], f"rest of {l.shape}, k {k}, T {T}")


def _check_sample(l: np.ndarray, T: float, top_k: int, top_p: float, min_p: float, dev=None, seed=7, row_of=None):
    n = l.shape[0] if row_of is None else len(row_of)
    uid, step = np.arange(n) * 3 + 1, (np.arange(n) * 7) % 50
    tok, lp = engine.sample_truncated(torch.from_numpy(l).cuda() if dev is None else dev, dev_i32(uid), dev_i32(step), T,
                                      seed, top_k, top_p, min_p, row_of=None if row_of is None else dev_i32(row_of))
    want, want_lp = truncated.sample(l, uid, step, T, seed, top_k, top_p, min_p, row_of)
    what = f"{l.shape} T {T} k {top_k} p {top_p} min_p {min_p}"
    np.testing.assert_array_equal(tok.cpu().numpy(), want, err_msg=what)
    got = lp.cpu().numpy()
    np.testing.assert_array_equal(np.isnan(got), np.isnan(want_lp))
    _close(np.nan_to_num(got), np.nan_to_num(want_lp), what)


KINDS = ["normal", "peak", "ties", "equal", "up", "down", "masked", "far"]
SIZES = [1, 2, 3, 5, 63, 64, 257, 1000, 1024, 1025, 4095, 4096, 4097, 8193, 12289, 20001]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("V", [1, 5, 1000, 4097, 20001])
def test_top_logits(kind, V):
    require_gpu()
    l = _rows(kind, 6, V, 1)
    for k in (1, 2, 64, 1000, 1024):
        _check_top(l, k, 1.0)
    _check_top(l, 33, 0.3)
    _check_top(l, 33, 5.0)


@pytest.mark.parametrize("V", SIZES)
def test_top_logits_sizes(V):
    require_gpu()
    for rows, k in ((1, 1), (3, min(V, 1024)), (2, 7), (5, 129)):
        _check_top(_rows("normal", rows, V, 2), k, 1.0)


@pytest.mark.parametrize("rows, V, k", [(3, 151936, 64), (2, 151936, 1024), (70, 50257, 20), (1, 151936, 1),
                                        (300, 9001, 50), (1, 1 << 20, 300)])
def test_top_logits_large(rows, V, k):
    require_gpu()
    _check_top(_rows("peak", rows, V, 3), k, 1.0)
    _check_top(_rows("up", rows, V, 3), k, 1.0)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T", [1.0, 0.7, 3.0])
def test_sample(kind, T):
    require_gpu()
    for V in (1, 5, 1000, 4097, 20001):
        l = _rows(kind, 6, V, 4)
        for top_k, top_p, min_p in ((0, 1.0, 0.0), (1, 1.0, 0.0), (40, 1.0, 0.0), (0, 0.9, 0.0), (0, 1.0, 0.05),
                                    (1024, 0.8, 0.01), (0, 0.3, 0.0), (0, 0.95, 0.1), (V, 0.5, 0.0), (3, 0.5, 0.5),
                                    (0, 1e-6, 0.0), (0, 1.0, 1.0)):
            _check_sample(l, T, top_k, top_p, min_p)


@pytest.mark.parametrize("V", SIZES)
def test_sample_sizes(V):
    require_gpu()
    l = _rows("normal", 4, V, 5)
    for top_k, top_p, min_p in ((0, 0.9, 0.0), (17, 0.9, 0.0), (0, 0.6, 0.02)):
        _check_sample(l, 1.0, top_k, top_p, min_p)


@pytest.mark.parametrize("rows, V", [(3, 151936), (130, 50257)])
@pytest.mark.parametrize("top_k, top_p, min_p", [(50, 0.9, 0.0), (0, 0.95, 0.0), (0, 1.0, 0.05), (0, 0.5, 0.0)])
def test_sample_large(rows, V, top_k, top_p, min_p):
    require_gpu()
    _check_sample(_rows("normal", rows, V, 6), 1.0, top_k, top_p, min_p)
    _check_sample(_rows("peak", rows, V, 6), 0.8, top_k, top_p, min_p)


@pytest.mark.parametrize("top_k, top_p, min_p", [(50, 0.9, 0.0), (700, 0.99, 0.0), (0, 0.95, 0.0), (0, 1.0, 0.05), (0, 0.5, 0.0),
                                                 (0, 0.7, 0.01), (0, 1.0, 0.0)])
def test_sample_many_rows(top_k, top_p, min_p):
    """Enough rows that none is cut into stretches."""
    require_gpu()
    row_of = np.arange(600) % 97
    l = _rows("normal", 97, 9001, 18)
    l[50:] = _rows("peak", 47, 9001, 18)
    l[7] = -np.inf
    _check_sample(l, 0.9, top_k, top_p, min_p, row_of=row_of)


@pytest.mark.parametrize("top_k, top_p, min_p", [(0, 0.6, 0.0), (20, 0.9, 0.0), (0, 1.0, 0.2)])
def test_sample_thousands_of_rows(top_k, top_p, min_p):
    require_gpu()
    _check_sample(_rows("normal", 97, 1501, 21), 1.1, top_k, top_p, min_p, row_of=np.arange(3001) % 97)


@pytest.mark.parametrize("rows", [3, 260])
@pytest.mark.parametrize("top_p, min_p", [(0.95, 0.0), (0.4, 0.0), (1.0, 0.1)])
def test_sample_long_rows(rows, top_p, min_p):
    """Rows of more than 2^18 tokens."""
    require_gpu()
    _check_sample(_rows("normal", 3, (1 << 18) + 77, 19), 1.0, 0, top_p, min_p, row_of=np.arange(rows) % 3)


def test_small_and_large_temperatures():
    require_gpu()
    l = _rows("normal", 4, 3001, 8)
    for T in (1e-3, 1e-30, 1e-38, 1e3, 1e30):
        if T > 1e-38:  # (a rest of that temperature is above the float32 range)
            _check_top(l, 25, T)
        for top_k, top_p, min_p in ((0, 0.9, 0.0), (30, 0.9, 0.0), (0, 1.0, 0.5)):
            _check_sample(l, T, top_k, top_p, min_p)


def test_border_is_decided_in_64_bits():
    """Rows whose mass reaches top_p to within float32 rounding: equal logits in numbers that make the border exact, and
    a border moved by 1e-9 to either side of a token's cumulative mass."""
    require_gpu()
    flat = np.zeros((32, 6000), np.float32)
    for top_p in (0.5, 0.25, 1 / 3, 0.125 + 2 ** -40):
        _check_sample(flat, 1.0, 0, top_p, 0.0)
    l = np.sort(_rows("normal", 1, 4000, 9), axis=1)[:, ::-1].repeat(64, 0).copy()
    w = np.exp(l[0].astype(np.float64) - l[0, 0])
    at = np.cumsum(w) / w.sum()
    for n in (3, 500, 2000):
        for shift in (-1e-9, 1e-9):
            _check_sample(l, 1.0, 0, float(at[n] + shift), 0.0)


def test_strides_row_map_and_status():
    require_gpu()
    V = 5003
    l = _rows("normal", 7, V, 10)
    wide = torch.full((7, V + 9), 99.0, device="cuda")  # what lies past a row must not be read as one
    wide[:, 5:V + 5] = torch.from_numpy(l).cuda()
    dev = wide[:, 5:V + 5]
    _check_top(l, 50, 1.0, dev)
    _check_sample(l, 1.0, 20, 0.9, 0.0, dev)
    _check_sample(l, 1.0, 0, 0.9, 0.0, dev)
    row_of = [0, 0, 6, 3, 3, 3, 1, 2, 0, 5]
    _check_sample(l, 0.9, 0, 0.8, 0.0, dev, row_of=row_of)
    _check_sample(l, 0.9, 9, 0.8, 0.0, dev, row_of=row_of)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    uid = dev_i32([0, 1])
    for top_k in (0, 5):
        status.zero_()
        engine.sample_truncated(dev[:2], uid, uid, 1.0, 3, top_k, 0.9, status=status)
        assert status.item() == 0
        empty = dev[:2].clone()
        empty[1] = -math.inf
        tok, lp = engine.sample_truncated(empty, uid, uid, 1.0, 3, top_k, 0.9, status=status)
        assert status.item() == 2 and tok[1].item() == -1 and math.isnan(lp[1].item()) and tok[0].item() >= 0
    tok, lp = engine.sample_truncated(dev, dev_i32([]), dev_i32([]), 1.0, 3)
    assert tok.numel() == 0 and lp.numel() == 0


def test_nothing_cut_is_the_untruncated_sampler():
    require_gpu()
    l = torch.from_numpy(_rows("normal", 64, 30011, 11)).cuda()
    uid, step = dev_i32(np.arange(64)), dev_i32(np.arange(64) + 5)
    for T in (1.0, 0.7):
        tok, lp = engine.sample(l, uid, step, T, 12)
        tok2, lp2 = engine.sample_truncated(l, uid, step, T, 12)
        assert torch.equal(tok, tok2)
        _close(lp2.cpu().numpy(), lp.cpu().double().numpy(), "log-prob")
        tok3, none = engine.sample_truncated(l, uid, step, T, 12, top_k=30011, with_logprob=False)
        assert torch.equal(tok, tok3) and none is None


def test_offsets_past_32_bits():
    """Rows that start more than 2^32 bytes into the logits."""
    require_gpu()
    V, ld = 3001, 1 << 28
    flat = torch.zeros(5 * ld + V, dtype=torch.float32, device="cuda")
    dev = flat.as_strided((6, V), (ld, 1))
    l = _rows("normal", 6, V, 12)
    dev.copy_(torch.from_numpy(l).cuda())
    _check_top(l, 10, 1.0, dev)
    _check_sample(l, 1.0, 10, 0.9, 0.0, dev)
    _check_sample(l, 1.0, 0, 0.9, 0.0, dev)


def test_equal_calls_give_equal_bits():
    require_gpu()
    l = torch.from_numpy(_rows("ties", 40, 50257, 13)).cuda()
    uid = dev_i32(np.arange(40))
    first = engine.top_logits(l, 200, 0.7), engine.sample_truncated(l, uid, uid, 0.7, 1, 0, 0.9)
    for _ in range(5):
        again = engine.top_logits(l, 200, 0.7), engine.sample_truncated(l, uid, uid, 0.7, 1, 0, 0.9)
        for a, b in zip(first, again):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("kind, V, k", [("peak", 151936, 1024), ("up", 151936, 900), ("normal", 50257, 1000)])
def test_equal_calls_give_equal_bits_for_many_entries(kind, V, k):
    """Lists of candidates too long to be cut at once, in an order that differs between calls."""
    require_gpu()
    l = torch.from_numpy(_rows(kind, 4, V, 20)).cuda().repeat(10, 1)
    uid = dev_i32(np.arange(40))
    first = engine.top_logits(l, k, 0.7), engine.sample_truncated(l, uid, uid, 0.7, 1, k, 0.9)
    for t in first[0]:
        assert torch.equal(t[:4], t[36:])
    for _ in range(5):
        again = engine.top_logits(l, k, 0.7), engine.sample_truncated(l, uid, uid, 0.7, 1, k, 0.9)
        for a, b in zip(first, again):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_other_stream_and_graph():
    require_gpu()
    l = torch.from_numpy(_rows("normal", 9, 20001, 14)).cuda()
    uid, step = dev_i32(np.arange(9)), dev_i32(np.arange(9))

    def calls():
        return (*engine.top_logits(l, 40, 1.0), *engine.sample_truncated(l, uid, step, 1.0, 2, 30, 0.9),
                *engine.sample_truncated(l, uid, step, 1.0, 2, 0, 0.9))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = calls()
    side.synchronize()
    for a, b in zip(calls(), got):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = calls()
    for seed in (15, 16, 17):
        l.copy_(torch.from_numpy(_rows("normal", 9, 20001, seed)).cuda())
        step += 1
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(calls(), held):
            assert torch.equal(a, b)


def test_calls_at_once_on_two_streams():
    """Calls that overlap in time have workspaces of their own: 20 of each kind on two streams, other rows on either."""
    require_gpu()
    sides = []
    for s in range(2):
        l = torch.from_numpy(_rows("normal", 300, 20011, 22 + s)).cuda()
        teacher = torch.from_numpy(_rows("peak", 300, 20011, 24 + s)).cuda()
        sides.append((l, teacher, dev_i32(np.arange(300) + s), torch.cuda.Stream()))

    def calls(l, teacher, uid):
        v, i, rest = engine.top_logits(teacher, 64, 1.0)
        return (v, i, rest, *engine.distill_loss_grad(l, v, i, rest), *engine.sample_truncated(l, uid, uid, 0.9, 3, 0, 0.6),
                *engine.sample_truncated(l, uid, uid, 0.9, 3, 600, 0.9))

    want = [calls(*s[:3]) for s in sides]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for k, s in enumerate(sides):
            with torch.cuda.stream(s[3]):
                got[k].append(calls(*s[:3]))
    torch.cuda.synchronize()
    for k in range(2):
        for g in got[k]:
            assert all(torch.equal(a, b) for a, b in zip(g, want[k]))


def test_two_graphs_replayed_in_turn():
    require_gpu()
    graphs = []
    for s in range(2):
        l = torch.from_numpy(_rows("normal", 40, 30011, 26 + s)).cuda()
        uid = dev_i32(np.arange(40) + s)
        run = lambda l=l, uid=uid: (*engine.top_logits(l, 700, 1.0), *engine.sample_truncated(l, uid, uid, 1.0, 5, 0, 0.5))
        run()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = run()
        graphs.append((graph, held, run))
    for _ in range(4):
        for graph, held, run in graphs:
            graph.replay()
            want = run()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(held, want))
