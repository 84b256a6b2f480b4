"""Refusals of the operators on rows of logits: the C ABI before any HIP call (no GPU needed) and engine's checks."""
import math

import pytest
import torch

from paper_2505_17218_amd import _lib as L
from paper_2505_17218_amd import engine

import os

pytestmark = pytest.mark.skipif(not os.path.exists(L.LIB_PATH), reason="libdash.so not built")

BIG = 0x10000000


def _status(f, *args):
    with pytest.raises(L.DashError) as e:
        f(*args)
    return e.value.status


def _sample(logits=BIG, ld=512, n=4, V=512, uid=0x2000, step=0x3000, T=1.0, top_k=5, top_p=0.9, min_p=0.0, out=0x4000,
            ws=0x10000, ws_bytes=1 << 30):
    L.dash_sample_truncated(logits, ld, n, V, None, uid, step, T, top_k, top_p, min_p, 1, out, None, None, ws, ws_bytes,
                            None)


@pytest.mark.parametrize("bad", [dict(logits=None), dict(uid=None), dict(step=None), dict(out=None), dict(n=-1),
                                 dict(V=0), dict(V=(1 << 28) + 1, ld=1 << 29), dict(ld=511), dict(T=0.0), dict(T=-1.0),
                                 dict(T=math.nan), dict(T=math.inf), dict(top_k=-1), dict(top_p=0.0), dict(top_p=1.1),
                                 dict(top_p=math.nan), dict(top_p=-0.5), dict(min_p=-0.1), dict(min_p=1.5),
                                 dict(min_p=math.nan)])
def test_sample_truncated_refuses(bad):
    assert _status(lambda: _sample(**bad)) == L.DASH_EINVAL


def test_sample_truncated_limits():
    assert _status(lambda: _sample(top_k=1025, V=4096, ld=4096)) == L.DASH_ENOTSUP
    assert _status(lambda: _sample(n=(1 << 21) + 1)) == L.DASH_ENOTSUP
    _sample(n=0)  # no rows: nothing to do
    need = L.dash_sample_truncated_workspace_bytes(4, 151936, 0)
    assert need > 0
    for ws, size in ((None, need), (0x10000, need - 1), (0x10000, 0)):
        assert _status(lambda: _sample(V=151936, ld=151936, top_k=0, ws=ws, ws_bytes=size)) == L.DASH_ECAPACITY
    assert _status(lambda: _sample(V=151936, ld=151936, top_k=0, ws=0x10080)) == L.DASH_EINVAL


def _top(logits=BIG, ld=512, rows=4, V=512, k=8, T=1.0, values=0x2000, indices=0x3000,
         ws=0x10000, ws_bytes=1 << 30):
    L.dash_top_logits(logits, ld, rows, V, k, T, values, indices, None, ws, ws_bytes, None)


@pytest.mark.parametrize("bad, want", [
    (dict(logits=None), L.DASH_EINVAL), (dict(values=None), L.DASH_EINVAL), (dict(indices=None), L.DASH_EINVAL),
    (dict(rows=-1), L.DASH_EINVAL), (dict(V=0), L.DASH_EINVAL), (dict(ld=511), L.DASH_EINVAL),
    (dict(k=0), L.DASH_EINVAL), (dict(T=0.0), L.DASH_EINVAL), (dict(T=math.inf), L.DASH_EINVAL),
    (dict(k=1025), L.DASH_ENOTSUP), (dict(rows=(1 << 21) + 1), L.DASH_ENOTSUP)])
def test_top_logits_refuses(bad, want):
    assert _status(lambda: _top(**bad)) == want
    _top(rows=0)


def test_workspaces_that_are_too_small():
    need = L.dash_top_logits_workspace_bytes(1, 151936, 64)
    assert need > 0
    for ws, size in ((None, need), (0x10000, need - 1)):
        assert _status(lambda: _top(rows=1, V=151936, ld=151936, k=64, ws=ws, ws_bytes=size)) == L.DASH_ECAPACITY
    assert _status(lambda: _top(rows=1, V=151936, ld=151936, k=64, ws=0x10010)) == L.DASH_EINVAL
    need = L.dash_distill_workspace_bytes(1, 151936)
    assert need > 0 and L.dash_distill_workspace_bytes(5000, 151936) == 0
    for f in (_loss, _both):
        a = _args(rows=1, V=151936, ld=151936, ldg=151936)
        assert _status(f, {**a, "ws_bytes": need - 1}) == L.DASH_ECAPACITY
        assert _status(f, {**a, "ws": None}) == L.DASH_ECAPACITY
        assert _status(f, {**a, "ws": 0x10010}) == L.DASH_EINVAL
    # sizes that the calls refuse need none
    assert L.dash_top_logits_workspace_bytes(0, 100, 5) == L.dash_top_logits_workspace_bytes(1, 100, 0) == 0
    assert L.dash_sample_truncated_workspace_bytes(-1, 100, 5) == L.dash_distill_workspace_bytes(3, 0) == 0


def _args(**kw):
    a = dict(logits=BIG, ld=512, rows=4, V=512, val=0x2000, idx=0x3000, rest=None, k=8, T=1.0, loss=0x4000, norm=0x5000,
             weight=None, grad=0x20000000, ldg=512, dtype=0, ws=0x10000, ws_bytes=1 << 30)
    a.update(kw)
    return a


def _loss(a):
    L.dash_distill_loss(a["logits"], a["ld"], a["rows"], a["V"], a["val"], a["idx"], a["rest"], a["k"], a["T"],
                        a["loss"], a["norm"], a["ws"], a["ws_bytes"], None)


def _grad(a):
    L.dash_distill_grad(a["logits"], a["ld"], a["rows"], a["V"], a["val"], a["idx"], a["rest"], a["k"], a["T"],
                        a["norm"], a["weight"], a["grad"], a["ldg"], a["dtype"], None)


def _both(a):
    L.dash_distill_loss_grad(a["logits"], a["ld"], a["rows"], a["V"], a["val"], a["idx"], a["rest"], a["k"], a["T"],
                             a["weight"], a["loss"], a["grad"], a["ldg"], a["dtype"], a["ws"], a["ws_bytes"], None)


COMMON = [(dict(logits=None), 1), (dict(val=None), 1), (dict(idx=None), 1), (dict(rows=-1), 1), (dict(V=0), 1),
          (dict(ld=511), 1), (dict(k=0), 1), (dict(k=-3), 1), (dict(T=0.0), 1), (dict(T=math.nan), 1),
          (dict(k=1025), 5), (dict(rows=(1 << 21) + 1), 5)]
GRADS = [(dict(grad=None), 1), (dict(ldg=511), 1), (dict(dtype=2), 1), (dict(dtype=-1), 1),
         (dict(grad=BIG + 4), 1), (dict(grad=BIG, dtype=1), 1), (dict(grad=BIG, ldg=513), 1),
         (dict(grad=BIG - 4, ldg=512), 1), (dict(grad=BIG + 4 * (3 * 512 + 511)), 1)]


@pytest.mark.parametrize("bad, want", COMMON + [(dict(loss=None), 1), (dict(norm=None), 1)])
def test_distill_loss_refuses(bad, want):
    assert _status(_loss, _args(**bad)) == want


@pytest.mark.parametrize("bad, want", COMMON + GRADS + [(dict(norm=None), 1)])
def test_distill_grad_refuses(bad, want):
    assert _status(_grad, _args(**bad)) == want


@pytest.mark.parametrize("bad, want", COMMON + GRADS + [(dict(loss=None), 1)])
def test_distill_loss_grad_refuses(bad, want):
    assert _status(_both, _args(**bad)) == want


def test_no_rows_is_no_work():
    for f in (_loss, _grad, _both):
        f(_args(rows=0))


def test_engine_refuses_host_tensors_and_wrong_types():
    l, i = torch.zeros(2, 8), torch.zeros(2, dtype=torch.int32)
    v, idx = torch.zeros(2, 3), torch.zeros(2, 3, dtype=torch.int32)
    for call in (lambda: engine.sample_truncated(l, i, i, 1.0, 0), lambda: engine.top_logits(l, 2),
                 lambda: engine.distill_loss(l, v, idx), lambda: engine.distill_loss_grad(l, v, idx),
                 lambda: engine.distill_grad(l, v, idx, torch.zeros(2, 4)), lambda: engine.top_logits(l.double(), 2),
                 lambda: engine.top_logits(l[0], 2)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.gpu
def test_engine_checks_shapes_and_strides():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    l = torch.zeros(4, 64, device="cuda")
    i = torch.zeros(4, dtype=torch.int32, device="cuda")
    v, idx = torch.zeros(4, 3, device="cuda"), torch.zeros(4, 3, dtype=torch.int32, device="cuda")
    norm = torch.zeros(4, 4, device="cuda")
    for call in (lambda: engine.top_logits(l.t(), 2), lambda: engine.top_logits(l[:, ::2], 2),
                 lambda: engine.top_logits(l[:1].expand(4, 64), 2), lambda: engine.top_logits(l.bfloat16(), 2),
                 lambda: engine.sample_truncated(l, i.long(), i, 1.0, 0),
                 lambda: engine.sample_truncated(l, i, i[:3], 1.0, 0),
                 lambda: engine.sample_truncated(l[:3], i, i, 1.0, 0),
                 lambda: engine.sample_truncated(l, i, i, 1.0, 0, row_of=i[:2]),
                 lambda: engine.sample_truncated(l, i.cpu(), i, 1.0, 0),
                 lambda: engine.distill_loss(l, v, idx.long()), lambda: engine.distill_loss(l, v[:3], idx),
                 lambda: engine.distill_loss(l, v, idx[:, :2]), lambda: engine.distill_loss(l, v, idx, norm),
                 lambda: engine.distill_loss(l, v.t().contiguous().t(), idx),
                 lambda: engine.distill_grad(l, v, idx, norm[:, :3].contiguous()),
                 lambda: engine.distill_loss_grad(l, v, idx, weight=norm),
                 lambda: engine.distill_loss_grad(l, v, idx, dtype=torch.float16),
                 lambda: engine.distill_loss_grad(l, v, idx, out=torch.zeros(4, 63, device="cuda")),
                 lambda: engine.distill_loss_grad(l, v, idx, out=torch.zeros(64, 4, device="cuda").t())):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: engine.distill_loss_grad(l, v, idx, out=torch.zeros(5, 64, device="cuda")[1:].view(4, 64)),):
        call()  # a view of its own memory is fine
    flat = torch.zeros(4 * 64 + 8, device="cuda")
    with pytest.raises(L.DashError):  # partly over the logits
        engine.distill_loss_grad(flat[:256].view(4, 64), v, idx, out=flat[8:].view(4, 64))
