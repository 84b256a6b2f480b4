"""Arguments of the operators on rows of logits that contradict each other or lie over each other are refused."""
import os

import pytest
import torch

from paper_2505_17218_amd import _lib as L
from paper_2505_17218_amd import engine


def test_a_gradient_buffer_of_another_type_than_asked_for():
    logits = torch.zeros(3, 8)
    for out, dtype in ((torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32)):
        with pytest.raises(ValueError):
            engine._grad_buffer(logits, torch.zeros(3, 8, dtype=out), dtype)
    for dtype, code in ((torch.float32, L.DASH_F32), (torch.bfloat16, L.DASH_BF16)):
        for out, asked in ((None, dtype), (torch.zeros(3, 8, dtype=dtype), dtype), (torch.zeros(3, 8, dtype=dtype), None)):
            got, kind = engine._grad_buffer(logits, out, asked)
            assert got.dtype == dtype and kind == code and (out is None or got is out)
    assert engine._grad_buffer(logits, None, None)[0].dtype == torch.float32
    with pytest.raises(ValueError):
        engine._grad_buffer(logits, None, torch.float16)


GRAD, ROWS, V, K, ROOM = 0x20000000, 4, 512, 8, 100  # ROOM: entries between two rows of the gradient
APART = dict(val=0x2000, idx=0x3000, rest=0x4000, norm=0x5000, weight=0x6000, loss=0x7000, ws=0x10000)


def _args(dtype, **kw):
    a = dict(APART)
    a.update(kw)
    return a, GRAD, V + ROOM, dtype


def _grad(a, grad, ldg, dtype):
    L.dash_distill_grad(0x10000000, V, ROWS, V, a["val"], a["idx"], a["rest"], K, 1.0, a["norm"], a["weight"], grad, ldg,
                        dtype, None)


def _both(a, grad, ldg, dtype):
    L.dash_distill_loss_grad(0x10000000, V, ROWS, V, a["val"], a["idx"], a["rest"], K, 1.0, a["weight"], a["loss"], grad,
                             ldg, dtype, a["ws"], 1 << 20, None)


@pytest.mark.skipif(not os.path.exists(L.LIB_PATH), reason="libdash.so not built")
@pytest.mark.parametrize("dtype, size", [(L.DASH_F32, 4), (L.DASH_BF16, 2)])
@pytest.mark.parametrize("f, names", [(_grad, ["val", "idx", "rest", "norm", "weight"]),
                                      (_both, ["val", "idx", "rest", "weight", "loss", "ws"])])
def test_a_gradient_over_another_array_of_the_call(f, names, dtype, size):
    """From one entry before it on, at a row's start and end, and from the room between two rows into the next."""
    need = L.dash_distill_workspace_bytes(ROWS, V)
    bytes_of = dict(val=4 * ROWS * K, idx=4 * ROWS * K, rest=4 * ROWS, norm=16 * ROWS, weight=4 * ROWS, loss=4 * ROWS, ws=need)
    stride, row = size * (V + ROOM), size * V
    for name in names:
        n = bytes_of[name]
        places = [GRAD, GRAD - n + 4, GRAD + row - 4, GRAD + stride, GRAD + stride - 4, GRAD + 3 * stride + row - 4]
        if name == "ws":  # aligned: the places that are
            places = [p & ~255 for p in (GRAD, GRAD + stride + 256)]
        for at in places:
            with pytest.raises(L.DashError) as e:
                f(*_args(dtype, **{name: at}))
            assert e.value.status == L.DASH_EINVAL and "overlaps the" in str(e.value), (name, hex(at), str(e.value))


@pytest.mark.gpu
def test_engine_refuses_a_gradient_over_what_it_reads():
    """A gradient next to its weights, and weights in the room between two of its rows, are fine."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rows, v = 4, 64
    logits, values = torch.randn(rows, v, device="cuda"), torch.randn(rows, 5, device="cuda")
    indices = torch.arange(5, dtype=torch.int32, device="cuda").repeat(rows, 1)
    flat = torch.ones(rows * (v + 8), device="cuda")
    wide = flat.view(rows, v + 8)[:, :v]
    _, norm = engine.distill_loss(logits, values, indices)
    for weight in (flat[:rows], flat[v + 6:v + 6 + rows], flat[3 * (v + 8) + v - 1:][:rows]):
        for call in (lambda: engine.distill_grad(logits, values, indices, norm, weight=weight, out=wide),
                     lambda: engine.distill_loss_grad(logits, values, indices, weight=weight, out=wide)):
            with pytest.raises(L.DashError):
                call()
    assert (flat == 1).all()
    _, want = engine.distill_loss_grad(logits, values, indices)
    for weight in (flat[v + 2:v + 2 + rows], flat[3 * (v + 8) + v:][:rows]):
        assert torch.equal(engine.distill_grad(logits, values, indices, norm, weight=weight, out=wide), want)
        assert torch.equal(engine.distill_loss_grad(logits, values, indices, weight=weight, out=wide)[1], want)
        assert (weight == 1).all()


@pytest.mark.skipif(not os.path.exists(L.LIB_PATH), reason="libdash.so not built")
@pytest.mark.parametrize("name", ["n", "vocab", "k"])
@pytest.mark.parametrize("f", [
    lambda n=4, vocab=64, k=5: L.dash_sample_truncated(0x10000000, 1 << 40, n, vocab, None, 0x2000, 0x3000, 1.0, k, 0.9, 0.0, 1,
                                                       0x4000, None, None, 0x10000, 1 << 40, None),
    lambda n=4, vocab=64, k=5: L.dash_sample_truncated_workspace_bytes(n, vocab, k),
    lambda n=4, vocab=64, k=5: L.dash_top_logits(0x10000000, 1 << 40, n, vocab, k, 1.0, 0x2000, 0x3000, None, 0x10000, 1 << 40,
                                                 None),
    lambda n=4, vocab=64, k=5: L.dash_top_logits_workspace_bytes(n, vocab, k),
    lambda n=4, vocab=64, k=5: L.dash_distill_loss(0x10000000, 1 << 40, n, vocab, 0x2000, 0x3000, None, k, 1.0, 0x4000, 0x5000,
                                                   0x10000, 1 << 40, None),
    lambda n=4, vocab=64, k=5: L.dash_distill_grad(0x10000000, 1 << 40, n, vocab, 0x2000, 0x3000, None, k, 1.0, 0x5000, None,
                                                   1 << 50, 1 << 40, L.DASH_F32, None),
    lambda n=4, vocab=64, k=5: L.dash_distill_loss_grad(0x10000000, 1 << 40, n, vocab, 0x2000, 0x3000, None, k, 1.0, None,
                                                        0x4000, 1 << 50, 1 << 40, L.DASH_F32, 0x10000, 1 << 40, None)])
def test_sizes_past_32_bits_do_not_wrap(f, name):
    for big in (2 ** 32, 2 ** 32 + 5, 2 ** 31, -2 ** 31 - 1, 2 ** 63 - 1):
        with pytest.raises(L.DashError) as e:
            f(**{name: big})
        assert e.value.status == L.DASH_EINVAL and "32 bits" in str(e.value)
