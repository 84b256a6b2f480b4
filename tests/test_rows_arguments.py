"""Arguments of the operators on rows of logits that contradict each other or lie over each other are refused."""
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
