"""The operators on rows of logits at temperatures near the largest float32, over logits that use the type's whole range.

Bounds as in test_gpu_truncated.py and test_gpu_distill.py: they count roundings relative to an exponent's size, so they do
not depend on the scale of logits and temperature."""
import numpy as np
import pytest
import torch

from gpu_util import require_gpu
from test_gpu_truncated import _check_sample

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
