"""Registers of the kernels on rows of logits, from the compiler's remarks (a gfx950 cross-compile, no GPU needed).

None uses scratch memory: a reload inside a loop that streams a row waits for every load in flight, and a launch with
scratch is slow to start.  The loops that need two work-groups of 1024 threads (or four of 512) on a CU stay within 64
vector registers, and the fused gradient's tiles within the 256 that two waves per SIMD have."""
import pytest

from test_kernel_resources import _resources, needs_hipcc


@needs_hipcc
@pytest.mark.parametrize("src, kernels, lean", [
    ("top_logits.hip", 5, ["top_part_k"]),
    ("truncate.hip", 32, ["draw_firstILb1ELb1ELb0ELb0E", "draw_firstILb1ELb1ELb1ELb0E"]),
    ("distill.hip", 7, ["distill_loss_k", "distill_part_k", "distill_grad_k"])])
def test_no_scratch_and_full_occupancy(src, kernels, lean):
    res = _resources(src, "off")
    assert len(res) == kernels, sorted(res)
    for name, r in res.items():
        assert r.get("ScratchSize [bytes/lane]", 0) == 0, (name, r)
        if any(k in name for k in lean):
            assert r["VGPRs"] <= 64, (name, r)
        assert r["VGPRs"] <= 256, (name, r)
