"""The distillation gradient may be written over the logits.  Its kernels must not tell the compiler that the two are apart:
no store to global memory in them carries a promise of that (`!noalias`) in the optimised IR (no GPU needed)."""
import re
import subprocess

from test_kernel_resources import _cmd, needs_hipcc


@needs_hipcc
def test_gradient_stores_may_alias_the_logits(tmp_path):
    ir = tmp_path / "distill.ll"
    r = subprocess.run([*_cmd("distill.hip", "off"), "-emit-llvm", "-S", "-o", str(ir)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    kernels = {m.group(1): m.group(0) for m in re.finditer(r"^define [^@]*@(\w+)\(.*?^}", ir.read_text(), re.M | re.S)}
    in_place = [k for k in kernels if "distill_grad_k" in k or "distill_loss_grad_k" in k]
    assert len(in_place) == 4, sorted(kernels)
    for k in in_place:
        stores = [line for line in kernels[k].splitlines() if " store " in line and "addrspace(1)" in line]
        assert len(stores) > 5
        assert not [line for line in stores if "!noalias" in line], k
