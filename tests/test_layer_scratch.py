"""Scratch memory of the kernels of selective state-space layers, from the built objects' metadata: none, but for fp32
rows in the kernels named here.  No GPU needed."""
import os

import pytest

from paper_2606_27748_amd import build as B
from tests.test_kernel_scratch import LLVM, scratch_bytes

# fp32 operands take twice the registers of bf16 ones: with states of 128 rows the sweeps' two waves of a SIMD want a few more.
ALLOWED = {"k_scan_sweepIfLi128ELi0E": 16, "k_scan_sweepIfLi128ELi1E": 16}


@pytest.mark.parametrize("source", ["flex_conv.hip", "flex_norm.hip", "flex_scan_fwd.hip", "flex_scan_bwd.hip"])
def test_no_spilled_registers(source, tmp_path):
    obj = os.path.join(B.BUILD, source.replace(".hip", ".o"))
    if not (os.path.exists(obj) and os.path.exists(f"{LLVM}/clang-offload-bundler")):
        pytest.skip("needs the built objects and the LLVM tools")
    over = {name: size for name, size in scratch_bytes(obj, str(tmp_path)).items()
            if size > max([v for k, v in ALLOWED.items() if k in name], default=0)}
    assert not over
