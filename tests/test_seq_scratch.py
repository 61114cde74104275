"""Scratch memory of the packed-sequence kernels, from the built objects' metadata: none, but for fp32 rows in the
kernels named here.  No GPU needed."""
import os

import pytest

from paper_2606_27748_amd import build as B
from tests.test_kernel_scratch import LLVM, scratch_bytes

# fp32 rows take twice the registers of bf16 ones.  The sweeps' six waves leave a wave 256 of them, the key sweep's
# two workgroups per CU as many; k_delta_grad takes all 512.
ALLOWED = {
    "k_delta_sweepIfLi128E": 72,
    "k_delta_rsweepIfLi64E": 12,
    "k_delta_rsweepIfLi128E": 436,
    "k_delta_gradIfLi128E": 384,
    "k_attn_dkvIfLi64E": 148,
}


@pytest.mark.parametrize("source", ["flex_attn_fwd.hip", "flex_attn_bwd.hip", "flex_delta_fwd.hip", "flex_delta_bwd.hip"])
def test_no_spilled_registers(source, tmp_path):
    obj = os.path.join(B.BUILD, source.replace(".hip", ".o"))
    if not (os.path.exists(obj) and os.path.exists(f"{LLVM}/clang-offload-bundler")):
        pytest.skip("needs the built objects and the LLVM tools")
    over = {name: size for name, size in scratch_bytes(obj, str(tmp_path)).items()
            if size > max([v for k, v in ALLOWED.items() if k in name], default=0)}
    assert not over
