"""No access of the attention side's kernels claims more alignment than its callers promise (CPU only: hipcc cross-compiles without a GPU)."""
import os
import shutil
import subprocess

import pytest

from tests.test_operand_alignment import CSRC, PROMISED, accesses


@pytest.mark.parametrize("source", ["rope.hip", "attn_decode.hip"])
def test_no_access_claims_more_than_the_contract(source, tmp_path):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    from paper_2508_02317_amd.build import HIPCC_FLAGS
    out = str(tmp_path / "kernels.ll")
    res = subprocess.run([hipcc, *[f for f in HIPCC_FLAGS if f != "-fPIC"], "--cuda-device-only", "-emit-llvm", "-S", os.path.join(CSRC, source), "-o", out],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    seen = list(accesses(open(out).read()))
    assert len(seen) > 20
    too_much = [i for i, a in seen if a > PROMISED]
    assert not too_much, too_much[:5]
