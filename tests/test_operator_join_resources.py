"""What the compiler made of the kernel that joins the sums of several rounds of rows (CPU only), as test_operator_resources asks of the others."""
import os
import shutil

import pytest

from paper_2508_11553_amd import build as sd_build
from tests.test_kernel_resources import resource_remarks


@pytest.mark.skipif(shutil.which(sd_build.HIPCC) is None and not os.path.exists(sd_build.HIPCC), reason="needs hipcc")
def test_no_registers_in_memory(tmp_path):
    found = {k: v for k, v in resource_remarks("weight_scores.hip", tmp_path).items() if "weight_join_kernel" in k}
    assert len(found) == 1
    for name, res in found.items():
        assert res["ScratchSize"] == 0 and res["VGPRs Spill"] == 0 and res["Occupancy"] >= 4, (name, res)
