"""What the compiler made of the kernels that close a rollout's loop (CPU only): none of them keeps registers in scratch memory or spills vector registers, and
each leaves room for as many waves as its launch counts on."""
import os
import shutil

import pytest

from paper_2508_11553_amd import build as sd_build
from tests.test_kernel_resources import resource_remarks


@pytest.mark.skipif(shutil.which(sd_build.HIPCC) is None and not os.path.exists(sd_build.HIPCC), reason="needs hipcc")
@pytest.mark.parametrize("source,least", [
    # sixteen waves of one workgroup at four to a SIMD, or eight of two
    ("sample.hip", {"sample_stretch_kernel": (4, 4), "sample_pick_kernel": (2, 4), "sample_choose_kernel": (4, 4)}),
    ("token_logprobs.hip", {"logprob_kernel": (4, 4), "logprob_join_kernel": (2, 1), "logprob_backward_kernel": (2, 4)}),
    ("plan_step.hip", {"plan_kernel": (1, 1), "plan_sums_kernel": (3, 1), "plan_fill_kernel": (1, 2)}),
])
def test_no_registers_in_memory(source, least, tmp_path):
    remarks = resource_remarks(source, tmp_path)
    for kernel, (instances, occupancy) in least.items():
        found = {k: v for k, v in remarks.items() if kernel in k}
        assert len(found) >= instances, (kernel, list(found))
        for name, res in found.items():
            assert res["ScratchSize"] == 0 and res["VGPRs Spill"] == 0, (name, res)
            assert res["Occupancy"] >= occupancy, (name, res)
