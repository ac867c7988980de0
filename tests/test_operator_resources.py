"""What the compiler made of the kernels around the decode step (CPU only): none of them keeps registers in scratch memory or spills
vector registers, and each leaves room for as many waves as its launch counts on."""
import os
import shutil

import pytest

from paper_2508_11553_amd import build as sd_build
from tests.test_kernel_resources import resource_remarks


@pytest.mark.skipif(shutil.which(sd_build.HIPCC) is None and not os.path.exists(sd_build.HIPCC), reason="needs hipcc")
@pytest.mark.parametrize("source,least", [
    ("norm_rope.hip", {"norm_rope_kernel": (8, 4), "norm_rope_backward_kernel": (4, 4), "norm_weight_kernel": (2, 4)}),
    # 16 waves of one workgroup at four to a SIMD; 8 of two workgroups
    ("weight_scores.hip", {"weight_whole_kernel": (12, 4), "weight_products_kernel": (12, 4), "weight_apply_kept_kernel": (3, 4), "weight_stats_kernel": (4, 4),
                           "weight_apply_kernel": (4, 4), "weight_rows_kernel": (1, 4)}),
    ("kv_evict.hip", {"evict_select_kernel": (1, 4), "evict_move_kernel": (4, 4)}),
])
def test_no_registers_in_memory(source, least, tmp_path):
    remarks = resource_remarks(source, tmp_path)
    for kernel, (instances, occupancy) in least.items():
        found = {k: v for k, v in remarks.items() if kernel in k}
        assert len(found) >= instances, (kernel, list(found))
        for name, res in found.items():
            assert res["ScratchSize"] == 0 and res["VGPRs Spill"] == 0, (name, res)
            assert res["Occupancy"] >= occupancy, (name, res)
