"""Host arithmetic of the operators around the decode step (CPU only: compiled from kernels.h for the host)."""
import os
import shutil
import subprocess

import pytest

from paper_2508_11553_amd import build as sd_build
from tests.test_abi import lib  # noqa: F401
from tests.test_kernel_resources import CSRC

PROGRAM = r'''
#include <cstdio>
#include <cstdlib>
#include "kernels.h"
static void fail(const char *what, unsigned long a, unsigned long b) { std::printf("%s %lu %lu\n", what, a, b); std::exit(1); }
int main()
{
    // division by a product: every divisor a call can bring, at the numerators next to its multiples and at the largest
    unsigned long state = 1;
    for (unsigned by = 1; by <= 5000; ++by) {
        const sd::Division d = sd::division_by(by);
        for (int i = 0; i < 200; ++i) {
            state = state * 6364136223846793005ul + 1442695040888963407ul;
            const unsigned x = (unsigned)(state >> 33), q = x / by * by;   // below 2^31
            for (unsigned y : {x, q, q ? q - 1 : 0u, 0x7fffffffu, 0x7fffffffu / by * by, 0u, by - 1, by < 0x7fffffffu ? by : 0u})
                if (d.of(y) != y / by) fail("division", y, by);
        }
    }
    for (unsigned by : {1u << 20, (1u << 20) + 1, 0x3fffffffu, 0x40000000u, 0x7ffffffeu, 0x7fffffffu})
        for (unsigned y : {0u, by - 1, by, 0x7fffffffu, 0x7ffffffeu, 12345u})
            if (sd::division_by(by).of(y) != y / by) fail("division", y, by);
    // tiles of products have room for the rows; waves for all rows in as few rounds as the most waves need
    for (long rows = 1; rows <= 16; ++rows)
        if (16 / sd::weight_pack(rows) < rows || (sd::weight_pack(rows) < 4 && 16 / (2 * sd::weight_pack(rows)) >= rows)) fail("pack", rows, sd::weight_pack(rows));
    for (long rows = 0; rows <= 5000; ++rows) {
        const int waves = sd::row_waves(rows);
        if (waves < 1 || waves > sd::kRowWaves) fail("waves", rows, waves);
        const auto rounds = [rows](int w) { return (rows + w * sd::kRowsOfWave - 1) / (w * sd::kRowsOfWave); };
        if (rounds(waves) != rounds(sd::kRowWaves) || (waves > 1 && rounds(waves - 1) == rounds(waves))) fail("rounds", rows, waves);
    }
    std::printf("ok");
}
'''


@pytest.mark.skipif(shutil.which(sd_build.HIPCC) is None and not os.path.exists(sd_build.HIPCC), reason="needs hipcc")
def test_rules_compiled_for_the_host(tmp_path):
    (tmp_path / "rules.hip").write_text(PROGRAM)
    r = subprocess.run([sd_build.HIPCC, "--offload-host-only", "-O1", "-std=c++17", f"-I{CSRC}", str(tmp_path / "rules.hip"), "-o", str(tmp_path / "rules")],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    out = subprocess.run([str(tmp_path / "rules")], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout == "ok", out.stdout


@pytest.mark.parametrize("heads", [2, 6, 8, 24, 64])
def test_weight_workspace_of_many_rows_serves_fewer(heads):
    import paper_2508_11553_amd as sd
    from tests.test_abi import good_shape
    for n in (1, 500, 5000, 131072):
        for batch in (1, 16, 300):
            s = good_shape(batch=batch, num_q_heads=heads, num_kv_heads=2, max_blocks_per_seq=8192, max_context_len=n)
            sizes = [sd.paged_weight_workspace_bytes(s, most) for most in range(70)]
            assert 0 < sizes[0] and sizes == sorted(sizes)


def test_calls_of_more_threads_than_a_launch_has(lib):
    """2^32 - 1 threads: a launch of more fails, and one that follows it would read what the first has not written."""
    from tests.test_abi import good_shape
    from tests.test_operator_refusals import append, evict, good_norm, gradient, rows, weights
    for d, T in ((64, 2 ** 30 // 12 + 1), (128, 2 ** 29 // 12 + 1)):      # d / 16 threads to a row, 12 rows to a token
        n, s = good_norm(head_dim=d), good_shape(head_dim=d)
        assert rows(lib, n, T=T) == -2 and append(lib, s, n, T=T) == -2 and gradient(lib, n, T=T) == -2
    assert evict(lib, good_shape(batch=2 ** 21, num_kv_heads=2)) == -2                    # 1024 to a (sequence, KV head)
    assert evict(lib, good_shape(batch=2 ** 14, num_kv_heads=2, max_blocks_per_seq=8192, max_context_len=131072), budget=131072, stride=131072, ostride=131072) == -2   # 64 to a page
    assert evict(lib, good_shape(batch=2 ** 31 - 1, num_q_heads=2 ** 31 - 1, num_kv_heads=2 ** 31 - 1)) == -2
    assert weights(lib, good_shape(batch=2 ** 21, num_kv_heads=2), total=2 ** 21) == -2
    assert weights(lib, good_shape(batch=2 ** 31 - 1, num_q_heads=2 ** 31 - 1, num_kv_heads=2 ** 31 - 1), total=2 ** 31 - 1) == -2
    long = good_shape(batch=2 ** 18, num_q_heads=64, num_kv_heads=2, max_blocks_per_seq=8192, max_context_len=131072)
    assert weights(lib, long, qs=32, total=2 ** 19, most=2, stride=131072, size=2 ** 60) == -2
