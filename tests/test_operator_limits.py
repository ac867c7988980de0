"""Sizes that the operators around the decode step refuse before anything is launched (CPU only)."""
import pytest

from tests.test_abi import good_shape, lib  # noqa: F401
from tests.test_operator_refusals import evict


@pytest.mark.parametrize("batch,pages", [(8193, 8191), (8191, 8193), (2731, 24573)])
def test_moves_of_one_thread_more_than_a_launch_has(lib, batch, pages):
    """2^26 - 1 new pages, a wave each, four waves to a workgroup: 2^24 workgroups of 256 threads, 2^32 in all."""
    assert batch * pages == 2 ** 26 - 1
    tokens = 16 * pages
    s = good_shape(batch=batch, num_q_heads=1, num_kv_heads=1, max_blocks_per_seq=pages, max_context_len=tokens)
    assert evict(lib, s, budget=tokens, stride=tokens, ostride=tokens) == -2
