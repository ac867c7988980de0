"""Sizes that the operators around the decode step refuse before anything is launched (CPU only)."""
import pytest

from tests.test_abi import good_shape, lib  # noqa: F401
from tests.test_operator_refusals import evict, weights


@pytest.mark.parametrize("batch,pages", [(8193, 8191), (8191, 8193), (2731, 24573)])
def test_moves_of_one_thread_more_than_a_launch_has(lib, batch, pages):
    """2^26 - 1 new pages, a wave each, four waves to a workgroup: 2^24 workgroups of 256 threads, 2^32 in all."""
    assert batch * pages == 2 ** 26 - 1
    tokens = 16 * pages
    s = good_shape(batch=batch, num_q_heads=1, num_kv_heads=1, max_blocks_per_seq=pages, max_context_len=tokens)
    assert evict(lib, s, budget=tokens, stride=tokens, ostride=tokens) == -2


@pytest.mark.parametrize("tokens", [2 ** 31 - 65535, 2 ** 31 - 1])
def test_sequences_whose_end_no_walk_can_pass(lib, tokens):
    """Walks go on by up to 65536 tokens at a time until they are past the last one: beyond 2^31 - 65536 a 32-bit position would wrap before."""
    s = good_shape(max_blocks_per_seq=2 ** 27, max_context_len=tokens)
    assert evict(lib, s, stride=2 ** 31) == -2
    assert weights(lib, s, stride=2 ** 31, size=2 ** 62) == -2
    assert weights(lib, s, qs=32, total=400, most=100, stride=2 ** 31, size=2 ** 62) == -2
