"""What paged_weight_accumulate asks for where a sequence has many query rows: a small part of 8 bytes for each of them and every 64 tokens (CPU only)."""
import pytest

import paper_2508_11553_amd as sd
from tests.test_abi import good_shape, lib  # noqa: F401


def up(n, to):
    return (n + to - 1) // to * to


@pytest.mark.parametrize("batch,kv_heads,group,tokens,most", [
    (8, 8, 4, 8192, 8192),      # whole prompts (the product of rows and 64-token stretches: 2 GB)
    (64, 8, 4, 8192, 8192),     # 16 GB
    (1, 8, 4, 131072, 131072),  # 64 GB
    (8, 8, 4, 8192, 64), (300, 2, 8, 5000, 40), (1, 1, 64, 1, 1), (3, 1, 17, 100, 1), (1, 2, 4, 100000, 5),
])
def test_bytes_of_many_rows(lib, batch, kv_heads, group, tokens, most):
    s = good_shape(batch=batch, num_q_heads=kv_heads * group, num_kv_heads=kv_heads, max_blocks_per_seq=8192, max_context_len=tokens)
    units, rows = batch * kv_heads, most * group
    few = units * up(tokens, 64) * 4 * 16 + units * 2 * up(tokens, 128) + 4096                 # that of 16 rows: products, and statistics of 128 tokens
    statistics = units * rows * 8 * -(-tokens // 1024) + (1 << 20)
    sums = units * -(-rows // 256) * up(tokens, 4) * 4 if rows > 256 else 0
    assert sd.paged_weight_workspace_bytes(s, most) <= max(few, max(statistics, sums) + units * rows * 8) + 1024


@pytest.mark.parametrize("kv_heads,group", [(1, 1), (8, 4), (2, 17), (1, 64)])
def test_a_larger_call_never_asks_for_less(lib, kv_heads, group):
    need = lambda batch, tokens, most: sd.paged_weight_workspace_bytes(  # noqa: E731
        good_shape(batch=batch, num_q_heads=kv_heads * group, num_kv_heads=kv_heads, max_blocks_per_seq=8192, max_context_len=tokens), most)
    batches, lengths, rows = (1, 2, 7, 63, 64, 65, 200), (1, 63, 64, 65, 1000, 1023, 1024, 1025, 4095, 4097, 20000, 131072), (1, 2, 4, 5, 16, 17, 33, 64, 65, 127, 250, 257, 300, 1000, 5000)
    for most in rows:
        for tokens in lengths:
            assert (x := [need(b, tokens, most) for b in batches]) == sorted(x)
    for batch in batches:
        for most in rows:
            assert (x := [need(batch, t, most) for t in lengths]) == sorted(x)
        for tokens in lengths:
            assert (x := [need(batch, tokens, m) for m in rows]) == sorted(x)
