"""Calls of many query rows with no more workspace than they ask for: the weights of whole prompts, bytes behind the workspace untouched."""
import numpy as np
import pytest

from tests.test_gpu_weight_scores import Cache, U, queries

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sd():
    import torch
    assert torch.cuda.is_available()
    import paper_2508_11553_amd as m
    m.load()
    return m


@pytest.mark.parametrize("lens,rows,hq,hkv,d,kv,bound", [
    ([1300, 700, 0, 65], [1300, 700, 0, 65], 8, 2, 64, "bf16", None),        # dealt out by the lengths, rounds of rows
    ([1, 200], [1, 200], 64, 1, 64, "bf16", None),
    ([300, 1000], [5, 9], 8, 2, 128, "fp8", 60000),                           # a loose bound on the lengths
    ([20000], [6], 4, 1, 64, "bf16", None),                                   # groups of more than one workgroup's
    ([150 + 3 * b for b in range(70)], [150 + 3 * b for b in range(70)], 4, 1, 64, "bf16", None),   # dealt out by the bound
    ([40 + b for b in range(66)], [3] * 66, 8, 1, 128, "fp8", 3000),
])
def test_no_more_than_they_ask_for(sd, lens, rows, hq, hkv, d, kv, bound):
    import torch
    c = Cache(lens, hkv, d, kv, 61, max_context_len=bound)
    q = queries(sum(rows), hq, d, 62)
    shape, stride, G = c.shape(sd, hq), (c.max_context_len + 3) // 4 * 4, hq // hkv
    starts = np.concatenate([[0], np.cumsum(rows)])
    dev = lambda a: torch.tensor(np.asarray(a, np.int32), device="cuda")  # noqa: E731
    ws = sd.paged_weight_workspace_bytes(shape, max(rows))
    work = torch.full((ws + 65536,), 0xa5, dtype=torch.uint8, device="cuda")
    out = torch.full((len(lens), hkv, stride), -3.0, device="cuda")
    sd.paged_weight_accumulate(shape, q, dev(starts), len(q), max(rows), c.pool, c.scales, dev(c.table), dev(lens), d ** -0.5, 1.0, 0, None, out, stride, work, ws)
    assert bool((work[ws:] == 0xa5).all())
    for b, L in enumerate(lens):
        assert bool((out[b, :, L:] == -3).all())
        k = torch.from_numpy(c.k[b]).cuda()
        end = torch.arange(L - rows[b] + 1, L + 1, device="cuda").repeat_interleave(G)[:, None]
        seen = torch.arange(L, device="cuda")[None] < end
        for g in range(hkv if rows[b] else 0):
            y = q[starts[b]:starts[b + 1], g * G:(g + 1) * G].double().reshape(-1, d)
            x, size = d ** -0.5 * (y @ k[:, g].T.contiguous()), d ** -0.5 * (y.abs() @ k[:, g].abs().T.contiguous())
            p = torch.softmax(x.masked_fill(~seen, float("-inf")), 1)
            off = 3 * (d + 4) * size.masked_fill(~seen, 0).amax(1, keepdim=True) * U + (64 + x.masked_fill(~seen, 0).abs().amax(1, keepdim=True)) * 2 * U
            want, tol = p.sum(0), (p * off + 1e-37 * seen).sum(0)   # (derived in test_gpu_weight_scores)
            assert bool(((out[b, g, :L].double() - want).abs() <= tol + 80 * U * want).all()), (b, g)
