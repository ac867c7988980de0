"""fp8 pages whose scale is below zero: a value is its code times its page's scale, whatever the scale's sign, as in the attention."""
import numpy as np
import pytest

from tests.test_gpu_weight_scores import Cache, check, expected, queries, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sd():
    import torch
    assert torch.cuda.is_available()
    import paper_2508_11553_amd as m
    m.load()
    return m


@pytest.mark.parametrize("which", ["all", "some"])
@pytest.mark.parametrize("lens,rows,hq,hkv,d", [
    ([300, 40, 1], None, 8, 2, 64),                          # one kernel
    ([9000, 100], None, 4, 1, 128),                          # products kept between two launches
    ([700, 300], [20, 33], 8, 2, 64),                        # rows held while K streams
    ([640, 500], [64, 100], 8, 1, 128),
    ([400 + b for b in range(66)], [5 + b % 3 for b in range(66)], 4, 1, 128),
])
def test_weights(sd, lens, rows, hq, hkv, d, which):
    c = Cache(lens, hkv, d, "fp8", 41, gain=4.0)   # scores of some hundreds: relative to the smallest one of a page the largest is infinite
    rng = np.random.default_rng(42)
    for b, n in enumerate(lens):
        for j in range((n + 15) // 16):
            turned = np.ones(hkv, bool) if which == "all" else rng.random(hkv) < 0.3
            c.scales[int(c.table[b, j]), np.flatnonzero(turned).tolist()] *= -1
            c.k[b][16 * j:16 * j + 16, turned] *= -1
    starts = np.arange(len(lens) + 1) if rows is None else np.concatenate([[0], np.cumsum(rows)])
    q = queries(int(starts[-1]), hq, d, 43, 30.0)
    got = run(sd, c, hq, q, None if rows is None else starts, d ** -0.5, 1.0, 0)
    check(got, expected(c, q.double().cpu().numpy(), starts, lens, d ** -0.5, 1.0, 0, None), lens)
