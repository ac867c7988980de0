"""Every row's weights sum to one, whatever the size of its scores: the scores of a KV head to its rows.

Tolerance, 256 x 2^-24 a row: what a score is off by does not enter, for both passes over K make the same products.  A weight 2^a of a sum carries the
rounding of its exponent, 2^-24 |a| ln 2, in each pass (up to 16 more in the first, whose reference lags), and the sum over t of p |a| is at most log2 L <= 10; two
exponentials of 2^-23, the reference's moves and the division add less than 40 x 2^-24; the additions of at most 100 tokens of a lane, its wave's and the
rows' as many roundings as they are.  A reference rounded in proportion to a score of 10^4 to 10^5 would be off by thousands.
"""
import numpy as np
import pytest

from tests.test_gpu_weight_scores import U, Cache, queries, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sd():
    import torch
    assert torch.cuda.is_available()
    import paper_2508_11553_amd as m
    m.load()
    return m


@pytest.mark.parametrize("kind", ["offset", "wide"])
@pytest.mark.parametrize("lens,rows,hq,hkv,d,kv", [
    ([300, 129, 70, 64], [20, 5, 33, 64], 8, 2, 64, "bf16"),
    ([290, 17, 200], [16, 16, 1], 16, 2, 128, "bf16"),
    ([257, 300], [40, 9], 4, 1, 128, "fp8"),
    ([310], [310], 8, 1, 64, "fp8"),                                          # several workgroups' rows, the whole sequence a window
    ([100 + b for b in range(66)], [6 - b % 5 for b in range(66)], 8, 2, 128, "bf16"),   # more sequences than a wave has lanes
    ([300, 40], [1, 1], 8, 2, 64, "bf16"),                                    # (one pass, products kept)
])
def test_weights_sum_to_the_rows(sd, lens, rows, hq, hkv, d, kv, kind):
    """Scores that share a large offset (many tokens of like weight), and scores far apart (one token has all)."""
    c = Cache(lens, hkv, d, kv, 31, gain=1.0 if kind == "offset" else 30.0)
    q = queries(sum(rows), hq, d, 32, 1.0 if kind == "offset" else 300.0)
    if kind == "offset":
        q[..., 0] = 1024.0
        for b, n in enumerate(lens):
            for t in range(n):
                c.pool[int(c.table[b, t // 16]), :, t % 16, 0] = 512.0 if kv == "bf16" else 0x7e   # (fp8: 448 times the page's scale, alike or far apart)
    starts = np.concatenate([[0], np.cumsum(rows)])
    got = run(sd, c, hq, q, starts, d ** -0.5, 1.0, 0).double().cpu().numpy()
    for b, (n, r) in enumerate(zip(lens, rows)):
        count = r * hq // hkv
        total = got[b, :, :n].sum(-1)
        assert (np.abs(total - count) <= 256 * U * count).all(), (b, (total - count) / count / U)
