"""Ranges of query rows that are longer than max_q_len: the rows within the bound stand at the positions that the whole range gives them."""
import numpy as np
import pytest

from tests.test_gpu_prefill import check as check_rows, gpu, make_bound, ref
from tests.test_gpu_weight_scores import U, Cache, check, queries, run
from tests.test_prefill_geometry import PLANS, context_bound, plan as route_of, program, stretch_case  # noqa: F401  (program is a fixture)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sd():
    import torch
    assert torch.cuda.is_available()
    import paper_2508_11553_amd as m
    m.load()
    return m


def weights_within(cache, q, starts, most, scale):
    """Scores and their tolerances (derived in test_gpu_weight_scores): row i of n stands at L - n + i, and those from `most` on add nothing."""
    out = []
    for b, L in enumerate(cache.lens):
        rows, n, hkv = q[starts[b]:starts[b + 1]], starts[b + 1] - starts[b], cache.hkv
        got, tol = np.zeros((hkv, L)), np.zeros((hkv, L))
        for i in range(min(n, most)):
            end = L - n + i + 1
            if end <= 0:
                continue
            for h in range(q.shape[1]):
                g = h // (q.shape[1] // hkv)
                k = cache.k[b][:end, g]
                x = scale * (k @ rows[i, h])
                size = abs(scale) * (np.abs(k) @ np.abs(rows[i, h])).max()
                p = np.exp(x - x.max())
                p /= p.sum()
                got[g, :end] += p
                tol[g, :end] += p * (3 * (cache.d + 4) * size * U + (64 + np.abs(x).max()) * 2 * U) + 1e-37
        out.append((got, tol + got * 80 * U))
    return out


@pytest.mark.parametrize("lens,rows,most,hq,hkv,d,kv", [
    ([300, 70, 4], [9, 2, 7], 2, 8, 2, 64, "bf16"),             # one kernel
    ([6000, 40], [9, 5], 3, 4, 1, 128, "bf16"),                 # products kept between two launches
    ([5000, 700], [5, 40], 1, 4, 1, 64, "fp8"),
    ([700, 300, 45], [90, 41, 50], 40, 8, 2, 64, "bf16"),       # rows held while K streams; the last one begins before its first token
    ([600, 500], [150, 100], 100, 8, 1, 128, "fp8"),            # several workgroups' rows
    ([90 + b % 7 for b in range(66)], [30 - b % 12 for b in range(66)], 20, 4, 1, 64, "bf16"),   # more sequences than a wave has lanes
])
def test_weights(sd, lens, rows, most, hq, hkv, d, kv):
    c = Cache(lens, hkv, d, kv, sum(rows))
    starts = np.concatenate([[0], np.cumsum(rows)])
    q = queries(int(starts[-1]), hq, d, 2, 1.5)
    got = run(sd, c, hq, q, starts, d ** -0.5, 1.0, 0, None, max_q_len=most)
    check(got, weights_within(c, q.double().cpu().numpy(), starts, most, d ** -0.5), lens)


@pytest.mark.parametrize("kv,d,plan", PLANS)
def test_attention(sd, program, kv, d, plan):
    """Every kernel of the causal pass, at its own size: what it writes are the rows within the bound, as the whole ranges have them, and no others."""
    lens, nq, Hq, Hkv = stretch_case(plan, d)
    bound, most = context_bound(plan[0], d), max(nq)
    more = list(nq)
    more[nq.index(most)] += 23   # one is longer than the bound
    assert route_of(program, lens, more, Hq, Hkv, d, kv, bound, most) == plan
    wl, q, q_start = make_bound(lens, more, Hq, Hkv, d, kv, bound, seed=900 + d)
    got, want = gpu(wl, q, q_start, max_q=most), ref(wl, q, q_start)
    within = np.concatenate([np.arange(n) < most for n in more])
    assert (~within).sum() == 23
    assert np.isnan(got[~within]).all()
    check_rows(got[within], want[within], kv)
    # a range that leaves the rows has none, though those within the bound lie inside
    few = nq[-1]
    outside = q_start.copy()
    outside[-1] = len(q) + 5
    got, inner = gpu(wl, q, outside, max_q=few), slice(0, q_start[-2])
    assert np.isnan(got[q_start[-2]:]).all()
    within = np.concatenate([np.arange(n) < few for n in more])[inner]
    check_rows(got[inner][within], want[inner][within], kv)
