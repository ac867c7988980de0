"""fp8 pages whose scale is below zero: a value is its code times its page's scale, whatever the scale's sign, as in the attention."""
import numpy as np
import pytest

from tests.test_gpu_evict import Case, kept_of
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


@pytest.mark.parametrize("which", ["all", "some", "zeros"])
@pytest.mark.parametrize("lens,hkv,d,budget", [([300, 45, 20], 2, 128, 37), ([1000, 500], 3, 64, 129), ([90, 8], 2, 64, 200)])
def test_evict(sd, lens, hkv, d, budget, which):
    """A new tile takes the largest magnitude of its rows' scales (its last tile is partly filled), and a row's codes times it are the row's values."""
    import torch
    c = Case(sd, lens, hkv, d, "fp8", budget, 51)
    gen = torch.Generator().manual_seed(52)
    for s in c.scales:
        turned = torch.ones(s.shape, dtype=torch.bool) if which == "all" else torch.rand(s.shape, generator=gen) < 0.4
        s.copy_(torch.where(turned, -s.cpu() if which != "zeros" else torch.zeros(s.shape), s.cpu()))
    dev = lambda a: torch.tensor(np.asarray(a, np.int32), device="cuda")  # noqa: E731
    kept, new_lens = torch.empty(len(lens), hkv, budget, dtype=torch.int32, device="cuda"), dev(lens)
    before, scales_before = [p.clone() for p in c.pools], [s.clone() for s in c.scales]
    sd.kv_evict(c.shape, budget, 2, 10, torch.from_numpy(c.scores).cuda(), c.stride, *c.pools, *c.scales, dev(c.table), dev(lens), dev(c.new_table), kept, new_lens)
    for b, L in enumerate(lens):
        n = min(L, budget)
        for g in range(hkv):
            at = kept_of(c.scores[b, g], L, budget, 2, 10)
            assert np.array_equal(kept[b, g, :n].cpu().numpy(), at)
            page, slot = (torch.from_numpy(x.astype(np.int64)) for x in (c.table[b, at // 16], at % 16))
            for pool, scales, old_pool, old_scales in zip(c.pools, c.scales, before, scales_before):
                codes, old = old_pool.cpu()[page, g, slot], old_scales.cpu()[page, g]
                for j in range((n + 15) // 16):
                    rows = slice(16 * j, min(16 * j + 16, n))
                    top = old[rows].abs().max()
                    to = int(c.new_table[b, j])
                    assert scales[to, g].cpu() == top
                    ratio = old[rows] / top if top > 0 else torch.ones_like(old[rows])
                    again = (codes[rows].view(torch.float8_e4m3fn).float() * ratio[:, None]).to(torch.float8_e4m3fn).view(torch.uint8)
                    assert torch.equal(pool[to, g, :len(ratio)].cpu(), torch.where((ratio == 1)[:, None], codes[rows], again)), (b, g, j)
