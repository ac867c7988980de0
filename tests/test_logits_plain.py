"""The plain forms that the kernels are compared with, against brute force and closed forms (CPU only)."""
import itertools

import numpy as np
import pytest

from tests import logits_plain as plain


@pytest.mark.parametrize("seed", range(6))
def test_shares_of_a_uniform_grid_are_the_probabilities(seed):
    """Over an even grid of uniform numbers every token comes as often as the truncated distribution says, to one step of the grid."""
    rng = np.random.default_rng(seed)
    vocab, grid = 12, 4000
    x = np.round(rng.normal(0, 2, vocab), 1).astype(np.float32)
    k, p, m = [(0, 1.0, 0.0), (5, 1.0, 0.0), (0, 0.7, 0.0), (0, 1.0, 0.2), (6, 0.8, 0.05), (1, 0.5, 0.0)][seed]
    t = 0.7
    w = np.exp((x.astype(np.float64) - x.max()) / t)
    order = sorted(range(vocab), key=lambda i: (-x[i], i))
    keep = order[:k] if k else order
    mass = np.cumsum([w[i] for i in keep])
    keep = [i for j, i in enumerate(keep) if mass[j] - w[i] < p * mass[-1]] if p < 1 else keep
    keep = [i for i in keep if w[i] >= m]
    want = np.zeros(vocab)
    want[keep] = w[keep] / w[keep].sum()
    got = np.zeros(vocab)
    for j in range(grid):
        token, lp, dlp = plain.sample(x, t, k, p, m, j / grid)
        got[token] += 1 / grid
        assert abs(lp - np.log(w[token] / w.sum())) < 1e-11 and abs(dlp - np.log(want[token])) < 1e-11
    assert abs(got - want).max() <= 1.0001 / grid


def test_rows_at_the_edges():
    inf = np.inf
    assert plain.sample(np.array([-inf, -inf]))[0] == -1
    assert plain.sample(np.array([-inf, 3.0, np.nan, -inf]), uniform=0.99)[:2] == (1, 0.0)
    assert plain.sample(np.array([inf, 0.0, inf]), uniform=0.6)[0] == 2
    assert plain.sample(np.array([1.0, 2.0, 2.0]), temperature=0.0)[0] == 1
    assert plain.sample(np.zeros(8), uniform=3 / 8)[0] == 3 and plain.sample(np.zeros(8), uniform=1.0)[0] == 7
    assert plain.sample(np.array([0.0, 1.0, 1.0]), top_k=1, uniform=0.9)[0] == 1
    assert plain.sample(np.array([0.0, 1.0, 1.0]), top_p=0.0, uniform=0.9)[0] == 1
    assert plain.sample(np.array([0.0, 1.0, 1.0]), min_p=1.0, uniform=0.9)[0] == 2


def test_gradient_is_that_of_the_log_probability_and_entropy():
    rng = np.random.default_rng(1)
    x, target, t, g, h = rng.normal(0, 2, 9), 4, 0.8, 0.7, -0.3
    d = plain.gradient(x, target, t, g, h)
    for j in range(9):
        e = np.zeros(9)
        e[j] = 1e-5
        f = [g * lp + h * H for lp, H, *_ in (plain.logprobs(x + e, target, t), plain.logprobs(x - e, target, t))]
        assert abs((f[0] - f[1]) / 2e-5 - d[j]) < 1e-9


def test_plan_keeps_every_page_once():
    rng = np.random.default_rng(2)
    for _ in range(200):
        B, blocks, pages = int(rng.integers(1, 9)), 6, 30
        order = list(rng.permutation(pages))
        lens = [int(rng.integers(0, 40)) for _ in range(B)]
        table = []
        for n in lens:
            need = (n + 15) // 16
            if need > len(order):
                need = 0
            row, order = order[:need], order[need:]
            table.append(row + [-1] * (blocks - need))
        lens = [n if table[b][0] >= 0 or n == 0 else 0 for b, n in enumerate(lens)]
        new = [int(x) for x in rng.integers(-1, 60, B)]
        free = list(order)
        got = plain.plan(new, [0] * B, lens, [0] * B, free, table, int(rng.integers(0, 200)), 16 * blocks)
        held = list(itertools.chain(*(table[b][:(n + 15) // 16] for b, n in enumerate(got["lens_out"]))))
        assert sorted(held + free) == sorted(range(pages))
        assert all(g in (0, n) for g, n in zip(got["granted"], new) if n > 0)
