"""Temperatures at the lower end of fp32, where log2(e) / temperature passes its range."""
import numpy as np
import pytest

from tests.test_gpu_sample import Batch, check, sd  # noqa: F401

pytestmark = pytest.mark.gpu

COLD = [4.3e-39, 4.2e-39, 1e-39, 1e-40, 1e-42, 1e-45]


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [5003, 30001])
@pytest.mark.parametrize("times", [2, 50])
def test_limits_among_thousands_of_equal_logits(sd, kind, vocab, times):  # noqa: F811
    """The largest logit is that of half the row: top_p keeps its share of them, the first by index."""
    rng = np.random.default_rng(vocab)
    x = np.where(rng.random((len(COLD), vocab)) < 0.5, 1.5, rng.normal(0, 0.3, (len(COLD), vocab)))
    rows = len(COLD) * times
    b, few = Batch(sd, np.tile(x, (times, 1)), kind), Batch(sd, x, kind)
    u = rng.random(rows).astype(np.float32)
    for use in (dict(top_p=[0.5] * rows), dict(top_p=[0.01] * rows), dict(top_p=[0.999] * rows, min_p=[0.1] * rows), dict(top_k=[2100] * rows), dict(top_k=[2100] * rows, top_p=[0.3] * rows)):
        t = COLD * times
        got = b.draw(u, temperature=t, **use)
        want = check(few, u[:len(COLD)], temperature=COLD, **{k: v[:len(COLD)] for k, v in use.items()})
        assert all(np.array_equal(y[:len(COLD)], z) for y, z in zip(got, want))
        first = [np.flatnonzero(few.x[r] == 1.5) for r in range(len(COLD))]
        for r in range(rows):   # all weigh alike: the draw is a count
            mine = first[r % len(COLD)]
            n = min(len(mine), use["top_k"][r]) if "top_k" in use else len(mine)
            n = int(np.ceil(np.float64(np.float32(use["top_p"][r])) * n)) if "top_p" in use else n
            assert got[0][r] == mine[int(np.float64(u[r]) * n)], (r, use)


@pytest.mark.parametrize("kind,unit", [("bf16", 2.0 ** -133), ("f32", 2.0 ** -149), ("f32", 2.0 ** -140)])
def test_logits_as_small_as_their_temperature(sd, kind, unit):  # noqa: F811
    """Steps of the smallest numbers of the type, a temperature of some of them: thousands of weights that differ."""
    rng = np.random.default_rng(1)
    rows, vocab = 6, 6007
    x = (rng.integers(0, 40, (rows, vocab)) * unit).astype(np.float32)
    b = Batch(sd, x, kind)
    t = [max(n * unit, 1e-45) for n in (1, 3, 10, 30, 100, 300)]
    for use in (dict(top_p=[0.9] * rows), dict(top_p=[0.999] * rows, min_p=[0.05] * rows), dict(min_p=[0.3] * rows), dict(top_k=[3000] * rows), dict()):
        check(b, rng.random(rows).astype(np.float32), temperature=t, **use)
