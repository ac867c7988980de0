"""Rows that are cut into parts (few rows of many logits, joined by a second kernel): padding, rows and whole parts with nothing, masked targets, what is not a number."""
import numpy as np
import pytest

from tests import logits_plain as plain
from tests.test_gpu_sample import Batch, sd  # noqa: F401
from tests.test_gpu_token_logprobs import backward, check_forward, check_gradient, forward

pytestmark = pytest.mark.gpu

CUT = [("bf16", 131075), ("f32", 70001), ("f32", 49153)]   # the last one just past the rule for 4 logits a vector


def without_the_lightest(x, targets, t, g, h, got):
    """`got` with the 64-bit form's values where p is below 2^-126, fp32's smallest number of full precision: the exponential gives 0 there, which leaves
    out at most 2^-126 |g + h (log p + H)| / T of the gradient."""
    got = got.copy()
    for r, row in enumerate(x):
        z = row.astype(np.float64) / t
        z = z - z.max()
        logp = z - np.log(np.exp(z).sum())
        light = (logp < -125.9 * np.log(2)) & (np.arange(len(row)) != targets[r])
        want = plain.gradient(row, targets[r], t, float(np.float32(g[r])), float(np.float32(h[r])))
        H = -np.where(np.exp(logp) > 0, np.exp(logp) * np.where(np.isfinite(logp), logp, 0), 0).sum()
        size = abs(g[r]) + abs(h[r]) * (np.where(np.isfinite(logp), abs(logp), 0) + H)
        assert (abs(got[r] - want)[light] <= 1.01 * (2.0 ** -125.9 * size / t)[light]).all()
        got[r][light] = want[light]
    return got


@pytest.mark.parametrize("kind,vocab", CUT)
@pytest.mark.parametrize("temperature", [None, 0.7])
def test_padding_masked_and_extreme_rows(sd, kind, vocab, temperature):  # noqa: F811
    rng = np.random.default_rng(vocab)
    rows = 13
    x = rng.normal(0, 2, (rows, vocab))
    x[0] = np.nan                                   # padding: never read
    x[1, 1::2] = -np.inf
    x[2] = -np.inf                                  # nothing at all
    x[3], x[3, vocab - 1] = -np.inf, 2.0            # all in the last part, or in the first one
    x[4], x[4, 0] = -np.inf, 2.0
    x[5], x[5, 9] = np.finfo(np.float32).min, 0.0
    x[6, vocab // 2] = 3.0e38
    x[7] = 1.5
    x[8, 3] = -np.inf                               # a masked target
    x[9, vocab // 3:] = -np.inf
    x[10, :2 * vocab // 3] = -np.inf
    x[11, vocab - 2] = 60.0
    x[12] = np.nan
    b = Batch(sd, x, kind)
    targets = np.array([-1, 4, 5, vocab - 1, 0, 9, vocab // 2, 100, 3, 7, vocab - 1, 1, vocab])
    t = None if temperature is None else [temperature] * rows
    got = forward(b, targets, t)
    assert got[0][0] == got[1][0] == got[0][12] == got[1][12] == 0
    assert got[0][2] == -np.inf and got[1][2] == 0 and got[0][8] == -np.inf
    assert all(got[0][r] == got[1][r] == 0 for r in (3, 4, 5, 6))
    keep = [1, 3, 4, 5, 6, 7, 8, 9, 10, 11]
    part = Batch(sd, x[keep], kind)
    mine = None if t is None else [temperature] * len(keep)
    with np.errstate(invalid="ignore"):
        check_forward(part, targets[keep], mine, (got[0][keep], got[1][keep]))
        g, h = rng.normal(0, 1, rows), rng.normal(0, 1, rows)
        d = backward(b, g, h)
        assert not d[0].any() and not d[2].any() and not d[12].any()
        d = without_the_lightest(part.x, targets[keep], float(np.float32(temperature or 1.0)), g[keep], h[keep], d[keep])
        check_gradient(part, targets[keep], mine, g[keep], h[keep], d)


@pytest.mark.parametrize("kind,vocab", CUT)
@pytest.mark.parametrize("bad", [np.nan, np.inf])
@pytest.mark.parametrize("where", [0, 0.5, 1])
def test_what_is_not_a_number_shows(sd, kind, vocab, bad, where):  # noqa: F811
    """In the target's part or in another one, with finite logits or nothing else in it."""
    at = int(where * (vocab - 1))
    x = np.zeros((4, vocab))
    x[1, at] = bad
    x[2], x[2, at], x[2, 5] = -np.inf, bad, 0.0
    b = Batch(sd, x, kind)
    lp, H = forward(b, [5, 5, 5, 5])
    assert np.isnan(lp[1:3]).all() and np.isnan(H[1:3]).all() and np.isfinite(lp[[0, 3]]).all() and np.isfinite(H[[0, 3]]).all()
    d = backward(b, [1.0] * 4, [1.0] * 4)
    assert all(np.isnan(d[r]).any() for r in (1, 2)) and np.isfinite(d[[0, 3]]).all()


@pytest.mark.parametrize("rows", [1, 2, 127, 128, 129])
def test_as_many_parts_as_the_workspace_holds(sd, rows):  # noqa: F811
    """From one row in as many parts as its vectors make to the most rows that are cut, and one more."""
    rng = np.random.default_rng(rows)
    vocab = 98313
    b = Batch(sd, rng.normal(0, 2, (rows, vocab)), "bf16")
    targets = rng.integers(0, vocab, rows)
    check = sorted({0, rows // 2, rows - 1})
    got = forward(b, targets)
    part = Batch(sd, b.x[check], "bf16")
    check_forward(part, targets[check], None, (got[0][check], got[1][check]))
