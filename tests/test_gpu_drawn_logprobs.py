"""The log probability that comes with a drawn token is the one that token_logprobs gives for it, but for what the header excepts."""
import numpy as np
import pytest

from tests import logits_plain as plain
from tests.test_gpu_sample import Batch, peaked, sd  # noqa: F401
from tests.test_gpu_token_logprobs import STEP, forward, log_sum_error

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", [(9, 131075), (200, 5003)])
def test_the_same_where_nothing_is_excepted(sd, kind, rows, vocab):  # noqa: F811
    """Cut rows and whole ones; masked logits, the largest logit taken, temperatures near both ends."""
    rng = np.random.default_rng(rows)
    x = peaked(rng, rows, vocab)
    x[:, 1::3] = -np.inf
    b = Batch(sd, x, kind)
    t = rng.uniform(0.5, 1.2, rows)
    t[:6] = 0.0, -1.0, np.nan, 2.0 ** -126, 2.0 ** 125, 1e-30
    tokens, lp, _ = b.draw(rng.random(rows).astype(np.float32), temperature=t, top_p=[0.95] * rows)
    got = forward(b, tokens, t)[0]
    for r in range(min(rows, 40)):
        with np.errstate(over="ignore", invalid="ignore"):
            want, _, z1, _, s2 = plain.logprobs(b.x[r], tokens[r], float(np.float32(t[r])) if t[r] > 0 else 1.0)
        assert abs(got[r] - lp[r]) <= log_sum_error(vocab, z1, s2) + STEP * (6 * (abs(want) + s2)) + 1e-9, r


def test_the_exceptions(sd):  # noqa: F811
    vocab = 1000
    x = np.full((6, vocab), -np.inf)
    x[0, :8], x[0, 3] = 0.0, np.nan                     # NaN: passed over; there the row is not a number
    x[1, :8], x[1, [2, 5]] = 0.0, np.inf                # two of +inf share all weight
    x[2, :2] = 0.0, 2.0 ** -140                         # a temperature below 2^-126: here as it is, there 2^-126
    x[3, :2] = 0.0, 3e38                                # one above 2^125
    x[4, :2] = -3e38, 3e38                              # further apart than fp32 reaches
    x[5, :2] = 0.0, 1.0                                 # (nothing excepted)
    t = [1.0, 1.0, 2.0 ** -140, 3e38, 1e38, 1.0]
    b = Batch(sd, x, "f32")
    tokens, lp, _ = b.draw([0.99] * 6, temperature=t)
    scored = forward(b, tokens, t)[0]
    assert list(tokens) == [7, 5, 1, 1, 1, 1]
    near = lambda got, want: abs(got - want) <= 8 * STEP  # noqa: E731
    one = -np.log1p(np.exp(-1.0))
    assert near(lp[0], -np.log(7)) and near(lp[1], -np.log(2)) and np.isnan(scored[:2]).all()
    assert near(lp[2], one) and near(scored[2], -np.log1p(np.exp(-2.0 ** -14)))
    assert near(lp[3], one) and near(scored[3], -np.log1p(np.exp(-float(np.float32(3e38)) / 2.0 ** 125)))
    assert near(lp[4], -np.log1p(np.exp(-6.0))) and scored[4] == 0
    assert near(lp[5], one) and near(scored[5], one)
