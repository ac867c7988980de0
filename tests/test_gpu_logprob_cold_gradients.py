"""The gradient of log probabilities at temperatures so low that a gradient over the temperature passes the range of fp32: what has no weight stays 0."""
import numpy as np
import pytest

from tests.test_gpu_sample import Batch, sd  # noqa: F401
from tests.test_gpu_token_logprobs import backward, forward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [5, 1003, 131075])
def test_gradients_past_the_range(sd, kind, vocab):  # noqa: F811
    """p is 1 at the largest logit and 0 elsewhere: a target there leaves no gradient at all, another one g / T at itself and as much less at the largest, infinite where
    that passes the range (the temperature is held to 2^-126)."""
    rng = np.random.default_rng(vocab)
    t = np.array([1e-45, 2.0 ** -126, 1e-38, 1e-45, 1e-38, 1e-38, 1e-30, 1.0], np.float32)
    rows = len(t)
    x = rng.normal(0, 1, (rows, vocab))
    x[:, 2], x[:, 3], x[5] = 9.0, -np.inf, 0.25
    b = Batch(sd, x, kind)
    targets = np.array([2, 2, 2, 4, 4, 0, 2, 2])
    g, h = np.array([8, 100, -3e38, 8, 1e-5, 0.0, 3e38, 1.0], np.float32), np.array([0, -5, 1e30, 7, 1e3, 0.0, 3e38, 0.1], np.float32)
    lp, H = forward(b, targets, t)
    assert (lp[:3] == 0).all() and (H[:5] == 0).all()
    for d in (backward(b, g, h), backward(b, g, None)):
        assert not np.isnan(d).any()
        assert not d[[0, 1, 2, 5, 6]].any() and not d[:, 3].any()
        others = [i for i in range(vocab) if i not in (2, 4)]
        assert not d[3:5, others].any()
        assert d[3, 4] == np.inf and d[3, 2] == -np.inf
        want = float(g[4]) / max(float(t[4]), 2.0 ** -126)
        # 1 / T from a rounded log2(e) / T and ln 2, the product and the type's rounding: half a step each
        assert abs(d[4, 4] / want - 1) <= 4 * 2.0 ** -24 + 2.0 ** -8 * (kind == "bf16") and d[4, 2] == -d[4, 4]
