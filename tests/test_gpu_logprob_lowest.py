"""Targets whose logit is the type's lowest number, as masks make them: their log probability is finite where fp32 holds it."""
import numpy as np
import pytest

from tests import logits_plain as plain
from tests.test_gpu_sample import Batch, sd  # noqa: F401
from tests.test_gpu_token_logprobs import STEP, backward, forward, log_sum_error

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,lowest", [("bf16", -float.fromhex("0x1.fep127")), ("f32", -float.fromhex("0x1.fffffep127"))])
@pytest.mark.parametrize("rows,vocab", [(6, 1003), (6, 131075), (600, 70)])
def test_masked_targets(sd, kind, lowest, rows, vocab):  # noqa: F811
    """In the uncut form, in parts, and with many rows.  A result is off by the sum's error, its logarithm's rounding and its own."""
    rng = np.random.default_rng(vocab)
    x = rng.normal(0, 2, (rows, vocab))
    x[:, 1::2] = lowest
    x[:, 3] = lowest / 4
    b = Batch(sd, x, kind)
    targets = np.where(np.arange(rows) % 2, 1, 3)
    for t in (None, 1.0, 0.7, 1.5, 1e30, 3e37):
        got = forward(b, targets, None if t is None else [t] * rows)
        for r in range(min(rows, 8)):
            with np.errstate(over="ignore"):
                want, _, z1, _, s2 = plain.logprobs(b.x[r], targets[r], float(np.float32(t or 1.0)))
            if abs(want) > float.fromhex("0x1.ffffffp127"):
                assert got[0][r] == -np.inf, (r, t, got[0][r], want)
            else:
                assert np.isfinite(got[0][r]) and abs(got[0][r] - want) <= log_sum_error(vocab, z1 if z1 < 1e3 else 0, s2) + STEP * 2 * (abs(want) + s2), (r, t, got[0][r], want)
    forward(b, targets, None)
    g = rng.normal(0, 1, rows)
    d = backward(b, g, np.ones(rows))
    assert np.isfinite(d).all()
    assert np.array_equal(d[np.arange(rows), targets], plain.bf16_values(plain.bf16_bits(g)) if kind == "bf16" else g.astype(np.float32))   # p is 0: the target's is g, the other masked ones' 0
    d[np.arange(rows), targets] = 0
    assert not d[:, 1::2].any()
