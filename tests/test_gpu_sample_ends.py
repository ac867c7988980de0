"""Draws that end with the last of all kept tokens, where a row with limits is gone over because its logits are nearly even."""
import numpy as np
import pytest

from tests.test_gpu_sample import Batch, check, sd  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", [(40, 20011), (40, 50000), (260, 4099)])
@pytest.mark.parametrize("middle", [0.0, 100.0, 1000.0])
def test_a_uniform_number_of_one_takes_the_last_kept_token(sd, kind, rows, vocab, middle):  # noqa: F811
    """Thousands are kept by top_p, of which min_p takes the lightest (or none); few rows and many, logits near 0 and far from it (whose positions are made another
    way); the largest number below one and what counts as it.  Every row is written."""
    rng = np.random.default_rng(vocab)
    x = (middle + rng.normal(0, 0.7, (rows, vocab))).astype(np.float32)
    if middle and kind == "bf16":
        x = (middle + np.round(rng.normal(0, 2, (rows, vocab))) * (0.5 if middle == 100.0 else 4.0)).astype(np.float32)   # (representable, and not all alike)
    b = Batch(sd, x, kind)
    t = 0.8 if middle < 1000 or kind == "f32" else 6.0
    u = np.ones(rows, np.float32)
    u[1::4] = 1 - 2.0 ** -24
    u[2::4] = 2.0
    p = 0.85 + 0.14 * rng.random(rows)
    for min_p in (None, [1e-9] * rows, [0.004] * rows, [0.03] * rows):
        some = slice(0, rows) if rows < 100 else slice(0, 24)
        got = b.draw(u, temperature=[t] * rows, top_p=p, min_p=min_p)
        assert (got[0] >= 0).all() and (got[1] <= 0).all() and (got[2] <= 0).all()
        part = Batch(sd, x[some], kind)
        same = check(part, u[some], temperature=[t] * len(u[some]), top_p=p[some], min_p=None if min_p is None else min_p[some])
        assert all(np.array_equal(y[some], z) for y, z in zip(got, same))


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [70, 2048, 6001])
def test_a_uniform_number_of_one_without_limits_takes_the_last_token(sd, kind, vocab):  # noqa: F811
    """Thousands of rows whose every token has weight: the kernel that sums a stretch and those that walk it come to the same sum, whatever limits are given that
    do not limit, for few rows and for many."""
    rng = np.random.default_rng(vocab)
    rows = 20000 if vocab < 5000 else 6000
    x = (rng.normal(0, 1, (rows, vocab)) + rng.normal(0, 10, (rows, 1))).astype(np.float32)
    t = rng.uniform(0.5, 1.5, rows)
    u = np.ones(rows, np.float32)
    b = Batch(sd, x, kind)
    want = b.draw(u, temperature=t)
    assert (want[0] == vocab - 1).all(), np.flatnonzero(want[0] != vocab - 1)[:5]
    many = b.draw(u, temperature=t, top_p=np.ones(rows))
    assert all(np.array_equal(y, z) for y, z in zip(many, want))
    for first in range(0, rows, rows // 8):
        at = slice(first, first + 256)
        few = Batch(sd, x[at], kind).draw(u[at], temperature=t[at], top_p=np.ones(256))
        assert all(np.array_equal(y, z[at]) for y, z in zip(few, want))
