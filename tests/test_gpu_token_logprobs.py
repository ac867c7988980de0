"""token_logprobs and its gradient against the plain form in 64 bits and against differences."""
import numpy as np
import pytest

from tests import logits_plain as plain
from tests.test_gpu_sample import Batch, peaked, sd  # noqa: F401

pytestmark = pytest.mark.gpu

STEP = 2.0 ** -24   # half a step of fp32


def forward(b, targets, temperature=None, entropy=True, stats=True):
    import torch
    sd = b.sd  # noqa: F811
    dev = lambda a, t: None if a is None else torch.tensor(np.asarray(a, t), device="cuda")  # noqa: E731
    b.targets, b.temperature = dev(targets, np.int32), dev(temperature, np.float32)
    b.lp, b.H, b.stats = (torch.full(s, 7.0, device="cuda") for s in ((b.rows,), (b.rows,), (b.rows, 2)))
    ws = sd.token_logprobs_workspace_bytes(b.desc)
    work = torch.full((ws,), 255, dtype=torch.uint8, device="cuda")
    sd.token_logprobs(b.desc, b.flat, b.targets, b.temperature, b.lp, b.H if entropy else None, b.stats if stats else None, work, ws)
    return b.lp.cpu().numpy(), b.H.cpu().numpy()


def backward(b, g, h, out=None):
    import torch
    g, h = torch.tensor(g, dtype=torch.float32, device="cuda"), None if h is None else torch.tensor(h, dtype=torch.float32, device="cuda")
    out = torch.full_like(b.flat, 3) if out is None else out
    b.sd.token_logprobs_backward(b.desc, b.flat, b.targets, b.temperature, b.stats, None if h is None else b.H, g, h, out)
    b.out = out
    flat = out.cpu().numpy()
    flat = plain.bf16_values(flat.view(np.uint16)) if flat.dtype == np.int16 else flat
    stride = b.desc.stride or b.vocab
    return np.stack([flat[r * stride:r * stride + b.vocab] for r in range(b.rows)])


def log_sum_error(vocab, z1, s2):
    """Relative error of a row's sum: every term has a rounded difference, factor and product (3 half steps of |z|) and an exponential of 1 step, the
    rescaled sums as much again; a lane adds at most vocab / 512 + 8 terms, then 10 times two halves."""
    return STEP * (2 * 3 * np.log(2) * (z1 + 1) + 4 + vocab / 512 + 8 + 3 * 10)


def check_forward(b, targets, temperature, got):
    for r in range(b.rows):
        t = np.float32(1.0 if temperature is None else temperature[r])
        lp, H, z1, z2, s2 = plain.logprobs(b.x[r], targets[r], float(t))
        err = log_sum_error(b.vocab, z1, s2)
        if np.isfinite(lp):
            assert abs(got[0][r] - lp) <= err + STEP * (4 * (abs(lp) + s2) + 2 * abs(lp)) + 1e-30, (r, got[0][r], lp)
        else:
            assert got[0][r] == lp
        # H = log S - T / S: T's terms have z's rounding besides
        assert abs(got[1][r] - H) <= err * (2 + z1) + STEP * (6 * np.log(2) * (z1 + z2) + 4 * s2 + 2 * H), (r, got[1][r], H)


def check_gradient(b, targets, temperature, g, h, got):
    half = 2.0 ** -8 if b.desc.dtype == b.sd.SD_BF16 else STEP
    for r in range(b.rows):
        t = float(np.float32(1.0 if temperature is None else temperature[r]))
        gr, hr = float(np.float32(g[r])), 0.0 if h is None else float(np.float32(h[r]))
        want = plain.gradient(b.x[r], targets[r], t, gr, hr)
        _, H, z1, z2, s2 = plain.logprobs(b.x[r], targets[r], t)
        x = b.x[r].astype(np.float64)
        z = np.where(np.isfinite(x), (x - x.max()) / t, -1e4) / np.log(2)
        p = np.exp2(z - s2)
        # p: z's three half steps, the sum's logarithm (its error, its rounding), one subtraction, an exponential of 1 step
        log_p = log_sum_error(b.vocab, z1, s2) + STEP * np.log(2) * (3 * abs(z) + 3 * s2 + abs(z - s2))
        H_err = log_sum_error(b.vocab, z1, s2) * (2 + z1) + STEP * (6 * (z1 + z2) + 4 * s2 + 2 * H)
        size = abs(gr) + abs(hr) * (abs(z - s2) * np.log(2) + H)
        err = p / t * (size * (log_p + 8 * STEP) + abs(hr) * (log_p + H_err))
        err[targets[r]] += 4 * STEP * abs(gr) / t
        bad = abs(got[r] - want) > half * abs(want) + err * (1 + half) + 1e-38
        assert not bad.any(), (r, np.nonzero(bad)[0][:5], got[r][bad][:5], want[bad][:5])


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [1, 2, 7, 8, 9, 63, 65, 511, 2048, 4099, 33001, 131072])
def test_rows(sd, kind, vocab):  # noqa: F811
    rng = np.random.default_rng(vocab)
    rows = 5
    b = Batch(sd, peaked(rng, rows, vocab) if vocab % 2 else rng.normal(0, 1, (rows, vocab)), kind, gap=[0, 3][vocab % 3 == 0])
    targets = rng.integers(0, vocab, rows)
    targets[0], targets[1] = 0, vocab - 1
    for temperature in (None, rng.uniform(0.4, 1.5, rows)):
        check_forward(b, targets, temperature, forward(b, targets, temperature))
        g, h = rng.normal(0, 1, rows), rng.normal(0, 0.1, rows)
        check_gradient(b, targets, temperature, g, h, backward(b, g, h))
        check_gradient(b, targets, temperature, g, None, backward(b, g, None))


@pytest.mark.parametrize("rows", [1, 2, 17, 200, 1025])
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_batches(sd, kind, rows):  # noqa: F811
    rng = np.random.default_rng(rows)
    vocab = 70001 if rows < 20 else 1111
    b = Batch(sd, peaked(rng, rows, vocab), kind)
    targets = np.where(rng.random(rows) < 0.5, b.x.argmax(1), rng.integers(0, vocab, rows))
    check_forward(b, targets, None, forward(b, targets))
    g, h = rng.normal(0, 1, rows) / rows, np.full(rows, -0.01 / rows)
    check_gradient(b, targets, None, g, h, backward(b, g, h))


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_padding_masked_and_extreme_rows(sd, kind):  # noqa: F811
    rng = np.random.default_rng(3)
    rows, vocab = 9, 4001
    x = rng.normal(0, 2, (rows, vocab))
    x[0] = np.nan                                # padding: never read
    x[1, 1::2] = -np.inf
    x[2] = -np.inf                               # nothing at all
    x[3], x[3, 7] = -np.inf, 2.0
    x[4], x[4, 9] = np.finfo(np.float32).min, 0.0
    x[5, 11] = 3.0e38
    x[6] = 1.5
    x[7, 3] = -np.inf                            # a masked target
    x[8] = np.nan
    b = Batch(sd, x, kind)
    targets = np.array([-1, 4, 5, 7, 9, 11, 100, 3, vocab])
    got = forward(b, targets)
    assert got[0][0] == got[1][0] == got[0][8] == got[1][8] == 0
    assert got[0][2] == -np.inf and got[1][2] == 0 and got[0][7] == -np.inf
    assert got[0][3] == got[1][3] == got[0][4] == got[1][4] == got[0][5] == got[1][5] == 0
    keep = [1, 3, 4, 5, 6, 7]
    part = Batch(sd, x[keep], kind)
    with np.errstate(invalid="ignore"):
        check_forward(part, targets[keep], None, (got[0][keep], got[1][keep]))
        g, h = rng.normal(0, 1, rows), rng.normal(0, 1, rows)
        d = backward(b, g, h)
        assert not d[0].any() and not d[2].any() and not d[8].any()
        check_gradient(part, targets[keep], None, g[keep], h[keep], d[keep])


@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_what_is_not_a_number_shows(sd, bad):  # noqa: F811
    x = np.zeros((3, 777))
    x[1, 700] = bad
    b = Batch(sd, x, "f32")
    lp, H = forward(b, [5, 5, 5])
    assert np.isnan(lp[1]) and np.isnan(H[1]) and np.isfinite(lp[[0, 2]]).all()
    d = backward(b, [1.0] * 3, [1.0] * 3)
    assert np.isnan(d[1]).any() and np.isfinite(d[[0, 2]]).all()


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_gradient_in_place_leaves_what_lies_between_the_rows(sd, kind):  # noqa: F811
    import torch
    rng = np.random.default_rng(4)
    rows, vocab = 7, 1003
    b = Batch(sd, peaked(rng, rows, vocab), kind, gap=6)
    targets = rng.integers(0, vocab, rows)
    targets[2] = -1
    forward(b, targets)
    g, h = rng.normal(0, 1, rows), rng.normal(0, 1, rows)
    apart = backward(b, g, h)
    gaps = [int(i) for r in range(rows) for i in range(r * (vocab + 6) + vocab, (r + 1) * (vocab + 6))]
    assert (b.out[gaps] == 3).all()
    before = b.flat.clone()
    again = backward(b, g, h, out=b.flat)
    assert np.array_equal(apart, again) and torch.equal(before[gaps], b.flat[gaps])


def test_gradient_against_differences(sd):  # noqa: F811
    """Of the fp32 results: differences over 2 * 2^-4 of a sum of log probabilities and entropies; their error is that of the results over the step,
    and the third derivative's share, at most step^2 (both functions have third derivatives below 2 (1 + log vocab) / T^3)."""
    rng = np.random.default_rng(6)
    vocab, e, t = 21, 2.0 ** -4, 1.3
    x = rng.normal(0, 1, vocab).astype(np.float32)
    rows = np.stack([x] + [x + s * e * np.eye(vocab)[j] for j in range(vocab) for s in (1, -1)])
    b = Batch(sd, rows, "f32")
    n = len(rows)
    lp, H = forward(b, [6] * n, [t] * n)
    g, h = 0.8, -0.5
    d = backward(b, [g] * n, [h] * n)[0]
    f = g * lp.astype(np.float64) + h * H
    want = (f[1::2] - f[2::2]) / (2 * e)
    assert abs(d - want).max() <= 1e-5 / e + e * e * 2 * (1 + np.log(vocab)) / t ** 3


def test_what_is_drawn_has_the_trainers_log_probability(sd):  # noqa: F811
    rng = np.random.default_rng(8)
    rows, vocab = 40, 20011
    b = Batch(sd, peaked(rng, rows, vocab), "bf16")
    t = rng.uniform(0.5, 1.2, rows)
    tokens, lp, _ = b.draw(rng.random(rows).astype(np.float32), temperature=t, top_p=[0.9] * rows)
    got = forward(b, tokens, t)
    for r in range(rows):
        want, H, z1, z2, s2 = plain.logprobs(b.x[r], tokens[r], float(np.float32(t[r])))
        assert abs(got[0][r] - lp[r]) <= log_sum_error(vocab, z1, s2) + STEP * (6 * (abs(want) + s2)) + 1e-9


def test_results_that_are_not_asked_for(sd):  # noqa: F811
    rng = np.random.default_rng(12)
    b = Batch(sd, peaked(rng, 4, 5000), "f32")
    full = forward(b, [1, 2, 3, 4])
    lp, H = forward(b, [1, 2, 3, 4], entropy=False, stats=False)
    assert np.array_equal(lp, full[0]) and (H == 7).all() and (b.stats == 7).all()


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_temperatures_at_the_ends_of_the_range(sd, kind):  # noqa: F811
    """The smallest leave the largest logits alone, however near the next ones are; the largest weigh all alike that are not masked; 0, below and NaN count as 1."""
    rng = np.random.default_rng(13)
    vocab = 1001
    x = np.tile(rng.normal(0, 2, vocab), (8, 1))
    x[:, 3::7] = -np.inf
    x[:, [5, 700]] = 9.0
    t = [1e-45, 1e-39, 2e-38, np.inf, 3e38, 0.0, -1.0, np.nan]
    b = Batch(sd, x, kind)
    targets = [5, 4, 700, 5, 700, 5, 5, 5]
    lp, H = forward(b, targets, t)
    some = np.isfinite(b.x[0]).sum()
    assert abs(lp[0] + np.log(2)) <= 4 * STEP and lp[1] < -1e30 and abs(lp[2] + np.log(2)) <= 4 * STEP and (abs(H[:3] - np.log(2)) <= 8 * STEP).all()
    assert (abs(lp[3:5] + np.log(some)) <= 16 * STEP * np.log(some)).all() and (abs(H[3:5] - np.log(some)) <= 16 * STEP * np.log(some)).all()
    assert lp[5] == lp[6] == lp[7] and H[5] == H[6] == H[7]
    one = forward(Batch(sd, x[5:], kind), targets[5:])
    assert np.array_equal(one[0], lp[5:]) and np.array_equal(one[1], H[5:])
    forward(b, targets, t)
    d = backward(b, [1e-30] * 8, [1e-30] * 8)
    assert np.isfinite(d).all() and not d[:, ~np.isfinite(b.x[0])].any()
