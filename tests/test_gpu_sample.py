"""sample_tokens against the plain form in 64 bits: which token, and its log probabilities."""
import numpy as np
import pytest

from tests import logits_plain as plain

pytestmark = pytest.mark.gpu

NONE = dict(temperature=None, top_k=None, top_p=None, min_p=None)


@pytest.fixture(scope="module")
def sd():
    import torch
    assert torch.cuda.is_available()
    import paper_2508_11553_amd as m
    m.load()
    return m


class Batch:
    """Rows of logits on the device (bf16 or fp32, rows `stride` elements apart) and the values that they hold."""

    def __init__(self, sd, x, kind, gap=0):
        import torch
        self.sd, (self.rows, self.vocab) = sd, x.shape
        stride = self.vocab + gap
        if kind == "bf16":
            bits = plain.bf16_bits(x)
            self.x = plain.bf16_values(bits)
            flat = np.full(self.rows * stride, 0x7f80, np.uint16)   # +inf between the rows: whoever reads it draws nothing else
            raw = bits
        else:
            self.x = x.astype(np.float32)
            flat = np.full(self.rows * stride, np.inf, np.float32)
            raw = self.x
        for r in range(self.rows):
            flat[r * stride:r * stride + self.vocab] = raw[r]
        self.flat = torch.from_numpy(flat.view(np.int16) if kind == "bf16" else flat).cuda()
        self.desc = sd.Logits(rows=self.rows, vocab=self.vocab, dtype=sd.SD_BF16 if kind == "bf16" else sd.SD_F32, stride=stride if gap else 0)
        self.ws = sd.sample_workspace_bytes(self.desc)
        self.work = torch.full((self.ws,), 255, dtype=torch.uint8, device="cuda")

    def draw(self, uniform, temperature=None, top_k=None, top_p=None, min_p=None):
        import torch
        dev = lambda a, t: None if a is None else torch.tensor(np.asarray(a, t), device="cuda")  # noqa: E731
        tokens = torch.full((self.rows,), -7, dtype=torch.int32, device="cuda")
        lp, dlp = torch.full((self.rows,), 7.0, device="cuda"), torch.full((self.rows,), 7.0, device="cuda")
        self.sd.sample_tokens(self.desc, self.flat, dev(temperature, np.float32), dev(top_k, np.int32), dev(top_p, np.float32), dev(min_p, np.float32),
                              dev(uniform, np.float32), tokens, lp, dlp, self.work, self.ws)
        return tokens.cpu().numpy(), lp.cpu().numpy(), dlp.cpu().numpy()


def check(b, uniform, **limits):
    """A rounding to fp32 is off by half a step, 2^-24 of the value; sums of whole weights have none."""
    limits = {**NONE, **limits}
    got = b.draw(uniform, **limits)
    for r in range(b.rows):
        mine = {k: np.float32(v[r]) if k != "top_k" else int(v[r]) for k, v in limits.items() if v is not None}
        token, lp, dlp = plain.sample(b.x[r], uniform=np.float32(uniform[r]), **mine)
        assert got[0][r] == token, (r, got[0][r], token, mine)
        for value, want in ((got[1][r], lp), (got[2][r], dlp)):
            assert value == want or abs(value - want) <= 2.0 ** -24 * abs(want) + 1e-9, (r, value, want)
    return got


def peaked(rng, rows, vocab):
    x = rng.normal(0, 2, (rows, vocab))
    for r in range(rows):
        at = rng.integers(0, vocab, min(30, vocab))
        x[r, at] = 10 - 1.5 * np.log(np.arange(1, len(at) + 1)) + rng.normal(0, 0.3, len(at))
    return x


VOCABS = [1, 2, 7, 8, 9, 63, 64, 65, 255, 1000, 4097, 16383, 50001]


@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("limits", ["none", "top_k", "top_p", "min_p", "all"])
def test_draws(sd, vocab, kind, limits):
    rng = np.random.default_rng(vocab * 10 + len(limits))
    rows = 6
    x = peaked(rng, rows, vocab) if vocab % 2 else rng.normal(0, 1, (rows, vocab))
    b = Batch(sd, x, kind, gap=[0, 3][vocab % 3 == 0])
    use = dict(temperature=rng.uniform(0.3, 1.5, rows))
    if limits in ("top_k", "all"):
        use["top_k"] = [1, 2, 17, max(1, vocab // 2), vocab, 0]
    if limits in ("top_p", "all"):
        use["top_p"] = [0.9, 0.1, 0.999, 0.5, 1.0, 0.97]
    if limits in ("min_p", "all"):
        use["min_p"] = [0.0, 0.01, 0.3, 0.001, 0.1, 0.02]
    for _ in range(3):
        check(b, rng.random(rows).astype(np.float32), **use)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 2, 5, 33, 129, 300])
def test_batches(sd, kind, rows):
    rng = np.random.default_rng(rows)
    b = Batch(sd, peaked(rng, rows, 2500 if rows > 5 else 131072), kind)
    check(b, rng.random(rows).astype(np.float32), temperature=rng.uniform(0, 1.2, rows), top_k=rng.integers(0, 80, rows), top_p=rng.uniform(0.5, 1.05, rows),
          min_p=rng.uniform(-0.02, 0.1, rows))


@pytest.mark.parametrize("vocab", [8, 1000, 32768])
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_ties_are_cut_by_index(sd, vocab, kind):
    """Few different values: every limit ends among equals."""
    rng = np.random.default_rng(vocab)
    rows = 8
    b = Batch(sd, rng.integers(-2, 3, (rows, vocab)).astype(np.float64), kind)
    u = rng.random(rows).astype(np.float32)
    u[:2] = 0.0, 1 - 2.0 ** -24
    k = [1, 2, 3, vocab // 5 + 1, vocab // 3, vocab // 2 + 1, vocab - 1, vocab]
    check(b, u, top_k=k)
    check(b, u, top_p=[0.01, 0.2, 0.3, 0.4, 0.5, 0.6, 0.9, 0.9999])
    check(b, u, top_k=k, top_p=[0.9] * rows)
    check(b, u, top_p=[0.9] * rows, min_p=[np.exp(-1.0), np.exp(-2.0), 1.0, 2.0, 0.5, 0.3, 0.1, 0.0])


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_equal_logits(sd, kind):
    """All weights are one: the token is the uniform number times the vocabulary, rounded down, at the borders too."""
    for vocab in (1, 2, 64, 1000, 65536, 100003):
        u = np.array([0, 0.25, 0.5, 0.75, 1 - 2.0 ** -24, 1.0], np.float32)
        for value in (0.0, -5.0, float(np.float32(-3.38e38))):
            b = Batch(sd, np.full((len(u), vocab), value), kind)
            got = check(b, u)
            assert list(got[0]) == [min(vocab - 1, int(float(x) * vocab)) for x in u]


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [9, 5000])
def test_masked_infinite_and_missing_logits(sd, kind, vocab):
    rng = np.random.default_rng(3)
    x = rng.normal(0, 2, (12, vocab))
    x[0] = -np.inf
    x[1] = np.nan
    x[2], x[2, vocab - 1] = -np.inf, -4.0
    x[3, ::2] = np.nan
    x[4, 1::2] = -np.inf
    x[5, [1, vocab - 2]] = np.inf
    x[6], x[6, 3] = np.finfo(np.float32).min, 1.0
    x[7], x[7, 2] = -np.inf, np.nan
    x[8], x[8, 5] = np.nan, np.inf
    x[9], x[9, 5] = -3.0e38, 3.0e38
    x[10] = np.where(np.arange(vocab) % 3 == 0, 0.0, -0.0)
    x[11, 4] = 300.0
    b = Batch(sd, x, kind)
    u = rng.random(12).astype(np.float32)
    with np.errstate(invalid="ignore"):
        for limits in (dict(), dict(top_k=[3] * 12), dict(top_p=[0.8] * 12), dict(min_p=[0.1] * 12), dict(temperature=[0.0] * 12), dict(temperature=[2.0] * 12, top_k=[vocab - 1] * 12, top_p=[0.99] * 12)):
            got = check(b, u, **limits)
            assert got[0][0] == got[0][1] == got[0][7] == -1 and got[0][2] == vocab - 1 and got[0][8] == 5


def test_parameters_out_of_range(sd):
    rng = np.random.default_rng(5)
    vocab = 700
    row = rng.normal(0, 2, vocab)
    nan, inf = np.nan, np.inf
    b = Batch(sd, np.tile(row, (8, 1)), "f32")
    u = np.full(8, 0.4, np.float32)
    t, lp, dlp = b.draw(u, temperature=[0.0, -1.0, nan, 1e-30, 1.0, 1.0, 1.0, 1.0])
    assert (t[:4] == row.argmax()).all() and (dlp[:4] == 0).all()
    assert lp[0] == lp[1] == lp[2] and lp[3] == 0.0     # that of temperature 1; at 1e-30 nothing else has weight
    t, lp, dlp = b.draw(u, top_p=[1.0, 2.0, nan, inf, 0.0, -1.0, 1e-20, 0.9])
    assert len(set(t[:4])) == 1 and (lp[:4] == dlp[:4]).all() and (t[4:7] == row.argmax()).all()
    t, lp, dlp = b.draw(u, top_k=[0, -1, vocab, vocab + 5, 2 ** 31 - 1, -2 ** 31, 1, 2])
    assert len(set(t[:6])) == 1 and (lp[:6] == dlp[:6]).all() and t[6] == row.argmax()
    t, lp, dlp = b.draw(u, min_p=[0.0, -1.0, nan, -inf, 1.0, 5.0, inf, 0.5])
    assert len(set(t[:4])) == 1 and (t[4:7] == row.argmax()).all()
    t, lp, dlp = b.draw([-1.0, nan, 0.0, -inf, 1.0, 2.0, inf, 0.5])
    assert len(set(t[:4])) == 1 and len(set(t[4:7])) == 1 and t[0] == 0 and t[4] == vocab - 1
    b.draw(u, temperature=[inf] * 8)
    assert b.draw(u, temperature=[inf] * 8)[0][0] == int(np.float32(0.4) * vocab)      # all weigh alike


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [3001, 131072])
def test_a_row_draws_the_same_in_every_batch(sd, kind, vocab):
    rng = np.random.default_rng(9)
    rows = 400
    x = peaked(rng, 8, vocab)[np.arange(rows) % 8]
    x[:, 0] += np.arange(rows) * 1e-3
    u, t = rng.random(rows).astype(np.float32), rng.uniform(0.5, 1.2, rows)
    p, k = rng.uniform(0.7, 1.1, rows), rng.integers(0, 60, rows)
    whole = Batch(sd, x, kind).draw(u, temperature=t, top_p=p, top_k=k)
    for first, n in ((0, 1), (7, 2), (20, 13), (100, 60), (150, 200)):
        at = slice(first, first + n)
        part = Batch(sd, x[at], kind, gap=5).draw(u[at], temperature=t[at], top_p=p[at], top_k=k[at])
        for a, b in zip(whole, part):
            assert np.array_equal(a[at], b)


def test_outputs_that_are_not_asked_for(sd):
    import torch
    rng = np.random.default_rng(11)
    b = Batch(sd, peaked(rng, 3, 900), "bf16")
    u = torch.tensor([0.1, 0.5, 0.9], device="cuda")
    tokens = torch.zeros(3, dtype=torch.int32, device="cuda")
    sd.sample_tokens(b.desc, b.flat, None, None, None, None, u, tokens, None, None, b.work, b.ws)
    assert np.array_equal(tokens.cpu().numpy(), b.draw(u.cpu().numpy())[0])


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [300, 5000, 40001])
def test_temperatures_and_logits_of_any_size(sd, kind, vocab):
    """Temperatures at which all logits weigh alike though they differ, or only the largest weighs anything; logits so large that their neighbours are
    whole temperatures away, or that differences pass the range of fp32; with every limit, few rows and many."""
    rng = np.random.default_rng(vocab)
    inf = np.inf
    temperature = [inf, 1e30, 1e38, 1e-30, 1e-40, 1e-45, 1.0, 1e8, 1e9, 3e37, 1.0, 0.5]
    rows = len(temperature)
    x = rng.normal(0, 2, (rows, vocab))
    x[6] *= 1e10
    x[7] *= 1e10
    x[8] = 1e10 + rng.integers(-3, 4, vocab) * 1e9
    x[9] = rng.choice([-3e38, 3e38, 0.0, 1e38], vocab)
    x[10] = 1e10 + rng.integers(0, 3, vocab)         # all equal once rounded
    x[11] = -1e30
    x[:, 5::11] = -inf
    times = 1 if vocab > 10000 else 25
    b = Batch(sd, np.tile(x, (times, 1)), kind)
    for limits in (dict(), dict(top_k=7), dict(top_k=vocab // 2), dict(top_p=0.6), dict(top_p=0.999), dict(min_p=0.3), dict(top_k=vocab // 3, top_p=0.7, min_p=0.01)):
        u = rng.random(rows * times).astype(np.float32)
        got = b.draw(u, temperature=temperature * times, **{k: [v] * (rows * times) for k, v in limits.items()})
        for r in range(rows * times if times == 1 else 3 * rows):
            token, lp, dlp = plain.sample(b.x[r], np.float32(temperature[r % rows]), uniform=u[r], **{k: np.float32(v) if k != "top_k" else v for k, v in limits.items()})
            assert got[0][r] == token, (r, limits, got[0][r], token)
            for value, want in ((got[1][r], lp), (got[2][r], dlp)):
                assert value == want or abs(value - want) <= 2.0 ** -24 * abs(want) + 1e-9, (r, limits, value, want)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", [(3, 2 ** 20 - 1), (2, 524289), (300, 270001)])
def test_the_largest_vocabularies(sd, kind, rows, vocab):
    """More lanes' maxima than the threads hold at once, more stretches than a wave has lanes; peaked rows and nearly even ones."""
    import torch
    rng = np.random.default_rng(rows)
    some = sorted({0, 1, rows - 1})
    x = np.zeros((rows, vocab), np.float32)
    for r in some:
        x[r] = rng.normal(0, 0.5 if r else 2, vocab)
    x[0, rng.integers(0, vocab, 30)] = 12 + rng.normal(0, 1, 30)
    x[0, vocab - 1] = 14.0
    b = Batch(sd, x, kind)
    for limits in (dict(), dict(top_k=40, top_p=0.9), dict(top_p=0.95), dict(top_k=vocab // 2), dict(min_p=0.2)):
        u = rng.random(rows).astype(np.float32)
        got = b.draw(u, **{k: [v] * rows for k, v in limits.items()})
        for r in some:
            token, lp, dlp = plain.sample(b.x[r], uniform=u[r], **{k: np.float32(v) if k != "top_k" else v for k, v in limits.items()})
            assert got[0][r] == token, (r, limits, got[0][r], token)
            for value, want in ((got[1][r], lp), (got[2][r], dlp)):
                assert abs(value - want) <= 2.0 ** -24 * abs(want) + 1e-9, (r, limits, value, want)
    del b
    torch.cuda.empty_cache()


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [257, 300, 700, 2047, 2048, 2049, 3100])
@pytest.mark.parametrize("step", [0, 0.25, 0.002])
def test_hundreds_are_kept(sd, kind, vocab, step):
    """Candidates by the hundred: a limit ends within a bin of nearly equal ones, among equal ones (logits in steps), or past all of them; each limit alone and with others."""
    rng = np.random.default_rng(vocab)
    rows = 7
    x = rng.normal(0, 0.6, (rows, vocab))
    if step:
        x = np.round(x / step) * step
    b = Batch(sd, x, kind)
    k = [256, 257, 300, min(500, vocab), vocab // 2 + 1, vocab - 1, 2]
    p = [0.5, 0.9, 0.99, 0.999, 0.3, 0.7, 0.97]
    m = [0.05, 0.1, 0.2, 0.01, 0.3, 0.02, 0.15]
    for use in (dict(top_k=k), dict(top_p=p), dict(top_k=k, top_p=p), dict(top_k=k, min_p=m), dict(top_p=p, min_p=m), dict(top_k=k, top_p=p, min_p=m), dict(min_p=m)):
        check(b, rng.random(rows).astype(np.float32), temperature=rng.uniform(0.4, 1.3, rows), **use)
