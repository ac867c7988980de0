"""TokenLogprobs (examples/captured_rollout.py) of logits, targets and temperatures that do not lie side by side: copies, or a refusal, never memory that is
not theirs.  On the CPU the entry points are stood in for by what they are documented to read and write; on the GPU they run."""
import importlib.util
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    spec = importlib.util.spec_from_file_location("captured_rollout_layouts", os.path.join(ROOT, "examples", "captured_rollout.py"))
    m = importlib.util.module_from_spec(spec)
    before = list(sys.path)
    spec.loader.exec_module(m)
    sys.path[:] = before
    return m


class Documented:
    """The calls as the header has them, on tensors of the host: rows at the shape's stride from the first element on, one element a row of the rest."""

    def __init__(self, sd):
        self.sd = sd

    def _of(self, desc, logits, targets, temperature):
        assert logits.dtype == {self.sd.SD_BF16: torch.bfloat16, self.sd.SD_F32: torch.float32}[desc.dtype]
        assert all(p is None or p.data_ptr() % 16 == 0 for p in (logits, targets, temperature))
        assert targets.dtype == torch.int32 and (temperature is None or temperature.dtype == torch.float32)
        assert desc.rows <= 1 or desc.stride == 0 or desc.stride >= desc.vocab
        x = self._rows(desc, logits).double()
        y = targets.as_strided((desc.rows,), (1,)).long()
        t = torch.ones(desc.rows) if temperature is None else temperature.as_strided((desc.rows,), (1,))
        return x, y, t.double()[:, None]

    @staticmethod
    def _rows(desc, x):   # (refused by torch where that passes what x's memory holds)
        return x.as_strided((desc.rows, desc.vocab), (desc.stride or desc.vocab, 1))

    def token_logprobs(self, desc, logits, targets, temperature, logprobs, entropy, stats, workspace, nbytes, stream=None):
        x, y, t = self._of(desc, logits, targets, temperature)
        logp = torch.log_softmax(x / t, 1)
        real = (y >= 0) & (y < desc.vocab)
        logprobs.copy_(torch.where(real, logp.gather(1, y.clamp(0, desc.vocab - 1)[:, None])[:, 0], 0.0))
        entropy.copy_(torch.where(real, -(logp.exp() * logp).sum(1), 0.0))

    def token_logprobs_backward(self, desc, logits, targets, temperature, stats, entropy, d_logprobs, d_entropy, d_logits, stream=None):
        x, y, t = self._of(desc, logits, targets, temperature)
        assert d_logits.dtype == logits.dtype and all(p.is_contiguous() and p.data_ptr() % 16 == 0 for p in (d_logprobs, d_entropy))
        x = x.requires_grad_()
        with torch.enable_grad():
            logp = torch.log_softmax(x / t, 1)
            real = (y >= 0) & (y < desc.vocab)
            chosen = logp.gather(1, y.clamp(0, desc.vocab - 1)[:, None])[:, 0]
            loss = torch.where(real, chosen * d_logprobs.double() - (logp.exp() * logp).sum(1) * d_entropy.double(), 0.0).sum()
        self._rows(desc, d_logits).copy_(torch.autograd.grad(loss, x)[0])


def views(dtype, device, vocab=37):
    """name -> (leaf, logits made of it, targets, temperature)."""
    gen = torch.Generator().manual_seed(3)
    base = lambda *shape: (2 * torch.randn(shape, generator=gen)).to(dtype).to(device).requires_grad_()  # noqa: E731
    i32, f32 = lambda x: torch.tensor(x, dtype=torch.int32, device=device), lambda x: torch.tensor(x, device=device)  # noqa: E731
    y, t = i32([3, vocab - 1, -1, 0, 7]), f32([0.5, 1.0, 2.0, 0.9, 1.3])
    made = {}
    for name, leaf, view in (("side by side", base(5, vocab), lambda x: x), ("a gap behind each row", base(5, vocab + 3), lambda x: x[:, :vocab]), ("every second logit", base(5, 2 * vocab), lambda x: x[:, ::2]),
                             ("an odd start", base(5, vocab + 3), lambda x: x[:, 3:]), ("rows of an odd start", base(6, vocab), lambda x: x[1:]), ("transposed", base(vocab, 5), lambda x: x.t()),
                             ("one row for all", base(1, vocab), lambda x: x.expand(5, vocab)), ("every second row", base(10, vocab), lambda x: x[::2]), ("rows that overlap", base(vocab + 4), lambda x: x.unfold(0, vocab, 1))):
        made[name] = leaf, view(leaf), y, t
    one = base(2, vocab)
    made["one row"] = one, one[1:].as_strided((1, vocab), (5, 1)), y[:1], t[:1]
    made["one logit a row"] = (lambda x: (x, x[:, 1:2], i32([0, 0, -1, 0, 1]), t))(base(5, 3))
    leaf = base(5, vocab)
    made["targets apart"] = leaf, leaf, torch.stack([y, y + 1], 1)[:, 0], t
    made["temperatures apart"] = leaf, leaf, y, torch.stack([t, 3 * t], 1)[:, 0]
    made["one temperature for all"] = leaf, leaf, y, f32([0.7]).expand(5)
    made["no temperature"] = leaf, leaf, y, None
    return made


NAMES = sorted(views(torch.float32, "cpu"))


def check(ex, leaf, logits, targets, temperature):
    """Half a step of the results' type, and in fp32 some tens of roundings (2^-24 each) of sums of 37 terms below 10."""
    g, h = torch.linspace(-1, 1.5, logits.shape[0], device=leaf.device), torch.linspace(0.3, -0.2, logits.shape[0], device=leaf.device)
    lp, entropy = ex.TokenLogprobs.apply(logits, targets, temperature)
    got = torch.autograd.grad((lp * g).sum() + (entropy * h).sum(), leaf)[0].double()
    t = 1.0 if temperature is None else temperature.double()[:, None]
    logp = torch.log_softmax(logits.double() / t, 1)
    real = (targets >= 0) & (targets < logits.shape[1])
    chosen = torch.where(real, logp.gather(1, targets.long().clamp(0, logits.shape[1] - 1)[:, None])[:, 0], 0.0)
    H = torch.where(real, -(logp.exp() * logp).sum(1), 0.0)
    want = torch.autograd.grad((chosen * g).sum() + (H * h).sum(), leaf)[0].double()
    assert (lp - chosen).abs().max() <= 64 * 10 * 2.0 ** -24 and (entropy - H).abs().max() <= 64 * 10 * 2.0 ** -24
    half = 2.0 ** -8 if leaf.dtype == torch.bfloat16 else 2.0 ** -24
    shared = 5 if logits.shape[0] == 5 and logits.shape[1] > 1 and logits.stride(0) < logits.shape[1] and logits.stride(1) == 1 else 1
    # (an element of several rows: five gradients below 4, each rounded, and four sums of them below 20)
    bound = half * (5 * 4 + 4 * 20) if shared > 1 else half * want.abs()
    assert ((got - want).abs() <= bound + shared * 64 * 10 * 2.0 ** -24).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("name", NAMES)
def test_documented_calls_read_what_is_theirs(ex, monkeypatch, name, dtype):
    calls = Documented(ex.sd)
    monkeypatch.setattr(ex.sd, "token_logprobs", calls.token_logprobs)
    monkeypatch.setattr(ex.sd, "token_logprobs_backward", calls.token_logprobs_backward)
    check(ex, *views(dtype, "cpu")[name])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("name", NAMES)
def test_layouts(ex, name, dtype):
    check(ex, *views(dtype, "cuda")[name])


def test_gradients_that_are_views(ex, monkeypatch):
    """What arrives at the results may be a part of another tensor, or one element for all rows."""
    calls = Documented(ex.sd)
    monkeypatch.setattr(ex.sd, "token_logprobs", calls.token_logprobs)
    monkeypatch.setattr(ex.sd, "token_logprobs_backward", calls.token_logprobs_backward)
    leaf, logits, targets, temperature = views(torch.float32, "cpu")["side by side"]
    lp, entropy = ex.TokenLogprobs.apply(logits, targets, temperature)
    joined = torch.cat([torch.zeros(1, requires_grad=True), lp, entropy])
    got = torch.autograd.grad(joined, leaf, torch.arange(11.0))[0]
    lp, entropy = ex.TokenLogprobs.apply(logits, targets, temperature)
    want = torch.autograd.grad((lp * torch.arange(1.0, 6)).sum() + (entropy * torch.arange(6.0, 11)).sum(), leaf)[0]
    assert torch.equal(got, want)
    lp, entropy = ex.TokenLogprobs.apply(logits, targets, temperature)
    assert torch.autograd.grad(lp.sum(), leaf)[0].abs().max() > 0      # (the entropy is not used)


def test_refusals(ex, monkeypatch):
    """What the calls do not take is refused before they see it."""
    def never(*args, **kw):
        raise AssertionError("called")
    monkeypatch.setattr(ex.sd, "token_logprobs", never)
    x, y, t = torch.zeros(4, 9), torch.zeros(4, dtype=torch.int32), torch.ones(4)
    for args in ((x.half(), y, t), (x.double(), y, t), (x, y.long(), t), (x, y.float(), t), (x, y, t.double()), (x, y, t.bfloat16())):
        with pytest.raises(TypeError):
            ex.TokenLogprobs.apply(*args)
    for args in ((x, y[:3], t), (x, y, t[:3]), (x[0], y, t), (x[None], y, t), (x, y[:, None], t), (x, y, t[:, None]), (torch.zeros(4, 0), y, t)):
        with pytest.raises(ValueError):
            ex.TokenLogprobs.apply(*args)


def test_rollouts_that_cannot_begin(ex):
    """A sequence without a token has no logits to draw from (those of the one before it would be taken), and each step of each sequence has a random number."""
    u = torch.zeros(4, 2)
    for prompts, max_new, uniform in (([[1, 2], []], 4, u), ([[], [3]], 4, u), ([], 4, u[:, :0]), ([[1], [2]], 0, u[:0]), ([[1], [2]], 5, u), ([[1], [2]], 4, u.t()), ([[1]], 4, u)):
        with pytest.raises(ValueError):
            ex.Rollout(None, prompts, max_new, 10, 0, uniform, None)
