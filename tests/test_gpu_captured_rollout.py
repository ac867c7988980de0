"""Sampling, the plan of a step and log probabilities together, as examples/captured_rollout.py uses them: every step's draws, tables and attention
against plain computations, the captured graph against eager steps, and the training step's log probabilities and gradient."""
import importlib.util
import os

import numpy as np
import pytest

from tests import logits_plain as plain
from tests.test_gpu_bounded_rollout import MAX_ABS, MEAN_ABS, ROOT, attend, normed
from tests.test_gpu_token_logprobs import STEP, log_sum_error

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ex():
    import torch
    assert torch.cuda.is_available()
    spec = importlib.util.spec_from_file_location("captured_rollout", os.path.join(ROOT, "examples", "captured_rollout.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


LENGTHS = [40, 3, 97, 16, 15, 33, 1, 64, 20]


def rollout(ex, spare, max_new=40, seed=1, vocab=523, limits=True):
    """Some rows take the largest logit, some have no limit; `spare` pages besides those of the prompts."""
    import torch
    gen = torch.Generator().manual_seed(seed)
    model = ex.Model(vocab, 64, 8, 2, 64, max_positions=512)
    prompts = [torch.randint(0, vocab, (n,), generator=gen).tolist() for n in LENGTHS]
    B, dev = len(prompts), lambda x: x.to("cuda")  # noqa: E731
    t = 0.5 + torch.rand(B, generator=gen)
    t[2] = 0.0
    k, p = torch.tensor([0, 5, 0, 50, 0, 1, 0, 20, 600], dtype=torch.int32), torch.tensor([1.0, 0.9, 1.0, 1.0, 0.8, 0.5, 0.95, 0.9, 0.99])
    pages = sum((n + 15) // 16 for n in LENGTHS) + spare
    return ex.Rollout(model, prompts, max_new, pages, stop=9, uniform=dev(torch.rand(max_new, B, generator=gen)), temperature=dev(t), top_k=dev(k) if limits else None,
                      top_p=dev(p) if limits else None)


@pytest.mark.parametrize("spare,waits", [(7, True), (40, False)])
def test_every_step(ex, spare, waits):
    import torch
    r = rollout(ex, spare)
    model, B = r.model, r.B
    free, table, lens = list(range(r.shape.num_pages)), [[0] * r.shape.max_blocks_per_seq for _ in range(B)], [0] * B
    r.prompt()
    want = plain.plan(LENGTHS, [0] * B, lens, lens, free, table, sum(LENGTHS), r.shape.max_context_len)
    lens = want["lens_out"]
    K, V = [], []
    for ids in r.prompts:
        _, k, v = normed(model, model.embedding[torch.tensor(ids, device="cuda")] @ model.projection, list(range(len(ids))))
        K.append(k)
        V.append(v)
    alive, stalled, token, count, errors, stalls = [True] * B, [False] * B, [0] * B, [0] * B, [], 0
    k, p, t, uniform = r.top_k.tolist(), r.top_p.cpu().numpy(), r.temperature.cpu().numpy(), r.uniform.cpu().numpy()
    for _ in range(60):
        logits = r.logits.float().cpu().numpy()
        r.step()
        asks = []
        for b in range(B):
            if alive[b] and not stalled[b]:
                token[b], lp, dlp = plain.sample(logits[b], t[b], k[b], p[b], 0.0, uniform[count[b], b])
                assert r.drawn[b].item() == token[b] == r.answers[b, count[b]].item()
                assert abs(r.logprobs[b, count[b]].item() - lp) <= STEP * abs(lp) + 1e-9 and abs(r.dlp[b].item() - dlp) <= STEP * abs(dlp) + 1e-9
                count[b] += 1
                ended = token[b] == r.stop or count[b] == r.max_new
                asks.append(-1 if ended else 1)
                alive[b] = not ended
            else:
                asks.append(int(alive[b]))
        before = lens
        want = plain.plan(asks, [0] * B, lens, lens, free, table, B, r.shape.max_context_len)
        lens = want["lens_out"]
        assert r.granted.tolist() == want["granted"] and r.lens.tolist() == lens and r.table.tolist() == table
        assert r.free.item() == len(free) and r.free_pages[:len(free)].tolist() == free
        held = [x for b in range(B) for x in table[b][:(lens[b] + 15) // 16]]
        assert sorted(held + free) == list(range(r.shape.num_pages))
        stalled = [alive[b] and not want["granted"][b] for b in range(B)]
        stalls += sum(stalled)
        assert r.waits.tolist() == stalled and r.alive.tolist() == alive
        x = model.embedding[torch.tensor(token, device="cuda")]
        q, k1, v1 = normed(model, x @ model.projection, before)
        out = r.attended.double().cpu()
        for b in range(B):
            if not want["granted"][b]:
                continue
            K[b], V[b] = torch.cat([K[b], k1[b:b + 1]]), torch.cat([V[b], v1[b:b + 1]])
            for g in range(2):
                errors.append((out[b, 4 * g:4 * g + 4] - attend(q[b, 4 * g:4 * g + 4], K[b][:, g], V[b][:, g], 0.125)).abs())
    e = torch.cat([x.reshape(-1) for x in errors])
    assert e.max() <= MAX_ABS and e.mean() <= MEAN_ABS
    assert not any(alive) or stalls
    assert (stalls > 0) == waits


def test_a_pool_that_no_sequence_can_end_in(ex):
    """Each holds some of the 7 pages and none gets its last: said instead of replayed for ever."""
    with pytest.raises(RuntimeError, match="waits"):
        rollout(ex, 7).run(look_every=5)


@pytest.mark.parametrize("spare,limits", [(14, True), (40, True), (40, False)])
def test_the_captured_step_is_the_eager_one(ex, spare, limits):
    import torch
    a, b = rollout(ex, spare, limits=limits), rollout(ex, spare, limits=limits)
    steps = a.run(look_every=5)
    b.prompt()
    for _ in range(steps):
        b.step()
    for name in ("answers", "logprobs", "states", "count", "table", "lens", "free"):
        x, y = getattr(a, name), getattr(b, name)
        x, y = (x[:, :-1], y[:, :-1]) if name in ("answers", "logprobs", "states") else (x, y)   # (the last column is nobody's)
        assert torch.equal(x, y), name
    assert not a.alive.any() and a.free.item() == a.shape.num_pages and sorted(a.free_pages.tolist()) == list(range(a.shape.num_pages))
    for made, row in zip(a.count.tolist(), a.answers.tolist()):
        assert all(0 <= x < 523 for x in row[:made]) and all(x == -1 for x in row[made:-1])
        assert made == a.max_new or row[made - 1] == a.stop


def test_two_graphs_in_turn(ex):
    """Two rollouts, each with its graph, replayed in turn: neither sees the other."""
    import torch
    alone = [rollout(ex, 40, seed=s) for s in (1, 2)]
    steps = [r.run(look_every=1) for r in alone]
    both = [rollout(ex, 40, seed=s) for s in (1, 2)]
    for r in both:
        r.prompt()
        r.step()
        r.capture()
    for i in range(1, max(steps)):
        for r, n in zip(both, steps):
            if i < n:
                r.graph.replay()
    for x, y in zip(alone, both):
        assert torch.equal(x.answers[:, :-1], y.answers[:, :-1]) and torch.equal(x.logprobs[:, :-1], y.logprobs[:, :-1])


def test_training_step(ex):
    """Log probabilities against 64 bits on the same logits; the gradient against autograd in 64 bits (the logits' gradient is rounded to bf16, 2^-8 of each, and
    the product's result once more): held to 2^-7 of its norm."""
    import torch
    r = rollout(ex, 40)
    r.run()
    n = r.max_new
    answers, old, states = r.answers[:, :n], r.logprobs[:, :n] + 0.02, r.states[:, :n]   # (as if drawn by a slightly different policy)
    gen = torch.Generator().manual_seed(5)
    advantage, temperature = torch.randn(r.B, generator=gen).cuda(), torch.where(r.temperature > 0, r.temperature, 1.0)
    loss, lp, grad = ex.learn(r.model, states, answers, old, advantage, temperature)
    real = (answers >= 0).cpu()
    logits = (states.reshape(r.B * n, -1) @ r.model.head).view(r.B, n, -1).float().cpu()
    for b in range(r.B):
        for i in range(n):
            if not real[b, i]:
                assert lp[b, i] == 0
                continue
            want, H, z1, z2, s2 = plain.logprobs(logits[b, i].numpy(), answers[b, i].item(), temperature[b].item())
            assert abs(lp[b, i].item() - want) <= log_sum_error(523, z1, s2) + STEP * (4 * (abs(want) + s2) + 2 * abs(want))
    x = logits.double().requires_grad_()
    logp = (x / temperature.double().cpu()[:, None, None]).log_softmax(-1)
    chosen = logp.gather(2, answers.long().cpu().clamp(min=0)[..., None])[..., 0]
    entropy = -(logp.exp() * logp).sum(-1)
    ratio, a = (chosen - old.double().cpu()).exp(), advantage.double().cpu()[:, None]
    gain = torch.minimum(ratio * a, ratio.clamp(0.8, 1.2) * a)
    want = -((gain + 0.01 * entropy) * real).sum() / real.sum()
    want.backward()
    d_head = states.reshape(r.B * n, -1).double().cpu().T @ x.grad.view(r.B * n, -1)
    assert abs(loss.item() - want.item()) <= 1e-5 * (1 + abs(want.item()))
    assert (grad.double().cpu() - d_head).norm() <= 2.0 ** -7 * d_head.norm()
