"""The operators together, as examples/bounded_rollout.py uses them: every step's attention against a dense 64-bit computation over the
tokens that the cache says it holds, the choice of those tokens, the pool's pages, and the gradients of the training step."""
import importlib.util
import os

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
MAX_ABS, MEAN_ABS = 1e-2, 1e-3   # as everywhere for bf16 pools


@pytest.fixture(scope="module")
def ex():
    import torch
    assert torch.cuda.is_available()
    spec = importlib.util.spec_from_file_location("bounded_rollout", os.path.join(ROOT, "examples", "bounded_rollout.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def normed(layer, qkv, positions):
    """Rotated queries and keys (rounded to bf16, as the cache holds them) and values in 64 bits; plain torch."""
    import torch
    d, T = layer.head_dim, qkv.shape[0]
    x = qkv.double().cpu().view(T, -1, d)
    q, k, v = x[:, :layer.heads], x[:, layer.heads:layer.heads + layer.kv_heads], x[:, layer.heads + layer.kv_heads:]
    row = layer.table.double().cpu()[positions][:, None]
    c, s = row[..., :d // 2], row[..., d // 2:]

    def one(x, w):
        z = x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt() * w.double().cpu()
        a, b = z[..., :d // 2], z[..., d // 2:]
        return torch.cat([a * c - b * s, b * c + a * s], dim=-1).bfloat16().double()

    return one(q, layer.q_weight), one(k, layer.k_weight), v


def attend(q, k, v, scale):
    """q [G][d], k and v [n][d] -> [G][d]"""
    return (scale * q @ k.T).softmax(-1) @ v


@pytest.mark.parametrize("heads,kv_heads,d", [(8, 2, 64), (14, 2, 128)])
def test_rollout_with_a_bounded_cache(ex, heads, kv_heads, d):
    import torch
    torch.manual_seed(1)
    lengths, hidden, budget, sinks, recent, slack = [90, 7, 150, 40], 64, 48, 3, 16, 8
    layer = ex.Layer(hidden, heads, kv_heads, d, max_positions=512)
    r = ex.Rollout(layer, lengths, budget, sinks, recent, slack, window=16)
    rows = torch.randn(sum(lengths), hidden, device="cuda").bfloat16()
    qkv = rows @ layer.projection
    q, k, v = normed(layer, qkv, [p for n in lengths for p in range(n)])
    out = r.prompt(rows).double().cpu()
    starts = np.concatenate([[0], np.cumsum(lengths)])
    K = [k[a:b] for a, b in zip(starts, starts[1:])]
    V = [v[a:b] for a, b in zip(starts, starts[1:])]
    G, scale, errors = heads // kv_heads, d ** -0.5, []
    for b, n in enumerate(lengths):
        for p in (0, 1, n // 2, n - 1):
            for g in range(kv_heads):
                want = attend(q[starts[b] + p, g * G:(g + 1) * G], K[b][:p + 1, g], V[b][:p + 1, g], scale)
                errors.append((out[starts[b] + p, g * G:(g + 1) * G] - want).abs())
    evictions, before = 0, list(r.lens)
    for step in range(60):
        x = torch.randn(len(lengths), hidden, device="cuda").bfloat16()
        held = None if r.cached is None else [[list(c) for c in heads_] for heads_ in r.cached]
        positions = list(r.positions)
        sq, sk, sv = normed(layer, x @ layer.projection, positions)
        out = r.step(x).double().cpu()
        for b in range(len(lengths)):
            K[b], V[b] = torch.cat([K[b], sk[b:b + 1]]), torch.cat([V[b], sv[b:b + 1]])
            for g in range(kv_heads):
                at = (list(range(positions[b])) if held is None else held[b][g]) + [positions[b]]
                errors.append((out[b, g * G:(g + 1) * G] - attend(sq[b, g * G:(g + 1) * G], K[b][at, g], V[b][at, g], scale)).abs())
        # what the cache holds: as much as it may, in order, its first and its newest tokens among it
        if r.lens != [n + 1 for n in before]:
            evictions += 1
            for b, n in enumerate(r.lens):
                for c in r.cached[b]:
                    assert len(c) == n <= budget and c == sorted(set(c)) and c[:min(sinks, n)] == list(range(min(sinks, n)))
                    if r.positions[b] > budget:
                        assert c[-recent:] == list(range(r.positions[b] - recent, r.positions[b]))
        before = list(r.lens)
        in_use = [p for pages in r.pages for p in pages]
        assert len(set(in_use)) == len(in_use) and sorted(in_use + r.free) == list(range(r.num_pages))
        assert max(r.lens) <= budget + slack
    assert evictions >= 5
    e = torch.cat([x.reshape(-1) for x in errors])
    assert e.max() <= MAX_ABS and e.mean() <= MEAN_ABS


def test_without_an_eviction_nothing_is_lost(ex):
    """A budget that is never reached: the same rows, bit for bit, as with a cache that is cut (until it is)."""
    import torch
    layer = ex.Layer(64, 8, 2, 64, max_positions=512)
    lengths = [30, 5, 21]
    torch.manual_seed(2)
    rows = [torch.randn(sum(lengths), 64, device="cuda").bfloat16()] + [torch.randn(3, 64, device="cuda").bfloat16() for _ in range(40)]
    wide, narrow = (ex.Rollout(layer, lengths, budget, 2, 8, 4, window=8) for budget in (400, 32))
    assert torch.equal(wide.prompt(rows[0]), narrow.prompt(rows[0]))
    for x in rows[1:]:
        same = narrow.cached is None
        a, b = wide.step(x), narrow.step(x)
        if same:
            assert torch.equal(a, b)
    assert wide.cached is None and wide.lens == wide.positions == [70, 45, 61] and narrow.cached is not None and max(narrow.lens) <= 36


def test_gradients_of_the_training_step(ex):
    """Through autograd: against plain fp32 torch on the same rows.  Gradients pass through bf16 (as the operator's outputs and the
    projection's gradient do), so they are held to 2 % of their norm."""
    import torch
    torch.manual_seed(3)
    layer = ex.Layer(96, 12, 3, 64, max_positions=300)
    rows, positions = torch.randn(257, 96, device="cuda").bfloat16(), torch.randint(0, 300, (257,), dtype=torch.int32, device="cuda")
    loss, *got = ex.learn(layer, rows, positions)
    p, qw, kw = (t.float().detach().requires_grad_() for t in (layer.projection, layer.q_weight, layer.k_weight))
    x = (rows.float() @ p).view(257, -1, 64)
    row = layer.table[positions.long()][:, None]
    c, s = row[..., :32], row[..., 32:]

    def one(x, w):
        z = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w
        return torch.cat([z[..., :32] * c - z[..., 32:] * s, z[..., 32:] * c + z[..., :32] * s], dim=-1)

    want = one(x[:, :12], qw).square().mean() + one(x[:, 12:15], kw).square().mean()
    want.backward()
    assert abs(loss - want) <= 2e-3 * want
    for g, w in zip(got, (p.grad, qw.grad, kw.grad)):
        assert (g.float() - w).norm() <= 0.02 * w.norm()
