"""A rollout whose cache is bounded: one attention layer, from its projections to the attention's rows.

Prompts go into the paged cache (qk_norm_rope_append), are attended (paged_prefill_attention), and the weights of their last
tokens start every cached token's score (paged_weight_accumulate).  Each further token is appended, attended
(paged_decode_attention) and added to the scores.  Whenever a sequence has outgrown its budget by `slack` tokens, kv_evict
moves the tokens that stay into other pages and the old ones go back to the pool; a token's position (its rotation) and its place
in the cache are then two things.  At the end the layer's norms and projection get their gradient from the whole trajectories, as a
training step would compute it (NormRope).

    python examples/bounded_rollout.py
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2508_11553_amd as sd  # noqa: E402

PAGE = 16


def rope_table(length, rotary_dim, theta=10000.0):
    """[length][rotary_dim] fp32: the cosines of the pairs' angles, then the sines."""
    freq = theta ** (-torch.arange(0, rotary_dim, 2, dtype=torch.float64) / rotary_dim)
    angle = torch.arange(length, dtype=torch.float64)[:, None] * freq
    return torch.cat([angle.cos(), angle.sin()], dim=1).float()


class NormRope(torch.autograd.Function):
    """qk_norm_rope on the rows of a fused projection [T][(heads + 2 kv_heads) d], with its gradient."""

    @staticmethod
    def forward(ctx, qkv, q_weight, k_weight, table, positions, norm):
        T, d = qkv.shape[0], norm.head_dim
        q, k = NormRope.parts(qkv, norm)
        q_out = torch.empty((T, norm.num_q_heads, d), dtype=qkv.dtype, device=qkv.device)
        k_out = torch.empty((T, norm.num_kv_heads, d), dtype=qkv.dtype, device=qkv.device)
        sd.qk_norm_rope(norm, q, k, q_weight, k_weight, table, positions, T, q_out, k_out)
        ctx.save_for_backward(qkv, q_weight, k_weight, table, positions)
        ctx.norm = norm
        return q_out, k_out

    @staticmethod
    def backward(ctx, dq_out, dk_out):
        qkv, q_weight, k_weight, table, positions = ctx.saved_tensors
        norm, T = ctx.norm, qkv.shape[0]
        q, k = NormRope.parts(qkv, norm)
        dqkv = torch.zeros_like(qkv)   # the values' part stays 0 here
        dq, dk = NormRope.parts(dqkv, norm)
        dq_weight, dk_weight = (torch.empty(norm.head_dim, device=qkv.device) for _ in range(2))
        ws = sd.qk_norm_rope_workspace_bytes(norm, T)
        workspace = torch.empty(ws, dtype=torch.uint8, device=qkv.device)
        sd.qk_norm_rope_backward(norm, dq_out.contiguous(), dk_out.contiguous(), q, k, q_weight, k_weight, table, positions, T, dq, dk, dq_weight,
                                 dk_weight, workspace, ws)
        return dqkv, dq_weight.to(q_weight.dtype), dk_weight.to(k_weight.dtype), None, None, None

    @staticmethod
    def parts(qkv, norm):
        a, b = norm.num_q_heads * norm.head_dim, (norm.num_q_heads + norm.num_kv_heads) * norm.head_dim
        return qkv[:, :a], qkv[:, a:b]


class Layer:
    """Projection and norms of one attention layer, random."""

    def __init__(self, hidden, heads, kv_heads, head_dim, max_positions, seed=0, device="cuda:0"):
        gen = torch.Generator().manual_seed(seed)
        width = (heads + 2 * kv_heads) * head_dim
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        self.projection = (torch.randn(hidden, width, generator=gen) / math.sqrt(hidden)).bfloat16().to(device)
        self.q_weight, self.k_weight = ((1 + 0.2 * torch.randn(head_dim, generator=gen)).bfloat16().to(device) for _ in range(2))
        self.table = rope_table(max_positions, head_dim).to(device)
        self.norm = sd.QkNorm(num_q_heads=heads, num_kv_heads=kv_heads, head_dim=head_dim, rotary_dim=head_dim, interleaved=0, table_len=max_positions,
                              weight_dtype=sd.SD_BF16, eps=1e-6, q_stride=width, k_stride=width, v_stride=width)

    def values(self, qkv):
        return qkv[:, (self.heads + self.kv_heads) * self.head_dim:]


class Rollout:
    """The cache of a batch of sequences, each held to `budget` tokens plus at most `slack`."""

    def __init__(self, layer, lengths, budget, sinks, recent, slack, window, decay=1.0, device="cuda:0"):
        self.layer, self.device = layer, torch.device(device)
        self.budget, self.sinks, self.recent, self.slack, self.window, self.decay = budget, sinks, recent, slack, window, decay
        self.positions, self.lens = list(lengths), list(lengths)   # tokens so far; of them in the cache
        B, d = len(lengths), layer.head_dim
        self.capacity = max(max(lengths), budget + slack + 1)
        self.blocks = (self.capacity + PAGE - 1) // PAGE
        self.num_pages = 2 * B * self.blocks   # an eviction needs new pages before it gives the old ones back
        self.free = list(range(self.num_pages))
        pool = (self.num_pages, layer.kv_heads, PAGE, d)
        self.k_pages, self.v_pages = (torch.empty(pool, dtype=torch.bfloat16, device=self.device) for _ in range(2))
        self.pages = [[] for _ in range(B)]
        self.stride = (self.capacity + 3) // 4 * 4
        self.scores = torch.zeros((B, layer.kv_heads, self.stride), device=self.device)
        self.cached = None   # [B][kv_heads][..]: the positions that the cache holds, for whoever wants to know
        for b, n in enumerate(lengths):
            self._grow(b, n)

    def _grow(self, b, tokens):
        while len(self.pages[b]) * PAGE < tokens:
            self.pages[b].append(self.free.pop())

    def _int(self, values):
        return torch.tensor(values, dtype=torch.int32, device=self.device)

    def _table(self):
        return self._int([p + [0] * (self.blocks - len(p)) for p in self.pages])

    def _shape(self):
        layer = self.layer
        return sd.Shape(batch=len(self.lens), num_q_heads=layer.heads, num_kv_heads=layer.kv_heads, head_dim=layer.head_dim, page_size=PAGE,
                        num_pages=self.num_pages, max_blocks_per_seq=self.blocks, kv_dtype=sd.SD_BF16, max_context_len=max(self.lens), chunk_tokens=0)

    def _append(self, hidden, seq_ids, positions, slots):
        """Projects the rows' hidden states and puts their keys and values into the cache; -> queries."""
        layer, T = self.layer, hidden.shape[0]
        qkv = hidden @ layer.projection
        q, k = NormRope.parts(qkv, layer.norm)
        q_out = torch.empty((T, layer.heads, layer.head_dim), dtype=torch.bfloat16, device=self.device)
        sd.qk_norm_rope_append(self._shape(), layer.norm, q, k, layer.values(qkv), layer.q_weight, layer.k_weight, layer.table, self._int(positions),
                               self._int(seq_ids), self._int(slots), T, q_out, self.k_pages, self.v_pages, self._table())
        return q_out

    def _accumulate(self, q, q_start, total, most, new, before):
        shape = self._shape()
        ws = sd.paged_weight_workspace_bytes(shape, most)
        workspace = torch.empty(ws, dtype=torch.uint8, device=self.device)
        sd.paged_weight_accumulate(shape, q, q_start, total, most, self.k_pages, None, self._table(), self._int(self.lens), self.layer.head_dim ** -0.5,
                                   self.decay, new, before, self.scores, self.stride, workspace, ws)

    def prompt(self, hidden):
        """hidden: the prompts' rows, one sequence after the other; -> the attention's rows."""
        lens = self.lens
        starts = [0]
        for n in lens:
            starts.append(starts[-1] + n)
        q = self._append(hidden, [b for b, n in enumerate(lens) for _ in range(n)], [p for n in lens for p in range(n)], [p for n in lens for p in range(n)])
        out = torch.empty(q.shape, device=self.device)
        sd.paged_prefill_attention(self._shape(), q, self._int(starts), starts[-1], max(lens), self.k_pages, self.v_pages, None, None, self._table(),
                                   self._int(lens), self.layer.head_dim ** -0.5, out)
        # the last tokens' weights stand for what later ones look at
        rows, w = [], [0]
        for b, n in enumerate(lens):
            rows += range(starts[b + 1] - min(n, self.window), starts[b + 1])
            w.append(len(rows))
        self._accumulate(q[torch.tensor(rows, device=self.device)], self._int(w), len(rows), min(self.window, max(lens)), 0, None)
        self._evict()
        return out

    def step(self, hidden):
        """One more token of every sequence; -> the attention's rows."""
        B = len(self.lens)
        slots = list(self.lens)
        for b in range(B):
            self.lens[b] += 1
            self._grow(b, self.lens[b])
        q = self._append(hidden, list(range(B)), self.positions, slots)
        if self.cached is not None:
            for b in range(B):
                self.cached[b] = [c + [self.positions[b]] for c in self.cached[b]]
        self.positions = [p + 1 for p in self.positions]
        shape = self._shape()
        out = torch.empty(q.shape, device=self.device)
        ws = sd.workspace_bytes(shape)
        workspace = torch.empty(ws, dtype=torch.uint8, device=self.device)
        sd.paged_decode_attention(shape, q, self.k_pages, self.v_pages, None, None, self._table(), self._int(self.lens), self.layer.head_dim ** -0.5, out,
                                  workspace, ws)
        self._accumulate(q, None, B, 1, 1, self.scores)
        self._evict()
        return out

    def _evict(self):
        if max(self.lens) <= self.budget + self.slack:
            return
        shape, old_table, old = self._shape(), self._table(), self.pages
        kept_lens = [min(n, self.budget) for n in self.lens]
        self.pages = [[] for _ in old]
        for b, n in enumerate(kept_lens):
            self._grow(b, n)
        kept = torch.empty((len(old), self.layer.kv_heads, self.budget), dtype=torch.int32, device=self.device)
        new_lens = torch.empty(len(old), dtype=torch.int32, device=self.device)
        sd.kv_evict(shape, self.budget, self.sinks, self.recent, self.scores, self.stride, self.k_pages, self.v_pages, None, None, old_table,
                    self._int(self.lens), self._table(), kept, new_lens, self.scores, self.stride)
        if self.cached is None:
            self.cached = [[list(range(n)) for _ in range(self.layer.kv_heads)] for n in self.lens]
        for b, rows in enumerate(kept.tolist()):
            self.cached[b] = [[c[i] for i in row[:kept_lens[b]]] for c, row in zip(self.cached[b], rows)]
        self.lens = kept_lens
        for pages in old:
            self.free += pages   # (the pool's next writer is on the same stream)


def learn(layer, hidden, positions):
    """Gradients of the projection and of the norms' weights for one pass over whole trajectories (here of the mean square of what
    the attention is given)."""
    projection, qw, kw = (t.detach().requires_grad_() for t in (layer.projection, layer.q_weight, layer.k_weight))
    q, k = NormRope.apply(hidden @ projection, qw, kw, layer.table, positions, layer.norm)
    loss = q.float().square().mean() + k.float().square().mean()
    loss.backward()
    return loss.detach(), projection.grad, qw.grad, kw.grad


def main():
    torch.manual_seed(0)
    layer = Layer(hidden=512, heads=28, kv_heads=4, head_dim=128, max_positions=4096)
    lengths = [700, 33, 1500, 260]
    rollout = Rollout(layer, lengths, budget=512, sinks=4, recent=128, slack=64, window=32)
    hidden = [torch.randn(sum(lengths), 512, device="cuda").bfloat16()]
    rollout.prompt(hidden[0])
    print("prompts of", lengths, "hold", rollout.lens, "tokens,", rollout.num_pages - len(rollout.free), "pages in use")
    for step in range(200):
        hidden.append(torch.randn(len(lengths), 512, device="cuda").bfloat16())
        rollout.step(hidden[-1])
    print("after 200 tokens more they hold", rollout.lens, "of", rollout.positions, "tokens,", rollout.num_pages - len(rollout.free), "pages in use")
    rows = torch.cat(hidden)
    positions = torch.tensor([p for n in lengths for p in range(n)] + [n + s for s in range(200) for n in lengths], dtype=torch.int32, device="cuda")
    loss, dp, dq, dk = learn(layer, rows, positions)
    print("loss %.4f, gradients' norms: projection %.3e, queries' norm %.3e, keys' norm %.3e" % (loss, dp.float().norm(), dq.float().norm(), dk.float().norm()))


if __name__ == "__main__":
    main()
