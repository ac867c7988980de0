"""A rollout whose whole step is one captured graph, and a training step on what it drew.

Between two decode steps nothing goes through the host: tokens are drawn from the logits (sample_tokens), sequences that ended give their pages
back and the others get places for their new tokens (kv_plan_step), keys and values go there (qk_norm_rope_append) and are attended
(paged_decode_attention).  Where the pool runs short a sequence waits with its token until another one ends.  At the end the log probabilities of all
that was drawn are computed again, with their gradient, and enter a clipped objective (TokenLogprobs).

    python examples/captured_rollout.py
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import paper_2508_11553_amd as sd  # noqa: E402
from bounded_rollout import PAGE, Layer, NormRope  # noqa: E402


def side_by_side(x):
    """x as the calls take it: without gaps, from 16 bytes on."""
    return x if x is None or (x.is_contiguous() and x.data_ptr() % 16 == 0) else x.clone(memory_format=torch.contiguous_format)


class TokenLogprobs(torch.autograd.Function):
    """Log probabilities of `targets` [T] (< 0: padding) under the rows of `logits` [T][vocab], and the rows' entropies."""

    @staticmethod
    def forward(ctx, logits, targets, temperature):
        if logits.dtype not in (torch.bfloat16, torch.float32) or targets.dtype != torch.int32 or (temperature is not None and temperature.dtype != torch.float32):
            raise TypeError("logits are bf16 or fp32, targets int32, temperatures fp32")
        if logits.dim() != 2 or logits.shape[1] == 0 or targets.shape != logits.shape[:1] or (temperature is not None and temperature.shape != targets.shape):
            raise ValueError("logits are [T][vocab], targets and temperatures [T]")
        rows, vocab = logits.shape
        # (the calls take rows of logits that lie apart, but no other gaps)
        taken = logits.stride(1) == 1 and logits.stride(0) >= vocab and logits.data_ptr() % 16 == 0
        logits = logits if taken else logits.clone(memory_format=torch.contiguous_format)
        targets, temperature = side_by_side(targets), side_by_side(temperature)
        desc = sd.Logits(rows=rows, vocab=vocab, dtype=sd.SD_BF16 if logits.dtype == torch.bfloat16 else sd.SD_F32, stride=logits.stride(0) if taken else 0)
        logprobs, entropy = (torch.empty(rows, device=logits.device) for _ in range(2))
        stats = torch.empty((rows, 2), device=logits.device)
        ws = sd.token_logprobs_workspace_bytes(desc)
        sd.token_logprobs(desc, logits, targets, temperature, logprobs, entropy, stats, torch.empty(ws, dtype=torch.uint8, device=logits.device), ws)
        ctx.save_for_backward(logits, targets, temperature, stats, entropy)
        ctx.desc = desc
        return logprobs, entropy

    @staticmethod
    def backward(ctx, d_logprobs, d_entropy):
        logits, targets, temperature, stats, entropy = ctx.saved_tensors
        d_logits = torch.empty_strided(logits.shape, logits.stride(), dtype=logits.dtype, device=logits.device)
        sd.token_logprobs_backward(ctx.desc, logits, targets, temperature, stats, entropy, side_by_side(d_logprobs), side_by_side(d_entropy), d_logits)
        return d_logits, None, None


class Model(Layer):
    """One attention layer between an embedding and a head, random."""

    def __init__(self, vocab, hidden, heads, kv_heads, head_dim, max_positions, seed=0, device="cuda:0"):
        super().__init__(hidden, heads, kv_heads, head_dim, max_positions, seed, device)
        gen = torch.Generator().manual_seed(seed + 1)
        self.vocab, self.hidden = vocab, hidden
        self.embedding = torch.randn(vocab, hidden, generator=gen).bfloat16().to(device)
        self.output = (torch.randn(heads * head_dim, hidden, generator=gen) / math.sqrt(heads * head_dim)).bfloat16().to(device)
        self.head = (2 * torch.randn(hidden, vocab, generator=gen) / math.sqrt(hidden)).bfloat16().to(device)


class Rollout:
    """A batch of sequences: `uniform` [max_new][B] are the random numbers, temperature, top_k and top_p [B] the rows' limits."""

    def __init__(self, model, prompts, max_new, pages, stop, uniform, temperature, top_k=None, top_p=None, device="cuda:0"):
        if not prompts or not all(len(p) for p in prompts) or max_new < 1:
            raise ValueError("every prompt has a token at least, and one is drawn for it")
        if uniform.shape != (max_new, len(prompts)):
            raise ValueError("uniform is [max_new][B]")
        self.model, self.stop, self.max_new, self.device = model, stop, max_new, torch.device(device)
        self.uniform, self.temperature, self.top_k, self.top_p = uniform, temperature, top_k, top_p
        B, d = len(prompts), model.head_dim
        self.B, self.prompts, self.graph = B, prompts, None
        blocks = (max(len(p) for p in prompts) + max_new + PAGE - 1) // PAGE
        self.shape = sd.Shape(batch=B, num_q_heads=model.heads, num_kv_heads=model.kv_heads, head_dim=d, page_size=PAGE, num_pages=pages, max_blocks_per_seq=blocks,
                              kv_dtype=sd.SD_BF16, max_context_len=PAGE * blocks, chunk_tokens=0)
        self.desc = sd.Logits(rows=B, vocab=model.vocab, dtype=sd.SD_BF16, stride=0)
        self.k_pages, self.v_pages = (torch.zeros((pages, model.kv_heads, PAGE, d), dtype=torch.bfloat16, device=device) for _ in range(2))
        i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=device)  # noqa: E731
        self.free_pages, self.free = torch.arange(pages, dtype=torch.int32, device=device), torch.full((1,), pages, dtype=torch.int32, device=device)
        self.table, self.lens, self.starts, self.granted, self.row_start = i32(B, blocks), i32(B), i32(B), i32(B), i32(B + 1)
        self.asks, self.token, self.drawn, self.count = i32(B), i32(B), i32(B), i32(B)
        self.alive, self.waits = torch.ones(B, dtype=torch.bool, device=device), torch.zeros(B, dtype=torch.bool, device=device)
        self.seq, self.rows = torch.arange(B, dtype=torch.int32, device=device), [i32(B) for _ in range(3)]
        self.lp, self.dlp = (torch.zeros(B, device=device) for _ in range(2))
        self.logits, self.state = (torch.zeros((B, n), dtype=torch.bfloat16, device=device) for n in (model.vocab, model.hidden))
        self.q, self.attended = torch.zeros((B, model.heads, d), dtype=torch.bfloat16, device=device), torch.zeros((B, model.heads, d), device=device)
        # what was drawn: tokens (-1: nothing), their log probabilities and the states that they were drawn from; a last column for nobody
        self.answers, self.logprobs = torch.full((B, max_new + 1), -1, dtype=torch.int32, device=device), torch.zeros((B, max_new + 1), device=device)
        self.states = torch.zeros((B, max_new + 1, model.hidden), dtype=torch.bfloat16, device=device)
        self.sizes = sd.sample_workspace_bytes(self.desc), sd.kv_plan_workspace_bytes(self.shape), sd.workspace_bytes(self.shape)
        self.spaces = [torch.empty(max(n, 16), dtype=torch.uint8, device=device) for n in self.sizes]

    def _plan(self, max_rows, seq_ids, slots, positions):
        sd.kv_plan_step(self.shape, self.asks, None, self.lens, self.lens, None, None, self.free_pages, self.free, self.free, self.table, max_rows, self.granted,
                        self.row_start, self.starts, seq_ids, slots, positions, self.spaces[1], self.sizes[1])

    def _append(self, x, positions, seq_ids, slots, q):
        model = self.model
        qkv = x @ model.projection
        qx, kx = NormRope.parts(qkv, model.norm)
        sd.qk_norm_rope_append(self.shape, model.norm, qx, kx, model.values(qkv), model.q_weight, model.k_weight, model.table, positions, seq_ids, slots, x.shape[0], q,
                               self.k_pages, self.v_pages, self.table)

    def _finish(self, x, attended):
        state = x + attended.flatten(1).bfloat16() @ self.model.output
        self.state.copy_(state)
        torch.mm(state, self.model.head, out=self.logits)

    def prompt(self):
        """The prompts into the cache; their last tokens' logits."""
        model, lengths = self.model, [len(p) for p in self.prompts]
        rows = sum(lengths)
        self.asks.copy_(torch.tensor(lengths, dtype=torch.int32))
        seq_ids, slots, positions = (torch.empty(rows, dtype=torch.int32, device=self.device) for _ in range(3))
        self._plan(rows, seq_ids, slots, positions)
        if self.granted.tolist() != lengths:
            raise RuntimeError("the pool does not hold the prompts")
        x = model.embedding[torch.tensor([t for p in self.prompts for t in p], device=self.device)]
        q = torch.empty((rows, model.heads, model.head_dim), dtype=torch.bfloat16, device=self.device)
        self._append(x, positions, seq_ids, slots, q)
        out = torch.empty(q.shape, device=self.device)
        sd.paged_prefill_attention(self.shape, q, self.row_start, rows, max(lengths), self.k_pages, self.v_pages, None, None, self.table, self.lens, model.head_dim ** -0.5, out)
        last = (self.row_start[1:] - 1).long()
        self._finish(x[last], out[last])

    def step(self):
        """Draws a token for every sequence that goes on and takes it into the cache."""
        model, B = self.model, self.B
        u = self.uniform.gather(0, self.count.clamp(max=self.max_new - 1).long()[None])[0]
        sd.sample_tokens(self.desc, self.logits, self.temperature, self.top_k, self.top_p, None, u, self.drawn, self.lp, self.dlp, self.spaces[0], self.sizes[0])
        # who waits still has its token; the others' are written down
        new = self.alive & ~self.waits
        at = torch.where(new, self.count, self.max_new).long()[:, None]
        self.answers.scatter_(1, at, self.drawn[:, None])
        self.logprobs.scatter_(1, at, self.lp[:, None])
        self.states.scatter_(1, at[:, :, None].expand(B, 1, model.hidden), self.state[:, None])
        self.token.copy_(torch.where(new, self.drawn, self.token))
        self.count.add_(new)
        ends = new & ((self.token == self.stop) | (self.count == self.max_new))
        self.alive.logical_and_(~ends)
        self.asks.copy_(self.alive.int() - ends.int())
        self._plan(B, *self.rows)
        served = self.granted > 0
        self.waits.copy_(self.alive & ~served)
        x = model.embedding[self.token.long()]
        self._append(x, self.starts, torch.where(served, self.seq, -1), self.starts, self.q)
        sd.paged_decode_attention(self.shape, self.q, self.k_pages, self.v_pages, None, None, self.table, self.lens, model.head_dim ** -0.5, self.attended, self.spaces[2],
                                  self.sizes[2])
        self._finish(x, self.attended)

    def capture(self):
        """After one step, so that the libraries have what they need: every further one replays its graph."""
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self.step()

    def run(self, look_every=16):
        """Until all sequences have ended; -> steps taken."""
        self.prompt()
        self.step()
        self.capture()
        steps = 1
        while True:
            alive, waits = self.alive.tolist(), self.waits.tolist()
            if not any(alive):
                return steps
            if all(w for a, w in zip(alive, waits) if a):
                raise RuntimeError("every sequence waits for pages")
            for _ in range(look_every):
                self.graph.replay()
            steps += look_every


def learn(model, states, answers, logprobs, advantage, temperature, clip=0.2, entropy_bonus=0.01):
    """The head's gradient of the clipped objective over all drawn tokens ([B][n], -1: none); -> (loss, log probabilities now, gradient)."""
    B, n = answers.shape
    head = model.head.detach().requires_grad_()
    lp, entropy = TokenLogprobs.apply(states.reshape(B * n, -1) @ head, answers.reshape(-1).contiguous(), temperature[:, None].expand(B, n).reshape(-1).contiguous())
    real = (answers >= 0).reshape(-1)
    a = advantage[:, None].expand(B, n).reshape(-1)
    ratio = torch.exp(torch.where(real, lp - logprobs.reshape(-1), 0.0))
    gain = torch.minimum(ratio * a, ratio.clamp(1 - clip, 1 + clip) * a)
    loss = -(torch.where(real, gain, 0.0).sum() + entropy_bonus * entropy.sum()) / real.sum()
    loss.backward()
    return loss.detach(), lp.detach().view(B, n), head.grad


def main():
    torch.manual_seed(0)
    model = Model(vocab=32000, hidden=512, heads=28, kv_heads=4, head_dim=128, max_positions=4096)
    B, max_new = 48, 200
    prompts = [torch.randint(0, 32000, (n,)).tolist() for n in torch.randint(5, 900, (B,)).tolist()]
    held = sum((len(p) + PAGE - 1) // PAGE for p in prompts)
    temperature = torch.full((B,), 0.8, device="cuda")
    rollout = Rollout(model, prompts, max_new, pages=held + 560, stop=7, uniform=torch.rand(max_new, B, device="cuda"), temperature=temperature,
                      top_p=torch.full((B,), 0.95, device="cuda"))
    steps = rollout.run()
    print("%d sequences drew %d tokens in %d steps, %d of %d pages free" % (B, int(rollout.count.sum()), steps, rollout.free.item(), held + 560))
    advantage = torch.randn(B, device="cuda")
    answers, logprobs, states = rollout.answers[:, :max_new], rollout.logprobs[:, :max_new], rollout.states[:, :max_new]
    loss, lp, grad = learn(model, states, answers, logprobs, advantage, temperature)
    print("loss %.4f, the gradient's norm %.3e, log probabilities differ by at most %.1e" % (loss, grad.float().norm(), (lp - logprobs)[answers >= 0].abs().max()))


if __name__ == "__main__":
    main()
