"""Sampling, log probabilities and the plan of a step where sizes are large, streams differ and graphs share a workspace."""
import numpy as np
import pytest

from tests.test_gpu_operator_streams import same

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sd():
    import torch
    assert torch.cuda.is_available()
    import paper_2508_11553_amd as m
    m.load()
    return m


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_rows_beyond_32_bit_offsets(sd, kind):
    """Five rows 2^30 + 9 elements apart, what lies between them never touched: tokens, log probabilities and the gradient in place as those of the rows side by side."""
    import torch
    rows, vocab, stride = 5, 3001, 2 ** 30 + 9
    gen = torch.Generator(device="cuda").manual_seed(1)
    dtype = torch.bfloat16 if kind == "bf16" else torch.float32
    near = (3 * torch.randn((rows, vocab), generator=gen, device="cuda")).to(dtype)
    far = torch.full(((rows - 1) * stride + vocab,), float("nan"), dtype=dtype, device="cuda")
    view = far.as_strided((rows, vocab), (stride, 1))
    view.copy_(near)
    u, t = torch.rand(rows, generator=gen, device="cuda"), 0.5 + torch.rand(rows, generator=gen, device="cuda")
    p = torch.full((rows,), 0.9, device="cuda")
    targets = torch.tensor([0, 7, -1, 3000, 55], dtype=torch.int32, device="cuda")
    g, h = torch.randn(rows, generator=gen, device="cuda"), torch.randn(rows, generator=gen, device="cuda")
    results = []
    for x, gap in ((near, 0), (far, stride)):
        s = sd.Logits(rows=rows, vocab=vocab, dtype=sd.SD_BF16 if kind == "bf16" else sd.SD_F32, stride=gap)
        n = max(sd.sample_workspace_bytes(s), sd.token_logprobs_workspace_bytes(s))
        work = torch.empty(n, dtype=torch.uint8, device="cuda")
        out = [torch.zeros(rows, dtype=torch.int32, device="cuda")] + [torch.zeros(rows, device="cuda") for _ in range(4)] + [torch.zeros((rows, 2), device="cuda")]
        plainly = torch.zeros(rows, dtype=torch.int32, device="cuda")
        sd.sample_tokens(s, x, t, None, p, None, u, out[0], out[1], out[2], work, n)
        sd.sample_tokens(s, x, t, None, None, None, u, plainly, None, None, work, n)
        sd.token_logprobs(s, x, targets, t, out[3], out[4], out[5], work, n)
        sd.token_logprobs_backward(s, x, targets, t, out[5], out[4], g, h, x)
        results.append(out + [plainly, (view if gap else near).clone()])
    assert all(same(*results))
    assert torch.isnan(far[vocab:stride]).all() and torch.isnan(far[3 * stride + vocab:4 * stride]).all()
    assert results[0][0].unique().numel() > 1 and results[0][-1][:2].abs().max() > 0


def test_many_rows_beyond_32_bit_offsets(sd):
    """More than 2^32 logits side by side: the last rows as those of a call of their own."""
    import torch
    vocab, rows, tail = 131072, 2 ** 15 + 40, 6
    x = torch.empty((rows, vocab), dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(2)
    x[:-tail] = 0
    x[-tail:] = 3 * torch.randn((tail, vocab), generator=gen, device="cuda")
    targets = torch.randint(0, vocab, (rows,), generator=gen, device="cuda").int()
    u = torch.rand(rows, generator=gen, device="cuda")
    results = []
    for first in (0, rows - tail):
        n = rows - first
        s = sd.Logits(rows=n, vocab=vocab, dtype=sd.SD_BF16, stride=0)
        size = max(sd.sample_workspace_bytes(s), sd.token_logprobs_workspace_bytes(s))
        work = torch.empty(size, dtype=torch.uint8, device="cuda")
        tokens, lp = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, device="cuda")
        k = torch.full((n,), 100, dtype=torch.int32, device="cuda")
        limited, scored, H = torch.zeros_like(tokens), torch.zeros_like(lp), torch.zeros_like(lp)
        sd.sample_tokens(s, x[first:], None, None, None, None, u[first:].clone(), tokens, lp, None, work, size)
        sd.sample_tokens(s, x[first:], None, k, None, None, u[first:].clone(), limited, None, None, work, size)
        sd.token_logprobs(s, x[first:], targets[first:].clone(), None, scored, H, None, work, size)
        results.append([y[-tail:].cpu().numpy() for y in (tokens, lp, limited, scored, H)])
        if not first:
            assert (abs(scored[:-tail] + np.log(vocab)) <= 1e-5).all() and torch.equal(tokens[:-tail], (u[:-tail].double() * vocab).int())
            assert torch.equal(limited[:-tail], (u[:-tail].double() * 100).int())      # of equal logits the first hundred
    for a, b in zip(*results[:2]):
        if a.dtype == np.int32:
            assert np.array_equal(a, b)
        else:   # (a row alone is cut into parts, whose sums are added in another order: each adds at most 2^17 / 512 half steps)
            assert abs(a - b).max() <= 2.0 ** -24 * (2 * 300 + 60) * 12
    assert np.array_equal(results[0][1], results[1][1])      # what is drawn does not depend on the batch


class Calls:
    """Every operator of the loop, small; run(stream) enqueues them, inputs: what they read, outputs: what they write."""

    def __init__(self, sd, rows=5, vocab=4099):
        import torch
        self.sd, self.rows = sd, rows
        empty = lambda *s, kind=torch.float32: torch.zeros(s, dtype=kind, device="cuda")  # noqa: E731
        i32 = torch.int32
        self.desc = sd.Logits(rows=rows, vocab=vocab, dtype=sd.SD_BF16, stride=0)
        self.x, self.u = empty(rows, vocab, kind=torch.bfloat16), empty(rows)
        self.t, self.k, self.p, self.m = torch.full((rows,), 0.9, device="cuda"), torch.full((rows,), 40, dtype=i32, device="cuda"), torch.full((rows,), 0.97, device="cuda"), torch.full((rows,), 0.001, device="cuda")
        self.g, self.h = empty(rows), empty(rows)
        self.tokens, self.more = empty(rows, kind=i32), empty(rows, kind=i32)
        self.lp, self.dlp, self.score, self.H, self.stats, self.d = empty(rows), empty(rows), empty(rows), empty(rows), empty(rows, 2), empty(rows, vocab, kind=torch.bfloat16)
        self.shapes = [sd.Shape(batch=B, num_q_heads=8, num_kv_heads=8, head_dim=64, page_size=16, num_pages=4000, max_blocks_per_seq=9, kv_dtype=sd.SD_BF16, max_context_len=144,
                                chunk_tokens=0) for B in (rows, 1200)]
        self.asks = [empty(s.batch, kind=i32) for s in self.shapes]
        self.places = [[empty(s.batch, kind=i32) for _ in range(3)] + [empty(s.batch + 1, kind=i32), empty(1, kind=i32), empty(4000, kind=i32), empty(s.batch, 9, kind=i32)]
                       + [empty(4000, kind=i32) for _ in range(3)] for s in self.shapes]
        self.sizes = [sd.sample_workspace_bytes(self.desc), sd.token_logprobs_workspace_bytes(self.desc)] + [sd.kv_plan_workspace_bytes(s) for s in self.shapes]
        self.work = empty(max(self.sizes), kind=torch.uint8)                 # one for all: the calls of a stream come one after the other
        self.inputs = [self.x, self.u, self.g, self.h] + self.asks
        self.outputs = [self.tokens, self.more, self.lp, self.dlp, self.score, self.H, self.stats, self.d] + [x for p in self.places for x in p]

    def run(self, stream=None):
        sd, w, n = self.sd, self.work, self.sizes
        sd.sample_tokens(self.desc, self.x, self.t, self.k, self.p, self.m, self.u, self.tokens, self.lp, self.dlp, w, n[0], stream=stream)
        sd.sample_tokens(self.desc, self.x, self.t, None, None, None, self.u, self.more, None, None, w, n[0], stream=stream)
        sd.token_logprobs(self.desc, self.x, self.tokens, self.t, self.score, self.H, self.stats, w, n[1], stream=stream)
        sd.token_logprobs_backward(self.desc, self.x, self.tokens, self.t, self.stats, self.H, self.g, self.h, self.d, stream=stream)
        for s, asks, (granted, starts, lens, row_start, free, pages, table, seq, slots, positions), size in zip(self.shapes, self.asks, self.places, n[2:]):
            sd.kv_plan_step(s, asks, None, lens, lens, None, None, pages, free, free, table, 4000, granted, row_start, starts, seq, slots, positions, w, size, stream=stream)

    def fresh(self, seed):
        import torch
        gen = torch.Generator(device="cuda").manual_seed(seed)
        new = [3 * torch.randn(self.x.shape, generator=gen, device="cuda"), torch.rand(self.rows, generator=gen, device="cuda")]
        new += [torch.randn(self.rows, generator=gen, device="cuda") for _ in range(2)]
        return new + [torch.randint(-1, 5, a.shape, generator=gen, device="cuda").int() for a in self.asks]

    def set(self, values):
        for x, y in zip(self.inputs, values):
            x.copy_(y)

    def clear(self):
        """Empty tables, all pages free."""
        import torch
        for x in self.outputs:
            x.zero_()
        for p in self.places:
            p[4].fill_(4000)
            p[5].copy_(torch.arange(4000, dtype=torch.int32, device="cuda"))

    def results(self):
        import torch
        torch.cuda.synchronize()
        return [x.clone() for x in self.outputs]


@pytest.mark.parametrize("given", [True, False])
def test_calls_follow_what_their_stream_holds(sd, given):
    """Behind work that takes some 50 ms on the side stream the inputs change there; the calls come after that change."""
    import torch
    c = Calls(sd)
    old, new = c.fresh(1), c.fresh(2)
    c.set(old)
    c.clear()
    c.run()
    stale = c.results()
    c.clear()
    c.set(new)
    c.run()
    want = c.results()
    assert not any(same(stale[2:8], want[2:8]))
    side = torch.cuda.Stream()
    a = torch.randn(8192, 8192, device="cuda").bfloat16()
    b = torch.empty_like(a)
    for _ in range(2):
        c.set(old)
        c.clear()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(40):
                torch.mm(a, a, out=b)
            c.set(new)
            if not given:
                c.run()
        if given:
            c.run(stream=side)
        side.synchronize()
        assert all(same(c.results(), want))


def test_two_graphs_share_a_workspace(sd):
    """Two sets of calls, captured each into a graph, their workspace the same: replayed in turn with other inputs, with eager calls between."""
    import torch
    calls = [Calls(sd), Calls(sd)]
    calls[1].work = calls[0].work
    graphs = []
    for c in calls:
        c.clear()
        c.run()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c.run()
        graphs.append(graph)
    for seed in range(3):
        want = []
        for i, c in enumerate(calls):
            c.set(c.fresh(10 * seed + i))
            c.clear()
            c.run()
            want.append(c.results())
            c.clear()
        torch.cuda.synchronize()
        for graph in graphs:
            graph.replay()
        for c, w in zip(calls, want):
            assert all(same(c.results(), w))


def test_two_streams_at_once(sd):
    """Two sets of calls, each with its own workspace, side by side."""
    import torch
    calls, streams = [Calls(sd) for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    want = []
    for i, c in enumerate(calls):
        c.set(c.fresh(i))
        c.clear()
        c.run()
        want.append(c.results())
    for _ in range(5):
        for c in calls:
            c.clear()
        torch.cuda.synchronize()
        for c, s in zip(calls, streams):
            c.run(stream=s)
        for c, w in zip(calls, want):
            assert all(same(c.results(), w))


def test_the_workspace_of_the_largest_call_and_no_byte_more(sd):
    """Bytes behind each call's workspace stay as they are, for a larger call's workspace too."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(4)
    for kind, flag in ((torch.bfloat16, sd.SD_BF16), (torch.float32, sd.SD_F32)):
        for rows, vocab in ((1, 1), (1, 2049), (3, 5000), (130, 300), (7, 131072)):
            x = (3 * torch.randn((rows, vocab), generator=gen, device="cuda")).to(kind)
            s = sd.Logits(rows=rows, vocab=vocab, dtype=flag, stride=0)
            u, p = torch.rand(rows, generator=gen, device="cuda"), torch.full((rows,), 0.8, device="cuda")
            tokens, out = torch.zeros(rows, dtype=torch.int32, device="cuda"), [torch.zeros(rows, device="cuda") for _ in range(3)]
            for n, call in ((sd.sample_workspace_bytes(s), lambda w, n: sd.sample_tokens(s, x, None, None, p, None, u, tokens, out[0], None, w, n)),
                            (sd.token_logprobs_workspace_bytes(s), lambda w, n: sd.token_logprobs(s, x, tokens, None, out[1], out[2], None, w, n))):
                work = torch.full((n + 4096,), 0xa5, dtype=torch.uint8, device="cuda")
                call(work, n)
                assert (work[n:] == 0xa5).all()
    s = sd.Shape(batch=5003, num_q_heads=8, num_kv_heads=8, head_dim=64, page_size=16, num_pages=20000, max_blocks_per_seq=3, kv_dtype=sd.SD_BF16, max_context_len=48, chunk_tokens=0)
    n = sd.kv_plan_workspace_bytes(s)
    work = torch.full((n + 4096,), 0xa5, dtype=torch.uint8, device="cuda")
    i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")  # noqa: E731
    lens, free = i32(5003), torch.full((1,), 20000, dtype=torch.int32, device="cuda")
    sd.kv_plan_step(s, i32(5003) + 2, None, lens, lens, None, None, torch.arange(20000, dtype=torch.int32, device="cuda"), free, free, i32(5003, 3), 10006, i32(5003), i32(5004), i32(5003),
                    i32(10006), i32(10006), i32(10006), work, n)
    assert (lens == 2).all() and free.item() == 20000 - 5003 and (work[n:] == 0xa5).all()
