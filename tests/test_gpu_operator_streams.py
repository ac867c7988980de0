"""The stream that a call is given, or the current one: where its inputs are still on their way there, a call on any other stream reads the old ones.
And graphs of the forms that test_gpu_operator_reach does not capture."""
import numpy as np
import pytest

from tests.test_gpu_norm_rope import Rows
from tests.test_gpu_operator_reach import shape_of
from tests.test_gpu_weight_scores import Cache, queries

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sd():
    import torch
    assert torch.cuda.is_available()
    import paper_2508_11553_amd as m
    m.load()
    return m


class Calls:
    """Every operator around the decode step, small; run(stream) enqueues them all, inputs: what they read, outputs: what they write."""

    def __init__(self, sd, B=3, hq=8, hkv=2, d=64, budget=64):
        import torch
        self.sd, self.B, self.hq, self.hkv, self.d, self.budget = sd, B, hq, hkv, d, budget
        self.lens = [500, 317, 900]
        c = Cache(self.lens, hkv, d, "bf16", 3)
        blocks = (budget + 15) // 16
        extra = torch.zeros(B * blocks, *c.pool.shape[1:], dtype=c.pool.dtype, device="cuda")
        self.pools = [torch.cat([torch.nan_to_num(c.pool), extra]) for _ in range(2)]
        self.bound = max(self.lens)
        self.shape = shape_of(sd, B, hq, hkv, d, c.pages + len(extra), c.max_blocks, self.bound)
        dev = lambda a: torch.tensor(np.asarray(a, np.int32), device="cuda")  # noqa: E731
        self.table, self.context = dev(c.table), dev(self.lens)
        at = np.arange(c.max_blocks)[None]
        self.new_table = dev(np.where(at < blocks, c.pages + np.arange(B)[:, None] * blocks + at, 0))
        self.r = Rows(sd, B, hq, hkv, d, d, False, 4)
        self.slots, self.starts = dev([n - 1 for n in self.lens]), dev([0, 80, 100, 200])
        self.window, self.most = queries(200, hq, d, 5), 100                 # 400 rows to a KV head: two rounds of them, joined by a launch
        empty = lambda *s, kind=torch.float32: torch.zeros(s, dtype=kind, device="cuda")  # noqa: E731
        self.q_out, self.q_rows, self.k_rows = empty(B, hq, d, kind=torch.bfloat16), empty(B, hq, d, kind=torch.bfloat16), empty(B, hkv, d, kind=torch.bfloat16)
        self.scores, self.more, self.out = empty(B, hkv, self.bound), empty(B, hkv, self.bound), empty(B, hkv, budget)
        self.kept, self.new_lens = empty(B, hkv, budget, kind=torch.int32), empty(B, kind=torch.int32)
        self.grads, self.dqw, self.dkw = torch.zeros_like(self.r.all), empty(d), empty(d)
        self.ws = max(sd.paged_weight_workspace_bytes(self.shape, n) for n in (1, self.most))
        self.gw = sd.qk_norm_rope_workspace_bytes(self.r.norm, B)
        self.work, self.grad_work = empty(self.ws, kind=torch.uint8), empty(self.gw, kind=torch.uint8)
        self.inputs = [self.r.all, self.window]
        self.outputs = [self.q_out, self.q_rows, self.k_rows, self.scores, self.more, self.out, self.kept, self.new_lens, self.grads, self.dqw, self.dkw] + self.pools

    def run(self, stream=None):
        sd, r, s = self.sd, self.r, self.shape
        norm = (r.q, r.k, r.qw, r.kw, r.table, r.positions)
        sd.qk_norm_rope(r.norm, *norm, self.B, self.q_rows, self.k_rows, stream=stream)
        sd.qk_norm_rope_append(s, r.norm, r.q, r.k, r.v, *norm[2:], None, self.slots, self.B, self.q_out, *self.pools, self.table, stream=stream)
        cache, step = (self.pools[0], None, self.table, self.context), (self.bound, self.work, self.ws)
        sd.paged_weight_accumulate(s, self.q_out, None, self.B, 1, *cache, 0.125, 0.9, 1, None, self.scores, *step, stream=stream)
        sd.paged_weight_accumulate(s, self.window, self.starts, 200, self.most, *cache, 0.125, 0.9, 0, self.scores, self.more, *step, stream=stream)
        sd.kv_evict(s, self.budget, 2, 16, self.more, self.bound, *self.pools, None, None, self.table, self.context, self.new_table, self.kept, self.new_lens, self.out,
                    self.budget, stream=stream)
        sd.qk_norm_rope_backward(r.norm, self.q_rows, self.k_rows, *norm, self.B, self.grads, self.grads[:, self.hq * self.d:], self.dqw, self.dkw, self.grad_work, self.gw,
                                 stream=stream)

    def fresh(self, seed):
        import torch
        gen = torch.Generator(device="cuda").manual_seed(seed)
        return [torch.randn(x.shape, generator=gen, device="cuda").bfloat16() for x in self.inputs]

    def set(self, values):
        for x, y in zip(self.inputs, values):
            x.copy_(y)

    def results(self):
        import torch
        torch.cuda.synchronize()
        return [x.clone() for x in self.outputs]

    def clear(self):
        for x in self.outputs[:-2]:
            x.zero_()


def same(a, b):
    import torch
    return [torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8)) for x, y in zip(a, b)]


@pytest.mark.parametrize("given", [True, False])
def test_calls_follow_what_their_stream_holds(sd, given):
    """Behind work that takes some 50 ms on the side stream the inputs change there; the calls come after that change."""
    import torch
    c = Calls(sd)
    old, new = c.fresh(1), c.fresh(2)
    c.set(old)
    c.run()
    stale = c.results()
    c.clear()
    c.set(new)
    c.run()
    want = c.results()
    assert not any(same(stale[:7], want[:7]))   # (the lengths do not depend on the inputs)
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


@pytest.mark.parametrize("given", [True, False])
def test_graphs(sd, given):
    """All of them captured, on the stream that they are given or on the current one: three replays with other inputs, each equal to the eager calls."""
    import torch
    c = Calls(sd)
    c.run()
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        c.run(stream=side if given else None)
    for seed in range(3):
        c.set(c.fresh(seed))
        c.run()
        want = c.results()
        c.clear()
        graph.replay()
        assert all(same(c.results(), want))
