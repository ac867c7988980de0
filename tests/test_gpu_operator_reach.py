"""Where the operators around the decode step reach: pools and scores beyond 32-bit offsets, replays of a captured graph, another stream."""
import numpy as np
import pytest

from tests.test_gpu_norm_rope import Rows
from tests.test_gpu_weight_scores import Cache, queries

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sd():
    import torch
    assert torch.cuda.is_available()
    import paper_2508_11553_amd as m
    m.load()
    return m


def shape_of(sd, B, hq, hkv, d, pages, blocks, bound, kv="bf16"):
    return sd.Shape(batch=B, num_q_heads=hq, num_kv_heads=hkv, head_dim=d, page_size=16, num_pages=pages, max_blocks_per_seq=blocks,
                    kv_dtype=sd.SD_FP8_E4M3 if kv == "fp8" else sd.SD_BF16, max_context_len=bound, chunk_tokens=0)


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
def test_pools_and_scores_beyond_32_bit_offsets(sd, kv):
    """The same sequences in the last pages of pools of more than 4 GB, with scores of more than 2^31 entries, as in small ones: bit for bit."""
    import torch
    B, hq, hkv, d, L, budget = 5, 8, 2, 128, 300, 70
    tile = 16 * d * (2 if kv == "bf16" else 1)
    many = (5 << 30) // (hkv * tile)
    blocks, kept = (L + 15) // 16, (budget + 15) // 16
    gen = torch.Generator().manual_seed(1)
    kind = torch.bfloat16 if kv == "bf16" else torch.uint8
    # (bytes below 0x78: finite codes, finite bf16)
    data = [(torch.randint(0, 0x78, (B * blocks, hkv, 16, d), generator=gen, dtype=torch.uint8) if kv == "fp8"
             else torch.randn(B * blocks, hkv, 16, d, generator=gen).bfloat16()) for _ in range(2)]
    scale_data = [torch.rand(B * blocks, hkv, generator=gen) + 0.01 for _ in range(2)]
    q = queries(B, hq, d, 2)
    results = []
    for pages, stride in ((B * (blocks + kept), L), (many, 1 << 28)):
        first = pages - B * (blocks + kept)
        pools = [torch.empty(pages, hkv, 16, d, dtype=kind, device="cuda") for _ in range(2)]
        scales = [torch.empty(pages, hkv, device="cuda") for _ in range(2)]
        for p, s, x, y in zip(pools, scales, data, scale_data):
            p[first:first + B * blocks], s[first:first + B * blocks] = x.cuda(), y.cuda()
            p[first + B * blocks:] = 0
        table = torch.zeros(B, blocks, dtype=torch.int32)
        table[:] = first + torch.arange(B * blocks).view(B, blocks)
        new = torch.zeros(B, blocks, dtype=torch.int32)
        new[:, :kept] = first + B * blocks + torch.arange(B * kept).view(B, kept)
        table, new, lens = table.cuda(), new.cuda(), torch.full((B,), L, dtype=torch.int32, device="cuda")
        shape = shape_of(sd, B, hq, hkv, d, pages, blocks, L, kv)
        scores = torch.empty(B * hkv * stride, device="cuda")
        assert pages < many or (pools[0].numel() * pools[0].element_size() > 1 << 32 and scores.numel() > 1 << 31)
        ks, vs = scales if kv == "fp8" else (None, None)
        ws = sd.paged_weight_workspace_bytes(shape, 1)
        work = torch.empty(ws, dtype=torch.uint8, device="cuda")
        sd.paged_weight_accumulate(shape, q, None, B, 1, pools[0], ks, table, lens, d ** -0.5, 1.0, 0, None, scores, stride, work, ws)
        one = [scores[i * stride:i * stride + L].clone() for i in range(B * hkv)]
        kept_at, new_lens = torch.empty(B, hkv, budget, dtype=torch.int32, device="cuda"), torch.empty_like(lens)
        sd.kv_evict(shape, budget, 4, 20, scores, stride, *pools, ks, vs, table, lens, new, kept_at, new_lens, scores, stride)
        two = [scores[i * stride:i * stride + budget].clone() for i in range(B * hkv)]
        got = one + two + [kept_at, new_lens] + [p[first + B * blocks:].clone() for p in pools]
        if kv == "fp8":
            got += [s[first + B * blocks:].clone() for s in scales]
        else:
            r = Rows(sd, 6, hq, hkv, d, d, False, 9)
            seq, slots = torch.tensor([0, 1, 2, 3, 4, 4], dtype=torch.int32, device="cuda"), torch.tensor([0, 17, 70, 250, 100, 299], dtype=torch.int32, device="cuda")
            q_out = torch.empty(6, hq, d, dtype=torch.bfloat16, device="cuda")
            sd.qk_norm_rope_append(shape, r.norm, r.q, r.k, r.v, r.qw, r.kw, r.table, r.positions, seq, slots, 6, q_out, *pools, table)
            got += [q_out] + [p[first:].clone() for p in pools]
        results.append(got)
        del pools, scales, scores
        torch.cuda.empty_cache()
    for a, b in zip(*results):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_replays_of_a_captured_graph(sd):
    """Append, weights (one row and a window), eviction and the gradient, captured once: three replays with other inputs between, each equal to
    the eager calls on the same inputs."""
    import torch
    B, hq, hkv, d, L, budget = 3, 8, 2, 64, 500, 64
    c = Cache([L, 317, 5000], hkv, d, "bf16", 3)
    kept_blocks = (budget + 15) // 16
    extra = B * kept_blocks
    pools = [torch.cat([c.pool, torch.zeros(extra, *c.pool.shape[1:], dtype=c.pool.dtype, device="cuda")]) for _ in range(2)]
    shape = shape_of(sd, B, hq, hkv, d, c.pages + extra, c.max_blocks, 5000)
    dev = lambda a: torch.tensor(np.asarray(a, np.int32), device="cuda")  # noqa: E731
    table, lens = dev(c.table), dev(c.lens)
    new = dev(np.where(np.arange(c.max_blocks)[None] < kept_blocks, c.pages + np.arange(B)[:, None] * kept_blocks + np.arange(c.max_blocks)[None], 0))
    r = Rows(sd, B, hq, hkv, d, d, False, 4)
    slots, starts = dev([n - 1 for n in c.lens]), dev([0, 20, 25, 60])
    window = queries(60, hq, d, 5)
    q_out, k_out = torch.zeros(B, hq, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(B, hkv, d, dtype=torch.bfloat16, device="cuda")
    scores, more = torch.zeros(B, hkv, 5000, device="cuda"), torch.zeros(B, hkv, 5000, device="cuda")
    kept, new_lens, out = torch.zeros(B, hkv, budget, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, hkv, budget, device="cuda")
    ws = max(sd.paged_weight_workspace_bytes(shape, n) for n in (1, 35))
    work = torch.empty(ws, dtype=torch.uint8, device="cuda")
    gw = sd.qk_norm_rope_workspace_bytes(r.norm, B)
    grad_work, grads = torch.empty(gw, dtype=torch.uint8, device="cuda"), torch.zeros_like(r.all)
    dqw, dkw = torch.zeros(d, device="cuda"), torch.zeros(d, device="cuda")
    outputs = [q_out, scores, more, kept, new_lens, out, grads, dqw, dkw] + pools

    def calls():
        sd.qk_norm_rope_append(shape, r.norm, r.q, r.k, r.v, r.qw, r.kw, r.table, r.positions, None, slots, B, q_out, *pools, table)
        sd.paged_weight_accumulate(shape, q_out, None, B, 1, pools[0], None, table, lens, 0.125, 0.9, 1, None, scores, 5000, work, ws)
        sd.paged_weight_accumulate(shape, window, starts, 60, 35, pools[0], None, table, lens, 0.125, 0.9, 0, scores, more, 5000, work, ws)
        sd.kv_evict(shape, budget, 2, 16, more, 5000, *pools, None, None, table, lens, new, kept, new_lens, out, budget)
        sd.qk_norm_rope_backward(r.norm, q_out, k_out, r.q, r.k, r.qw, r.kw, r.table, r.positions, B, grads, grads[:, hq * d:], dqw, dkw, grad_work, gw)

    calls()   # once outside
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for seed in range(3):
        torch.manual_seed(seed)
        r.all.copy_(torch.randn_like(r.all.float()).bfloat16())
        window.copy_(torch.randn_like(window.float()).bfloat16())
        k_out.copy_(torch.randn_like(k_out.float()).bfloat16())
        calls()
        torch.cuda.synchronize()
        want = [x.clone() for x in outputs]
        for x in outputs[:9]:
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outputs, want):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_another_stream(sd):
    import torch
    c = Cache([900, 40], 2, 64, "bf16", 6)
    q = queries(2, 8, 64, 7)
    from tests.test_gpu_weight_scores import check, expected, run
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = run(sd, c, 8, q, None, 0.125, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    side.synchronize()
    check(got, expected(c, q.double().cpu().numpy(), [0, 1, 2], [900, 40], 0.125, 1.0, 1, None), [900, 40])
