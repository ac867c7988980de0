"""The operators around the decode step at the ends of their ranges: very long sequences, loose bounds on the query rows, large budgets."""
import pytest

from tests.test_gpu_operator_reach import shape_of
from tests.test_gpu_weight_scores import U, queries

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sd():
    import torch
    assert torch.cuda.is_available()
    import paper_2508_11553_amd as m
    m.load()
    return m


def weights_of(q, k, scale):
    """-> sums of the rows' weights over k [L][d] and their tolerances (derived in test_gpu_weight_scores), q [rows][d]; 64 bits"""
    x = scale * (q @ k.T)
    size = abs(scale) * (q.abs() @ k.abs().T).amax(1, keepdim=True)
    p = (x - x.amax(1, keepdim=True)).exp()
    p /= p.sum(1, keepdim=True)
    tol = (p * (3 * (k.shape[1] + 4) * size * U + (64 + x.abs().amax(1, keepdim=True)) * 2 * U) + 1e-37).sum(0)
    return p.sum(0), tol + p.sum(0) * 80 * U


@pytest.mark.parametrize("heads", [4, 8, 16, 32])
@pytest.mark.parametrize("L", [524288, 600001, 1100000])
def test_weights_of_more_than_half_a_million_tokens(sd, heads, L):
    """A wave of the first step takes as many pages as it has lanes, and then there are more workgroups.  Every page of a small pool many times."""
    import torch
    d, pages, blocks = 64, 500, (L + 15) // 16
    gen = torch.Generator().manual_seed(heads)
    pool = torch.randn(pages, 1, 16, d, generator=gen).bfloat16().cuda()
    table = torch.randint(0, pages, (1, blocks), generator=gen, dtype=torch.int32).cuda()
    q = queries(1, heads, d, 3)
    shape = shape_of(sd, 1, heads, 1, d, pages, blocks, L)
    stride = (L + 3) // 4 * 4
    out = torch.full((stride,), float("nan"), device="cuda")
    ws = sd.paged_weight_workspace_bytes(shape, 1)
    work = torch.empty(ws, dtype=torch.uint8, device="cuda").fill_(255)
    sd.paged_weight_accumulate(shape, q, None, 1, 1, pool, None, table, torch.tensor([L], dtype=torch.int32, device="cuda"), d ** -0.5, 1.0, 0, None, out, stride, work, ws)
    k = pool[:, 0].double()[table[0].long()].reshape(-1, d)[:L]
    want, tol = weights_of(q[0].double(), k, d ** -0.5)
    assert bool(((out[:L].double() - want).abs() <= tol).all())


@pytest.mark.parametrize("heads,kv_heads", [(8, 2), (16, 1), (32, 1)])
@pytest.mark.parametrize("total", [0, 1, 2, 5])
def test_a_bound_on_the_query_rows_that_few_rows_come_near(sd, heads, kv_heads, total):
    """The bytes that the bound asks for serve a call of fewer rows, which may take another path."""
    import torch
    d, L, most = 64, [3000, 41], 40
    blocks = (max(L) + 15) // 16
    gen = torch.Generator().manual_seed(total)
    pool = torch.randn(2 * blocks, kv_heads, 16, d, generator=gen).bfloat16().cuda()
    table = torch.randperm(2 * blocks, generator=gen).view(2, blocks).int().cuda()
    shape = shape_of(sd, 2, heads, kv_heads, d, 2 * blocks, blocks, max(L))
    q = queries(max(total, 1), heads, d, 8)
    first = total // 2
    starts = torch.tensor([0, first, total], dtype=torch.int32, device="cuda")
    before = torch.rand(2, kv_heads, max(L), device="cuda")
    out = torch.full_like(before, float("nan"))
    ws = sd.paged_weight_workspace_bytes(shape, most)
    work = torch.empty(ws, dtype=torch.uint8, device="cuda").fill_(255)
    sd.paged_weight_accumulate(shape, q, starts, total, most, pool, None, table, torch.tensor(L, dtype=torch.int32, device="cuda"), d ** -0.5, 0.5, 0, before, out, max(L), work, ws)
    for b, (lo, hi) in enumerate(((0, first), (first, total))):
        k = pool.double()[table[b].long()].transpose(1, 2).reshape(-1, kv_heads, d)[:L[b]]
        for g in range(kv_heads):
            want, tol = 0.5 * before[b, g, :L[b]].double(), 8 * U * torch.ones(L[b], dtype=torch.float64, device="cuda")
            for i in range(lo, hi):
                end, rows = L[b] - hi + i + 1, q[i, g * (heads // kv_heads):(g + 1) * (heads // kv_heads)].double()
                p, t = weights_of(rows, k[:end, g].contiguous(), d ** -0.5)
                want[:end] += p
                tol[:end] += t
            assert bool(((out[b, g, :L[b]].double() - want).abs() <= tol + 8 * U * want).all()), (b, g)


def test_the_largest_budget(sd):
    """2^31 - 1 places, of which a sequence fills 300."""
    import torch
    hkv, d, L, budget, blocks = 1, 64, 300, 2 ** 31 - 1, 19
    pools = [torch.randn(2 * blocks, hkv, 16, d, device="cuda").bfloat16() for _ in range(2)]
    old = pools[0][:blocks].clone()
    table, new = (torch.arange(i * blocks, (i + 1) * blocks, dtype=torch.int32, device="cuda").view(1, blocks) for i in range(2))
    lens, new_lens = torch.tensor([L], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    kept = torch.zeros(budget, dtype=torch.int32, device="cuda")
    sd.kv_evict(shape_of(sd, 1, 4, hkv, d, 2 * blocks, blocks, L), budget, 4, 20, torch.rand(1, hkv, L, device="cuda"), L, *pools, None, None, table, lens, new, kept, new_lens)
    assert torch.equal(kept[:L], torch.arange(L, dtype=torch.int32, device="cuda")) and int(kept[L:].max()) == int(kept[L:].min()) == -1
    assert int(new_lens) == L and torch.equal(pools[0][blocks:].view(-1, d)[:L], old.view(-1, d)[:L])


@pytest.mark.parametrize("batch", [1, 2, 63, 64, 65, 130])
@pytest.mark.parametrize("bound", [700, 20000])
def test_windows_of_as_many_sequences_as_a_wave_holds_and_more(sd, batch, bound):
    """Up to 64 sequences are dealt out by their lengths, more by the bound; lengths of zero, below the window and far below the bound."""
    import torch
    heads, kv_heads, d, most, longest = 8, 2, 64, 7, 700
    gen = torch.Generator().manual_seed(batch)
    lens = [int(x) for x in torch.randint(0, longest + 1, (batch,), generator=gen)]
    lens[0], lens[-1] = longest, 3 if batch > 1 else longest
    n = [int(x) for x in torch.randint(0, most + 1, (batch,), generator=gen)]
    starts = [sum(n[:i]) for i in range(batch + 1)]
    blocks = (bound + 15) // 16
    pool = torch.randn(batch * 44, kv_heads, 16, d, generator=gen).bfloat16().cuda()
    table = torch.full((batch, blocks), -1, dtype=torch.int32)
    table[:, :44] = torch.randperm(batch * 44, generator=gen).view(batch, 44)
    shape = shape_of(sd, batch, heads, kv_heads, d, batch * 44, blocks, bound)
    q = queries(max(starts[-1], 1), heads, d, 8)
    ws = sd.paged_weight_workspace_bytes(shape, most)
    work = torch.empty(ws, dtype=torch.uint8, device="cuda").fill_(255)
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    out = torch.full((batch, kv_heads, bound), -1.0, device="cuda")
    sd.paged_weight_accumulate(shape, q, dev(starts), starts[-1], most, pool, None, table.cuda(), dev(lens), d ** -0.5, 1.0, 0, None, out, bound, work, ws)
    for b, L in enumerate(lens):
        assert bool((out[b, :, L:] == -1).all())
        k = pool[table[b, :44].long().cuda()].double().transpose(1, 2).reshape(-1, kv_heads, d)[:L]
        for g in range(kv_heads):
            want, tol = torch.zeros(L, dtype=torch.float64, device="cuda"), torch.full((L,), 1e-37, dtype=torch.float64, device="cuda")
            for i in range(n[b]):
                end = L - n[b] + i + 1
                if end > 0:
                    p, t = weights_of(q[starts[b] + i, 4 * g:4 * g + 4].double(), k[:end, g].contiguous(), d ** -0.5)
                    want[:end] += p
                    tol[:end] += t
            assert bool(((out[b, g, :L].double() - want).abs() <= tol).all()), (b, g)


@pytest.mark.parametrize("batch,heads,most,d,kv", [(3, 8, 300, 64, "bf16"), (2, 16, 65, 128, "fp8"), (66, 16, 40, 64, "bf16"), (1, 64, 100, 64, "fp8")])
def test_rows_of_several_workgroups(sd, batch, heads, most, d, kv):
    """One KV head, up to 6400 rows: sequences with all of the bound's rows, with one and with none, windows longer than the sequence, scores in place."""
    import torch
    gen = torch.Generator().manual_seed(most)
    lens = [most + 500 - 37 * (b % 13) for b in range(batch)]
    n = [(most, 1, 0, most // 2, most)[b % 5] for b in range(batch)]
    lens[-1] = most - 7 if batch > 1 else lens[-1]   # rows of negative positions
    starts = [sum(n[:i]) for i in range(batch + 1)]
    bound, per = (max(lens) + 3) // 4 * 4, (max(lens) + 15) // 16
    tile = torch.randn(batch * per, 1, 16, d, generator=gen)
    scales = torch.rand(batch * per, 1, generator=gen) * 0.5 + 0.75 if kv == "fp8" else None
    pool = tile.to(torch.float8_e4m3fn if kv == "fp8" else torch.bfloat16).cuda()
    values = pool.double() * (scales.cuda().double()[:, :, None, None] if kv == "fp8" else 1.0)
    table = torch.randperm(batch * per, generator=gen).view(batch, per).int().cuda()
    shape = shape_of(sd, batch, heads, 1, d, batch * per, per, bound, kv)
    q = queries(starts[-1], heads, d, 9)
    scores = torch.rand(batch, 1, bound, device="cuda") * 3
    before = scores.clone().double()
    ws = sd.paged_weight_workspace_bytes(shape, most)
    work = torch.empty(ws, dtype=torch.uint8, device="cuda").fill_(255)
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    sd.paged_weight_accumulate(shape, q, dev(starts), starts[-1], most, pool.view(torch.uint8) if kv == "fp8" else pool, scales.cuda() if kv == "fp8" else None, table, dev(lens),
                               d ** -0.5, 0.75, 3, scores, scores, bound, work, ws)
    for b, L in enumerate(lens):
        k = values[table[b].long(), 0].reshape(-1, d)[:L]
        want = 0.75 * before[b, 0, :L]
        want[L - 3:] = 0
        tol = 8 * U * want + 1e-37
        pos = torch.arange(L - n[b], L, device="cuda").repeat_interleave(heads)
        x = d ** -0.5 * (q[starts[b]:starts[b + 1]].double().reshape(-1, d) @ k.T)
        size = d ** -0.5 * (q[starts[b]:starts[b + 1]].double().abs().reshape(-1, d) @ k.abs().T)
        seen = torch.arange(L, device="cuda")[None] <= pos[:, None]
        x, size, seen = x[pos >= 0], size[pos >= 0], seen[pos >= 0]
        if len(x):
            p = torch.softmax(x.masked_fill(~seen, float("-inf")), 1)
            off = 3 * (d + 4) * size.masked_fill(~seen, 0).amax(1, keepdim=True) * U + (64 + x.masked_fill(~seen, 0).abs().amax(1, keepdim=True)) * 2 * U
            want, tol = want + p.sum(0), tol + (p * off + 1e-37 * seen).sum(0)
        got = scores[b, 0, :L].double()
        assert bool(((got - want).abs() <= tol + 80 * U * want).all()), b
        assert torch.equal(scores[b, 0, L:].double(), before[b, 0, L:])


@pytest.mark.parametrize("batch", [65, 100, 256, 257])
@pytest.mark.parametrize("bound", [400, 900])
def test_every_sequence_once_whatever_the_order(sd, batch, bound):
    """More (sequence, KV head)s than compute units: the longer sequences' workgroups come first, up to 256 sequences."""
    import torch
    heads, kv_heads, d, longest = 8, 4, 64, 400
    gen = torch.Generator().manual_seed(batch)
    lens = torch.randint(0, longest + 1, (batch,), generator=gen)
    lens[0], lens[1], lens[-1] = 0, 1, longest
    per, blocks = 25, (bound + 15) // 16
    pool = torch.randn(batch * per, kv_heads, 16, d, generator=gen).bfloat16().cuda()
    table = torch.full((batch, blocks), -1, dtype=torch.int32)
    table[:, :per] = torch.randperm(batch * per, generator=gen).view(batch, per)
    q = queries(batch, heads, d, 8)
    shape = shape_of(sd, batch, heads, kv_heads, d, batch * per, blocks, bound)
    ws = sd.paged_weight_workspace_bytes(shape, 1)
    work = torch.empty(ws, dtype=torch.uint8, device="cuda").fill_(255)
    out = torch.full((batch, kv_heads, bound), -1.0, device="cuda")
    sd.paged_weight_accumulate(shape, q, None, batch, 1, pool, None, table.cuda(), lens.int().cuda(), d ** -0.5, 1.0, 0, None, out, bound, work, ws)
    for b, L in enumerate(lens.tolist()):
        assert bool((out[b, :, L:] == -1).all())
        k = pool[table[b, :per].long().cuda()].double().transpose(1, 2).reshape(-1, kv_heads, d)[:L]
        for g in range(kv_heads if L else 0):
            want, tol = weights_of(q[b, 2 * g:2 * g + 2].double(), k[:, g].contiguous(), d ** -0.5)
            assert bool(((out[b, g, :L].double() - want).abs() <= tol).all()), (b, g)
