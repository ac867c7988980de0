"""kv_evict against a plain implementation: positions, lengths, scores, rows and fp8 codes are equal, not close."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sd():
    import torch
    assert torch.cuda.is_available()
    import paper_2508_11553_amd as m
    m.load()
    return m


def kept_of(scores, L, budget, sinks, recent):
    """Positions that stay of one (sequence, head): a stable order by descending score, NaN last."""
    if L <= budget:
        return np.arange(L)
    middle = np.arange(sinks, L - recent)
    x = scores[middle]
    order = np.lexsort((middle, np.where(np.isnan(x), 0, -x), np.isnan(x)))
    chosen = middle[order[:budget - sinks - recent]]
    return np.sort(np.concatenate([np.arange(sinks), chosen, np.arange(L - recent, L)]))


class Case:
    def __init__(self, sd, lens, hkv, d, kv, budget, seed, max_context_len=None):
        import torch
        rng = np.random.default_rng(seed)
        self.lens, self.hkv, self.d, self.kv, self.budget = lens, hkv, d, kv, budget
        held = [max(0, n) for n in lens]
        self.bound = max(held) if max_context_len is None else max_context_len
        old = [(n + 15) // 16 for n in held]
        new = [(min(n, budget, self.bound) + 15) // 16 for n in held]
        self.max_blocks = max(1, max(old), (self.bound + 15) // 16)
        self.pages = sum(old) + sum(new) + 2
        order = rng.permutation(self.pages)
        self.table, self.new_table = (np.full((len(lens), self.max_blocks), -1, np.int32) for _ in range(2))
        at = 0
        for table, counts in ((self.table, old), (self.new_table, new)):
            for b, n in enumerate(counts):
                table[b, :n] = order[at:at + n]
                at += n
        shape = (self.pages, hkv, 16, d)
        self.scales = None
        if kv == "bf16":
            self.pools = [torch.from_numpy(rng.normal(size=shape).astype(np.float32)).bfloat16().cuda() for _ in range(2)]
        else:   # every finite code, and scales of all sizes
            codes = [rng.integers(0, 256, shape).astype(np.uint8) for _ in range(2)]
            self.pools = [torch.from_numpy(np.where((c & 0x7f) == 0x7f, 0x3c, c).astype(np.uint8)).cuda() for c in codes]
            self.scales = [torch.from_numpy(np.exp(2 * rng.normal(size=shape[:2])).astype(np.float32)).cuda() for _ in range(2)]
        self.stride = (self.bound + 3) // 4 * 4
        self.scores = np.exp(3 * rng.normal(size=(len(lens), hkv, self.stride))).astype(np.float32)
        self.shape = sd.Shape(batch=len(lens), num_q_heads=hkv, num_kv_heads=hkv, head_dim=d, page_size=16, num_pages=self.pages, max_blocks_per_seq=self.max_blocks,
                              kv_dtype=sd.SD_BF16 if kv == "bf16" else sd.SD_FP8_E4M3, max_context_len=self.bound, chunk_tokens=0)

    def run_and_check(self, sd, sinks, recent, out_stride=None, in_place=False):
        import torch
        B, hkv, budget = len(self.lens), self.hkv, self.budget
        dev = lambda a: torch.tensor(np.asarray(a, np.int32), device="cuda")  # noqa: E731
        scores = torch.from_numpy(self.scores).cuda()
        kept = torch.full((B, hkv, budget), -7, dtype=torch.int32, device="cuda")
        lens = dev(self.lens)
        new_lens = lens if in_place else dev([-9] * B)
        out_stride = self.stride if in_place else out_stride or min(budget, self.bound)
        out = scores if in_place else torch.full((B, hkv, out_stride), -5.0, device="cuda")
        before = [p.clone() for p in self.pools]
        scales_before = [s.clone() for s in self.scales] if self.scales else None
        sd.kv_evict(self.shape, budget, sinks, recent, scores, self.stride, *self.pools, *(self.scales or (None, None)), dev(self.table), lens, dev(self.new_table),
                    kept, new_lens, out, out_stride)
        got_kept, got_out = kept.cpu().numpy(), out.cpu().numpy()
        L = [min(max(n, 0), self.bound) for n in self.lens]
        assert new_lens.cpu().tolist() == [min(n, budget) for n in L]
        touched = np.zeros((self.pages, hkv, 16), bool)
        tiles = np.zeros((self.pages, hkv), bool)
        where = []   # (destination page, slot, head, source page, source slot)
        for b in range(B):
            n = min(L[b], budget)
            for g in range(hkv):
                want = kept_of(self.scores[b, g], L[b], budget, sinks, recent)
                assert len(want) == n
                assert np.array_equal(got_kept[b, g, :n], want), (b, g)
                assert (got_kept[b, g, n:] == -1).all()
                assert np.array_equal(got_out[b, g, :n], self.scores[b, g, want], equal_nan=True)
                rest = got_out[b, g, n:]
                assert np.array_equal(rest, self.scores[b, g, n:], equal_nan=True) if in_place else (rest == -5).all()
                at = np.arange(n)
                where.append(np.stack([self.new_table[b, at // 16], at % 16, np.full(n, g), self.table[b, want // 16], want % 16], 1).reshape(-1, 5))
        to_page, to_slot, head, page, slot = (torch.from_numpy(x.astype(np.int64)).cuda() for x in np.concatenate(where).T)
        touched[to_page.cpu(), head.cpu(), to_slot.cpu()] = True
        tiles[to_page.cpu(), head.cpu()] = True
        touched, tiles = torch.from_numpy(touched).cuda(), torch.from_numpy(tiles).cuda()
        for i, pool in enumerate(self.pools):
            rows = before[i][page, head, slot]
            if self.scales:
                old = scales_before[i][page, head]
                top = torch.zeros_like(scales_before[i]).view(-1).scatter_reduce(0, to_page * hkv + head, old, "amax").view(self.pages, hkv)
                assert torch.equal(self.scales[i], torch.where(tiles, top, scales_before[i]))
                ratio = old / top[to_page, head]
                again = (rows.view(torch.float8_e4m3fn).float() * ratio[:, None]).to(torch.float8_e4m3fn).view(torch.uint8)
                rows = torch.where((ratio == 1)[:, None], rows, again)
            bits = (lambda x: x) if self.scales else (lambda x: x.view(torch.int16))
            assert torch.equal(bits(pool[to_page, head, to_slot]), bits(rows))
            assert torch.equal(bits(pool)[~touched], bits(before[i])[~touched])   # nothing else is written


CASES = [  # lens, kv heads, d, kv, budget, sinks, recent
    ([1], 1, 64, "bf16", 1, 0, 0),
    ([2], 1, 128, "bf16", 1, 0, 0),
    ([5, 0, 17, 3], 2, 64, "bf16", 3, 1, 1),
    ([40, 16, 17, 100, 15], 3, 128, "bf16", 16, 2, 5),
    ([1000, 999, 500, 501, 502], 4, 128, "bf16", 500, 4, 100),
    ([1025, 2049, 3000], 2, 64, "fp8", 1024, 0, 0),
    ([700, 20, 333], 8, 128, "fp8", 100, 7, 50),
    ([5000, 4000, 300], 2, 64, "bf16", 1111, 16, 1000),
    ([70000], 2, 64, "bf16", 4097, 4, 64),               # more than 16 bits of positions
    ([65536, 65537, 4096], 1, 64, "bf16", 600, 4, 64),
    ([140000, 5, 66000], 1, 64, "fp8", 70000, 0, 1000),
    ([4096, 4095, 130], 2, 64, "bf16", 129, 0, 64),
    ([4097, 4095, 130], 2, 64, "fp8", 129, 1, 64),
    ([16384, 16383, 8192, 600], 1, 64, "bf16", 511, 4, 64),
    ([16385, 16383, 8192, 600], 1, 64, "bf16", 511, 4, 64),
    ([300, 200], 2, 128, "fp8", 64, 0, 64),                # nothing left to choose: the last 64
    ([300, 200], 2, 128, "bf16", 64, 64, 0),               # the first
    ([300, 200], 2, 128, "bf16", 64, 20, 44),
    ([90, 200], 2, 128, "fp8", 1000, 4, 100),              # nothing to cut
]


@pytest.mark.parametrize("lens,hkv,d,kv,budget,sinks,recent", CASES)
def test_evict(sd, lens, hkv, d, kv, budget, sinks, recent):
    Case(sd, lens, hkv, d, kv, budget, sum(lens)).run_and_check(sd, sinks, recent)
    Case(sd, lens, hkv, d, kv, budget, sum(lens) + 1).run_and_check(sd, sinks, recent, in_place=True)


@pytest.mark.parametrize("longest", [3000, 9000, 20000])
@pytest.mark.parametrize("kind", ["equal", "zeros", "few", "nan", "inf", "close", "negative", "ascending", "descending"])
def test_scores_that_are_hard_to_tell_apart(sd, kind, longest):
    c = Case(sd, [longest, 130, 1200], 3, 64, "bf16", 128, 77)
    rng = np.random.default_rng(1)
    x = c.scores
    if kind == "equal":
        x[:] = 0.25
    elif kind == "zeros":
        x[:] = np.where(rng.random(x.shape) < 0.5, np.float32(0.0), np.float32(-0.0))
        x[..., ::97] = 1.0
    elif kind == "few":
        x[:] = rng.integers(0, 3, x.shape)
    elif kind == "nan":
        x[rng.random(x.shape) < 0.99] = np.nan     # fewer numbers than places: NaN fill the rest, the first of them
    elif kind == "inf":
        x[rng.random(x.shape) < 0.01] = np.inf
        x[rng.random(x.shape) < 0.95] = -np.inf
    elif kind == "close":                          # neighbouring floats
        x[:] = (np.float32(1.0).view(np.int32) + rng.integers(0, 5000, x.shape).astype(np.int32)).view(np.float32)
    elif kind == "negative":
        x[:] = -x
    elif kind == "ascending":
        x[:] = np.arange(x.shape[-1])
    else:
        x[:] = -np.arange(x.shape[-1])
    c.run_and_check(sd, 3, 20)
    c.run_and_check(sd, 0, 0, in_place=True)


def test_lengths_outside_the_bound(sd):
    c = Case(sd, [64, 64, 64, 64], 2, 64, "bf16", 32, 5)
    c.lens = [-4, 64, 2 ** 31 - 1, 10]
    c.run_and_check(sd, 2, 8)
    c.lens = [-4, 64, 2 ** 31 - 1, 10]
    c.run_and_check(sd, 2, 8, in_place=True)


def test_without_scores_out_and_with_a_wide_one(sd):
    import torch
    c = Case(sd, [500, 40], 2, 64, "bf16", 100, 6)
    c.run_and_check(sd, 4, 30, out_stride=137)
    dev = lambda a: torch.tensor(np.asarray(a, np.int32), device="cuda")  # noqa: E731
    kept, lens = torch.empty(2, 2, 100, dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
    sd.kv_evict(c.shape, 100, 4, 30, torch.from_numpy(c.scores).cuda(), c.stride, *c.pools, None, None, dev(c.table), dev(c.lens), dev(c.new_table), kept, lens)
    assert np.array_equal(kept[0, 1].cpu().numpy(), kept_of(c.scores[0, 1], 500, 100, 4, 30)) and lens.tolist() == [100, 40]


def test_shared_pages_are_left_alone(sd):
    """Two trajectories on one prefix: each gets its own cut, the prefix's pages keep their rows (checked by run_and_check)."""
    c = Case(sd, [320, 320], 2, 128, "bf16", 96, 9)
    c.table[1, :10] = c.table[0, :10]
    c.run_and_check(sd, 4, 40)
