"""paged_weight_accumulate against the definition in 64 bits.

Tolerance.  A score x = scale <q, k> is made of exact products summed in fp32: it is off by at most (d + 4) 2^-24 scale sum |q k|.  A weight
exp(x - max) / sum carries twice that, once more for its row's sum (an average of such errors), and the roundings of the
exponential (2^-22 with that of its argument, which is at most the score's size), of the additions and the division, together below
(64 + max |x|) 2^-23.  Scores are the sum of the rows' weights and one product.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def sd():
    import torch
    assert torch.cuda.is_available()
    import paper_2508_11553_amd as m
    m.load()
    return m


class Cache:
    """K of sequences of the given lengths over a pool whose unused slots hold NaN."""

    def __init__(self, lens, hkv, d, kv, seed, max_context_len=None, gain=1.0):
        import torch
        self.lens, self.hkv, self.d, self.kv = list(lens), hkv, d, kv
        rng = np.random.default_rng(seed)
        held = [max(0, n) for n in lens]
        blocks = [(n + 15) // 16 for n in held]
        self.max_context_len = max(held) if max_context_len is None else max_context_len
        self.max_blocks = max(1, max(blocks), (self.max_context_len + 15) // 16)
        self.pages = sum(blocks) + 2
        self.table = np.full((len(lens), self.max_blocks), -1, np.int32)
        order = rng.permutation(self.pages)
        at = 0
        for b, n in enumerate(blocks):
            self.table[b, :n] = order[at:at + n]
            at += n
        pool = torch.full((self.pages, hkv, 16, d), float("nan"))
        scales = torch.full((self.pages, hkv), float("nan"))
        self.k = []
        for b, n in enumerate(held):
            rows = torch.from_numpy(rng.normal(size=(n, hkv, d)).astype(np.float32) * gain)
            if kv == "bf16":
                rows = rows.bfloat16().float()
                for t in range(n):
                    pool[self.table[b, t // 16], :, t % 16] = rows[t]
                self.k.append(rows.double().numpy())
            else:
                full = np.zeros((n, hkv, d))
                for j in range(blocks[b]):
                    tile = rows[16 * j:16 * j + 16]
                    s = tile.abs().amax((0, 2)) / 448 * float(np.exp(rng.normal()))
                    code = (tile / s[None, :, None]).clamp(-448, 448).to(torch.float8_e4m3fn)
                    scales[self.table[b, j]] = s
                    pool[self.table[b, j], :, :len(tile)] = code.float().transpose(0, 1)
                    full[16 * j:16 * j + len(tile)] = (code.double() * s.double()[None, :, None]).numpy()
                self.k.append(full)
        self.pool = pool.bfloat16().cuda() if kv == "bf16" else pool.to(torch.float8_e4m3fn).view(torch.uint8).cuda()
        self.scales = None if kv == "bf16" else scales.cuda()

    def shape(self, sd, hq):
        return sd.Shape(batch=len(self.lens), num_q_heads=hq, num_kv_heads=self.hkv, head_dim=self.d, page_size=16, num_pages=self.pages,
                        max_blocks_per_seq=self.max_blocks, kv_dtype=sd.SD_BF16 if self.kv == "bf16" else sd.SD_FP8_E4M3, max_context_len=self.max_context_len,
                        chunk_tokens=0)


def expected(cache, q, starts, L, scale, decay, new, before):
    """-> scores and their tolerances, lists of [Hkv][L_b]; q: [rows][Hq][d] in 64 bits"""
    out = []
    for b in range(len(L)):
        rows = q[starts[b]:starts[b + 1]]
        n, hkv = len(rows), cache.hkv
        k = cache.k[b][:L[b]]
        old = np.zeros((hkv, L[b])) if before is None else before[b, :, :L[b]] * decay
        old[:, max(0, L[b] - new):] = 0
        got, tol = old.copy(), np.abs(old) * 4 * U
        for i in range(n):
            pos = L[b] - n + i
            if pos < 0:
                continue
            for h in range(q.shape[1]):
                g = h // (q.shape[1] // hkv)
                x = scale * (k[:pos + 1, g] @ rows[i, h])
                size = abs(scale) * (np.abs(k[:pos + 1, g]) @ np.abs(rows[i, h])).max()
                p = np.exp(x - x.max())
                p /= p.sum()
                got[g, :pos + 1] += p
                tol[g, :pos + 1] += p * (3 * (cache.d + 4) * size * U + (64 + np.abs(x).max()) * 2 * U) + 1e-37
        out.append((got, tol + np.abs(got) * 80 * U))
    return out


def run(sd, cache, hq, q, starts, scale, decay=1.0, new=1, before=None, lens=None, max_q_len=None, in_place=False, stride=None, stream=None):
    import torch
    B = len(cache.lens)
    shape = cache.shape(sd, hq)
    stride = stride or (cache.max_context_len + 3) // 4 * 4
    most = 1 if starts is None else max(np.diff(starts).max(), 0) if max_q_len is None else max_q_len
    ws = sd.paged_weight_workspace_bytes(shape, int(most))
    work = torch.empty(ws, dtype=torch.uint8, device="cuda").fill_(255)   # (fp32 NaN)
    out = before if in_place else torch.full((B, cache.hkv, stride), float("nan"), device="cuda")
    dev = lambda a: torch.tensor(np.asarray(a, np.int32), device="cuda")  # noqa: E731
    sd.paged_weight_accumulate(shape, q, None if starts is None else dev(starts), len(q), int(most), cache.pool, cache.scales, dev(cache.table),
                               dev(cache.lens if lens is None else lens), scale, decay, new, before, out, stride, work, ws, stream=stream)
    return out


def check(got, want, L):
    got = got.double().cpu().numpy()
    for b, (w, tol) in enumerate(want):
        bad = ~(np.abs(got[b, :, :L[b]] - w) <= tol)
        assert not bad.any(), (b, np.argwhere(bad)[:3], got[b, :, :L[b]][bad][:3], w[bad][:3], tol[bad][:3])


def queries(n, hq, d, seed, gain=1.0):
    import torch
    return (torch.randn(n, hq, d, generator=torch.Generator().manual_seed(seed)) * gain).bfloat16().cuda()


DECODE = [  # lens, heads, kv heads, d, kv
    ([1], 1, 1, 64, "bf16"),
    ([1, 2, 15, 16, 17, 63, 64, 65], 8, 2, 128, "bf16"),
    ([0, 3, 0, 255, 256, 257], 28, 4, 128, "bf16"),
    ([300, 1, 511, 512, 513], 16, 1, 64, "bf16"),        # 16 heads: a whole tile
    ([1023, 1024, 1025, 100], 12, 4, 64, "fp8"),
    ([2500, 37, 1], 64, 8, 128, "fp8"),
    ([5000, 4097], 8, 2, 128, "bf16"),
    ([20011], 4, 1, 128, "bf16"),                         # several chunks of 64 blocks
    ([130, 700, 0], 40, 2, 64, "bf16"),                  # 20 heads to a KV head: two tiles of rows
    ([90, 600], 64, 1, 128, "fp8"),                       # 64
    ([6000, 100, 4100], 12, 1, 128, "bf16"),              # 12 heads, long
    ([9000, 15], 7, 1, 64, "fp8"),
    ([6500, 3], 8, 2, 64, "bf16"),
]

MANY = [  # batches of more (sequence, KV head) pairs than half the compute units: a long sequence, many short ones
    (8192, 16, 2, 64, "bf16"), (8193, 16, 2, 64, "fp8"), (8192, 8, 2, 64, "fp8"), (4096, 24, 2, 64, "bf16"), (4097, 24, 2, 64, "bf16"), (2049, 10, 2, 128, "fp8"), (700, 6, 2, 128, "bf16"),
]


@pytest.mark.parametrize("lens,hq,hkv,d,kv", DECODE)
@pytest.mark.parametrize("decay", [1.0, 0.9])
def test_decode_step(sd, lens, hq, hkv, d, kv, decay):
    import torch
    c = Cache(lens, hkv, d, kv, len(lens) + hq)
    q = queries(len(lens), hq, d, 1, 2.0)
    stride = (c.max_context_len + 3) // 4 * 4 + 8
    before = torch.rand(len(lens), hkv, stride, device="cuda")
    for b, n in enumerate(lens):
        before[b, :, max(0, n - 1):] = float("nan")     # the newest token's entry and all behind it hold anything
    got = run(sd, c, hq, q, None, d ** -0.5, decay, 1, before, stride=stride)
    L = [max(0, n) for n in lens]
    check(got, expected(c, q.double().cpu().numpy(), np.arange(len(lens) + 1), L, d ** -0.5, decay, 1, before.double().cpu().numpy()), L)
    for b, n in enumerate(L):
        assert got[b, :, n:].isnan().all()
    again = run(sd, c, hq, q, None, d ** -0.5, decay, 1, before, in_place=True, stride=stride)
    for b, n in enumerate(L):
        assert torch.equal(again[b, :, :n], got[b, :, :n])


@pytest.mark.parametrize("longest,hq,hkv,d,kv", MANY)
def test_many_sequences(sd, longest, hq, hkv, d, kv):
    rng = np.random.default_rng(longest)
    lens = rng.integers(0, 60, 86).tolist()
    lens[7], lens[8], lens[9], lens[50] = 0, longest, 513, longest // 2
    c = Cache(lens, hkv, d, kv, 11)
    q = queries(len(lens), hq, d, 12, 2.0)
    check(run(sd, c, hq, q, None, d ** -0.5), expected(c, q.double().cpu().numpy(), np.arange(len(lens) + 1), lens, d ** -0.5, 1.0, 1, None), lens)


WINDOWS = [  # lens, rows of each, heads, kv heads, d, kv
    ([40, 1, 17], [2, 1, 17], 4, 2, 64, "bf16"),
    ([5, 300], [9, 4], 4, 1, 64, "bf16"),                 # more rows than tokens: those of negative positions add nothing
    ([333, 0, 64, 65], [32, 3, 0, 65], 8, 2, 128, "bf16"),
    ([1500, 700], [33, 64], 32, 8, 128, "bf16"),
    ([2100, 15], [16, 15], 28, 4, 128, "fp8"),
    ([1030], [7], 40, 1, 64, "fp8"),
    ([300, 290], [2, 3], 8, 2, 64, "bf16"),               # one tile of rows: 3 queries of 4 heads
    ([1100], [300], 4, 4, 128, "bf16"),
]


@pytest.mark.parametrize("lens,rows,hq,hkv,d,kv", WINDOWS)
def test_windows(sd, lens, rows, hq, hkv, d, kv):
    import torch
    c = Cache(lens, hkv, d, kv, sum(rows))
    starts = np.concatenate([[0], np.cumsum(rows)])
    q = queries(int(starts[-1]), hq, d, 2, 1.5)
    stride = (c.max_context_len + 3) // 4 * 4
    before = torch.rand(len(lens), hkv, stride, device="cuda")
    for new, scores in ((0, before), (5, before), (0, None)):
        got = run(sd, c, hq, q, starts, d ** -0.5, 0.7, new, scores)
        check(got, expected(c, q.double().cpu().numpy(), starts, lens, d ** -0.5, 0.7, new, None if scores is None else scores.double().cpu().numpy()), lens)


def test_lengths_outside_the_bound_and_ranges_outside_the_rows(sd):
    import torch
    c = Cache([100, 100, 100, 100, 100], 2, 64, "bf16", 5)
    starts = [0, 3, 6, 9, 12, 99]     # the last range leaves the 14 rows
    q = queries(14, 4, 64, 3)
    before = torch.rand(5, 2, 100, device="cuda")
    for lens in ([100, -5, 2 ** 31 - 1, 0, 100],):
        got = run(sd, c, 4, q, starts, 0.125, 1.0, 0, before, lens=lens, max_q_len=3)
        L = [min(max(n, 0), 100) for n in lens]
        want = expected(c, q.double().cpu().numpy(), [0, 3, 6, 9, 12], L[:4], 0.125, 1.0, 0, before.double().cpu().numpy())
        check(got[:4], want, L)
        assert torch.equal(got[4], before[4])


@pytest.mark.parametrize("scale", [0.0, -0.1, 3.0])
def test_scales_of_any_sign(sd, scale):
    c = Cache([70, 600], 2, 64, "bf16", 6)
    q = queries(2, 8, 64, 4)
    check(run(sd, c, 8, q, None, scale), expected(c, q.double().cpu().numpy(), [0, 1, 2], [70, 600], scale, 1.0, 1, None), [70, 600])
    if scale == 0.0:
        q = queries(40, 8, 64, 4)
        check(run(sd, c, 8, q, [0, 20, 40], scale), expected(c, q.double().cpu().numpy(), [0, 20, 40], [70, 600], scale, 1.0, 1, None), [70, 600])


@pytest.mark.parametrize("starts", [None, [0, 40]])
def test_a_score_that_is_not_finite_stays_in_its_head(sd, starts):
    """Infinite and NaN keys reach the weights of their KV head, and no other."""
    import torch
    c = Cache([400], 3, 64, "bf16", 7)
    page = int(c.table[0, 3])
    c.pool[page, 0, 5, 0] = float("nan")
    c.pool[page, 1, 5, 0] = float("inf")
    q = queries(1 if starts is None else 40, 6, 64, 5)
    q[..., 0] = 1.0
    got = run(sd, c, 6, q, starts, 0.125)
    assert got[0, 0].isnan().all() and got[0, 1].isnan().all()
    n = 1 if starts is None else 40
    want = expected(c, q.double().cpu().numpy(), [0, n], [400], 0.125, 1.0, 1, None)
    bad = np.abs(got[0, 2].double().cpu().numpy() - want[0][0][2]) > want[0][1][2]
    assert not bad.any()
    # -inf: a token that no row looks at
    c.pool[page, 0, 5, 0] = float("-inf")
    got = run(sd, c, 6, q, starts, 0.125)
    assert got[0, 0, 53] == 0 and got[0, 0].isfinite().all()


@pytest.mark.parametrize("lens,hq,hkv,d,starts", [([700], 8, 2, 64, None), ([6000], 4, 1, 128, None), ([5000], 8, 1, 64, None), ([4500], 12, 1, 64, None),
                                                  ([900], 8, 2, 64, [0, 40]), ([900], 8, 2, 128, [0, 3]), ([300, 20] * 40, 8, 2, 64, None)])
def test_stretches_of_tokens_without_any_weight(sd, lens, hq, hkv, d, starts):
    """Keys whose scores are -inf, single ones, whole pages, the first and the last of a sequence: weight 0, and the others' weights as if
    those tokens were not there.  A row that has nothing else is NaN (0 / 0), as the definition is."""
    c = Cache(lens, hkv, d, "bf16", 21)
    L = lens[0]
    gone = np.zeros(L, bool)
    gone[:67] = gone[90:112] = gone[113] = gone[130:134] = gone[L // 2:L // 2 + 70] = True
    for t in np.flatnonzero(gone):
        c.pool[int(c.table[0, t // 16]), 0, t % 16, 3] = float("-inf")
    n = len(lens) if starts is None else starts[-1]
    q = queries(n, hq, d, 22)
    q[..., 3] = 0.5
    got = run(sd, c, hq, q, starts, d ** -0.5)[0].double().cpu().numpy()
    k, G = c.k[0][:, 0].copy(), hq // hkv
    k[gone, 3] = 0
    want, tol = np.zeros(L), np.zeros(L)
    rows = q.double().cpu().numpy()[:1 if starts is None else n]
    for i, row in enumerate(rows):
        end = L - len(rows) + 1 + i
        for h in range(G):
            x = np.where(gone[:end], -np.inf, d ** -0.5 * (k[:end] @ row[h]))
            size = d ** -0.5 * (np.abs(k[:end]) @ np.abs(row[h])).max()
            p = np.exp(x - x.max())
            want[:end] += p / p.sum()
            tol[:end] += p / p.sum() * (3 * (d + 4) * size * U + (64 + size) * 2 * U) + 1e-37
    assert (got[0, :L][gone] == 0).all()
    assert (np.abs(got[0, :L] - want) <= tol + want * 80 * U).all()
    if hkv > 1:
        assert (got[1, :L] > 0).all()
    for t in range(L):
        c.pool[int(c.table[0, t // 16]), 0, t % 16, 3] = float("-inf")
    got = run(sd, c, hq, q, starts, d ** -0.5)[0]
    assert got[0, :L].isnan().all() and (hkv == 1 or got[1, :L].isfinite().all())


def test_weights_of_a_decode_step_sum_to_the_heads(sd):
    """Every row's weights sum to one: the scores of a KV head to its query heads, whatever the lengths."""
    lens = [1, 7, 4000, 16383]
    c = Cache(lens, 2, 128, "fp8", 8)
    got = run(sd, c, 14, queries(4, 14, 128, 6, 3.0), None, 128 ** -0.5).double()
    for b, n in enumerate(lens):
        assert np.allclose(got[b, :, :n].sum(-1).cpu().numpy(), 7, rtol=0, atol=7 * 64 * 2 * U)


def test_a_large_bound_over_short_sequences(sd):
    c = Cache([33, 200], 2, 64, "bf16", 9, max_context_len=100000)
    q = queries(2, 4, 64, 7)
    check(run(sd, c, 4, q, None, 0.125), expected(c, q.double().cpu().numpy(), [0, 1, 2], [33, 200], 0.125, 1.0, 1, None), [33, 200])
    q = queries(20, 4, 64, 7)
    check(run(sd, c, 4, q, [0, 10, 20], 0.125), expected(c, q.double().cpu().numpy(), [0, 10, 20], [33, 200], 0.125, 1.0, 1, None), [33, 200])
