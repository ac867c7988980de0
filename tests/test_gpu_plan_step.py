"""kv_plan_step against the plain form: whole numbers, equal to the last."""
import numpy as np
import pytest

from tests import logits_plain as plain

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sd():
    import torch
    assert torch.cuda.is_available()
    import paper_2508_11553_amd as m
    m.load()
    return m


NAMES = ("granted", "row_start", "starts", "lens_out", "next_out", "seq_ids", "slots", "positions")


class Plan:
    """A cache's tables: `lens` tokens a sequence on pages of a random order, `spare` free pages."""

    def __init__(self, sd, lens, blocks, spare, seed, limit=None):
        import torch
        self.sd, self.B, self.blocks = sd, len(lens), blocks
        rng = np.random.default_rng(seed)
        used = [(max(0, min(n, 16 * blocks)) + 15) // 16 for n in lens]
        self.pages = sum(used) + spare
        order = [int(x) for x in rng.permutation(self.pages)]
        self.table = []
        for n in used:
            row, order = order[:n], order[n:]
            self.table.append(row + [-1] * (blocks - n))
        self.free = order
        self.lens, self.next = list(lens), [int(n + x) for n, x in zip(lens, rng.integers(0, 3, self.B) * 500)]
        self.limit = 16 * blocks if limit is None else limit
        self.shape = sd.Shape(batch=self.B, num_q_heads=8, num_kv_heads=8, head_dim=128, page_size=16, num_pages=self.pages, max_blocks_per_seq=blocks, kv_dtype=sd.SD_BF16,
                              max_context_len=self.limit, chunk_tokens=0)
        self.ws = sd.kv_plan_workspace_bytes(self.shape)
        dev = lambda a: torch.tensor(np.asarray(a, np.int32), device="cuda")  # noqa: E731
        self.d = dict(block_table=dev(self.table).reshape(self.B, blocks), free_pages=dev(self.free + [-9] * (self.pages - len(self.free))), free=dev([len(self.free)]),
                      lens=dev(self.lens), next=dev(self.next), work=torch.full((self.ws,), 255, dtype=torch.uint8, device="cuda"))

    def step(self, new, shared=None, max_rows=None, in_place=True, positions=True):
        """Plans on the device and in plain Python, compares everything."""
        import torch
        d, B = self.d, self.B
        max_rows = sum(n for n in new if n > 0) if max_rows is None else max_rows
        dev = lambda a: torch.tensor(np.asarray(a, np.int32), device="cuda")  # noqa: E731
        out = {name: torch.full((max_rows if name in NAMES[-3:] else B + (name == "row_start"),), -77, dtype=torch.int32, device="cuda") for name in NAMES}
        if in_place:
            out["lens_out"], out["next_out"] = d["lens"], d["next"]
        free_out = d["free"] if in_place else dev([-5])
        self.sd.kv_plan_step(self.shape, dev(new), None if shared is None else dev(shared), d["lens"], out["lens_out"], d["next"] if positions else None,
                             out["next_out"] if positions else None, d["free_pages"], d["free"], free_out, d["block_table"], max_rows, out["granted"], out["row_start"], out["starts"],
                             out["seq_ids"], out["slots"], out["positions"] if positions else None, d["work"], self.ws)
        stack_before, held = list(self.free), len(self.free)
        want = plain.plan(new, shared or [0] * B, self.lens, self.next if positions else self.lens, self.free, self.table, max_rows, self.limit)
        for name in NAMES:
            if not positions and name in ("next_out", "positions"):
                continue
            assert out[name].tolist() == want[name], name
        assert free_out.item() == len(self.free)
        assert d["block_table"].tolist() == self.table
        stack = d["free_pages"].tolist()
        assert stack[:held] == stack_before          # not written below what was free before
        assert stack[held:len(self.free)] == self.free[held:]
        self.lens = want["lens_out"]
        self.next = want["next_out"] if positions else self.next
        if not in_place:
            d["lens"], d["next"], d["free"] = out["lens_out"], out["next_out"], free_out
        return want


def pages_once(p, shared=0):
    held = [x for b in range(p.B) for x in p.table[b][:(p.lens[b] + 15) // 16]]
    assert sorted(held + p.free) == list(range(p.pages))


@pytest.mark.parametrize("batch", [1, 2, 63, 64, 65, 700, 1023, 1024, 1025, 2500])
@pytest.mark.parametrize("most", [1, 40])
def test_steps_of_a_rollout(sd, batch, most):
    """Several steps one after the other, in place, some sequences waiting or finished; every page stays where it belongs, once."""
    rng = np.random.default_rng(batch + most)
    p = Plan(sd, rng.integers(0, 100, batch), 20, batch * 2, batch)
    for i in range(4):
        new = np.where(rng.random(batch) < 0.15, -1, np.where(rng.random(batch) < 0.15, 0, rng.integers(1, most + 1, batch)))
        p.step([int(n) for n in new], max_rows=[None, batch * most + 5][i % 2], in_place=i != 2)
        pages_once(p)


@pytest.mark.parametrize("lens,new", [([0], [1]), ([0], [16]), ([0], [17]), ([15], [1]), ([16], [1]), ([16], [0]), ([16], [-1]), ([0], [-1]), ([0, 0], [0, 0]), ([31, 32, 33], [1, 1, 1]),
                                      ([5, 40, 7], [-1, -1, -1]), ([160, 0], [-1, 160]), ([1], [159]), ([1], [160])])
def test_page_borders(sd, lens, new):
    p = Plan(sd, lens, 10, 3, 1)
    p.step(new)
    pages_once(p)


def test_long_resumes(sd):
    rng = np.random.default_rng(4)
    lens = rng.integers(0, 3000, 37)
    p = Plan(sd, lens, 800, 20000, 5)
    new = [int(n) for n in rng.integers(1, 9000, 37)]
    new[3], new[9], new[20] = -1, 0, -1
    p.step(new)
    pages_once(p)
    p.step([1] * 37, max_rows=64)


@pytest.mark.parametrize("spare", [0, 1, 5, 17])
def test_a_pool_that_runs_short(sd, spare):
    """The first in the batch are served; who needs no page goes on; pages that come back in the same call are used."""
    rng = np.random.default_rng(spare)
    p = Plan(sd, rng.integers(0, 64, 90), 12, spare, spare)
    for _ in range(3):
        want = p.step([int(n) for n in rng.choice([-1, 0, 1, 1, 1, 30], 90)])
        pages_once(p)
    assert any(n == 0 for n in want["granted"])


def test_rows_and_lengths_past_their_bounds(sd):
    p = Plan(sd, [10, 150, 159, 160, 20], 10, 50, 2)
    want = p.step([5, 11, 1, 1, 3], max_rows=100)
    assert want["granted"] == [5, 0, 1, 0, 3]                # 161 tokens do not fit 10 pages
    want = p.step([7, 1, 0, 0, 4], max_rows=8)
    assert want["granted"] == [7, 1, 0, 0, 0]                # 12 rows do not fit 8
    p = Plan(sd, [10, 99, -5, 300], 10, 50, 3, limit=100)    # a length below 0 counts as 0, one above the bound as the bound
    assert p.step([1, 2, 3, 1], max_rows=8)["granted"] == [1, 0, 3, 0]
    p.step([-1, 0, -1, -1], max_rows=0)
    p = Plan(sd, [3, 3], 4, 4, 3)
    assert p.step([2 ** 31 - 1, 1], max_rows=4)["granted"] == [0, 1]


def test_shared_pages_stay(sd):
    """A finished sequence gives back the pages behind its shared prefix only."""
    p = Plan(sd, [100, 100, 40, 100], 10, 4, 6)
    held = len(p.free)
    p.step([-1, -1, -1, 1], shared=[48, 0, 64, 100], max_rows=4)
    # 7 pages less 3 shared; 7; of 3 pages, 2 full ones shared (its 64 count as its 40); none is taken: 100 + 1 tokens fit 7 pages
    assert len(p.free) == held + 4 + 7 + 1


def test_without_positions(sd):
    p = Plan(sd, [3, 40, 17], 6, 8, 7)
    p.step([1, 30, -1], positions=False)


def test_a_batch_of_nothing(sd):
    p = Plan(sd, [7], 4, 1, 8)
    p.shape.batch = 0
    sd.kv_plan_step(p.shape, None, None, None, None, None, None, None, None, None, None, 0, None, None, None, None, None, None, None, 0)


@pytest.mark.parametrize("batch", [4095, 4096, 4097, 8191, 12345, 40000])
def test_batches_that_take_several_turns(sd, batch):
    """More sequences than one workgroup holds at once, and more than the second kernel keeps sums of."""
    rng = np.random.default_rng(batch)
    p = Plan(sd, rng.integers(0, 40, batch), 4, batch // 3, batch)
    for i in range(2):
        new = np.where(rng.random(batch) < 0.2, -1, np.where(rng.random(batch) < 0.2, 0, rng.integers(1, 12, batch)))
        p.step([int(n) for n in new], shared=[int(n) for n in rng.integers(0, 20, batch) // 16 * 16] if i else None, max_rows=[None, batch * 4 + 3][i])
        if i == 0:
            pages_once(p)


def test_the_last_free_page_and_none_at_all(sd):
    """Two sequences ask for the one page that is left: the first gets it; with none left only those that need none go on."""
    p = Plan(sd, [16, 16, 5], 4, 1, 1)
    assert p.step([1, 1, 1])["granted"] == [1, 0, 0 + 1]
    assert p.step([1, 1, 1])["granted"] == [1, 0, 1]
    assert p.step([1, 1, -1])["granted"] == [1, 1, 0]
    pages_once(p)


def test_counts_out_of_range(sd):
    """A count of free pages below zero counts as none, one above the pool as the pool; entries outside it are only moved, never followed."""
    import torch
    for count, granted in ((-5, [0, 1]), (10 ** 9, [1, 1])):
        p = Plan(sd, [16, 3], 4, 6, 2)
        d, B = p.d, 2
        out = {name: torch.zeros(8, dtype=torch.int32, device="cuda") for name in NAMES}
        new, free_in, free_out = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([1, 1], [count], [0]))
        sd.kv_plan_step(p.shape, new, None, d["lens"], out["lens_out"], None, None, d["free_pages"], free_in, free_out, d["block_table"], 4, out["granted"], out["row_start"],
                        out["starts"], out["seq_ids"], out["slots"], out["positions"], d["work"], p.ws)
        assert out["granted"][:B].tolist() == granted
        assert free_out.item() == (0 if count < 0 else p.pages - 1)
    p = Plan(sd, [40, 16], 4, 0, 3)
    p.d["block_table"][0, :3] = torch.tensor([-7, 2 ** 31 - 1, 1000], dtype=torch.int32, device="cuda")
    p.table[0][:3] = [-7, 2 ** 31 - 1, 1000]
    p.step([-1, 17], max_rows=17)


def test_places_of_a_quantised_cache(sd):
    """The plan's starts and row_start as kv_append_fp8 takes them, its slots as kv_append does: what every sequence then holds is what it holds on pages chosen by hand."""
    import torch
    B, heads, d, blocks, pages = 6, 2, 64, 9, 60
    gen = torch.Generator(device="cuda").manual_seed(3)
    i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")  # noqa: E731
    dev = lambda a: torch.tensor(np.asarray(a, np.int32), device="cuda")  # noqa: E731
    shapes = [sd.Shape(batch=B, num_q_heads=heads, num_kv_heads=heads, head_dim=d, page_size=16, num_pages=pages, max_blocks_per_seq=blocks, kv_dtype=kind, max_context_len=16 * blocks,
                       chunk_tokens=0) for kind in (sd.SD_FP8_E4M3, sd.SD_BF16)]
    own, hand = i32(B, blocks), torch.arange(B * blocks, dtype=torch.int32, device="cuda").view(B, blocks)
    pools = [[torch.zeros((pages, heads, 16, d), dtype=t, device="cuda") for t in (torch.uint8, torch.uint8, torch.int16, torch.int16)] +
             [torch.zeros((pages, heads), device="cuda") for _ in range(2)] for _ in range(2)]
    lens, free_pages, free, work = i32(B), torch.randperm(pages, generator=gen, device="cuda").int(), dev([pages]), torch.empty(4096, dtype=torch.uint8, device="cuda")
    granted, row_start, starts, every = i32(B), i32(B + 1), i32(B), dev(range(B))
    held = [0] * B
    for new in ([40, 3, 16, 0, 100, 1], [1, 17, -1, 5, 1, 1], [7, 1, 33, 1, -1, 15], [1, 1, 1, 1, 20, 1]):
        rows = sum(n for n in new if n > 0)
        seq, slots = i32(rows), i32(rows)
        sd.kv_plan_step(shapes[0], dev(new), None, lens, lens, None, None, free_pages, free, free, own, rows, granted, row_start, starts, seq, slots, None, work, 4096)
        k, v = (torch.randn((rows, heads, d), generator=gen, device="cuda").bfloat16() for _ in range(2))
        host = dict(seq=[b for b, n in enumerate(new) for _ in range(max(n, 0))], slots=[held[b] + i for b, n in enumerate(new) for i in range(max(n, 0))],
                    start=list(held), row0=[sum(max(n, 0) for n in new[:b]) for b in range(B + 1)])
        for (kq, vq, kb, vb, ks, vs), table, places in ((pools[0], own, (seq, slots, starts, row_start)), (pools[1], hand, [dev(host[n]) for n in ("seq", "slots", "start", "row0")])):
            sd.kv_append_fp8(shapes[0], k, v, every, places[2], places[3], B, max(new), kq, vq, ks, vs, table)
            sd.kv_append(shapes[1], k, v, places[0], places[1], rows, kb, vb, table)
        held = [0 if n < 0 else h + n for h, n in zip(held, new)]
        assert lens.tolist() == held
        for b, n in enumerate(held):
            used = (n + 15) // 16
            for i, (x, y) in enumerate(zip(*pools)):
                x, y = x[own[b, :used].long()], y[hand[b, :used].long()]
                if x.dim() == 4:
                    x, y = (z.transpose(1, 2).reshape(-1, heads, d)[:n] for z in (x, y))
                assert torch.equal(x, y), (new, b, i)
