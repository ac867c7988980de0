"""kv_plan_step where one workgroup ends to do a whole call (256 sequences, 1024 rows), and where it has more pages than threads to take or to give back."""
import numpy as np
import pytest

from tests.test_gpu_plan_step import Plan, pages_once, sd  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("batch", [255, 256, 257])
@pytest.mark.parametrize("max_rows", [1023, 1024, 1025])
def test_borders_of_the_small_call(sd, batch, max_rows):  # noqa: F811
    rng = np.random.default_rng(batch + max_rows)
    p = Plan(sd, rng.integers(0, 200, batch), 40, 2000, batch)
    for i in range(4):
        new = np.where(rng.random(batch) < 0.2, -1, np.where(rng.random(batch) < 0.15, 0, rng.integers(1, 6, batch)))
        p.step([int(n) for n in new], max_rows=max_rows, in_place=i != 2, positions=i != 1)
        pages_once(p)


@pytest.mark.parametrize("batch", [1, 8, 31, 64, 256])
@pytest.mark.parametrize("ends", [1, 3, 100])
def test_thousands_of_pages_come_back(sd, batch, ends):  # noqa: F811
    """Long sequences end in a small call, some of their first pages another's; counts of every remainder by four.  What is taken comes from what came back, or what comes
    back stays on what was free."""
    rng = np.random.default_rng(batch * 10 + ends)
    ends = min(ends, batch)
    for spare in (0, 3, 700):
        lens = rng.integers(0, 600, batch)
        gone = rng.choice(batch, ends, replace=False)
        lens[gone] = rng.integers(9000, 24000, ends) if ends < 50 else rng.integers(500, 3000, ends)
        shared = [0] * batch
        for b in gone[::2]:
            shared[b] = int(rng.integers(0, lens[b] + 40))
        new = [1] * batch
        for b in gone:
            new[b] = -1
        p = Plan(sd, lens, 1600, spare, batch + spare)
        back = sum((int(lens[b]) + 15) // 16 - min(shared[b], int(lens[b])) // 16 for b in gone)
        free = len(p.free)
        want = p.step(new, shared=shared, max_rows=min(1024, batch + 7))
        assert len(p.free) == free + back - sum(bool(n) and s % 16 == 0 for n, s in zip(want["granted"], want["starts"]))
        p.step([3] * batch, max_rows=1024)


@pytest.mark.parametrize("spare", [0, 100, 400])
def test_more_pages_are_taken_than_threads(sd, spare):  # noqa: F811
    """304 pages by 1024 rows of 256 sequences, all of which stand at a page's border, and those of a sequence that ends besides."""
    lens = [16 * (i % 5) for i in range(256)]
    new = [17] * 48 + [1] * 208
    p = Plan(sd, lens, 12, spare, 9)
    p.step(new, max_rows=1024)
    pages_once(p)
    lens[7] = 16 * 350 - 3
    new[7] = -1
    p = Plan(sd, lens, 350, spare, 9)
    p.step(new, max_rows=1024)
    pages_once(p)


@pytest.mark.parametrize("others", [9, 300])
def test_what_waits_holds_back_what_follows(sd, others):  # noqa: F811
    """The first asks for more pages than there are: in every call those behind it that need a page wait, those that need none go on.  In pieces all are served; a length
    that no sequence may have is not counted."""
    lens = [0] + [16 if i % 10 == 0 else 17 + i % 10 for i in range(others)]
    ones = [1] * others
    p = Plan(sd, lens, 100, 80, 4)
    assert p.step([1601] + ones, max_rows=4000)["granted"] == [0] + ones
    p = Plan(sd, lens, 100, 80, 4)
    for _ in range(2):
        goes = [int(n % 16 != 0) for n in p.lens[1:]]
        assert p.step([1584] + ones, max_rows=4000)["granted"] == [0] + goes and 0 in goes
    assert p.step([80] + ones, max_rows=4000)["granted"] == [80] + ones
