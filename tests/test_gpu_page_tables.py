"""Page tables built on the GPU against lists, number by number."""
import random

import pytest
import torch

import four_bits as plain
from paper_2604_13847_amd import binding as sb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Both:
    def __init__(self, S, max_pages, num_pages, page, seed=0):
        order = list(range(num_pages))
        random.Random(seed).shuffle(order)
        self.plain, self.pool = plain.Pool(S, max_pages, num_pages, page, order), sb.PagePool.empty(S, max_pages, num_pages, page)
        self.pool.free_pages.copy_(ints(order))
        self.num_pages = num_pages

    def step(self, cached, added, total=None):
        total = sum(max(n, 0) for n in added) if total is None else total
        want = self.plain.step(cached, added, total)
        got = sb.sb_cache_tables(self.pool, ints(cached), ints(added), total)
        for name, a, b in zip(("cu_new", "positions", "slots", "missing"), got, want):
            assert a.tolist() == ([b] if name == "missing" else b), name
        self.same()
        return got

    def same(self):
        p = self.pool
        assert p.held.tolist() == [len(r) for r in self.plain.rows]
        assert p.page_table.tolist() == [r + [-1] * (self.plain.max_pages - len(r)) for r in self.plain.rows]
        n = int(p.free_count[0])
        assert p.free_pages[:n].tolist() == self.plain.free
        assert sorted(self.plain.free + sum(self.plain.rows, [])) == list(range(self.num_pages))


@pytest.mark.parametrize("S,page,longest", [(1, 16, 40), (3, 64, 700), (64, 16, 300), (1023, 16, 60), (1024, 32, 90), (1025, 16, 60), (2500, 128, 500)])
def test_a_life_of_requests(S, page, longest):
    """Requests come, grow by one token, by drafted ones of which some are rejected, by prompts, and leave."""
    rng = random.Random(S)
    most = -(-2 * longest // page) + 2
    x = Both(S, most, S * most // 2 + 5, page, seed=S)
    cached = [0] * S
    for step in range(6):
        added = [rng.choice([0, 1, 1, 4, rng.randint(0, longest), -1 if c else 0]) if c + longest <= most * page else -1 for c in cached]
        x.step(cached, added)
        # of what was added some is rejected
        cached = [0 if n < 0 else c + n - (rng.randint(0, n) if rng.random() < 0.3 else 0) for c, n in zip(cached, added)]
        if step % 2:
            x.step(cached, [0] * S)


def test_a_step_and_its_undoing_leave_everything_as_it_was():
    x = Both(70, 40, 2000, 16)
    cached = [(37 * i) % 500 for i in range(70)]
    x.step([0] * 70, cached)
    before = [t.clone() for t in (x.pool.page_table, x.pool.held, x.pool.free_pages, x.pool.free_count)]
    for added in ([4] * 70, [-1 if i % 3 == 0 else 100 for i in range(70)], [-1] * 70, [-1] * 69 + [130]):
        x.step(cached, added)
        x.step(cached, [0] * 70)
        now = [x.pool.page_table, x.pool.held, x.pool.free_pages, x.pool.free_count]
        n = int(x.pool.free_count[0])
        assert torch.equal(before[0], now[0]) and torch.equal(before[1], now[1]) and torch.equal(before[2][:n], now[2][:n]) and torch.equal(before[3], now[3])


@pytest.mark.parametrize("pages", [0, 1, 7, 30])
def test_too_few_pages(pages):
    """The first rows get what there is; the rest of the entries stay -1, and the call says how many lacked."""
    x = Both(5, 20, pages, 16)
    x.step([0] * 5, [33, 100, 0, 64, 170])
    x.step([33, 100, 0, 64, 170], [20, 1, 40, -1, 1])
    x.step([53, 101, 40, 0, 171], [-1, -1, 0, 5, 1])


def test_lengths_that_the_table_cannot_hold_and_counts_that_cannot_be():
    x = Both(3, 4, 50, 16)
    x.step([0, 60, 1000], [200, 10, 5])
    x.step([-5, 60, 0], [3, 2 ** 31 - 100, 0], total=40)
    pool = sb.PagePool.empty(2, 4, 10, 16)
    pool.held.copy_(ints([-3, 99]))   # taken as 0 and 4
    pool.free_count.fill_(1000)       # taken as 10
    sb.sb_cache_tables(pool, ints([0, 64]), ints([1, 0]), 1)
    assert pool.held.tolist()[0] == 1 and int(pool.free_count[0]) == 9 and int(pool.page_table[0, 0]) == 9


def test_counts_that_cannot_be_are_put_right():
    """Also where a row neither gives back nor lacks a page."""
    pool = sb.PagePool.empty(4, 4, 30, 16)
    sb.sb_cache_tables(pool, ints([0] * 4), ints([64, 64, 64, 0]), 192)
    table = pool.page_table.clone()
    pool.held.copy_(ints([99, 4, 2 ** 31 - 1, -2 ** 31]))
    missing = sb.sb_cache_tables(pool, ints([64, 64, 50, 0]), ints([0, 5000, 0, 0]), 0)[3]
    assert pool.held.tolist() == [4, 4, 4, 0] and torch.equal(pool.page_table, table) and int(pool.free_count[0]) == 18 and int(missing[0]) == 0


def test_sums_of_tokens_stop_at_31_bits():
    pool = sb.PagePool.empty(3, 2, 10, 16)
    cu = sb.sb_cache_tables(pool, ints([0] * 3), ints([2 ** 31 - 1] * 3), 5)[0]
    assert cu.tolist() == [0] + [2 ** 31 - 1] * 3


@pytest.mark.parametrize("total", [0, 1, 4095, 4096, 4097, 30000])
def test_token_counts_about_the_second_launch(total):
    """All tokens by the tables' launch, or by one of their own; rows of the arrays behind the last sequence say that there is no token."""
    x = Both(9, 2000, 2500, 16)
    part = [total // 9 + (i < total % 9) for i in range(9)]
    x.step([5 * i for i in range(9)], part, total=total + 37)
    x.step([0] * 9, [3] * 9, total=11)  # fewer rows than tokens


def test_no_sequences_and_outputs_left_out():
    pool = sb.PagePool.empty(0, 3, 5, 16)
    cu, pos, slots, missing = sb.sb_cache_tables(pool, ints([]), ints([]), 4)
    assert cu.tolist() == [0] and pos.tolist() == [0] * 4 and slots.tolist() == [-1] * 4 and missing.tolist() == [0]
    pool = sb.PagePool.empty(2, 3, 5, 16)
    cached, added, cu = ints([0, 0]), ints([20, 1]), ints([7, 7, 7])
    stream = torch.cuda.current_stream().cuda_stream
    sb._call("sb_cache_tables", sb.C.addressof(pool.c), cached.data_ptr(), added.data_ptr(), 0, cu.data_ptr(), None, None, None, stream)
    assert cu.tolist() == [0, 20, 21] and pool.held.tolist() == [2, 1]
    slots = torch.zeros(21, dtype=torch.int64, device=DEV)
    sb._call("sb_cache_tables", sb.C.addressof(pool.c), cached.data_ptr(), added.data_ptr(), 21, cu.data_ptr(), None, slots.data_ptr(), None, stream)
    assert slots.tolist() == [4 * 16 + i for i in range(16)] + [3 * 16 + i for i in range(4)] + [2 * 16]


def test_slots_behind_31_bits():
    """Pages whose tokens' numbers pass 32 bits (no cache of that size is needed for the tables)."""
    pool = sb.PagePool.empty(1, 4, 3000000, 1024)
    slots = sb.sb_cache_tables(pool, ints([0]), ints([1500]), 1500)[2]
    assert slots[0] == 2999999 * 1024 and slots[1499] == 2999998 * 1024 + 475


def test_a_captured_step_on_another_stream():
    """One captured call serves steps of other lengths; its tables are the eager call's."""
    S = 40
    x = Both(S, 30, 900, 16)
    cached, added = ints([0] * S), ints([0] * S)
    out = sb.sb_cache_tables(x.pool, cached, added, 6000)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        sb.sb_cache_tables(x.pool, cached, added, 6000, *out)
    rng = random.Random(3)
    have = [0] * S
    for _ in range(5):
        n = [rng.choice([1, 4, rng.randint(0, 120)]) if c < 300 else -1 for c in have]
        cached.copy_(ints(have))
        added.copy_(ints(n))
        graph.replay()
        torch.cuda.synchronize()
        want = x.plain.step(have, n, 6000)
        assert [o.tolist() for o in out] == [want[0], want[1], want[2], [want[3]]]
        x.same()
        have = [0 if a < 0 else c + a for c, a in zip(have, n)]
