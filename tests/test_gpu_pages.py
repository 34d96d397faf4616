"""Page tables kept on the GPU against the same rules on the host, whole numbers throughout."""
import random

import pytest
import torch

import paper_2604_02570_amd as W
from f8_ref import Tables

pytestmark = pytest.mark.gpu
KEPT = -77


class Device:
    """A page pool's memory on the GPU next to its twin on the host."""

    def __init__(self, batch, page_rows, max_pages, n_pages, free, seed=0):
        order = random.Random(seed).sample(range(n_pages), free)
        self.host = Tables(batch, page_rows, max_pages, n_pages, order)
        self.batch, self.ctx = batch, W.wsvd_create(0)
        self.up()
        self.pool = W.make_page_pool(self.table, self.free, batch, page_rows, max_pages, n_pages)

    def up(self):
        i = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        h = self.host
        self.table, self.free, self.lens, self.n_free = i(h.table), i(h.free), i(h.lens), i([h.n_free])

    def same(self):
        h = self.host
        assert self.lens.tolist() == h.lens and self.n_free.tolist() == [h.n_free]
        assert self.free.tolist()[: h.n_free] == h.free[: h.n_free]
        R = h.R
        for b, n in enumerate(h.lens):
            k = min(-(-n // R), h.max_pages)
            assert self.table[b].tolist()[:k] == h.table[b][:k], b

    def grow(self, new, spare=0, in_place=True, one=False):
        n = sum(new)
        cu, positions, slots = (torch.full((k,), KEPT, dtype=torch.int32, device="cuda") for k in (self.batch + 2, n + spare + 1, n + spare + 1))
        lens, n_free = (self.lens, self.n_free) if in_place else (torch.full_like(self.lens, KEPT), torch.full_like(self.n_free, KEPT))
        W.wsvd_pages_grow(self.ctx, self.pool, None if one else torch.tensor(new, dtype=torch.int32, device="cuda"), n + spare, self.lens, self.n_free, lens,
                          n_free, cu, positions, slots)
        self.lens, self.n_free = lens, n_free
        want = self.host.grow(new)
        assert cu.tolist() == want[0] + [KEPT]
        assert positions.tolist() == want[1] + [KEPT] * (spare + 1)
        assert slots.tolist() == want[2] + [KEPT] * (spare + 1)
        self.same()
        return want[3]

    def release(self, done, in_place=True):
        lens, n_free = (self.lens, self.n_free) if in_place else (torch.full_like(self.lens, KEPT), torch.full_like(self.n_free, KEPT))
        W.wsvd_pages_release(self.ctx, self.pool, torch.tensor(done, dtype=torch.int32, device="cuda"), self.lens, self.n_free, lens, n_free)
        self.lens, self.n_free = lens, n_free
        self.host.release(done)
        self.same()

    def close(self, status=0):
        got = W.wsvd_check(self.ctx)
        W.wsvd_destroy(self.ctx)
        assert got == status, W.status_str(got)


@pytest.mark.parametrize("batch,page_rows,most", [(1, 16, 40), (5, 64, 300), (64, 16, 90), (300, 112, 250), (1500, 16, 30)])
@pytest.mark.parametrize("in_place", [True, False])
def test_steps_of_sequences_that_come_and_go(batch, page_rows, most, in_place):
    rng = random.Random(batch + page_rows)
    max_pages = 6 * most // page_rows + 2
    D = Device(batch, page_rows, max_pages, batch * max_pages + 3, batch * max_pages + 3)
    for step in range(6):
        D.release([int(rng.random() < 0.3) for _ in range(batch)], in_place)
        D.grow([rng.choice([0, 1, 1, 1, rng.randint(1, most)]) for _ in range(batch)], spare=rng.choice([0, 5]), in_place=in_place)
    D.release([1] * batch, in_place)
    assert sorted(D.free.tolist()) == list(range(batch * max_pages + 3))
    D.close()


def test_lengths_in_place_beside_a_free_list_that_is_not():
    D = Device(5, 16, 300, 1500, 1500)
    for step in range(3):
        new, n_free = [700, 1, 0, 1300, 40], torch.full_like(D.n_free, KEPT)
        W.wsvd_pages_grow(D.ctx, D.pool, torch.tensor(new, dtype=torch.int32, device="cuda"), sum(new), D.lens, D.n_free, D.lens, n_free)
        D.host.grow(new)
        D.n_free = n_free
        D.same()
    D.close()


def test_one_token_each():
    D = Device(40, 16, 8, 400, 390)
    D.grow([3 * (i % 7) for i in range(40)])
    for _ in range(20):
        D.grow([1] * 40, one=True)
    D.close()


@pytest.mark.parametrize("batch", [3, 1100])
def test_long_prompts(batch):
    """Many workgroups, prompts of one sequence across them; more than 1024 sequences, some of them empty."""
    D = Device(batch, 64, 2000, 6000, 6000)
    D.grow([100000 if b == batch // 2 else 7 * (b % 3) for b in range(batch)], in_place=True)
    D.grow([20000 if b == batch // 2 else 1 for b in range(batch)], spare=9, in_place=False)
    D.release([int(b == batch // 2) for b in range(batch)])
    D.grow([70001 if b == batch - 1 else 0 for b in range(batch)])
    D.close()


@pytest.mark.parametrize("free", [0, 3, 9])
@pytest.mark.parametrize("many", [False, True])
def test_a_free_list_that_ends(free, many):
    """Entries and slots that it cannot serve are -1 and reported; releasing leaves them out."""
    D = Device(6, 16, 300, 900, free)
    assert D.grow([5, 40, 0, 33, 4000 if many else 20, 1])
    assert W.wsvd_check(D.ctx) == W.E_CAPACITY
    D.release([0, 1, 0, 1, 1, 1])
    D.release([1] * 6)
    assert D.host.n_free == free
    D.close()


def test_rows_above_the_pages():
    D = Device(3, 16, 2, 20, 20)
    assert D.grow([30, 40, 32])
    assert W.wsvd_check(D.ctx) == W.E_CAPACITY
    D.close()


def test_numbers_out_of_range_are_reported():
    """Negative lengths and counts, lengths above the table, more tokens than there is room for: taken as the nearest that is allowed."""
    i = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    ctx, B, R, P = W.wsvd_create(0), 4, 16, 3
    table, free = torch.full((B, P), 5, dtype=torch.int32, device="cuda"), torch.arange(40, dtype=torch.int32, device="cuda")
    pool = W.make_page_pool(table, free, B, R, P, 40)

    def grow(new, n, lens, n_free, status=(W.E_SHAPE,)):
        out = [i([KEPT] * B), i([KEPT]), i([KEPT] * (B + 1)), i([KEPT] * (n + 1)), i([KEPT] * (n + 1))]
        W.wsvd_pages_grow(ctx, pool, i(new), n, i(lens), i([n_free]), *out)
        assert W.wsvd_check(ctx) in status
        assert out[3][n] == KEPT and out[4][n] == KEPT
        return [x.tolist() for x in out]
    lens, n_free, cu, positions, slots = grow([1, -3, 2, 0], 3, [-5, 4, 16, 1000], 40)
    assert lens == [1, 4, 18, 48] and n_free == [38] and cu == [0, 1, 1, 3, 3] and positions[:3] == [0, 16, 17] and slots[:3] == [39 * R, 38 * R, 38 * R + 1]
    lens, n_free, cu, positions, slots = grow([2, 2, 2, 2], 5, [0, 0, 0, 0], 10 ** 9)
    assert lens == [2, 2, 1, 0] and n_free == [37] and cu == [0, 2, 4, 5, 5] and positions[:5] == [0, 1, 0, 1, 0]
    most = 2 ** 31 - 1
    lens, n_free, cu, positions, slots = grow([most] * 4, 6, [0] * 4, -4, (W.E_SHAPE, W.E_CAPACITY))
    assert lens == [6, 0, 0, 0] and n_free == [0] and cu == [0, 6, 6, 6, 6] and slots[:6] == [-1] * 6
    free[39] = 40                                                       # no page
    _, _, _, _, slots = grow([1, 0, 0, 0], 1, [0] * 4, 40)
    assert slots[0] == -1
    W.wsvd_destroy(ctx)


def test_counts_that_pass_32_bits_in_sum():
    B, n = 3000, 500
    ctx = W.wsvd_create(0)
    i = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    table, free = torch.zeros(B, 40, dtype=torch.int32, device="cuda"), torch.arange(90, dtype=torch.int32, device="cuda")
    pool = W.make_page_pool(table, free, B, 16, 40, 90)
    out = [i([KEPT] * B), i([KEPT]), i([KEPT] * (B + 1)), i([KEPT] * (n + 1)), i([KEPT] * (n + 1))]
    W.wsvd_pages_grow(ctx, pool, i([7] + [1 << 30] * (B - 1)), n, i([0] * B), i([90]), *out)
    assert W.wsvd_check(ctx) == W.E_SHAPE
    lens, n_free, cu, positions, slots = [x.tolist() for x in out]
    assert lens == [7, 493] + [0] * (B - 2) and n_free == [90 - 1 - 31] and cu == [0, 7] + [n] * (B - 1)
    assert positions == list(range(7)) + list(range(493)) + [KEPT]
    W.wsvd_destroy(ctx)


@pytest.mark.parametrize("batch,max_pages", [(2, 3000), (40, 300), (1300, 20)])
@pytest.mark.parametrize("where", ["nowhere", "first", "last", "some"])
def test_entries_that_are_no_page_are_left_out(batch, max_pages, where):
    """Many workgroups: the pages' order is that of sequences and rows, with and without such entries among them."""
    D = Device(batch, 16, max_pages, batch * max_pages, batch * max_pages)
    rng = random.Random(batch)
    D.grow([16 * max_pages - rng.randrange(50) if b % 3 < 2 else 0 for b in range(batch)])
    spots = [(b, i) for b in range(batch) for i in range(max_pages) if b % 3 < 2 and 16 * i < D.host.lens[b]]
    for b, i in {"nowhere": [], "first": spots[:1], "last": spots[-1:], "some": spots[3::41]}[where]:
        D.host.table[b][i] = rng.choice([-1, D.host.n_pages, -2 ** 31])
    D.table.copy_(torch.tensor(D.host.table, dtype=torch.int32))
    D.release([1] * batch)
    D.close()


def test_a_page_given_back_twice_is_reported():
    i = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    ctx = W.wsvd_create(0)
    table, free = i([[3, 4], [3, 4]]), i([0, 1, 2, KEPT, KEPT])
    pool, n_free = W.make_page_pool(table, free, 2, 16, 2, 5), i([3])
    lens = i([20, 20])
    W.wsvd_pages_release(ctx, pool, i([1, 1]), lens, n_free, lens, n_free)
    assert W.wsvd_check(ctx) == W.E_SHAPE and n_free.tolist() == [5] and free.tolist() == [0, 1, 2, 3, 4] and lens.tolist() == [0, 0]
    W.wsvd_destroy(ctx)


def test_steps_in_a_graph():
    """A step's two calls captured on another stream and replayed, with eager work between: the tables go on by themselves."""
    B, R, P = 12, 16, 40
    D = Device(B, R, P, B * P, B * P)
    done, new = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(2))
    cu, positions, slots = (torch.zeros(k, dtype=torch.int32, device="cuda") for k in (B + 1, 600, 600))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        on = torch.cuda.current_stream()
        W.wsvd_pages_release(D.ctx, D.pool, done, D.lens, D.n_free, D.lens, D.n_free, on)
        W.wsvd_pages_grow(D.ctx, D.pool, new, 600, D.lens, D.n_free, D.lens, D.n_free, cu, positions, slots, on)
    rng = random.Random(3)
    for step in range(8):
        ends, more = [int(rng.random() < 0.2) for _ in range(B)], [rng.choice([0, 1, 1, 50]) for _ in range(B)]
        done.copy_(torch.tensor(ends, dtype=torch.int32))
        new.copy_(torch.tensor(more, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        D.host.release(ends)
        want = D.host.grow(more)
        n = sum(more)
        assert cu.tolist() == want[0] and positions.tolist()[:n] == want[1] and slots.tolist()[:n] == want[2]
        D.same()
    D.close()
