"""Rows taken back: pages that only they reach return to the free list, none is lost, and the rows before them are attended as they were."""
import random

import pytest
import torch

import paper_2604_02570_amd as W
from dense_ref import attend_fast, check, prefix, randn
from f8_ref import F8Pool
from test_gpu_dense import gen
from test_gpu_dense_f8 import Layer
from test_gpu_pages import KEPT, Device as PageTables

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Device(PageTables):
    def keep(self, kept, in_place=True):
        lens, n_free = (self.lens, self.n_free) if in_place else (torch.full_like(self.lens, KEPT), torch.full_like(self.n_free, KEPT))
        W.wsvd_pages_keep(self.ctx, self.pool, ints(kept), self.lens, self.n_free, lens, n_free)
        self.lens, self.n_free = lens, n_free
        h = self.host
        for b, k in enumerate(kept):
            k, n = max(k, 0), min(h.lens[b], h.max_pages * h.R)
            for i in range(-(-min(k, n) // h.R), -(-n // h.R)):
                if 0 <= h.table[b][i] < h.n_pages:
                    h.free[h.n_free] = h.table[b][i]
                    h.n_free += 1
            h.lens[b] = min(h.lens[b], k)
        self.same()

    def pages(self):
        """Every page there is: of the sequences, then free."""
        R, lens = self.host.R, self.lens.tolist()
        return sorted(p for b, row in enumerate(self.table.tolist()) for p in row[: -(-lens[b] // R)]) + self.free.tolist()[: int(self.n_free)]


def test_drafts_that_are_not_accepted():
    """Two sequences whose drafts begin a page; one accepts none of them, one some.  No page is lost over many steps."""
    D = Device(2, 16, 6, 12, 12)
    D.grow([15, 30])
    for step in range(9):
        n = D.host.lens[:]
        D.grow([5, 5])
        D.keep([n[0], n[1] + (step % 2)])
        assert sorted(D.pages()) == list(range(12))
    D.release([1, 1])
    assert sorted(D.free.tolist()) == list(range(12))
    D.close()


@pytest.mark.parametrize("batch,page_rows,most", [(1, 16, 40), (5, 64, 300), (64, 16, 90), (300, 112, 250), (1500, 16, 30)])
@pytest.mark.parametrize("in_place", [True, False])
def test_steps_with_rows_taken_back(batch, page_rows, most, in_place):
    rng = random.Random(batch + page_rows)
    max_pages = 6 * most // page_rows + 2
    total = batch * max_pages + 3
    D = Device(batch, page_rows, max_pages, total, total)
    for step in range(6):
        D.release([int(rng.random() < 0.2) for _ in range(batch)], in_place)
        D.grow([rng.choice([0, 1, rng.randint(1, most)]) for _ in range(batch)], in_place=in_place)
        D.keep([rng.choice([0, n, n + 1, 2 ** 31 - 1, max(n - 1, 0), rng.randint(0, n)]) for n in D.host.lens], in_place)
        assert sorted(D.pages()) == list(range(total))
    D.keep([0] * batch, in_place)
    assert sorted(D.free.tolist()) == list(range(total))
    D.close()


@pytest.mark.parametrize("batch,max_pages", [(2, 3000), (40, 300), (1300, 20)])
@pytest.mark.parametrize("holes", [False, True])
def test_many_pages(batch, max_pages, holes):
    """Many workgroups, with and without entries that are no page among those that go and those that stay."""
    D = Device(batch, 16, max_pages, batch * max_pages, batch * max_pages)
    rng = random.Random(batch)
    D.grow([16 * max_pages - rng.randrange(50) if b % 3 < 2 else 0 for b in range(batch)])
    if holes:
        spots = [(b, i) for b in range(batch) for i in range(max_pages) if b % 3 < 2 and 16 * i < D.host.lens[b]]
        for b, i in spots[3::41]:
            D.host.table[b][i] = rng.choice([-1, D.host.n_pages, -2 ** 31])
        D.table.copy_(ints(D.host.table))
    D.keep([rng.randint(0, 16 * max_pages) for _ in range(batch)])
    D.release([1] * batch)
    D.close()


def test_lengths_kept_where_they_are_written():
    """kept_lens may be seq_lens_out."""
    D = Device(3, 16, 4, 12, 12)
    D.grow([40, 17, 16])
    kept = ints([20, 90, 0])
    W.wsvd_pages_keep(D.ctx, D.pool, kept, D.lens, D.n_free, kept, D.n_free)
    assert kept.tolist() == [20, 17, 0] and int(D.n_free) == 12 - 2 - 2
    D.close()


def test_negative_rows_are_reported():
    D = Device(3, 16, 4, 12, 12)
    D.grow([40, 17, 16])
    D.keep([40, -1, -2 ** 31])
    assert D.host.lens == [40, 0, 0]
    D.close(W.E_SHAPE)


def test_lengths_above_the_table():
    """Rows that no page was left for go without one."""
    D = Device(2, 16, 2, 20, 20)
    assert D.grow([30, 40])
    assert W.wsvd_check(D.ctx) == W.E_CAPACITY
    D.keep([30, 17])
    assert int(D.n_free) == 16
    D.keep([16, 16])
    assert int(D.n_free) == 18
    D.close()


@pytest.mark.parametrize("hq,hkv,d,dtype", [(8, 2, 128, "bf16"), (4, 4, 64, "f16")])
def test_drafts_through_append_and_attention(hq, hkv, d, dtype):
    """Pages, append and attention of draft tokens, of which a part is accepted: rows, scales and outputs follow the definition, step by step."""
    g, B, R, P, n_pages = gen(4), 3, 16, 12, 30
    L, pool = Layer(B, hq, hkv, d, dtype), F8Pool(g, [0] * B, hkv, d, R, dtype, max_pages=P, spare=n_pages)
    cache = L.cache(pool)
    free, n_free, lens = torch.arange(n_pages, dtype=torch.int32, device="cuda"), ints([n_pages]), [0] * B
    tables = W.make_page_pool(L.table, free, B, R, P, n_pages)
    new, accepted = [[15, 33, 3], [5, 4, 6], [3, 2, 9], [8, 1, 2], [4, 20, 4]], [[15, 33, 3], [0, 4, 1], [2, 0, 9], [5, 1, 0], [4, 7, 4]]
    for n, kept in zip(new, accepted):
        T, ld = sum(n), (hq + 2 * hkv) * d
        x, cu = randn(g, dtype, T, ld), torch.empty(B + 1, dtype=torch.int32, device="cuda")
        xd, out = x.cuda(), torch.empty(T, hq * d, dtype=x.dtype, device="cuda")
        W.wsvd_pages_grow(L.ctx, tables, ints(n), T, L.lens, n_free, L.lens, n_free, cu)
        W.wsvd_dense_append_paged_f8(L.ctx, L.desc, None, 0, xd[:, hq * d:], ld, xd[:, (hq + hkv) * d:], ld, T, cu, None, None, None, 0, None, 0, cache)
        W.wsvd_dense_prefill_attn_paged_f8(L.ctx, L.desc, xd, ld, T, cu, cache, out, hq * d)
        pool.table = L.table.cpu()
        at = prefix(n).tolist()
        for b in range(B):
            y = x[at[b]:at[b + 1]].view(n[b], hq + 2 * hkv, d)
            pool.append(b, lens[b], y[:, hq:hq + hkv], y[:, hq + hkv:])
            lens[b] += n[b]
            k, v = pool.rows(b, lens[b])
            want, size = attend_fast(y[:, :hq], k, v, list(range(lens[b] - n[b], lens[b])), L.scale)
            check(out[at[b]:at[b + 1]].cpu().view(n[b], hq, d), want, size, dtype, True)
        L.holds(pool)
        lens = [a - m + k for a, m, k in zip(lens, n, kept)]
        W.wsvd_pages_keep(L.ctx, tables, ints(lens), L.lens, n_free, L.lens, n_free)
        assert L.lens.tolist() == lens
        held = [p for b in range(B) for p in L.table[b, : -(-lens[b] // R)].tolist()]
        assert sorted(held + free[: int(n_free)].tolist()) == list(range(n_pages))
    L.close()


@pytest.mark.parametrize("B,P", [(12, 40), (300, 60)])
def test_in_a_graph(B, P):
    """A step of drafts captured on another stream and replayed with eager work between, as one workgroup and as several: every replay as the rules
    have it."""
    R = 16
    D = Device(B, R, P, B * P, B * P)
    new, kept = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(2))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        on = torch.cuda.current_stream()
        W.wsvd_pages_grow(D.ctx, D.pool, new, 20 * B, D.lens, D.n_free, D.lens, D.n_free, stream=on)
        W.wsvd_pages_keep(D.ctx, D.pool, kept, D.lens, D.n_free, D.lens, D.n_free, on)
    rng = random.Random(3)
    for step in range(8):
        more = [rng.choice([0, 1, 20]) for _ in range(B)]
        stay = [n + rng.randint(0, m) for n, m in zip(D.host.lens, more)]
        new.copy_(ints(more)), kept.copy_(ints(stay))
        graph.replay()
        torch.cuda.synchronize()
        D.host.grow(more)
        h = D.host
        for b, k in enumerate(stay):
            for i in range(-(-k // R), -(-h.lens[b] // R)):
                h.free[h.n_free] = h.table[b][i]
                h.n_free += 1
            h.lens[b] = k
        D.same()
        assert sorted(D.pages()) == list(range(B * P))
    D.close()
