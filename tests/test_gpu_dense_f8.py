"""Dense layers over 8-bit pages on the GPU: the append that quantises, bit for bit, and the attentions over codes, against plain 64-bit forms."""
import math

import pytest
import torch

import paper_2604_02570_amd as W
from dense_ref import DTYPES, F64, attend, attend_fast, check, half_step, prefix, randn, rotate
from f8_ref import BIAS, F8Pool
from test_gpu_dense import BASE, Layer as DenseLayer, gen

pytestmark = pytest.mark.gpu


class Layer(DenseLayer):
    def cache(self, pool, lens=None):
        flat = lambda x: x.reshape(*x.shape[:2], -1).cuda()
        self.k, self.v, self.ks, self.vs = flat(pool.codes["k"]), flat(pool.codes["v"]), pool.scales["k"].cuda(), pool.scales["v"].cuda()
        self.lens = torch.tensor(pool.lens if lens is None else lens, dtype=torch.int32).cuda()
        self.table = pool.table.cuda()
        self.view = W.make_paged_cache(self.k, self.v, self.ks, self.vs, self.lens, self.table, pool.R, pool.max_pages, pool.n_pages)
        return self.view

    def holds(self, pool):
        """Every byte of the pools, those that nobody has written among them."""
        for x, codes, scales in (("k", self.k, self.ks), ("v", self.v, self.vs)):
            assert torch.equal(scales.cpu(), pool.scales[x]), (x, "scales")
            got, want = codes.cpu().view_as(pool.codes[x]), pool.codes[x]
            none = lambda y: (y & 0x7F) == 0x7F                        # (a NaN has two codes)
            same = (got == want) | (none(got) & none(want))
            assert bool(same.all()), (x, int((~same).sum()), (~same).nonzero()[:4].tolist())


# ------------------------------------------------------------------------------------------------ append
HEADS = [(8, 8, 64), (28, 4, 128), (3, 1, 128), (32, 8, 128), (16, 2, 64), (16, 1, 64)]


def append_case(hq, hkv, d, dtype, before, new, page_rows, *, make=None, positions=None, rope=True, ld_extra=0, with_q=True, spare=0, in_place=False,
                growth=0.0, times=1, packed=None):
    """growth: the new rows are 2^growth times as large as those that were there."""
    g, T = gen(5 + d + sum(new)), sum(new)
    L = Layer(len(new), hq, hkv, d, dtype)
    pool = F8Pool(g, [a + b for a, b in zip(before, new)], hkv, d, page_rows, dtype)
    for b, a in enumerate(before):
        pool.append(b, 0, randn(g, dtype, a, hkv, d), randn(g, dtype, a, hkv, d))
    x = randn(g, dtype, T + spare, (hq + 2 * hkv) * d + ld_extra) if make is None else make(g, T + spare, (hq + 2 * hkv) * d + ld_extra)
    x = (x.float() * 2.0 ** growth).to(DTYPES[dtype])
    inv = BASE ** (-torch.arange(0, d, 2, dtype=F64) / d)
    rows = torch.cat([torch.arange(a, a + n) for a, n in zip(before, new)])
    pos = rows if positions is None else positions
    cache = L.cache(pool)
    xd, ld = x.cuda(), (hq + 2 * hkv) * d + ld_extra
    q_out = torch.full((T + spare, hq * d), 7.0, dtype=DTYPES[dtype], device="cuda") if with_q else None
    k_out = torch.full((T + spare, hkv * d + 8), 7.0, dtype=DTYPES[dtype], device="cuda")
    if in_place:
        q_out, k_out, qld, kld = xd, xd[:, hq * d:], ld, ld
    else:
        qld, kld = hq * d, hkv * d + 8
    one = packed is False or (packed is None and all(n == 1 for n in new) and not spare)
    for _ in range(times):
        W.wsvd_dense_append_paged_f8(L.ctx, L.desc, xd if with_q else None, ld, xd[:, hq * d:], ld, xd[:, (hq + hkv) * d:], ld, T + spare,
                                     None if one else prefix(new).cuda(), None if positions is None else positions.int().cuda(),
                                     inv.cuda() if rope else None, q_out, qld, k_out, kld, cache)
    torch.cuda.synchronize()
    y = x[:T, : (hq + 2 * hkv) * d].view(T, hq + 2 * hkv, d)
    want = rotate(y[:, :hq + hkv], pos, inv) if rope else y[:, :hq + hkv].to(F64)
    pair = torch.hypot(want[..., : d // 2], want[..., d // 2:]).repeat(1, 1, 2)
    tol = half_step(dtype) * want.abs() + (2.0 ** -21 * pair if rope else 0) + (2.0 ** -25 if dtype == "f16" and rope else 0)
    near = lambda got, part: bool(((got.cpu().to(F64) - want[:, part]).abs() <= tol[:, part]).all())
    if make is None:
        if with_q:
            assert near(q_out[:T, : hq * d].reshape(T, hq, d), slice(0, hq))
        assert near(k_out[:T, : hkv * d].reshape(T, hkv, d), slice(hq, hq + hkv))
    if not in_place:
        assert (k_out[:, hkv * d:] == 7).all() and (k_out[T:] == 7).all()
        assert not with_q or (q_out[T:] == 7).all()
    # the pools hold what the rule makes of the keys that were returned, and of the values; nothing else has changed
    k, t = k_out[:T, : hkv * d].reshape(T, hkv, d).cpu(), 0
    for b, (a, n) in enumerate(zip(before, new)):
        pool.append(b, a, k[t:t + n], y[t:t + n, hq + hkv:])
        t += n
    L.holds(pool)
    L.close()
    return pool


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("growth", [0.0, 3.0, -9.0])
def test_append_one_token_each(hq, hkv, d, dtype, growth):
    append_case(hq, hkv, d, dtype, [0, 15, 16, 63, 64, 200], [1] * 6, 64, growth=growth)


@pytest.mark.parametrize("hq,hkv,d,dtype", [(28, 4, 128, "bf16"), (8, 8, 64, "f16"), (16, 1, 64, "bf16")])
@pytest.mark.parametrize("page_rows,growth", [(16, 0.0), (112, 1.0)])
def test_append_packed_sequences(hq, hkv, d, dtype, page_rows, growth):
    append_case(hq, hkv, d, dtype, [0, 5, 0, 17, 30, 47], [33, 0, 1, 130, 0, 2], page_rows, ld_extra=24, spare=3, growth=growth)


@pytest.mark.parametrize("new", [[900, 1, 1500, 16, 1700], [61] * 67 + [0, 37]])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_append_large_calls(new, dtype):
    # several tokens a workgroup: blocks across their borders
    assert sum(new) >= 4096
    append_case(2, 1, 64, dtype, [(13 * i) % 37 for i in range(len(new))], new, 32, spare=2)


def test_append_many_short_sequences():
    append_case(2, 1, 64, "bf16", [(7 * i) % 40 for i in range(700)], [(i % 12) for i in range(700)], 16)


def test_append_one_token_of_many_sequences():
    append_case(2, 1, 64, "f16", [(7 * i) % 40 for i in range(333)], [1] * 333, 16)
    append_case(2, 1, 64, "f16", [(7 * i) % 40 for i in range(333)], [1] * 333, 16, packed=True)


def test_append_far_positions():
    append_case(8, 2, 64, "f16", [3, 0, 19], [1, 1, 1], 64, positions=torch.tensor([900001, 5, 131072]))
    append_case(8, 2, 128, "bf16", [3, 0], [40, 9], 64, positions=torch.arange(49) * 21000 + 7)


def test_append_without_rotation_and_without_queries():
    append_case(4, 2, 128, "bf16", [9, 0], [5, 20], 16, rope=False)
    append_case(4, 2, 64, "f16", [9, 0], [5, 20], 16, with_q=False)


def test_append_in_place():
    append_case(8, 2, 128, "bf16", [9, 0], [5, 20], 16, in_place=True)
    append_case(8, 2, 64, "f16", [9, 1], [1, 1], 16, in_place=True)


def test_append_again_changes_nothing():
    append_case(8, 2, 128, "bf16", [9, 0], [5, 20], 16, growth=2.0, times=3)


SPECIAL = {"zeros": lambda x, i: x * 0, "infinite": lambda x, i: x.masked_fill(i % 37 == 5, math.inf).masked_fill(i % 41 == 7, -math.inf),
           "none": lambda x, i: x.masked_fill(i % 53 == 3, math.nan), "nothing finite": lambda x, i: torch.full_like(x, math.nan),
           "largest": lambda x, i: x.clamp(-1, 1) * 3.3e38, "smallest": lambda x, i: x * 2.0 ** -130, "tiny": lambda x, i: x * 2.0 ** -105,
           "spread": lambda x, i: x * torch.exp2((i % 47).float() - 23)}


@pytest.mark.parametrize("name", SPECIAL)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128])
def test_append_special_numbers(name, dtype, d):
    """Without rotation, so that keys are quantised as they are given; behind rows of size 1, and at a block's start."""
    def make(g, n, width):
        x = torch.randn(n, width, generator=g)
        y = SPECIAL[name](x, torch.arange(n * width).view(n, width))
        if name in ("largest", "smallest") and dtype == "f16":
            y = y.clamp(-65504, 65504) if name == "largest" else x * 2.0 ** -23
        return y.to(DTYPES[dtype])
    append_case(2, 2, d, dtype, [5, 0, 16], [20, 7, 1], 32, make=make, rope=False)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_append_token_by_token(dtype):
    """40 calls of one token, of sizes from 2^-6 to 2^6: every byte after each."""
    hq, hkv, d, g = 2, 2, 64, gen(11)
    L, pool = Layer(2, hq, hkv, d, dtype), F8Pool(g, [40, 57], hkv, d, 16, dtype)
    cache = L.cache(pool)
    for step in range(40):
        L.lens.copy_(torch.tensor([step + 1, step + 18], dtype=torch.int32))
        size = torch.exp2(torch.randint(-6, 7, (2, 1, 1), generator=g).float())
        k, v = ((torch.randn(2, hkv, d, generator=g) * size).to(DTYPES[dtype]) for _ in "kv")
        if step == 0:                                                   # the second sequence's first 17 rows
            a, b = randn(g, dtype, 17, hkv, d), randn(g, dtype, 17, hkv, d)
            pool.append(1, 0, a, b)
            L.cache(pool)
            cache = L.view
            L.lens.copy_(torch.tensor([1, 18], dtype=torch.int32))
        W.wsvd_dense_append_paged_f8(L.ctx, L.desc, None, 0, k.cuda(), hkv * d, v.cuda(), hkv * d, 2, None, None, None, None, 0, None, 0, cache)
        for b, row in ((0, step), (1, step + 17)):
            pool.append(b, row, k[b:b + 1], v[b:b + 1])
        L.holds(pool)
    L.close()


@pytest.mark.parametrize("lens,entry,status", [([5, 40], None, W.E_CAPACITY), ([1, 3], None, W.E_SHAPE), ([5, 20], 99, W.E_SHAPE), ([5, 20], -1, W.E_SHAPE)])
def test_append_bad_rows_and_pages_store_nothing(lens, entry, status):
    """The second sequence's rows lie past its pages, before its first row, or on no page: the others are stored, queries are rotated."""
    hq, hkv, d, new, g = 2, 1, 64, [3, 9], gen(3)
    L, pool = Layer(2, hq, hkv, d, "bf16"), F8Pool(g, [16, 32], hkv, d, 16, "bf16")
    if entry is not None:
        pool.table[1, 0] = entry                                        # rows 11 .. 15; 16 .. 19 have a page
    x = randn(g, "bf16", 12, 4 * d)
    out = torch.empty(12, hq * d, dtype=torch.bfloat16, device="cuda")
    W.wsvd_dense_append_paged_f8(L.ctx, L.desc, x.cuda(), 4 * d, x.cuda()[:, 2 * d:], 4 * d, x.cuda()[:, 3 * d:], 4 * d, 12, prefix(new).cuda(), None, None, out,
                                 hq * d, None, 0, L.cache(pool, lens))
    k, v = x[:, 2 * d:3 * d].view(12, 1, d), x[:, 3 * d:].view(12, 1, d)
    rows = list(range(lens[0] - 3, lens[0])) + list(range(lens[1] - 9, lens[1]))
    start = 0
    while start < 12:                                                   # the calls' rows block by block, as far as they are somewhere
        b = 0 if start < 3 else 1
        stop = start + 1
        while stop < (3 if b == 0 else 12) and rows[stop] % 16 and rows[stop] >= 1:
            stop += 1
        if 0 <= rows[start] < 16 * pool.max_pages and 0 <= int(pool.table[b, rows[start] // 16]) < pool.n_pages:
            pool.append(b, rows[start], k[start:stop], v[start:stop])
        start = stop
    L.holds(pool)
    assert torch.equal(out.cpu(), x[:, :2 * d])
    L.close(status)


# ------------------------------------------------------------------------------------------------ decode
def decode_case(lens, hq, hkv, d, dtype, page_rows, *, scale=0.0, ld_extra=0, q_scale=1.0, max_len=None, min_chunk=0, peaked=False, spread=3):
    g = gen(9 + sum(lens))
    L, pool = Layer(len(lens), hq, hkv, d, dtype, scale), F8Pool(g, lens, hkv, d, page_rows, dtype).random(g, spread)
    W.wsvd_ctx_set_option(L.ctx, "min_chunk", min_chunk)
    q = randn(g, dtype, len(lens), hq * d + ld_extra, scale=q_scale)
    out = torch.full((len(lens), hq, d), 7.0, dtype=DTYPES[dtype], device="cuda")
    W.wsvd_dense_decode_attn_paged_f8(L.ctx, L.desc, q.cuda(), hq * d + ld_extra, L.cache(pool), max_len or max(lens), out)
    got = out.cpu()
    for b, n in enumerate(lens):
        k, v = pool.rows(b)
        want, size = attend_fast(q[b:b + 1, : hq * d].view(1, hq, d), k, v, [n - 1], L.scale)
        check(got[b:b + 1], want, size, dtype, False)
    L.close()
    return got


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_decode_lengths_around_tiles(hq, hkv, d, dtype):
    decode_case([0, 1, 15, 16, 17, 31, 32, 33, 64, 100, 129, 257], hq, hkv, d, dtype, 16)


@pytest.mark.parametrize("page_rows", [16, 48, 128])
def test_decode_split_and_joined(page_rows):
    decode_case([2100, 0, 700, 1300, 5], 8, 2, 128, "bf16", page_rows)


@pytest.mark.parametrize("d,dtype", [(64, "f16"), (128, "bf16")])
def test_decode_one_long_sequence(d, dtype):
    decode_case([9001], 4, 1, d, dtype, 64)


@pytest.mark.parametrize("hq,hkv,d,min_chunk", [(8, 2, 128, 128), (16, 1, 64, 256), (4, 4, 64, 64)])
def test_decode_small_chunks(hq, hkv, d, min_chunk):
    decode_case([900, 130, 64, 0, 2049], hq, hkv, d, "bf16", 16, min_chunk=min_chunk)


@pytest.mark.parametrize("batch,hq,hkv,d", [(70, 8, 8, 64), (140, 8, 4, 64), (1100, 2, 1, 64), (70, 16, 16, 128)])
def test_decode_many_units(batch, hq, hkv, d):
    decode_case([(7 * i) % 50 for i in range(batch)], hq, hkv, d, "bf16", 16)


def test_decode_strides_and_scale():
    decode_case([33, 70], 12, 4, 64, "f16", 32, scale=0.3, ld_extra=40)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_decode_peaked_scores(dtype):
    decode_case([300, 64, 1000], 8, 2, 128, dtype, 16, scale=1.0, q_scale=0.5)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_decode_scales_far_apart(dtype):
    decode_case([300, 64, 1000], 8, 2, 64, dtype, 16, spread=9, q_scale=0.3)


@pytest.mark.parametrize("d,dtype", [(64, "f16"), (128, "bf16")])
def test_decode_chunks_of_many_tiles(d, dtype):
    # a wave looks its tiles up 32 at a time
    decode_case([9001, 20000, 8192 + 8192], 2, 1, d, dtype, 16, min_chunk=32768)


LONG = [([9000, 0, 4000, 17], 8, 2, 64, "f16"), ([3000, 2900], 28, 4, 128, "bf16"), ([2500], 16, 1, 128, "f16"), ([5000, 1, 700, 6001, 6000, 0, 3, 2048], 7, 1, 64, "bf16"),
        ([33000], 13, 1, 128, "bf16"), ([1700] * 16, 10, 2, 64, "f16"), ([4100], 16, 16, 128, "bf16"), ([2, 40000], 8, 8, 64, "f16")]


@pytest.mark.parametrize("lens,hq,hkv,d,dtype", LONG)
def test_decode_sequences_of_many_chunks(lens, hq, hkv, d, dtype):
    # joined by workgroups of their own, next to sequences that are not
    decode_case(lens, hq, hkv, d, dtype, 64, ld_extra=16)


@pytest.mark.parametrize("lens,hq,hkv,d,dtype", [LONG[0], LONG[1]])
def test_decode_sequences_of_many_chunks_values_that_are_none(lens, hq, hkv, d, dtype):
    g = gen(8)
    L, pool = Layer(len(lens), hq, hkv, d, dtype), F8Pool(g, lens, hkv, d, 64, dtype).random(g)
    last = 2 if len(lens) > 2 else 1
    pool.set("v", 0, lens[0] - 1, hkv - 1, 5, 0x7F), pool.set("v", 0, 3, 0, d - 1, 0xFF), pool.set("k", last, 1500, 0, 7, 0x7F)
    q, out = randn(g, dtype, len(lens), hq * d), torch.empty(len(lens), hq, d, dtype=DTYPES[dtype], device="cuda")
    W.wsvd_dense_decode_attn_paged_f8(L.ctx, L.desc, q.cuda(), hq * d, L.cache(pool), max(lens), out)
    want = torch.zeros(len(lens), hq, d, dtype=torch.bool)
    want[0, hq - hq // hkv:, 5] = True
    want[0, : hq // hkv, d - 1] = want[last, : hq // hkv] = True
    assert torch.equal(out.cpu().isnan(), want)
    L.close()


def test_decode_of_many_chunks_leaves_the_workspace_as_it_was():
    """Calls of other forms over one workspace, again and again: every call's bits stay what they were, also with the sequences in another order."""
    g, lens, hq, hkv, d = gen(77), [9000, 64, 4000, 0], 8, 2, 128
    pool, L = F8Pool(g, lens, hkv, d, 16, "bf16").random(g), Layer(4, hq, hkv, d, "bf16")
    q, qc, outs = randn(g, "bf16", 4, hq * d), randn(g, "bf16", 40, hq * d), []
    for order in ([0, 1, 2, 3], [2, 0, 3, 1], [0, 1, 2, 3]):
        cache = L.cache(pool, [lens[i] for i in order])
        L.table.copy_(pool.table[order])
        out, few, chunk = (torch.empty(n, hq * d, dtype=torch.bfloat16, device="cuda") for n in (4, 3, 40))
        W.wsvd_dense_decode_attn_paged_f8(L.ctx, L.desc, q[order].contiguous().cuda(), hq * d, cache, 9000, out)
        W.wsvd_dense_prefill_attn_paged_f8(L.ctx, L.desc, qc.cuda(), hq * d, 3, prefix([2, 1, 0, 0]).cuda(), cache, few, hq * d)
        W.wsvd_dense_prefill_attn_paged_f8(L.ctx, L.desc, qc.cuda(), hq * d, 40, prefix([39, 1, 0, 0]).cuda(), cache, chunk, hq * d)
        again = torch.empty_like(out)
        W.wsvd_dense_decode_attn_paged_f8(L.ctx, L.desc, q[order].contiguous().cuda(), hq * d, cache, 9000, again)
        assert torch.equal(out, again)
        outs.append((out.cpu()[[order.index(i) for i in range(4)]], few.cpu(), chunk.cpu()))
    assert torch.equal(outs[0][0], outs[1][0]) and all(torch.equal(a, b) for a, b in zip(outs[0], outs[2]))
    L.close()


def test_joined_calls_in_graphs_that_share_a_workspace():
    """Two graphs of long sequences' decode and few tokens over one workspace, replayed in turn with eager calls between, lengths changing."""
    g, hq, hkv, d = gen(91), 8, 2, 64
    pool, L = F8Pool(g, [9000, 4000], hkv, d, 64, "f16").random(g), Layer(2, hq, hkv, d, "f16")
    cache, q, cu = L.cache(pool), randn(g, "f16", 6, hq * d).cuda(), prefix([4, 2]).cuda()

    def calls(out, few, stream=None):
        W.wsvd_dense_decode_attn_paged_f8(L.ctx, L.desc, q, hq * d, cache, 9000, out, stream)
        W.wsvd_dense_prefill_attn_paged_f8(L.ctx, L.desc, q, hq * d, 6, cu, cache, few, hq * d, stream)

    new = lambda: (torch.zeros(2, hq * d, dtype=torch.float16, device="cuda"), torch.zeros(6, hq * d, dtype=torch.float16, device="cuda"))
    want = new()
    calls(*want)
    graphs = []
    for _ in range(2):
        outs, graph = new(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            calls(*outs, torch.cuda.current_stream())
        graphs.append((graph, outs))
    for lens in ([9000, 4000], [9000, 4000], [8999, 30], [2000, 0], [9000, 4000]):
        L.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        eager = new()
        calls(*eager)
        for graph, outs in graphs:
            for x in outs:
                x.fill_(3)
            graph.replay()
            assert all(torch.equal(a, b) for a, b in zip(outs, eager)), lens
        torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, want))
    L.close()


def test_decode_of_nothing():
    L, pool = Layer(3, 4, 2, 64, "bf16"), F8Pool(gen(2), [0, 0, 0], 2, 64, 16, "bf16")
    out = torch.full((3, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    W.wsvd_dense_decode_attn_paged_f8(L.ctx, L.desc, randn(gen(3), "bf16", 3, 256).cuda(), 256, L.cache(pool), 0, out)
    assert (out == 0).all()
    L.close()


@pytest.mark.parametrize("what", ["decode", "chunk"])
def test_sequences_that_share_pages(what):
    """A prefix that two sequences have in common: its pages are in both rows of the table."""
    g, hq, hkv, d = gen(5), 4, 2, 128
    L, pool = Layer(3, hq, hkv, d, "bf16"), F8Pool(g, [100, 70, 100], hkv, d, 16, "bf16").random(g)
    pool.table[1, :4] = pool.table[0, :4]
    pool.table[2] = pool.table[0]
    T = 3 if what == "decode" else 9
    q, out = randn(g, "bf16", T, hq * d), torch.empty(T, hq * d, dtype=torch.bfloat16, device="cuda")
    if what == "decode":
        W.wsvd_dense_decode_attn_paged_f8(L.ctx, L.desc, q.cuda(), hq * d, L.cache(pool), 100, out)
    else:
        W.wsvd_dense_prefill_attn_paged_f8(L.ctx, L.desc, q.cuda(), hq * d, T, prefix([3, 3, 3]).cuda(), L.cache(pool), out, hq * d)
    m = T // 3
    for b, n in enumerate(pool.lens):
        k, v = pool.rows(b)
        want, size = attend_fast(q[b * m:(b + 1) * m].view(m, hq, d), k, v, list(range(n - m, n)), L.scale)
        check(out[b * m:(b + 1) * m].cpu().view(m, hq, d), want, size, "bf16", what == "chunk")
    L.close()


def test_decode_longer_than_the_bound_is_reported():
    g = gen(4)
    L, pool = Layer(1, 4, 2, 64, "bf16"), F8Pool(g, [100], 2, 64, 16, "bf16").random(g)
    q, out = randn(g, "bf16", 1, 256), torch.empty(1, 4, 64, dtype=torch.bfloat16, device="cuda")
    W.wsvd_dense_decode_attn_paged_f8(L.ctx, L.desc, q.cuda(), 256, L.cache(pool), 50, out)
    k, v = pool.rows(0, 50)
    want, size = attend(q.view(1, 4, 64), k, v, [49], L.scale)
    check(out.cpu(), want, size, "bf16", False)
    L.close(W.E_SHAPE)


@pytest.mark.parametrize("what", ["decode", "chunk"])
def test_bad_page_is_reported(what):
    g = gen(6)
    L, pool = Layer(2, 4, 2, 64, "bf16"), F8Pool(g, [40, 20], 2, 64, 16, "bf16", fill=0).random(g)
    pool.scales["k"].fill_(120), pool.scales["v"].fill_(120)
    pool.table[0, 1] = pool.n_pages                                     # read as page 0
    cache = L.cache(pool)
    pool.table[0, 1] = 0
    if what == "decode":
        q, out = randn(g, "bf16", 2, 256), torch.empty(2, 4, 64, dtype=torch.bfloat16, device="cuda")
        W.wsvd_dense_decode_attn_paged_f8(L.ctx, L.desc, q.cuda(), 256, cache, 48, out)
    else:
        q, out = randn(g, "bf16", 7, 256), torch.empty(7, 256, dtype=torch.bfloat16, device="cuda")
        W.wsvd_dense_prefill_attn_paged_f8(L.ctx, L.desc, q.cuda(), 256, 7, prefix([3, 4]).cuda(), cache, out, 256)
    at = 0
    for b, (n, nq) in enumerate(((40, 1), (20, 1)) if what == "decode" else ((40, 3), (20, 4))):
        k, v = pool.rows(b)
        want, size = attend(q[at:at + nq].view(nq, 4, 64), k, v, list(range(n - nq, n)), L.scale)
        check(out.cpu().view(-1, 4, 64)[at:at + nq], want, size, "bf16", what == "chunk")
        at += nq
    L.close(W.E_SHAPE)


@pytest.mark.parametrize("d,dtype", [(64, "f16"), (128, "bf16")])
@pytest.mark.parametrize("min_chunk", [0, 128])
def test_decode_values_that_are_none(d, dtype, min_chunk):
    """A value that is none makes none of its dim for the heads of its kv head; a key that is none of all that they have."""
    g, hq, hkv, lens = gen(8), 6, 2, [300, 33]
    L, pool = Layer(2, hq, hkv, d, dtype), F8Pool(g, lens, hkv, d, 16, dtype).random(g)
    W.wsvd_ctx_set_option(L.ctx, "min_chunk", min_chunk)
    pool.set("v", 0, 299, 1, 5, 0x7F), pool.set("v", 0, 17, 0, d - 1, 0xFF), pool.set("k", 1, 32, 0, 7, 0x7F)
    q, out = randn(g, dtype, 2, hq * d), torch.empty(2, hq, d, dtype=DTYPES[dtype], device="cuda")
    W.wsvd_dense_decode_attn_paged_f8(L.ctx, L.desc, q.cuda(), hq * d, L.cache(pool), 300, out)
    got = out.cpu()
    none = torch.zeros(2, hq, d, dtype=torch.bool)
    none[0, 3:, 5] = none[0, :3, d - 1] = none[1, :3] = True
    assert torch.equal(torch.isnan(got), none)
    for b, n in enumerate(lens):
        k, v = pool.rows(b)
        want, size = attend(q[b:b + 1].view(1, hq, d), k.nan_to_num(0), v.nan_to_num(0), [n - 1], L.scale)
        fine = ~none[b:b + 1]
        check(got[b:b + 1][fine], want[fine], size[fine], dtype, False)
    L.close()


# ------------------------------------------------------------------------------------------------ tokens behind cached ones
def chunk_case(lens, new, hq, hkv, d, dtype, page_rows, *, scale=0.0, ld_extra=0, spare=0, q_scale=1.0, on_gpu=False, none=()):
    g = gen(21 + sum(lens))
    T = sum(new)
    L, pool = Layer(len(lens), hq, hkv, d, dtype, scale), F8Pool(g, lens, hkv, d, page_rows, dtype).random(g)
    for at in none:
        pool.set(*at)
    q = randn(g, dtype, T + spare, hq * d + ld_extra, scale=q_scale)
    out = torch.full((T + spare, hq * d + 8), 7.0, dtype=DTYPES[dtype], device="cuda")
    W.wsvd_dense_prefill_attn_paged_f8(L.ctx, L.desc, q.cuda(), hq * d + ld_extra, T + spare, prefix(new).cuda(), L.cache(pool), out, hq * d + 8)
    got, at = out.cpu(), 0
    assert (got[:, hq * d:] == 7).all() and (got[T:] == 7).all()
    for b, (n, m) in enumerate(zip(lens, new)):
        if m == 0:
            continue
        k, v = pool.rows(b)
        mine, queries = got[at:at + m, : hq * d].reshape(m, hq, d), q[at:at + m, : hq * d].reshape(m, hq, d)
        if on_gpu:
            queries, k, v = queries.cuda(), k.cuda(), v.cuda()
            rows = torch.arange(n, device="cuda")
            hidden = rows[None, :] > rows[n - m:, None]
            want, size = torch.empty(m, hq, d, dtype=F64), torch.empty(m, hq, d, dtype=F64)
            for h in range(hq):
                w = torch.softmax((queries[:, h].to(F64) @ k[:, h * hkv // hq].t().contiguous() * L.scale).masked_fill(hidden, -math.inf), 1)
                want[:, h], size[:, h] = (w @ v[:, h * hkv // hq].contiguous()).cpu(), (w @ v[:, h * hkv // hq].abs().contiguous()).cpu()
        else:
            last = list(range(n - m, n))
            bad = torch.zeros(m, hq, d, dtype=torch.bool)
            for x, bb, row, h, dim, _ in none:
                if bb == b and x == "v":
                    for i in range(m):
                        if row <= last[i]:
                            bad[i, h * hq // hkv:(h + 1) * hq // hkv, dim] = True
            want, size = attend_fast(queries, k, v.nan_to_num(0), last, L.scale)
            assert torch.equal(torch.isnan(mine), bad)
            mine, want, size = mine[~bad], want[~bad], size[~bad]
        check(mine, want, size, dtype, True)
        at += m
    L.close()


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_chunk_behind_cached_rows(hq, hkv, d, dtype):
    chunk_case([70, 33, 16, 200, 1, 129], [5, 33, 0, 70, 1, 16], hq, hkv, d, dtype, 16, spare=2)


@pytest.mark.parametrize("page_rows", [16, 48, 112, 256])
def test_chunk_page_sizes_and_strides(page_rows):
    chunk_case([300, 64, 63, 65], [100, 64, 1, 2], 8, 2, 128, "bf16", page_rows, ld_extra=40, scale=0.2)


@pytest.mark.parametrize("hq,hkv,d,dtype", [(4, 1, 128, "bf16"), (8, 2, 64, "f16"), (2, 2, 128, "f16")])
def test_chunk_shared_by_workgroups(hq, hkv, d, dtype):
    chunk_case([3000, 900], [7, 40], hq, hkv, d, dtype, 64)


FEW = [([700, 64, 0, 1501, 17], [5, 1, 0, 3, 4], 8, 8, 64, "f16"), ([700, 64, 33, 1501, 5], [5, 1, 0, 3, 5], 8, 2, 128, "bf16"), ([3000], [7], 32, 8, 128, "bf16"),
       ([2999, 40], [6, 2], 7, 1, 64, "bf16"), ([100, 100], [3, 1], 16, 1, 128, "f16"), ([2500, 7, 9, 64], [40, 0, 0, 1], 4, 2, 64, "f16"), ([9001], [1], 3, 1, 64, "f16"), ([20, 12], [20, 12], 4, 2, 128, "bf16")]


@pytest.mark.parametrize("lens,new,hq,hkv,d,dtype", FEW)
@pytest.mark.parametrize("page_rows", [16, 112])
def test_chunk_of_a_few_tokens(lens, new, hq, hkv, d, dtype, page_rows):
    # (token, head) pairs as columns, tiles of 16 that end inside a token's heads
    chunk_case(lens, new, hq, hkv, d, dtype, page_rows, spare=1, ld_extra=16)


@pytest.mark.parametrize("lens,new,hq,hkv,d,dtype", [FEW[1], FEW[2], FEW[4]])
def test_chunk_of_a_few_tokens_values_that_are_none(lens, new, hq, hkv, d, dtype):
    """Of rows that some of a tile's columns see and others do not, of rows that all see, and of the same dim twice."""
    n, m = lens[0], new[0]
    chunk_case(lens, new, hq, hkv, d, dtype, 16, none=[("v", 0, n - 1, 0, 3, 0x7F), ("v", 0, n - 2, 0, d - 1, 0xFF), ("v", 0, n - m + 1, 0, d - 1, 0x7F), ("v", 0, n - m, 0, 17, 0xFF),
                                                       ("v", 0, n - 4, hkv - 1, 33, 0x7F), ("v", 0, 2, hkv - 1, 40, 0x7F)])


JOINED = [([8000], [4], 28, 4, 128, "bf16"), ([9000, 30, 5000, 0], [8, 1, 3, 0], 8, 2, 64, "f16"), ([16000], [5], 16, 16, 64, "bf16"), ([7000, 3], [3, 3], 16, 1, 128, "f16"),
          ([3001, 3000], [9, 7], 7, 1, 64, "f16"), ([20000], [1], 8, 8, 128, "bf16")]


@pytest.mark.parametrize("lens,new,hq,hkv,d,dtype", JOINED)
def test_chunk_of_a_few_tokens_behind_many_rows(lens, new, hq, hkv, d, dtype):
    # the chunks of a tile joined by workgroups of their own, a pair each
    chunk_case(lens, new, hq, hkv, d, dtype, 64, spare=1, ld_extra=16)


@pytest.mark.parametrize("lens,new,hq,hkv,d,dtype", [JOINED[0], JOINED[1], JOINED[4]])
def test_chunk_of_a_few_tokens_behind_many_rows_values_that_are_none(lens, new, hq, hkv, d, dtype):
    n, m = lens[0], new[0]
    chunk_case(lens, new, hq, hkv, d, dtype, 64, none=[("v", 0, n - 1, 0, 3, 0x7F), ("v", 0, n - 2, 0, d - 1, 0xFF), ("v", 0, n - m, 0, 17, 0xFF), ("v", 0, n // 2, hkv - 1, 33, 0x7F)])


MANY = [(40, 8, 16, 4, 64, "bf16"), (40, 7, 16, 4, 128, "f16"), (20, 16, 16, 8, 128, "bf16"), (150, 5, 7, 1, 64, "f16"), (10, 30, 15, 15, 64, "bf16"), (17, 3, 112, 8, 128, "f16")]


@pytest.mark.parametrize("batch,most,hq,hkv,d,dtype", MANY)
def test_chunk_of_a_few_tokens_of_many_sequences(batch, most, hq, hkv, d, dtype):
    # tiles of 32 pairs where those of 16 would be more than the chip has CUs: sequences that fill one set and part of the other, one set, one pair, none
    lens = [(67 * i) % 300 + most for i in range(batch)]
    lens[1], lens[2] = 2100, most
    chunk_case(lens, [(1, most, 0, most - 1, most)[i % 5] for i in range(batch)], hq, hkv, d, dtype, 48, spare=1, ld_extra=16)


@pytest.mark.parametrize("batch,most,hq,hkv,d,dtype", [MANY[0], MANY[1]])
def test_chunk_of_a_few_tokens_of_many_sequences_values_that_are_none(batch, most, hq, hkv, d, dtype):
    lens = [(67 * i) % 300 + most for i in range(batch)]
    n = lens[1]
    chunk_case(lens, [most] * batch, hq, hkv, d, dtype, 16, none=[("v", 1, n - 1, 0, 3, 0x7F), ("v", 1, n - 2, 0, d - 1, 0xFF), ("v", 1, n - most + 1, 0, d - 1, 0x7F), ("v", 1, n - most, 0, 17, 0xFF),
                                                                  ("v", 1, n - 5, hkv - 1, 33, 0x7F), ("v", 1, 2, hkv - 1, 40, 0x7F)])


def test_chunk_of_a_few_tokens_gives_a_sequence_the_same_bits_in_every_place():
    g, lens, new, hq, hkv, d = gen(45), [700, 33, 2100, 0, 64], [3, 2, 4, 0, 1], 8, 2, 128
    pool = F8Pool(g, lens, hkv, d, 16, "bf16").random(g)
    q = [randn(g, "bf16", m, hq * d) for m in new]
    L, outs = Layer(5, hq, hkv, d, "bf16"), []
    for order in ([0, 1, 2, 3, 4], [4, 2, 0, 1, 3], [0, 1, 2, 3, 4]):
        cache = L.cache(pool, [lens[i] for i in order])
        L.table.copy_(pool.table[order])
        out = torch.empty(10, hq * d, dtype=torch.bfloat16, device="cuda")
        W.wsvd_dense_prefill_attn_paged_f8(L.ctx, L.desc, torch.cat([q[i] for i in order]).cuda(), hq * d, 10, prefix([new[i] for i in order]).cuda(), cache, out, hq * d)
        at = dict(zip(order, prefix([new[i] for i in order]).tolist()))
        outs.append(torch.cat([out.cpu()[at[i]:at[i] + new[i]] for i in range(5)]))
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    L.close()


def test_chunk_many_sequences():
    chunk_case([(7 * i) % 90 + 5 for i in range(150)], [i % 6 for i in range(150)], 4, 2, 64, "bf16", 16, spare=1)


def test_chunk_queries_that_see_nothing_give_zeros():
    """More queries than rows: the first ones lie before the sequence's first row."""
    g = gen(31)
    L, pool = Layer(2, 4, 2, 64, "bf16"), F8Pool(g, [3, 0], 2, 64, 16, "bf16").random(g)
    q, out = randn(g, "bf16", 12, 256), torch.full((12, 256), 7.0, dtype=torch.bfloat16, device="cuda")
    W.wsvd_dense_prefill_attn_paged_f8(L.ctx, L.desc, q.cuda(), 256, 12, prefix([8, 4]).cuda(), L.cache(pool), out, 256)
    k, v = pool.rows(0)
    want, size = attend(q[:8].view(8, 4, 64), k, v, list(range(-5, 3)), L.scale)
    check(out[:8].cpu().view(8, 4, 64), want, size, "bf16", True)
    assert (out[:5] == 0).all() and (out[8:] == 0).all()
    L.close()


@pytest.mark.parametrize("d,dtype", [(64, "f16"), (128, "bf16")])
@pytest.mark.parametrize("lens,new", [([300, 40], [130, 40]), ([2000, 40], [20, 3])])
def test_chunk_values_that_are_none(d, dtype, lens, new):
    """They make none of their dim for the queries that see them, and have no effect on the others."""
    n = lens[0]
    chunk_case(lens, new, 4, 2, d, dtype, 16, none=[("v", 0, n - 1, 0, 3, 0x7F), ("v", 0, n - 10, 1, d - 1, 0xFF), ("v", 0, n - 17, 1, 33, 0x7F), ("v", 0, 2, 0, 40, 0x7F),
                                                    ("v", 1, 38, 1, 0, 0xFF)])


@pytest.mark.parametrize("hq,hkv,d,dtype", [(8, 4, 64, "f16"), (16, 8, 128, "bf16")])
def test_chunk_two_tiles_a_workgroup(hq, hkv, d, dtype):
    chunk_case([8300, 8200], [8300 if d == 64 else 8000, 8177], hq, hkv, d, dtype, 64, on_gpu=True)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_chunk_peaked_scores(dtype):
    chunk_case([500, 90], [120, 90], 8, 2, 128, dtype, 16, scale=1.0, q_scale=0.5)


# ------------------------------------------------------------------------------------------------ large pools, streams, graphs
def test_pools_past_32_bits():
    """Pages whose codes begin past 2^32 bytes."""
    hq, hkv, d, R, g = 2, 1, 128, 4096, gen(41)
    pool = F8Pool(g, [70], hkv, d, R, "bf16", spare=0)
    n_pages = (1 << 32) // (R * d) + 2
    L = Layer(1, hq, hkv, d, "bf16")
    k, v = (torch.zeros(n_pages, hkv, R * d, dtype=torch.uint8, device="cuda") for _ in "kv")
    ks, vs = (torch.zeros(n_pages, hkv, R // 16, dtype=torch.uint8, device="cuda") for _ in "kv")
    lens, table = torch.tensor([70], dtype=torch.int32, device="cuda"), torch.tensor([[n_pages - 1]], dtype=torch.int32, device="cuda")
    cache = W.make_paged_cache(k, v, ks, vs, lens, table, R, 1, n_pages)
    x = randn(g, "bf16", 70, (hq + 2 * hkv) * d)
    xd, ld = x.cuda(), (hq + 2 * hkv) * d
    W.wsvd_dense_append_paged_f8(L.ctx, L.desc, None, 0, xd[:, hq * d:], ld, xd[:, (hq + hkv) * d:], ld, 70, prefix([70]).cuda(), None, None, None, 0, None, 0, cache)
    pool.append(0, 0, x[:, hq * d:(hq + hkv) * d].view(70, hkv, d), x[:, (hq + hkv) * d:].view(70, hkv, d))
    for x8, got in (("k", k), ("v", v)):
        assert torch.equal(got[n_pages - 1, :, : 5 * 16 * d].cpu().view(hkv, 5, -1)[:, :4], pool.codes[x8][0, :, :4])
    q, out = xd[:, :hq * d], torch.empty(70, hq * d, dtype=torch.bfloat16, device="cuda")
    W.wsvd_dense_prefill_attn_paged_f8(L.ctx, L.desc, q, ld, 70, prefix([70]).cuda(), cache, out, hq * d)
    kk, vv = pool.rows(0)
    want, size = attend_fast(x[:, : hq * d].view(70, hq, d), kk, vv, list(range(70)), L.scale)
    check(out.cpu().view(70, hq, d), want, size, "bf16", True)
    one = torch.empty(1, hq, d, dtype=torch.bfloat16, device="cuda")
    W.wsvd_dense_decode_attn_paged_f8(L.ctx, L.desc, q[69:], ld, cache, 70, one)
    check(one.cpu(), want[69:], size[69:], "bf16", False)
    L.close()


def test_decode_gives_a_sequence_the_same_bits_in_every_place():
    g, lens, hq, hkv, d = gen(43), [700, 33, 2100, 0, 64], 8, 2, 128
    pool = F8Pool(g, lens, hq // 4, d, 16, "bf16").random(g)
    q = randn(g, "bf16", 5, hq * d)
    L, outs = Layer(5, hq, hkv, d, "bf16"), []
    for order in ([0, 1, 2, 3, 4], [4, 2, 0, 1, 3], [0, 1, 2, 3, 4]):
        cache = L.cache(pool, [lens[i] for i in order])
        L.table.copy_(pool.table[order])
        out = torch.empty(5, hq, d, dtype=torch.bfloat16, device="cuda")
        W.wsvd_dense_decode_attn_paged_f8(L.ctx, L.desc, q[order].cuda(), hq * d, cache, 2100, out)
        outs.append(out.cpu()[[order.index(i) for i in range(5)]])
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    L.close()
