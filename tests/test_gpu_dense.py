"""Dense-layer operators on the GPU (rotary append to a paged cache, decode attention over it, attention of packed prompts and
of tokens behind cached ones) against plain 64-bit forms."""
import math

import pytest
import torch

import paper_2604_02570_amd as W
from dense_ref import DTYPES, F64, Pool, attend, attend_fast, check, half_step, prefix, randn, rotate

pytestmark = pytest.mark.gpu
BASE = 10000.0


class Layer:
    """Descriptor, context and workspace of one dense layer."""

    def __init__(self, batch, hq, hkv, d, dtype, scale=0.0):
        self.desc = W.dense_desc(batch, hq, hkv, d, dtype, scale)
        self.scale = scale or 1.0 / math.sqrt(d)
        self.ctx = W.wsvd_create(0)
        self.ws = torch.empty(W.wsvd_dense_workspace_bytes(self.desc), dtype=torch.uint8, device="cuda")
        W.wsvd_set_workspace(self.ctx, self.ws)

    def cache(self, pool, lens=None):
        self.k, self.v = pool.k.cuda(), pool.v.cuda()
        self.lens = torch.tensor(pool.lens if lens is None else lens, dtype=torch.int32).cuda()
        self.table = pool.table.cuda()
        return W.make_paged_cache(self.k, self.v, None, None, self.lens, self.table, pool.R, pool.max_pages, pool.n_pages)

    def close(self, status=0):
        got = W.wsvd_check(self.ctx)
        W.wsvd_destroy(self.ctx)
        assert got == status, W.status_str(got)


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


# ------------------------------------------------------------------------------------------------ append
HEADS = [(8, 8, 64), (28, 4, 128), (3, 1, 128), (32, 8, 128), (16, 2, 64), (16, 1, 64)]


def append_case(hq, hkv, d, dtype, before, new, page_rows, *, positions=None, rope=True, ld_extra=0, keep_k=True, with_q=True, spare=0,
                in_place=False):
    g, T = gen(5 + d + sum(new)), sum(new)
    L = Layer(len(new), hq, hkv, d, dtype)
    pool = Pool(g, [a + b for a, b in zip(before, new)], hkv, d, page_rows, dtype, fill_rows=False)
    x = randn(g, dtype, T + spare, (hq + 2 * hkv) * d + ld_extra)
    inv = BASE ** (-torch.arange(0, d, 2, dtype=F64) / d)
    rows = torch.cat([torch.arange(a, a + n) for a, n in zip(before, new)])
    pos = rows if positions is None else positions
    cache = L.cache(pool)
    xd, ld = x.cuda(), (hq + 2 * hkv) * d + ld_extra
    q_out = torch.full((T + spare, hq * d), 7.0, dtype=DTYPES[dtype], device="cuda") if with_q else None
    k_out = torch.full((T + spare, hkv * d + 8), 7.0, dtype=DTYPES[dtype], device="cuda") if keep_k else None
    if in_place:
        q_out, k_out, qld, kld = xd, xd[:, hq * d:], ld, ld
    else:
        qld, kld = hq * d, hkv * d + 8
    one = all(n == 1 for n in new) and not spare
    W.wsvd_dense_append_paged(L.ctx, L.desc, xd if with_q else None, ld, xd[:, hq * d:], ld, xd[:, (hq + hkv) * d:], ld, T + spare,
                              None if one else prefix(new).cuda(), None if positions is None else positions.int().cuda(),
                              inv.cuda() if rope else None, q_out, qld, k_out, kld, cache)
    torch.cuda.synchronize()
    y = x[:T, : (hq + 2 * hkv) * d].view(T, hq + 2 * hkv, d)
    want = rotate(y[:, :hq + hkv], pos, inv) if rope else y[:, :hq + hkv].to(F64)
    # rounding of the result, and fp32 products of a pair: 3 roundings of at most sqrt(2) * the pair's length
    pair = torch.hypot(want[..., : d // 2], want[..., d // 2:]).repeat(1, 1, 2)
    tol = half_step(dtype) * want.abs() + (2.0 ** -21 * pair if rope else 0) + (2.0 ** -25 if dtype == "f16" and rope else 0)
    near = lambda got, part: bool(((got.cpu().to(F64) - want[:, part]).abs() <= tol[:, part]).all())
    if with_q:
        assert near(q_out[:T, : hq * d].reshape(T, hq, d), slice(0, hq))
        if spare and not in_place:
            assert (q_out[T:] == 7).all()
    if keep_k:
        assert near(k_out[:T, : hkv * d].reshape(T, hkv, d), slice(hq, hq + hkv))
        if not in_place:
            assert (k_out[:, hkv * d:] == 7).all() and (k_out[T:] == 7).all()
    # the pools: new rows hold the keys and values, everything else is as it was
    expect = Pool(gen(0), [0], hkv, d, page_rows, dtype)
    expect.table, expect.k, expect.v = pool.table, torch.full_like(pool.k, math.nan), torch.full_like(pool.v, math.nan)
    kept = L.k.cpu(), L.v.cpu()
    touched = torch.zeros(pool.k.shape[0], pool.k.shape[2], dtype=torch.bool)
    t = 0
    for b, (a, n) in enumerate(zip(before, new)):
        for i in range(n):
            page, at = int(pool.table[b, (a + i) // page_rows]), (a + i) % page_rows
            touched[page, at] = True
            assert bool(((kept[0][page, :, at].to(F64) - want[t, hq:]).abs() <= tol[t, hq:]).all()), (b, i)
            assert torch.equal(kept[1][page, :, at], y[t, hq + hkv:]), (b, i)
            t += 1
    for x in kept:
        assert torch.isnan(x.transpose(1, 2)[~touched]).all()
    L.close()


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_append_one_token_each(hq, hkv, d, dtype):
    append_case(hq, hkv, d, dtype, [0, 63, 64, 1000], [1, 1, 1, 1], 64, keep_k=False)


@pytest.mark.parametrize("hq,hkv,d,dtype", [(28, 4, 128, "bf16"), (8, 8, 64, "f16"), (16, 1, 64, "bf16")])
@pytest.mark.parametrize("page_rows", [16, 112])
def test_append_packed_sequences(hq, hkv, d, dtype, page_rows):
    append_case(hq, hkv, d, dtype, [0, 5, 0, 17, 300], [33, 0, 1, 130, 0], page_rows, ld_extra=24, spare=3)


def test_append_many_tokens_and_sequences():
    # four tokens per workgroup, more than 64 sequences, some without tokens, workgroups across their borders
    new = [(7 * i) % 61 for i in range(75)]
    assert sum(new) >= 2048
    append_case(4, 2, 64, "bf16", [(13 * i) % 97 for i in range(75)], new, 32, spare=2)


def test_append_far_positions():
    # an angle of 1e7 radians in fp32 would be off by 0.5
    pos = torch.tensor([131071, 1000003, 16777213, 3])
    append_case(4, 2, 128, "bf16", [10, 20, 30, 0], [1, 1, 1, 1], 16, positions=pos)


def test_append_without_rotation_and_without_queries():
    append_case(4, 2, 128, "f16", [3], [40], 16, rope=False)
    append_case(4, 2, 64, "bf16", [3, 9], [4, 2], 16, with_q=False)


def test_append_in_place():
    append_case(6, 2, 128, "bf16", [3, 9], [4, 90], 16, in_place=True)


def test_append_bad_rows_and_pages_store_nothing():
    for new_lens, table_value, status in (([70], None, W.E_CAPACITY), ([2], None, W.E_SHAPE), ([60], 1 << 20, W.E_SHAPE), ([60], -1, W.E_SHAPE)):
        g = gen(3)
        L = Layer(1, 4, 2, 64, "bf16")
        pool = Pool(g, [60], 2, 64, 16, "bf16", fill_rows=False)          # 4 pages: rows 0 .. 63
        if table_value is not None:
            pool.table[0, 3] = table_value
        cache = L.cache(pool, lens=new_lens)
        x = randn(g, "bf16", 8, 8 * 64).cuda()
        inv = BASE ** (-torch.arange(0, 64, 2, dtype=F64) / 64)
        W.wsvd_dense_append_paged(L.ctx, L.desc, None, 0, x[:, 256:], 512, x[:, 384:], 512, 8, prefix([8]).cuda(), None, inv.cuda(), None, 0,
                                  None, 0, cache)
        torch.cuda.synchronize()
        stored = {70: 2, 2: 2, 60: 0}[new_lens[0]] if table_value is None else 0     # rows 62, 63; rows 0, 1; rows 52 .. 59 are in page 3
        if table_value is None:
            assert int((~torch.isnan(L.v[:, 0, :, 0])).sum()) == stored
        else:
            assert int((~torch.isnan(L.v[:, 0, :, 0])).sum()) == 0
        L.close(status)


# ------------------------------------------------------------------------------------------------ decode
def decode_case(hq, hkv, d, dtype, lens, page_rows, *, max_len=None, scale=0.0, ld_extra=0, q_scale=1.0, max_pages=None, min_chunk=0, status=0):
    g = gen(11 + hq + d + sum(lens))
    L = Layer(len(lens), hq, hkv, d, dtype, scale)
    W.wsvd_ctx_set_option(L.ctx, "min_chunk", min_chunk)
    pool = Pool(g, lens, hkv, d, page_rows, dtype, max_pages=max_pages)
    q = randn(g, dtype, len(lens), hq * d + ld_extra, scale=q_scale)
    cache = L.cache(pool)
    out = torch.full((len(lens), hq, d), math.nan, dtype=DTYPES[dtype], device="cuda")
    qd = q.cuda()
    for _ in range(2):                                             # the second call on a used workspace
        out.fill_(math.nan)
        W.wsvd_dense_decode_attn_paged(L.ctx, L.desc, qd, hq * d + ld_extra, cache, max(lens) if max_len is None else max_len, out)
    got = out.cpu()
    for b, n in enumerate(lens):
        n = n if max_len is None else min(n, max_len)
        k, v = pool.rows(b, n)
        want, size = attend_fast(q[b:b + 1, : hq * d].view(1, hq, d), k, v, [n - 1], L.scale)
        if n == 0:
            assert (got[b] == 0).all()
        else:
            check(got[b:b + 1], want, size, dtype, weights_rounded=False)
    L.close(status)
    return got


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_decode_lengths_around_tiles(hq, hkv, d, dtype):
    decode_case(hq, hkv, d, dtype, [0, 1, 2, 15, 16, 17, 31, 32, 33, 127, 128, 129, 0], 16)


@pytest.mark.parametrize("page_rows", [16, 48, 64, 112, 256])
def test_decode_split_and_joined(page_rows):
    decode_case(14, 2, 128, "bf16", [5000, 1, 0, 2049, 255, 256, 257], page_rows)


@pytest.mark.parametrize("d,dtype", [(64, "f16"), (128, "bf16"), (64, "bf16")])
def test_decode_one_long_sequence(d, dtype):
    decode_case(2, 1, d, dtype, [20011], 16)


def test_decode_more_than_64_sequences():
    decode_case(4, 2, 64, "bf16", [(97 * i) % 401 for i in range(150)], 16, max_pages=32)


@pytest.mark.parametrize("hq,hkv,d,dtype", [(4, 4, 64, "bf16"), (16, 1, 128, "f16"), (7, 1, 128, "bf16")])
def test_decode_small_chunks(hq, hkv, d, dtype):
    """Chunks of 128 rows: one or two folds, groups that end in the middle, empty last chunks."""
    decode_case(hq, hkv, d, dtype, [1, 129, 1024, 1025, 0, 2200, 7 * 128 + 1], 16, min_chunk=128)
    decode_case(hq, hkv, d, dtype, [8300], 32, min_chunk=128)


@pytest.mark.parametrize("batch,hq,hkv,d", [(70, 8, 8, 64), (64, 16, 8, 128), (150, 8, 8, 64), (33, 64, 32, 128), (9, 128, 128, 64)])
def test_decode_many_units(batch, hq, hkv, d):
    """Two and four waves a workgroup (eight where a sequence is longer); one sequence is long enough to be cut all the same."""
    decode_case(hq, hkv, d, "bf16", [(61 * i) % 150 for i in range(batch - 1)] + [1023], 64, max_pages=65)
    decode_case(hq, hkv, d, "bf16", [(61 * i) % 50 for i in range(batch - 1)] + [4100], 64, max_pages=65)


def test_decode_strides_and_scale():
    decode_case(6, 2, 128, "f16", [300, 40], 32, ld_extra=40, scale=0.25)


def test_decode_peaked_scores():
    # scores up to some hundreds: the reference moves, all but a few weights vanish
    decode_case(4, 1, 128, "bf16", [3000, 700], 64, q_scale=4.0)


def test_decode_longer_than_the_bound_is_reported():
    decode_case(4, 2, 64, "bf16", [600, 90], 16, max_len=512, status=W.E_SHAPE)


def test_decode_does_not_depend_on_other_sequences_order():
    a = decode_case(8, 2, 128, "bf16", [900, 3000, 17], 16)
    b = decode_case(8, 2, 128, "bf16", [900, 3000, 17], 16)
    assert torch.equal(a, b)


def test_decode_infinite_scores():
    # a key of -inf scores has no weight; nothing but such keys counts as nothing to see
    def tweak(pool, q):
        q[:] = q.abs()
        k, v = pool.rows(0)
        k[5] = -math.inf
        pool.put(0, 0, k, v)
        k, v = pool.rows(1)
        k[:] = -math.inf
        pool.put(1, 0, k, v)
    g = gen(1)
    L = Layer(2, 4, 2, 64, "bf16")
    pool = Pool(g, [40, 3], 2, 64, 16, "bf16")
    q = randn(g, "bf16", 2, 256)
    tweak(pool, q)
    cache, out = L.cache(pool), torch.empty(2, 4, 64, dtype=torch.bfloat16, device="cuda")
    W.wsvd_dense_decode_attn_paged(L.ctx, L.desc, q.cuda(), 256, cache, 40, out)
    k, v = pool.rows(0)
    keep = [i for i in range(40) if i != 5]
    want, size = attend_fast(q[:1].view(1, 4, 64), k[keep], v[keep], [38], L.scale)
    check(out[:1].cpu(), want, size, "bf16", False)
    assert (out[1] == 0).all()
    L.close()


@pytest.mark.parametrize("d,dtype", [(128, "bf16"), (64, "f16")])
def test_decode_infinite_values(d, dtype):
    """Infinite values that are seen come out infinite, NaN comes out NaN, and only in their own dims; one head and several chunks."""
    g = gen(4)
    L = Layer(2, 4, 2, d, dtype)
    pool = Pool(g, [1300, 20], 2, d, 16, dtype)
    k, v = pool.rows(0)
    v[17, 0, 3], v[900, 1, 5], v[1299, 1, 7], v[40, 0, 9] = math.inf, -math.inf, math.nan, math.inf
    pool.put(0, 0, k, v)
    k1, v1 = pool.rows(1)
    v1[19, 0, 0] = -math.inf
    pool.put(1, 0, k1, v1)
    q = randn(g, dtype, 2, 4 * d)
    cache, out = L.cache(pool), torch.empty(2, 4, d, dtype=DTYPES[dtype], device="cuda")
    W.wsvd_dense_decode_attn_paged(L.ctx, L.desc, q.cuda(), 4 * d, cache, 1300, out)
    got = out.cpu()
    for b, (kk, vv) in enumerate(((k, v), (k1, v1))):
        want, size = attend(q[b:b + 1].view(1, 4, d), kk, vv, [kk.shape[0] - 1], L.scale)
        fine = torch.isfinite(want)
        assert not fine.all() and torch.equal(torch.isnan(want[0]), torch.isnan(got[b]))
        infinite = torch.isinf(want[0])
        assert torch.equal(want[0][infinite], got[b][infinite].to(F64))
        check(torch.where(fine[0], got[b], 0), torch.where(fine[0], want[0], 0), torch.where(fine[0], size[0], 0), dtype, True)
    L.close()


def test_decode_bad_page_is_reported():
    g = gen(2)
    L = Layer(1, 4, 2, 64, "bf16")
    pool = Pool(g, [100], 2, 64, 16, "bf16")
    pool.table[0, 2] = pool.n_pages
    cache, out = L.cache(pool), torch.empty(1, 4, 64, dtype=torch.bfloat16, device="cuda")
    W.wsvd_dense_decode_attn_paged(L.ctx, L.desc, randn(g, "bf16", 1, 256).cuda(), 256, cache, 100, out)
    L.close(W.E_SHAPE)


# ------------------------------------------------------------------------------------------------ prompts
def prompt_case(hq, hkv, d, dtype, nq, nk=None, *, causal=True, page_rows=0, ld_extra=0, q_scale=1.0, spare=0, tweak=None, loops=False):
    g = gen(23 + hq + d + sum(nq))
    L = Layer(len(nq), hq, hkv, d, dtype)
    T = sum(nq)
    q = randn(g, dtype, T + spare, hq * d + ld_extra, scale=q_scale)
    lens = nq if nk is None else nk
    if page_rows:
        pool = Pool(g, lens, hkv, d, page_rows, dtype)
        rows = [pool.rows(b) for b in range(len(nq))]
    else:
        k, v = (randn(g, dtype, max(1, sum(lens)), hkv * d + e) for e in (ld_extra, 2 * ld_extra))
        if tweak:
            tweak(k, v)
        at = prefix(lens).tolist()
        rows = [tuple(x[at[b]:at[b + 1], : hkv * d].reshape(-1, hkv, d) for x in (k, v)) for b in range(len(nq))]
    out = torch.full((T + spare, hq * d + ld_extra), 7.0, dtype=DTYPES[dtype], device="cuda")
    qd, cu = q.cuda(), prefix(nq).cuda()
    if page_rows:
        W.wsvd_dense_prefill_attn_paged(L.ctx, L.desc, qd, hq * d + ld_extra, T + spare, cu, L.cache(pool), out, hq * d + ld_extra)
    else:
        kd, vd = k.cuda(), v.cuda()
        W.wsvd_dense_prefill_attn(L.ctx, L.desc, qd, hq * d + ld_extra, kd, hkv * d + ld_extra, vd, hkv * d + 2 * ld_extra, T + spare,
                                  sum(lens) if nk is not None else T + spare, cu, None if nk is None else prefix(nk).cuda(), causal, out,
                                  hq * d + ld_extra)
    got = out.cpu()
    assert (got[T:] == 7).all() and (got[:, hq * d:] == 7).all()
    at = prefix(nq).tolist()
    for b, n in enumerate(nq):
        if n == 0:
            continue
        t = lens[b]
        last = torch.arange(t - n, t) if causal else torch.full((n,), t - 1)
        x = q[at[b]:at[b + 1], : hq * d].view(n, hq, d)
        kk, vv = rows[b]
        if tweak:                                                  # numbers that are none: only where they are seen
            want, size = attend(x, kk, vv, last, L.scale)
        else:
            want, size = attend_fast(x, kk, vv, last, L.scale)
        o = got[at[b]:at[b + 1], : hq * d].view(n, hq, d)
        if tweak:
            fine = torch.isfinite(want)
            assert torch.equal(torch.isnan(want), torch.isnan(o)) and torch.equal(want[~fine & ~torch.isnan(want)], o[~fine & ~torch.isnan(want)].to(F64))
            check(torch.where(fine, o, 0), torch.where(fine, want, 0), torch.where(fine, size, 0), dtype, True)
        else:
            check(o, want, size, dtype, weights_rounded=True)
    L.close()
    return got


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_prompt_lengths_around_tiles(hq, hkv, d, dtype):
    prompt_case(hq, hkv, d, dtype, [1, 0, 2, 31, 32, 33, 63, 64, 65, 129], spare=2)


@pytest.mark.parametrize("hq,hkv,d,dtype", [(4, 4, 128, "bf16"), (7, 1, 128, "f16"), (4, 2, 64, "bf16")])
@pytest.mark.parametrize("causal", [True, False])
def test_prompt_long_and_ragged(hq, hkv, d, dtype, causal):
    prompt_case(hq, hkv, d, dtype, [700, 3, 257], causal=causal)


@pytest.mark.parametrize("causal", [True, False])
def test_prompt_keys_of_another_number(causal):
    # more keys than queries, fewer (the first queries see nothing), none
    prompt_case(4, 2, 128, "bf16", [10, 70, 100, 5, 64], [200, 30, 100, 0, 1], causal=causal)
    prompt_case(3, 1, 64, "f16", [4, 9], [0, 0], causal=causal)


def test_prompt_strides():
    prompt_case(6, 2, 128, "bf16", [70, 30], ld_extra=24)
    prompt_case(6, 6, 64, "f16", [70, 30], ld_extra=8)


def test_prompt_many_sequences():
    prompt_case(2, 2, 64, "bf16", [(11 * i) % 37 for i in range(140)])


def test_prompt_peaked_scores():
    prompt_case(2, 1, 128, "bf16", [400], q_scale=4.0)


@pytest.mark.parametrize("hq,hkv,d,dtype", [(4, 2, 128, "bf16"), (2, 2, 64, "f16"), (7, 1, 128, "f16"), (8, 1, 64, "bf16")])
def test_prompt_hidden_values_have_no_effect(hq, hkv, d, dtype):
    # infinities and NaN among the values (and NaN keys): earlier queries do not see them, later ones do
    def tweak(k, v):
        v[20, 3], v[37, 5], v[50, 0], v[50, 1] = math.inf, -math.inf, math.nan, math.inf
        k[66] = math.nan
        v[69, d - 1] = math.inf
    prompt_case(hq, hkv, d, dtype, [70], tweak=tweak)


@pytest.mark.parametrize("page_rows", [16, 112, 128])
@pytest.mark.parametrize("hq,hkv,d,dtype", [(28, 4, 128, "bf16"), (4, 4, 64, "f16"), (5, 1, 128, "f16")])
def test_chunk_behind_cached_rows(page_rows, hq, hkv, d, dtype):
    prompt_case(hq, hkv, d, dtype, [1, 0, 40, 129, 3], [300, 50, 40, 500, 17], page_rows=page_rows, spare=1)


def test_chunk_bad_page_is_reported():
    g = gen(2)
    L = Layer(1, 4, 2, 64, "bf16")
    pool = Pool(g, [100], 2, 64, 16, "bf16")
    pool.table[0, 2] = -1
    out = torch.empty(4, 256, dtype=torch.bfloat16, device="cuda")
    W.wsvd_dense_prefill_attn_paged(L.ctx, L.desc, randn(g, "bf16", 4, 256).cuda(), 256, 4, prefix([4]).cuda(), L.cache(pool), out, 256)
    L.close(W.E_SHAPE)


# few tiles over many keys: several workgroups share a tile's keys, their parts are joined by a second launch
@pytest.mark.parametrize("hq,hkv,d,dtype", [(4, 1, 128, "bf16"), (4, 4, 64, "f16"), (7, 1, 128, "f16"), (16, 2, 64, "bf16")])
def test_chunk_shared_by_workgroups(hq, hkv, d, dtype):
    prompt_case(hq, hkv, d, dtype, [5, 0, 1, 70], [2600, 900, 3, 1201], page_rows=16)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("hq,hkv,d,dtype", [(3, 1, 128, "bf16"), (2, 2, 64, "f16")])
def test_prompt_shared_by_workgroups(causal, hq, hkv, d, dtype):
    prompt_case(hq, hkv, d, dtype, [9, 40, 6], [1500, 20, 2049], causal=causal)
    prompt_case(hq, hkv, d, dtype, [1100], causal=causal)


def test_prompt_shared_by_workgroups_hidden_values():
    # numbers that are none at the end of the keys, where only the last queries see them, and beyond what any query of a tile sees
    def tweak(k, v):
        v[1598, 3], v[1599, 64], v[1400, 7] = math.inf, math.nan, -math.inf
        k[1597] = math.nan
    prompt_case(2, 1, 128, "bf16", [6], [1600], tweak=tweak)
    prompt_case(2, 1, 64, "f16", [300], [1600], tweak=lambda k, v: v[1597:, 5].fill_(math.inf))


def test_workspace_serves_decode_and_prompts_in_turn():
    """Partial results that a prompt leaves in the workspace lie where a decode call's workgroups hand theirs over."""
    g = gen(31)
    hq, hkv, d = 8, 1, 64
    L = Layer(1, hq, hkv, d, "bf16")
    pool = Pool(g, [4000], hkv, d, 16, "bf16")
    cache = L.cache(pool)
    k, v = pool.rows(0)
    q = randn(g, "bf16", 20, hq * d)
    qd, cu = q.cuda(), prefix([20]).cuda()
    out, one = torch.empty(20, hq * d, dtype=torch.bfloat16, device="cuda"), torch.empty(1, hq, d, dtype=torch.bfloat16, device="cuda")
    for _ in range(3):
        W.wsvd_dense_prefill_attn_paged(L.ctx, L.desc, qd, hq * d, 20, cu, cache, out, hq * d)
        W.wsvd_dense_decode_attn_paged(L.ctx, L.desc, qd[19:], hq * d, cache, 4000, one)
        want, size = attend_fast(q.view(20, hq, d), k, v, torch.arange(3980, 4000), L.scale)
        check(out.view(20, hq, d).cpu(), want, size, "bf16", True)
        check(one.cpu(), want[19:], size[19:], "bf16", False)
        out.zero_(), one.zero_()
    L.close()


# ------------------------------------------------------------------------------------------------ streams and graphs
def test_decode_step_in_a_graph_on_another_stream():
    """Append and attention captured on a stream of their own; replays after the lengths and inputs have changed give what eager
    calls give."""
    g = gen(9)
    hq, hkv, d, B = 8, 2, 128, 3
    L = Layer(B, hq, hkv, d, "bf16")
    lens = [200, 1, 1030]
    pool = Pool(g, [n + 8 for n in lens], hkv, d, 16, "bf16")
    cache = L.cache(pool, lens=lens)
    x, out = torch.zeros(B, (hq + 2 * hkv) * d, dtype=torch.bfloat16, device="cuda"), torch.empty(B, hq * d, dtype=torch.bfloat16, device="cuda")
    q_rot, inv = torch.empty_like(out), (BASE ** (-torch.arange(0, d, 2, dtype=F64) / d)).cuda()
    ld = x.shape[1]

    def step(stream):
        W.wsvd_dense_append_paged(L.ctx, L.desc, x, ld, x[:, hq * d:], ld, x[:, (hq + hkv) * d:], ld, B, None, None, inv, q_rot, hq * d, None, 0,
                                  cache, stream)
        W.wsvd_dense_decode_attn_paged(L.ctx, L.desc, q_rot, hq * d, cache, pool.max_pages * 16, out, stream)

    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step(torch.cuda.current_stream())
    for i in range(4):
        L.lens += 1
        x.copy_(randn(g, "bf16", B, ld))
        out.fill_(math.nan)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        replayed = out.clone()
        out.fill_(math.nan)
        with torch.cuda.stream(side):
            step(side)
        torch.cuda.synchronize()
        assert torch.equal(out, replayed) and torch.isfinite(replayed).all(), i
    L.close()


# ------------------------------------------------------------------------------------------------ two tiles a workgroup
def spread(lengths, batch):
    """The lengths among sequences of none: so many that workgroups take two tiles each."""
    out = [0] * batch
    for i, n in enumerate(lengths):
        out[(i * 997 + 3) % batch] = n
    return out


@pytest.mark.parametrize("hq,hkv,d,dtype", [(4, 4, 128, "bf16"), (7, 1, 128, "f16"), (4, 2, 64, "bf16"), (16, 1, 64, "f16")])
def test_prompt_two_tiles_a_workgroup(hq, hkv, d, dtype):
    # even and odd numbers of tiles, last ones of few rows, one tile alone
    prompt_case(hq, hkv, d, dtype, spread([700, 129, 128, 1, 257, 384, 33, 511], 2100 // hkv), spare=3)


def test_prompt_two_tiles_a_workgroup_keys_of_another_number():
    # more keys than queries; fewer, so that the second tile sees nothing, or the first only part of its keys; none
    nq, nk = [300, 300, 300, 300, 140, 520], [800, 130, 300, 0, 10, 391]
    prompt_case(3, 1, 128, "bf16", spread(nq, 2100), spread(nk, 2100))
    prompt_case(2, 2, 64, "f16", spread(nq, 1100), spread(nk, 1100))


@pytest.mark.parametrize("hq,hkv,d,dtype,page_rows", [(2, 1, 128, "bf16", 16), (1, 1, 64, "f16", 112), (5, 1, 128, "f16", 128)])
def test_chunk_two_tiles_a_workgroup(hq, hkv, d, dtype, page_rows):
    # more than 64 blocks of keys: where they lie is looked up again for the second tile
    prompt_case(hq, hkv, d, dtype, spread([260, 300, 129, 2], 2100), spread([4700, 300, 4300, 70], 2100), page_rows=page_rows)


@pytest.mark.parametrize("hq,hkv,d,dtype", [(1, 1, 128, "bf16"), (2, 1, 64, "f16")])
def test_prompt_two_tiles_a_workgroup_hidden_values(hq, hkv, d, dtype):
    # numbers that are none late in the sequence (the first tile of a pair sees them, the second does not), early, and in between
    def tweak(k, v):
        v[350, 3], v[399, 60], v[130, 5], v[2, 7] = math.inf, math.nan, -math.inf, math.inf
        k[380] = math.nan
    prompt_case(hq, hkv, d, dtype, spread([400], 2100), tweak=tweak)
    prompt_case(hq, hkv, d, dtype, spread([300], 2100), tweak=lambda k, v: v[297:, 5].fill_(math.inf))
