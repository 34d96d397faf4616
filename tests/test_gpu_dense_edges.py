"""Dense-layer operators on the GPU where single numbers decide: weights far below the largest, infinite values and scores, what other
calls left in the workspace; and the forms that only large calls take.  Against plain 64-bit forms."""
import math

import pytest
import torch

import paper_2604_02570_amd as W
from dense_ref import DTYPES, F64, Pool, attend, attend_fast, check, half_step, prefix, randn, rotate
from test_gpu_dense import Layer, gen

pytestmark = pytest.mark.gpu
LN2 = math.log(2.0)                             # as the softmax scale: scores count in powers of two


def run_decode(dtype, q, keys, values, *, scale=0.0, min_chunk=0, page_rows=16, L=None):
    """q [B, Hq, d]; keys, values: a tensor [rows, Hkv, d] for every sequence."""
    B, hq, d = q.shape
    own = L is None
    L = L or Layer(B, hq, keys[0].shape[1], d, dtype, scale)
    W.wsvd_ctx_set_option(L.ctx, "min_chunk", min_chunk)
    lens = [k.shape[0] for k in keys]
    pool = Pool(gen(17), lens, keys[0].shape[1], d, page_rows, dtype, fill_rows=False)
    for b, (k, v) in enumerate(zip(keys, values)):
        pool.put(b, 0, k, v)
    out = torch.full((B, hq, d), 7.0, dtype=DTYPES[dtype], device="cuda")
    W.wsvd_dense_decode_attn_paged(L.ctx, L.desc, q.cuda(), hq * d, L.cache(pool), max(lens), out)
    got = out.cpu()
    if own:
        L.close()
    return got


def run_prompt(dtype, q, k, v, nq, nk, *, scale=0.0, causal=True, page_rows=0, batch=0):
    """q [tokens, Hq, d], k, v [rows, Hkv, d], packed; batch: sequences of nothing behind them up to this number."""
    nq, nk = [list(n) + [0] * (batch - len(n)) for n in (nq, nk)]
    T, hq, d = q.shape
    hkv = k.shape[1]
    L = Layer(len(nq), hq, hkv, d, dtype, scale)
    out = torch.full((T, hq * d), 7.0, dtype=DTYPES[dtype], device="cuda")
    if page_rows:
        pool, at = Pool(gen(18), nk, hkv, d, page_rows, dtype, fill_rows=False), prefix(nk).tolist()
        for b in range(len(nk)):
            pool.put(b, 0, k[at[b]:at[b + 1]], v[at[b]:at[b + 1]])
        W.wsvd_dense_prefill_attn_paged(L.ctx, L.desc, q.cuda(), hq * d, T, prefix(nq).cuda(), L.cache(pool), out, hq * d)
    else:
        W.wsvd_dense_prefill_attn(L.ctx, L.desc, q.cuda(), hq * d, k.cuda(), hkv * d, v.cuda(), hkv * d, T, k.shape[0], prefix(nq).cuda(),
                                  prefix(nk).cuda(), causal, out, hq * d)
    got = out.cpu().view(T, hq, d)
    L.close()
    return got


def same_kind(got, want):
    """Infinite where the formula is infinite, NaN where it is NaN; returns where it is a number."""
    assert torch.equal(torch.isnan(want), torch.isnan(got))
    infinite = torch.isinf(want)
    assert torch.equal(want[infinite], got[infinite].to(F64))
    return torch.isfinite(want)


# ------------------------------------------------------------------------------------------------ weights far below the largest
def sink(dtype, rows, hq, hkv, d, gap, at, dims=None):
    """A key `gap` powers of two above the others, whose scores spread a little, and whose value is 0: the output is what the small
    weights make it.  Queries of 1 in their first dim."""
    g = gen(rows + d)
    q = torch.zeros(1, hq, d, dtype=DTYPES[dtype])
    q[..., 0] = 1.0
    k, v = torch.zeros(rows, hkv, d, dtype=DTYPES[dtype]), 1.0 + randn(g, dtype, rows, hkv, d, scale=0.25)
    k[..., 0] = randn(g, dtype, rows, hkv, scale=0.5)
    k[at, :, 0], v[at] = gap, 0.0
    return q, k, v


def check_small_weights(got, want, size, dtype, rounded, rows, v):
    """As everywhere; and where the type's small numbers run out, a weight is off by at most 2^-36 of the largest."""
    lost = rows * 2.0 ** -36 * v.to(F64).abs().max()
    check(got, want, size + (lost * 2.0 ** 12 if dtype == "f16" else 0.0), dtype, rounded)


@pytest.mark.parametrize("rows,min_chunk", [(640, 0), (1100, 128), (65001, 0)])
@pytest.mark.parametrize("gap", [18.0, 25.5, 27.0])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_decode_weights_far_below_the_largest(dtype, gap, rows, min_chunk):
    for at in (0, rows // 2, rows - 1) if rows < 2000 else (0,):
        q, k, v = sink(dtype, rows, 4, 1, 64, gap, at)
        got = run_decode(dtype, q, [k], [v], scale=LN2, min_chunk=min_chunk)
        want, size = attend_fast(q, k, v, [rows - 1], LN2)
        check_small_weights(got, want, size, dtype, False, rows, v)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_decode_peaked_scores_over_many_rows(dtype):
    g = gen(77)
    q, k, v = randn(g, dtype, 1, 8, 128, scale=4.0), randn(g, dtype, 20011, 2, 128), randn(g, dtype, 20011, 2, 128)
    want, size = attend_fast(q, k, v, [20010], 128 ** -0.5)
    check_small_weights(run_decode(dtype, q, [k], [v]), want, size, dtype, False, 20011, v)


def large_scores(dtype, queries, rows, d, most, growth):
    """Values of 1 and scores of `most` powers of two and more, in the steps of which 32 bits hold them: they grow by 0.5 every `growth` rows,
    then jump about."""
    g = gen(rows)
    q = torch.zeros(queries, 2, d, dtype=DTYPES[dtype])
    q[..., 0], q[..., 1] = 2.0 ** math.floor(math.log2(most) / 2), 1.0
    k = torch.zeros(rows, 1, d, dtype=DTYPES[dtype])
    k[..., 0], k[..., 1] = most / q[0, 0, 0].item(), torch.arange(rows)[:, None] // growth * 0.5
    k[rows // 2:, 0, 1] = (torch.randint(0, 60, (rows - rows // 2,), generator=g) * 0.5).to(DTYPES[dtype])
    return q, k, torch.ones(rows, 1, d, dtype=DTYPES[dtype])


@pytest.mark.parametrize("rows,min_chunk", [(900, 0), (1500, 128)])
@pytest.mark.parametrize("growth", [1, 8, 60])
@pytest.mark.parametrize("most", [2.0 ** 15, 2.0 ** 21, 2.0 ** 24, 2.0 ** 25, 2.0 ** 26, 2.0 ** 27, 2.0 ** 28, 2.0 ** 30])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_decode_large_scores(dtype, most, growth, rows, min_chunk):
    """Weights stay inside the type whatever the scores' own steps are: a mean of ones is 1, up to the weights' rounding."""
    q, k, v = large_scores(dtype, 1, rows, 64, most, growth)
    got = run_decode(dtype, q, [k], [v], scale=LN2, min_chunk=min_chunk)
    assert ((got.to(F64) - 1).abs() <= torch.finfo(DTYPES[dtype]).eps).all()


@pytest.mark.parametrize("queries,rows,page_rows", [(300, 700, 0), (5, 2600, 0), (300, 700, 16), (5, 2600, 112)])
@pytest.mark.parametrize("gap", [18.0, 25.5, 27.0])
@pytest.mark.parametrize("d,dtype", [(64, "f16"), (128, "f16"), (128, "bf16")])
def test_prompt_weights_far_below_the_largest(d, dtype, gap, queries, rows, page_rows):
    """Tiles of one workgroup, and of several."""
    for at in (0, rows - queries - 3):
        q, k, v = sink(dtype, rows, 2, 1, d, gap, at)
        q = q.expand(queries, 2, d).contiguous()
        got = run_prompt(dtype, q, k, v, [queries], [rows], scale=LN2, page_rows=page_rows)
        want, size = attend_fast(q, k, v, torch.arange(rows - queries, rows), LN2)
        check_small_weights(got, want, size, dtype, True, rows, v)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_prompt_peaked_scores_of_both_types(dtype):
    g = gen(78)
    q, k, v = randn(g, dtype, 900, 4, 128, scale=4.0), randn(g, dtype, 900, 1, 128), randn(g, dtype, 900, 1, 128)
    want, size = attend_fast(q, k, v, torch.arange(900), 128 ** -0.5)
    check_small_weights(run_prompt(dtype, q, k, v, [900], [900]), want, size, dtype, True, 900, v)


@pytest.mark.parametrize("queries,rows,page_rows", [(200, 700, 0), (5, 2600, 0), (200, 700, 16)])
@pytest.mark.parametrize("growth", [1, 8, 60])
@pytest.mark.parametrize("most", [2.0 ** 15, 2.0 ** 21, 2.0 ** 24, 2.0 ** 25, 2.0 ** 26, 2.0 ** 27])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_prompt_large_scores(dtype, most, growth, queries, rows, page_rows):
    q, k, v = large_scores(dtype, queries, rows, 128, most, growth)
    got = run_prompt(dtype, q, k, v, [queries], [rows], scale=LN2, page_rows=page_rows)
    assert ((got.to(F64) - 1).abs() <= torch.finfo(DTYPES[dtype]).eps).all()


# ------------------------------------------------------------------------------------------------ infinite scores and values
@pytest.mark.parametrize("queries,rows,page_rows,batch", [(70, 70, 0, 0), (70, 90, 16, 0), (6, 1600, 0, 0), (6, 1600, 16, 0), (300, 300, 0, 2100)])
@pytest.mark.parametrize("d,dtype", [(64, "f16"), (128, "bf16")])
def test_prompt_nothing_but_scores_of_minus_infinity_gives_zeros(d, dtype, queries, rows, page_rows, batch):
    """Whatever the values hold: tiles of one workgroup, of several, two tiles a workgroup."""
    g = gen(5)
    q, k, v = randn(g, dtype, queries, 2, d).abs(), torch.full((rows, 1, d), -math.inf, dtype=DTYPES[dtype]), randn(g, dtype, rows, 1, d)
    v[3, 0, 1], v[3, 0, 2], v[rows // 2, 0, 5], v[rows - queries, 0, d - 1] = math.inf, math.nan, -math.inf, math.nan
    assert (run_prompt(dtype, q, k, v, [queries], [rows], page_rows=page_rows, batch=batch) == 0).all()


@pytest.mark.parametrize("min_chunk", [0, 128])
def test_decode_nothing_but_scores_of_minus_infinity_gives_zeros(min_chunk):
    g = gen(6)
    q, k, v = randn(g, "bf16", 1, 2, 64).abs(), torch.full((700, 1, 64), -math.inf, dtype=torch.bfloat16), randn(g, "bf16", 700, 1, 64)
    v[3, 0, 1], v[300, 0, 2], v[699, 0, 5] = math.inf, math.nan, -math.inf
    assert (run_decode("bf16", q, [k], [v], min_chunk=min_chunk) == 0).all()


def infinite_values(dtype, rows, d, gap, top, odd):
    """One key `gap` powers of two above the others, and values that are no numbers at a key of a small weight."""
    g = gen(rows + d)
    q = torch.zeros(1, 4, d, dtype=DTYPES[dtype])
    q[..., 0] = 1.0
    k, v = torch.zeros(rows, 2, d, dtype=DTYPES[dtype]), randn(g, dtype, rows, 2, d)
    k[..., 0] = randn(g, dtype, rows, 2, scale=0.5)
    k[top, :, 0] = gap
    v[odd, 0, 3], v[odd, 0, 6], v[odd, 1, 4], v[odd, 1, 5] = math.inf, -math.inf, -math.inf, math.nan
    return q, k, v


@pytest.mark.parametrize("rows,min_chunk", [(33, 0), (600, 0), (1500, 128)])
@pytest.mark.parametrize("gap", [40.0, 200.0])
@pytest.mark.parametrize("d,dtype", [(64, "f16"), (128, "bf16"), (128, "f16")])
def test_decode_infinite_values_of_small_weights(d, dtype, gap, rows, min_chunk):
    """A weight too small for the type, or for 32 bits, is not 0: infinite values come out infinite, whichever key comes first and
    whichever workgroup has it."""
    for top, odd in ((0, rows - 1), (rows - 1, 0), (rows // 2, 7), (1, 2)):
        q, k, v = infinite_values(dtype, rows, d, gap, top, odd)
        want, size = attend(q, k, v, [rows - 1], LN2)
        got = run_decode(dtype, q, [k], [v], scale=LN2, min_chunk=min_chunk)
        fine = same_kind(got, want)
        assert torch.isinf(want).sum() == 2 * 3 and torch.isnan(want).sum() == 2
        check(torch.where(fine, got, 0), torch.where(fine, want, 0), torch.where(fine, size, 0), dtype, False)


@pytest.mark.parametrize("d,dtype", [(64, "f16"), (128, "bf16")])
def test_decode_numbers_beside_infinite_values(d, dtype):
    """What is a number comes out as exactly as without infinite values beside it."""
    g = gen(8)
    for rows in (2, 5, 40):
        q, k, v = randn(g, dtype, 1, 16, d), randn(g, dtype, rows, 2, d), randn(g, dtype, rows, 2, d)
        v[1, 0, 3], v[0, 1, 9], v[1, 1, 9] = math.inf, math.inf, -math.inf
        want, size = attend(q, k, v, [rows - 1], d ** -0.5)
        got = run_decode(dtype, q, [k], [v])
        fine = same_kind(got, want)
        check(torch.where(fine, got, 0), torch.where(fine, want, 0), torch.where(fine, size, 0), dtype, False)


def test_decode_infinite_value_under_a_score_of_minus_infinity():
    """0 times infinity, as the formula has it."""
    g = gen(9)
    q, k, v = randn(g, "bf16", 1, 2, 64).abs(), randn(g, "bf16", 40, 1, 64), randn(g, "bf16", 40, 1, 64)
    k[11], v[11, 0, 5] = -math.inf, math.inf
    want, _ = attend(q, k, v, [39], 0.125)
    assert torch.isnan(want[..., 5]).all()
    same_kind(run_decode("bf16", q, [k], [v]), want)


@pytest.mark.parametrize("queries,rows,page_rows,batch", [(40, 200, 0, 0), (40, 200, 16, 0), (5, 1600, 0, 0), (300, 400, 0, 2100)])
@pytest.mark.parametrize("gap", [40.0, 200.0])
@pytest.mark.parametrize("d,dtype", [(64, "f16"), (128, "bf16")])
def test_prompt_infinite_values_of_small_weights(d, dtype, gap, queries, rows, page_rows, batch):
    for top, odd in ((0, rows - queries), (rows - queries, 0), (rows - queries - 1, 1)):
        q, k, v = infinite_values(dtype, rows, d, gap, top, odd)
        q = q.expand(queries, 4, d).contiguous()
        want, size = attend(q, k, v, torch.arange(rows - queries, rows), LN2)
        got = run_prompt(dtype, q, k, v, [queries], [rows], scale=LN2, page_rows=page_rows, batch=batch)
        fine = same_kind(got, want)
        assert torch.isinf(want).any() and torch.isnan(want).any()
        check(torch.where(fine, got, 0), torch.where(fine, want, 0), torch.where(fine, size, 0), dtype, True)


@pytest.mark.parametrize("queries,rows", [(30, 70), (5, 1600)])
def test_prompt_infinite_value_under_a_score_of_minus_infinity(queries, rows):
    """0 times infinity, as the formula has it, for the queries that see the key, at every place of a block."""
    g = gen(10)
    q, k, v = randn(g, "bf16", queries, 2, 64).abs(), randn(g, "bf16", rows, 1, 64), randn(g, "bf16", rows, 1, 64)
    for i, key in enumerate((0, 3, 5, 14, 22, 31, 32, 45, 63, rows - 2)):
        k[key], v[key, 0, 5 + i], v[key, 0, 40] = -math.inf, -math.inf if i % 2 else math.inf, math.inf
        v[key + 1, 0, 30 + i] = math.inf
    want, _ = attend(q, k, v, torch.arange(rows - queries, rows), 0.125)
    same_kind(run_prompt("bf16", q, k, v, [queries], [rows]), want)


# ------------------------------------------------------------------------------------------------ what is left in the workspace
def left_behind(L, pattern):
    """The area behind the counters as another layer's plain 32-bit sums may leave it."""
    words = L.ws.view(torch.int32)
    words[16384:] = pattern


# 32-bit numbers of every kind that a sum can be
@pytest.mark.parametrize("pattern", [0x53504C54, 0x4C4C5701, 0x3F800000, -0x40000000, 0x7F800000, 0x7FC00000, -1 << 22, 1])
def test_decode_over_what_sums_leave_in_the_workspace(pattern):
    g = gen(41)
    hq, hkv, d, rows = 4, 2, 64, 3000
    q, k, v = randn(g, "bf16", 1, hq, d), randn(g, "bf16", rows, hkv, d), randn(g, "bf16", rows, hkv, d)
    want, size = attend_fast(q, k, v, [rows - 1], d ** -0.5)
    L = Layer(1, hq, hkv, d, "bf16")
    left_behind(L, pattern)
    for _ in range(2):
        check(run_decode("bf16", q, [k], [v], L=L), want, size, "bf16", False)
    L.close()


@pytest.mark.parametrize("name,over", [("c3_small", dict(context=1500, batch=2)), ("c4_small", dict()), ("c2_small", dict(context=900)), ("c1", dict())])
def test_one_workspace_serves_latent_and_dense_layers_in_turn(name, over):
    """Latent appends, split attention and decode steps between dense prompts whose tiles are shared and dense decode calls that are cut, on
    one context: the latent calls as on a context of their own, bit for bit, the dense ones against the formula."""
    import wsvd_inputs as WI
    from cases import build_case
    from harness import as_dtype_dev, q_to_device
    from test_gpu_parity import layer_for
    c = build_case(name, extra_cap=128, **over)
    sp = c.sp
    alone, shared = layer_for(c), layer_for(c)
    g = gen(51)
    hq, hkv, d, rows, tokens = 4, 1, 128, 2600, 9
    k, v, q = randn(g, "bf16", rows, hkv, d), randn(g, "bf16", rows, hkv, d), randn(g, "bf16", tokens, hq, d)
    want, size = attend_fast(q, k, v, torch.arange(rows - tokens, rows), d ** -0.5)
    desc = W.dense_desc(1, hq, hkv, d, "bf16")
    shared.ws = torch.empty(max(W.wsvd_dense_workspace_bytes(desc), shared.ws.numel()), dtype=torch.uint8, device="cuda")
    W.wsvd_set_workspace(shared.ctx, shared.ws)
    pool = Pool(gen(17), [rows], hkv, d, 16, "bf16", fill_rows=False)
    pool.put(0, 0, k, v)
    kd, vd, lens, table, qd, cu = pool.k.cuda(), pool.v.cuda(), torch.tensor([rows], dtype=torch.int32).cuda(), pool.table.cuda(), q.cuda(), prefix([tokens]).cuda()
    cache = W.make_paged_cache(kd, vd, None, None, lens, table, 16, pool.max_pages, pool.n_pages)
    many, one = (torch.empty(n, hq, d, dtype=torch.bfloat16, device="cuda") for n in (tokens, 1))
    x = as_dtype_dev(WI.bf16_exact(c.x_new[0]) if sp.factor_dtype == "bf16" else c.x_new[0], sp.factor_dtype)
    ql, qs, _ = q_to_device(c.q32[0], sp.q_dtype)
    B = [as_dtype_dev(b, sp.factor_dtype) for b in (c.BK, c.BV)]
    A = {}
    for L in (alone, shared):
        L.upload(c.cache)
        A[L] = [L.pack_A(a, sp.factor_dtype) for a in (c.AK, c.AV)]

    def dense():
        many.zero_(), one.zero_()
        W.wsvd_dense_prefill_attn_paged(shared.ctx, desc, qd, hq * d, tokens, cu, cache, many, hq * d)
        W.wsvd_dense_decode_attn_paged(shared.ctx, desc, qd[tokens - 1:], hq * d, cache, rows, one)
        W.wsvd_dense_prefill_attn_paged(shared.ctx, desc, qd, hq * d, tokens, cu, cache, many, hq * d)
        check(many.cpu(), want, size, "bf16", True)
        check(one.cpu(), want[tokens - 1:], size[tokens - 1:], "bf16", False)

    longest = int(c.lens.max())
    for i in range(4):
        outs = []
        for L in (alone, shared):
            W.wsvd_ctx_set_option(L.ctx, "step_launches", 0 if i % 2 else 2)
            if L is shared:
                dense()
            assert L.append(x, None, *A[L]) == 0
            if L is shared:
                dense()
            o = [L.attend(ql, qs, *B, longest + 2 * i + 1)]
            if L is shared:
                dense()
            got, st = L.step(x, *A[L], ql, qs, *B, longest + 2 * i + 2)
            assert st == 0, W.status_str(st)
            outs.append(o + [got])
        for a, b in zip(*outs):
            assert (a == b).all(), i
        for a, b in ((alone.k_codes, shared.k_codes), (alone.v_codes, shared.v_codes)):
            assert torch.equal(a, b)
    alone.close(), shared.close()


# ------------------------------------------------------------------------------------------------ forms that large calls take
def large_append(hq, hkv, d, dtype, before, new, page_rows, ld_extra=0):
    """Every token of a large append against the rotation in 64 bits; rows of nobody stay as they were."""
    g, T, B = gen(sum(new) + d), sum(new), len(new)
    L = Layer(B, hq, hkv, d, dtype)
    pool = Pool(g, [a + n for a, n in zip(before, new)], hkv, d, page_rows, dtype, fill_rows=False)
    cache = L.cache(pool)
    ld = (hq + 2 * hkv) * d + ld_extra
    x = randn(g, dtype, T, ld)
    inv = 10000.0 ** (-torch.arange(0, d, 2, dtype=F64) / d)
    q_out, k_out = (torch.full((T, h * d + 8), 7.0, dtype=DTYPES[dtype], device="cuda") for h in (hq, hkv))
    xd = x.cuda()
    W.wsvd_dense_append_paged(L.ctx, L.desc, xd, ld, xd[:, hq * d:], ld, xd[:, (hq + hkv) * d:], ld, T, prefix(new).cuda(), None, inv.cuda(),
                              q_out, hq * d + 8, k_out, hkv * d + 8, cache)
    y = x[:, : (hq + 2 * hkv) * d].view(T, hq + 2 * hkv, d)
    b = torch.repeat_interleave(torch.arange(B), torch.tensor(new))
    pos = torch.tensor(before)[b] + torch.arange(T) - prefix(new).long()[b]
    want = rotate(y[:, :hq + hkv], pos, inv)
    pair = torch.hypot(want[..., : d // 2], want[..., d // 2:]).repeat(1, 1, 2)
    # the result's rounding, and fp32 products of a pair: 3 roundings of at most sqrt(2) times the pair's length
    tol = half_step(dtype) * want.abs() + 2.0 ** -21 * pair + (2.0 ** -25 if dtype == "f16" else 0)
    near = lambda got, part: bool(((got.to(F64) - want[:, part]).abs() <= tol[:, part]).all())
    assert near(q_out[:, : hq * d].cpu().view(T, hq, d), slice(0, hq))
    assert near(k_out[:, : hkv * d].cpu().view(T, hkv, d), slice(hq, hq + hkv))
    assert (q_out[:, hq * d:] == 7).all() and (k_out[:, hkv * d:] == 7).all()
    page, row = pool.table[b, pos // page_rows].long(), pos % page_rows
    k, v = L.k.cpu(), L.v.cpu()
    assert near(k[page, :, row], slice(hq, hq + hkv)) and torch.equal(v[page, :, row], y[:, hq + hkv:])
    touched = torch.zeros(k.shape[0], page_rows, dtype=torch.bool)
    touched[page, row] = True
    for x in (k, v):
        assert torch.isnan(x.transpose(1, 2)[~touched]).all()
    L.close()


@pytest.mark.parametrize("hq,hkv,d,dtype,tokens", [
    (16, 2, 128, "bf16", 2307),                 # two tokens a workgroup
    (16, 2, 128, "f16", 9901),                  # the same, past the caches
    (28, 4, 128, "bf16", 2049),                 # one token, within them
    (32, 32, 128, "bf16", 2113),                # one token, past them
    (32, 32, 64, "f16", 4501),
    (4, 2, 64, "f16", 2050),                    # four tokens
    (4, 2, 64, "bf16", 48901),                  # four tokens, past the caches
])
def test_append_forms_of_large_calls(hq, hkv, d, dtype, tokens):
    part = [tokens // 7, 0, tokens // 3 + 1, 1]
    large_append(hq, hkv, d, dtype, [5, 90, 0, 333, 18], part + [tokens - sum(part)], 48, ld_extra=8)


@pytest.mark.parametrize("min_chunk", [0, 128])
def test_decode_gives_a_sequence_the_same_bits_in_every_place(min_chunk):
    """The same sequences in another order, in other pages: their outputs move with them, bit for bit."""
    g = gen(3)
    hq, hkv, d, lens = 8, 2, 128, [900, 3000, 17, 0, 1300, 1, 640]
    q, k, v = randn(g, "bf16", len(lens), hq, d), [randn(g, "bf16", n, hkv, d) for n in lens], [randn(g, "bf16", n, hkv, d) for n in lens]
    first = run_decode("bf16", q, k, v, min_chunk=min_chunk)
    for order in ([6, 5, 4, 3, 2, 1, 0], [2, 0, 5, 1, 6, 3, 4]):
        again = run_decode("bf16", q[order], [k[i] for i in order], [v[i] for i in order], min_chunk=min_chunk, page_rows=32)
        assert torch.equal(again, first[order])


@pytest.mark.parametrize("hq,hkv,d,dtype,nq,nk,page_rows,batch", [
    (4, 4, 128, "bf16", [700, 3, 257], [700, 3, 257], 0, 0), (28, 4, 128, "bf16", [333, 90], [1834, 400], 16, 0),
    (8, 1, 64, "f16", [5, 70], [2600, 1200], 16, 0), (2, 1, 128, "f16", [300, 129, 511], [300, 129, 511], 0, 2100)])
def test_prompts_repeat_themselves_bit_for_bit(hq, hkv, d, dtype, nq, nk, page_rows, batch):
    """Whole tiles, shared ones, two a workgroup: nothing depends on which workgroup comes first."""
    g = gen(4)
    q, k, v = randn(g, dtype, sum(nq), hq, d), randn(g, dtype, sum(nk), hkv, d), randn(g, dtype, sum(nk), hkv, d)
    first = run_prompt(dtype, q, k, v, nq, nk, page_rows=page_rows, batch=batch)
    for _ in range(3):
        assert torch.equal(run_prompt(dtype, q, k, v, nq, nk, page_rows=page_rows, batch=batch), first)


@pytest.mark.parametrize("d,dtype", [(64, "f16"), (128, "bf16")])
def test_infinite_values_change_no_other_output(d, dtype):
    """With and without them: other dims, other heads and queries that do not see them come out with the same bits."""
    g = gen(61)
    rows, queries = 700, 150
    q, k, v = randn(g, dtype, queries, 4, d), randn(g, dtype, rows, 2, d), randn(g, dtype, rows, 2, d)
    odd = v.clone()
    key = rows - queries + 60                                      # the first 60 queries do not see it
    odd[key, 1, 3], odd[key, 1, 9], odd[key, 1, d - 1] = math.inf, math.nan, -math.inf
    touched = torch.zeros(queries, 4, d, dtype=torch.bool)
    touched[60:, 2:, 3], touched[60:, 2:, 9], touched[60:, 2:, d - 1] = True, True, True
    for page_rows in (0, 16):
        plain, other = (run_prompt(dtype, q, k, x, [queries], [rows], page_rows=page_rows) for x in (v, odd))
        assert torch.equal(plain[~touched], other[~touched]) and not torch.isfinite(other[touched]).any()
    for min_chunk in (0, 128):
        plain, other = (run_decode(dtype, q[-1:], [k], [x], min_chunk=min_chunk) for x in (v, odd))
        assert torch.equal(plain[~touched[-1:]], other[~touched[-1:]]) and not torch.isfinite(other[touched[-1:]]).any()
