"""The calls of the 8-bit cache together, as a server makes them: requests that come and go, steps in graphs, tables on the GPU; and the
numbers at the ends of the types' ranges through append and attention."""
import math
import os
import sys

import pytest
import torch

import paper_2604_02570_amd as W
from dense_ref import DTYPES, F64, attend_fast, check, prefix, randn, rotate
from f8_ref import BIAS, F8Pool, exponent, quantised
from test_gpu_dense import BASE, gen
from test_gpu_dense_f8 import Layer

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu


def test_requests_that_come_and_go():
    """The example, request by request, against a plain 64-bit layer without quantisation."""
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import serving_with_8bit_cache as example
    finally:
        sys.path.pop(0)
    r = example.run()
    layer, w, inv = r["layer"], r["layer"].w_qkv.cpu().to(F64), r["layer"].inv_freq.cpu()
    hq, hkv, d = layer.hq, layer.hkv, layer.d
    assert len(r["requests"]) == 12
    for q in r["requests"]:
        x = torch.cat(q["x"]).cpu().to(F64)
        y = (x @ w).view(-1, hq + 2 * hkv, d)
        n = torch.arange(y.shape[0])
        want, size = attend_fast(rotate(y[:, :hq], n, inv), rotate(y[:, hq:hq + hkv], n, inv), y[:, hq + hkv:], n, 1.0 / math.sqrt(d))
        got = torch.cat(q["out"]).cpu().to(F64).view(-1, hq, d)
        # A code is off by half a step, 2^-4, of its number: a value's error enters at that size, and a score of about 1, a sum of d
        # products whose keys are off by 2^-4 each (independent, 2^-4 * 2^-1 in the mean square), by less than 2^-2: 2^-1 of the mean of |v| at
        # most (the definition itself is checked bit for bit elsewhere; this finds rows and pages that are mixed up, whose error is of |v|'s size).
        err = (got - want).abs()
        assert (err <= 2.0 ** -4 * want.abs() + 2.0 ** -1 * size + 2.0 ** -8).all()
        assert err.mean() <= 2.0 ** -4 * size.mean()
    assert layer.lens.tolist() == [sum(t.shape[0] for t in q["x"]) for q in r["running"]]
    used = sum(-(-n // layer.page_rows) for n in layer.lens.tolist())
    held = [p for b, n in enumerate(layer.lens.tolist()) for p in layer.table[b, : -(-n // layer.page_rows)].tolist()]
    assert int(layer.n_free) == layer.n_pages - used and sorted(held + layer.free[: layer.n_pages - used].tolist()) == list(range(layer.n_pages))
    example.close(r)


@pytest.mark.parametrize("hq,hkv,d,dtype", [(8, 2, 128, "bf16"), (4, 4, 64, "f16")])
def test_step_in_a_graph_on_another_stream(hq, hkv, d, dtype):
    """Tables, append and attention captured on a stream of their own; replays, with eager work between, give what the definition gives."""
    g, B, R, P = gen(9), 3, 16, 90
    lens = [200, 1, 1030]
    L, pool = Layer(B, hq, hkv, d, dtype), F8Pool(g, [n + 8 for n in lens], hkv, d, R, dtype, max_pages=P, spare=9)
    for b, n in enumerate(lens):
        pool.append(b, 0, randn(g, dtype, n, hkv, d), randn(g, dtype, n, hkv, d))
    cache = L.cache(pool, lens)
    used = [-(-n // R) for n in lens]
    mine = {int(pool.table[b, i]) for b in range(B) for i in range(used[b])}
    rest = [p for p in range(pool.n_pages) if p not in mine]
    free, n_free = torch.tensor(rest + [0] * len(mine), dtype=torch.int32, device="cuda"), torch.tensor([len(rest)], dtype=torch.int32, device="cuda")
    tables = W.make_page_pool(L.table, free, B, R, P, pool.n_pages)
    x, out = torch.zeros(B, (hq + 2 * hkv) * d, dtype=DTYPES[dtype], device="cuda"), torch.empty(B, hq, d, dtype=DTYPES[dtype], device="cuda")
    q_rot, k_rot, inv = torch.empty(B, hq * d, dtype=x.dtype, device="cuda"), torch.empty(B, hkv * d, dtype=x.dtype, device="cuda"), (BASE ** (-torch.arange(0, d, 2, dtype=F64) / d)).cuda()
    ld = x.shape[1]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        on = torch.cuda.current_stream()
        W.wsvd_pages_grow(L.ctx, tables, None, B, L.lens, n_free, L.lens, n_free, stream=on)
        W.wsvd_dense_append_paged_f8(L.ctx, L.desc, x, ld, x[:, hq * d:], ld, x[:, (hq + hkv) * d:], ld, B, None, None, inv, q_rot, hq * d, k_rot, hkv * d, cache, on)
        W.wsvd_dense_decode_attn_paged_f8(L.ctx, L.desc, q_rot, hq * d, cache, P * R, out, on)
    for i in range(5):
        new = randn(g, dtype, B, ld, scale=2.0 ** (i - 1))
        x.copy_(new)
        out.fill_(math.nan)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        pool.table = L.table.cpu()
        for b in range(B):
            pool.append(b, lens[b], k_rot[b:b + 1].view(1, hkv, d).cpu(), new[b:b + 1, (hq + hkv) * d:].view(1, hkv, d))
            lens[b] += 1
        L.holds(pool)
        for b in range(B):
            k, v = pool.rows(b, lens[b])
            want, size = attend_fast(q_rot[b:b + 1].view(1, hq, d).cpu(), k, v, [lens[b] - 1], L.scale)
            check(out[b:b + 1].cpu(), want, size, dtype, False)
        torch.matmul(x[:, :64].float(), x[:, :64].float().t())         # the program's own work between replays
    assert L.lens.tolist() == lens
    L.close()


@pytest.mark.parametrize("dtype,size_k,size_v", [("f16", 1.0, 2.0 ** -21), ("f16", 2.0 ** -19, 1.0), ("f16", 0.01, 20000.0), ("bf16", 1.0, 1e37), ("bf16", 1.0, 2.0 ** -90),
                                                 ("bf16", 2.0 ** -60, 1.0)])
@pytest.mark.parametrize("d", [64, 128])
def test_numbers_at_the_ends_of_the_types(dtype, size_k, size_v, d):
    """Rows as small and as large as the type holds: what is stored is a number of the type, and attention takes it as it is."""
    hq, hkv, n, g = 4, 2, 70, gen(12)
    most = torch.finfo(DTYPES[dtype]).max
    L, pool = Layer(1, hq, hkv, d, dtype), F8Pool(g, [n], hkv, d, 16, dtype)
    k, v = ((torch.randn(n, hkv, d, generator=g) * s).clamp(-most, most).to(DTYPES[dtype]) for s in (size_k, size_v))
    q = (torch.randn(n, hq, d, generator=g) * min(1 / size_k, 1000.0)).to(DTYPES[dtype])
    cache, cu = L.cache(pool), prefix([n]).cuda()
    kd, vd, qd = k.cuda(), v.cuda(), q.cuda()
    W.wsvd_dense_append_paged_f8(L.ctx, L.desc, None, 0, kd, hkv * d, vd, hkv * d, n, cu, None, None, None, 0, None, 0, cache)
    pool.append(0, 0, k, v)
    L.holds(pool)
    kk, vv = pool.rows(0)
    for x in (kk, vv):
        assert torch.equal(x.to(DTYPES[dtype]).to(F64), x)
    want, size = attend_fast(q, kk, vv, list(range(n)), L.scale)
    out, one = torch.empty(n, hq * d, dtype=DTYPES[dtype], device="cuda"), torch.empty(1, hq, d, dtype=DTYPES[dtype], device="cuda")
    W.wsvd_dense_prefill_attn_paged_f8(L.ctx, L.desc, qd, hq * d, n, cu, cache, out, hq * d)
    W.wsvd_dense_decode_attn_paged_f8(L.ctx, L.desc, qd[n - 1:], hq * d, cache, n, one)
    check(out.view(n, hq, d).cpu(), want, size, dtype, True)
    check(one.cpu(), want[n - 1:], size[n - 1:], dtype, False)
    L.close()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_infinite_queries(dtype):
    """Scores of -inf alone count as nothing to see, whatever the values are; an infinite weight is none, for its head alone."""
    hq, hkv, d, n, g = 3, 1, 64, 40, gen(13)
    L, pool = Layer(1, hq, hkv, d, dtype), F8Pool(g, [n], hkv, d, 16, dtype).random(g)
    for row in range(n):
        pool.set("k", 0, row, 0, 9, 0xB8)                               # -1 times the scale
    pool.set("v", 0, 11, 0, 3, 0x7F)
    q = randn(g, dtype, 2, hq * d)
    q[:, 9], q[:, d + 9] = math.inf, -math.inf                          # the first head's scores are all -inf, the second's +inf
    out, one = torch.empty(2, hq * d, dtype=DTYPES[dtype], device="cuda"), torch.empty(1, hq, d, dtype=DTYPES[dtype], device="cuda")
    cache, qd = L.cache(pool), q.cuda()
    W.wsvd_dense_prefill_attn_paged_f8(L.ctx, L.desc, qd, hq * d, 2, prefix([2]).cuda(), cache, out, hq * d)
    W.wsvd_dense_decode_attn_paged_f8(L.ctx, L.desc, qd[1:], hq * d, cache, n, one)
    k, v = pool.rows(0)
    want, size = attend_fast(q.view(2, hq, d)[:, 2:].clone(), k, v.nan_to_num(0), [n - 2, n - 1], L.scale)
    for got, w, s in ((out.view(2, hq, d).cpu(), want, size), (one.cpu(), want[1:], size[1:])):
        assert (got[:, 0] == 0).all() and torch.isnan(got[:, 1]).all()
        assert torch.isnan(got[:, 2, 3]).all()
        fine = [i for i in range(d) if i != 3]
        check(got[:, 2:, fine], w[..., fine], s[..., fine], dtype, True)
    L.close()


def test_two_contexts_on_two_streams():
    """Contexts are independent: two layers at work side by side give what they give one after the other."""
    g, hq, hkv, d, lens = gen(14), 8, 2, 128, [2100, 33, 700]
    pool = F8Pool(g, lens, hkv, d, 16, "bf16").random(g)
    layers, outs, queries = [Layer(3, hq, hkv, d, "bf16") for _ in range(2)], [], [randn(g, "bf16", 3, hq * d).cuda() for _ in range(2)]
    caches = [L.cache(pool) for L in layers]
    for L, c, q in zip(layers, caches, queries):
        out = torch.empty(3, hq, d, dtype=torch.bfloat16, device="cuda")
        W.wsvd_dense_decode_attn_paged_f8(L.ctx, L.desc, q, hq * d, c, 2100, out)
        outs.append(out)
    streams, again = [torch.cuda.Stream() for _ in range(2)], [torch.empty_like(o) for o in outs]
    torch.cuda.synchronize()
    for _ in range(20):
        for L, c, q, s, out in zip(layers, caches, queries, streams, again):
            W.wsvd_dense_decode_attn_paged_f8(L.ctx, L.desc, q, hq * d, c, 2100, out, s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, again))
    for L in layers:
        L.close()


def test_workspace_serves_16_bit_and_8_bit_calls_in_turn():
    """Partial results that a chunk leaves in the workspace lie where a decode call's workgroups hand theirs over."""
    from dense_ref import Pool
    from test_gpu_dense import Layer as DenseLayer
    g, hq, hkv, d = gen(15), 8, 1, 64
    L, pool = Layer(1, hq, hkv, d, "bf16"), F8Pool(g, [6000], hkv, d, 16, "bf16").random(g)
    cache = L.cache(pool)
    D = DenseLayer(1, hq, hkv, d, "bf16")
    plain = Pool(g, [6000], hkv, d, 16, "bf16")
    dense = D.cache(plain)
    q = randn(g, "bf16", 20, hq * d)
    qd, cu = q.cuda(), prefix([20]).cuda()
    refs = [attend_fast(q.view(20, hq, d), *p.rows(0), torch.arange(5980, 6000), L.scale) for p in (pool, plain)]
    out, one = torch.empty(20, hq * d, dtype=torch.bfloat16, device="cuda"), torch.empty(1, hq, d, dtype=torch.bfloat16, device="cuda")
    for _ in range(2):
        for (want, size), c, many, single in ((refs[0], cache, W.wsvd_dense_prefill_attn_paged_f8, W.wsvd_dense_decode_attn_paged_f8),
                                              (refs[1], dense, W.wsvd_dense_prefill_attn_paged, W.wsvd_dense_decode_attn_paged)):
            many(L.ctx, L.desc, qd, hq * d, 20, cu, c, out, hq * d)
            single(L.ctx, L.desc, qd[19:], hq * d, c, 6000, one)
            check(out.view(20, hq, d).cpu(), want, size, "bf16", True)
            check(one.cpu(), want[19:], size[19:], "bf16", False)
            out.zero_(), one.zero_()
    D.close()
    L.close()


def test_append_fills_what_prompts_left_begun():
    """A prompt in pieces of odd lengths gives the rows of one call where no scale has to grow, and reads back as the definition has it."""
    hq, hkv, d, g, dtype = 2, 2, 64, gen(16), "bf16"
    pieces = [5, 11, 1, 16, 30, 1, 1, 63]
    n = sum(pieces)
    x = randn(g, dtype, n, (hq + 2 * hkv) * d)
    x[0::16] *= 8                                                      # each block's first row is its largest
    ld, stored = x.shape[1], []
    for split in ([n], pieces):
        L, pool, at = Layer(1, hq, hkv, d, dtype), F8Pool(gen(17), [n], hkv, d, 32, dtype), 0
        cache, xd = L.cache(pool), x.cuda()
        for m in split:
            L.lens.fill_(at + m)
            W.wsvd_dense_append_paged_f8(L.ctx, L.desc, None, 0, xd[at:, hq * d:], ld, xd[at:, (hq + hkv) * d:], ld, m, prefix([m]).cuda(), None, None, None, 0, None, 0,
                                         cache)
            at += m
        torch.cuda.synchronize()
        stored.append([t.cpu() for t in (L.k, L.v, L.ks, L.vs)])
        pool.append(0, 0, x[:, hq * d:(hq + hkv) * d].view(n, hkv, d), x[:, (hq + hkv) * d:].view(n, hkv, d))
        L.holds(pool)
        L.close()
    assert all(torch.equal(a, b) for a, b in zip(*stored))
