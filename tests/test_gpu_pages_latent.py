"""Page tables from the free list under latent layers, whose appends advance their lengths themselves, and under a dense layer in 8 bits beside them."""
import os
import sys

import pytest
import torch

import paper_2604_02570_amd as W
from dense_ref import attend_fast, check, prefix, randn
from f8_ref import F8Pool
from test_gpu_dense import gen
from test_gpu_dense_f8 import Layer

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu


def latent_layer(pages):
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import dense_and_latent_layers as example
    finally:
        sys.path.pop(0)
    torch.manual_seed(5)
    return example.LatentLayer(pages, 256, 4, 2, 128, 32)


class Pages:
    def __init__(self, batch, page_rows, max_pages, n_pages):
        self.batch, self.page_rows, self.max_pages, self.n_pages, self.rows = batch, page_rows, max_pages, n_pages, page_rows * max_pages
        self.table = torch.full((batch, max_pages), -1, dtype=torch.int32, device="cuda")


def test_latent_layers_and_a_dense_one_over_a_growing_table():
    """Lengths grow into memory of their own where the latent append advances them; the dense layer takes the advanced ones.  The outputs are those
    of a latent layer whose table was full from the start, bit for bit, and those of the definition."""
    B, R, P, d_model, hq, hkv, d, g = 3, 64, 5, 256, 4, 2, 128, gen(3)
    grown, full = Pages(B, R, P, B * P), Pages(B, R, P, B * P)
    full.table.copy_(torch.randperm(B * P, generator=g).to(torch.int32).view(B, P))
    latent, want = latent_layer(grown), latent_layer(full)
    free, n_free = torch.randperm(B * P, generator=g).to(torch.int32).cuda(), torch.tensor([B * P], dtype=torch.int32, device="cuda")
    tables, after = W.make_page_pool(grown.table, free, B, R, P, B * P), torch.empty(B, dtype=torch.int32, device="cuda")
    L, pool = Layer(B, hq, hkv, d, "bf16"), F8Pool(g, [0] * B, hkv, d, R, "bf16", max_pages=P, spare=B * P)
    L.cache(pool)
    cache = W.make_paged_cache(L.k, L.v, L.ks, L.vs, latent.lens, grown.table, R, P, B * P)
    lens = [0] * B
    outs, out = [torch.empty(B, hq, d, dtype=torch.float32, device="cuda") for _ in range(2)], torch.empty(B, hq, d, dtype=torch.bfloat16, device="cuda")
    for new in ([70, 5, 130], [30, 61, 1], *[[1] * B] * 5):
        T, cu = sum(new), torch.empty(B + 1, dtype=torch.int32, device="cuda")
        x, y = randn(g, "bf16", T, d_model).cuda(), randn(g, "bf16", T, (hq + 2 * hkv) * d)
        W.wsvd_pages_grow(latent.ctx, tables, torch.tensor(new, dtype=torch.int32, device="cuda"), T, latent.lens, n_free, after, n_free, cu)
        if T > B:
            latent.fill(x, new), want.fill(x, new)
        else:
            latent.step(x, outs[0]), want.step(x, outs[1])
            assert torch.equal(outs[0], outs[1])
        assert torch.equal(latent.lens, after) and torch.equal(latent.lens, want.lens)
        yd, ld = y.cuda(), y.shape[1]
        W.wsvd_dense_append_paged_f8(L.ctx, L.desc, None, 0, yd[:, hq * d:], ld, yd[:, (hq + hkv) * d:], ld, T, cu, None, None, None, 0, None, 0, cache)
        pool.table, at = grown.table.cpu(), prefix(new).tolist()
        for b in range(B):
            z = y[at[b]:at[b + 1]].view(new[b], hq + 2 * hkv, d)
            pool.append(b, lens[b], z[:, hq:hq + hkv], z[:, hq + hkv:])
            lens[b] += new[b]
        L.holds(pool)
    W.wsvd_dense_decode_attn_paged_f8(L.ctx, L.desc, yd, ld, cache, grown.rows, out)
    for b in range(B):
        k, v = pool.rows(b, lens[b])
        o, size = attend_fast(y[b:b + 1, : hq * d].view(1, hq, d), k, v, [lens[b] - 1], L.scale)
        check(out[b:b + 1].cpu(), o, size, "bf16", False)
    for layer in (latent, want):
        assert W.wsvd_check(layer.ctx) == 0
        W.wsvd_destroy(layer.ctx)
    L.close()
