#!/usr/bin/env python3
"""Continuous batching over an 8-bit cache whose page tables live on the GPU.

An attention layer serves requests that come and go in a few slots.  Its cache holds E4M3 codes with a scale for each block of 16 rows and
kv head; pages are dealt out from a free list on the device.  A step is

  1. pages of finished sequences back to the free list, pages for the step's new tokens (wsvd_pages_release, wsvd_pages_grow);
  2. rotary embedding, keys and values quantised into the pages (wsvd_dense_append_paged_f8);
  3. attention: of a mixed step's packed tokens, pieces of prompts beside single tokens (wsvd_dense_prefill_attn_paged_f8), or,
     once every slot goes on by one token, of those (wsvd_dense_decode_attn_paged_f8), as a graph that is replayed: the host
     sends no table and no length.

Weights are random.  Run it from the repository's root:  python3 examples/serving_with_8bit_cache.py
"""
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch

import paper_2604_02570_amd as W

BF16, I32, U8 = torch.bfloat16, torch.int32, torch.uint8


def ints(*shape):
    return torch.zeros(*shape, dtype=I32, device="cuda")


class Layer:
    """x -> attention output, over a cache of `slots` sequences."""

    def __init__(self, slots, d_model, q_heads, kv_heads, d, page_rows, max_pages, n_pages):
        self.slots, self.hq, self.hkv, self.d, self.rows = slots, q_heads, kv_heads, d, page_rows * max_pages
        self.w_qkv = (torch.randn(d_model, (q_heads + 2 * kv_heads) * d, device="cuda") * d_model ** -0.5).to(BF16)
        self.inv_freq = 10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64, device="cuda") / d)
        self.desc = W.dense_desc(slots, q_heads, kv_heads, d, "bf16")
        self.ctx = W.wsvd_create(0)
        self.workspace = torch.empty(W.wsvd_dense_workspace_bytes(self.desc), dtype=U8, device="cuda")
        W.wsvd_set_workspace(self.ctx, self.workspace)
        # the page tables: nobody has a page, all are free
        self.table, self.free, self.n_free, self.lens = ints(slots, max_pages), torch.randperm(n_pages, device="cuda").to(I32), ints(1) + n_pages, ints(slots)
        self.tables = W.make_page_pool(self.table, self.free, slots, page_rows, max_pages, n_pages)
        codes, scales = W.wsvd_dense_f8_cache_bytes(self.desc, page_rows, n_pages)
        self.pools = [torch.zeros(n, dtype=U8, device="cuda") for n in (codes, codes, scales, scales)]
        self.cache = W.make_paged_cache(*self.pools, self.lens, self.table, page_rows, max_pages, n_pages)
        self.page_rows, self.n_pages = page_rows, n_pages

    def append(self, x, cu, stream=None):
        y, wq, wkv = x @ self.w_qkv, self.hq * self.d, self.hkv * self.d
        W.wsvd_dense_append_paged_f8(self.ctx, self.desc, y, y.shape[1], y[:, wq:], y.shape[1], y[:, wq + wkv:], y.shape[1], x.shape[0], cu, None,
                                     self.inv_freq, y, y.shape[1], None, 0, self.cache, stream)
        return y

    def mixed(self, x, done, new):
        """A step of packed tokens, new[b] of slot b, after the sequences with done[b] have left."""
        n, cu, out = x.shape[0], ints(self.slots + 1), torch.empty(x.shape[0], self.hq * self.d, dtype=BF16, device="cuda")
        done, new = (torch.tensor(v, dtype=I32, device="cuda") for v in (done, new))
        W.wsvd_pages_release(self.ctx, self.tables, done, self.lens, self.n_free, self.lens, self.n_free)
        W.wsvd_pages_grow(self.ctx, self.tables, new, n, self.lens, self.n_free, self.lens, self.n_free, cu)
        y = self.append(x, cu)
        W.wsvd_dense_prefill_attn_paged_f8(self.ctx, self.desc, y, y.shape[1], n, cu, self.cache, out, out.shape[1])
        return out

    def step(self, x, out, stream=None):
        """One token of every slot."""
        W.wsvd_pages_grow(self.ctx, self.tables, None, self.slots, self.lens, self.n_free, self.lens, self.n_free, stream=stream)
        y = self.append(x, None, stream)
        W.wsvd_dense_decode_attn_paged_f8(self.ctx, self.desc, y, y.shape[1], self.cache, self.rows, out, stream)


def run(steps=8, seed=0):
    """Serves the requests; returns what a check needs: the layer and, request by request, hidden states and outputs in order."""
    torch.manual_seed(seed)
    slots, d_model, piece = 6, 512, 48
    layer = Layer(slots, d_model, 8, 2, 128, 32, 12, 40)
    waiting = [(70, 3), (5, 9), (200, 2), (33, 1), (130, 6), (1, 4), (90, 0), (17, 0), (60, 0), (49, 0), (150, 0), (20, 0)]     # prompt, tokens after it (0: to the end)
    requests, running = [], [None] * slots
    while waiting or any(r and r["left"] for r in running):
        done = [int(r is not None and r["left"] == 0 and r["more"] == 0 and not r["stays"]) for r in running]
        for b, end in enumerate(done):
            if end:
                running[b] = None
        for b in range(slots):
            if running[b] is None and waiting:
                prompt, after = waiting.pop(0)
                running[b] = dict(left=prompt, more=after, stays=after == 0, x=[], out=[])
                requests.append(running[b])
        new = [0 if r is None else min(r["left"], piece) if r["left"] else int(r["more"] > 0) for r in running]
        x = torch.randn(sum(new), d_model, device="cuda").to(BF16)
        out, at = layer.mixed(x, done, new), 0
        for r, n in zip(running, new):
            if n:
                r["x"].append(x[at:at + n]), r["out"].append(out[at:at + n])
                r["left" if r["left"] else "more"] -= n
                at += n
    assert all(r["stays"] for r in running)

    # from here on every slot goes on by one token a step: one graph, replayed
    x, out = torch.zeros(slots, d_model, dtype=BF16, device="cuda"), torch.empty(slots, layer.hq * layer.d, dtype=BF16, device="cuda")
    x @ layer.w_qkv                                                    # the library product's own set-up stays out of the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.step(x, out, torch.cuda.current_stream())
    for _ in range(steps):
        x.copy_(torch.randn(slots, d_model, device="cuda").to(BF16))
        graph.replay()
        for b, r in enumerate(running):
            r["x"].append(x[b:b + 1].clone()), r["out"].append(out[b:b + 1].clone())
    status = W.wsvd_check(layer.ctx)
    assert status == W.OK, W.status_str(status)
    return dict(layer=layer, requests=requests, running=running)


def close(result):
    torch.cuda.synchronize()
    W.wsvd_destroy(result["layer"].ctx)


if __name__ == "__main__":
    r = run()
    layer = r["layer"]
    print("requests served:", len(r["requests"]), " rows per slot:", layer.lens.tolist(), " free pages:", int(layer.n_free), "of", layer.n_pages)
    print("bytes of a cached token: %.1f, in 16 bits %d" % (2 * layer.hkv * (layer.d + 1 / 16), 2 * layer.hkv * layer.d * 2))
    print("all finite:", all(bool(torch.isfinite(t).all()) for q in r["requests"] for t in q["out"]))
    close(r)
