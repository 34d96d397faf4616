#!/usr/bin/env python3
"""A decoder that keeps one attention layer dense and one compressed, over the same page table.

A rank budget rarely treats all layers alike: some keep plain keys and values, the others a low-rank latent per head.  Both kinds of
cache are paged and share table, page size and lengths; only the pools differ.  The script serves a few prompts of different
lengths with such a pair of layers and random weights:

  1. the first piece of every prompt, packed: rotary append and causal attention of the packed tokens (dense layer);
  2. the second piece behind the cached first one: rotary append and attention over the pages (dense layer);
  3. both pieces into the latent layer's pools, sequence by sequence, with their attention;
  4. single tokens, one step of both layers captured in a graph and replayed.

Run it from the repository's root:  python3 examples/dense_and_latent_layers.py
"""
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch

import paper_2604_02570_amd as W

BF16 = torch.bfloat16


def randn(*shape, scale=1.0):
    return (torch.randn(*shape, device="cuda") * scale).to(BF16)


def prefix(lengths):
    return torch.tensor([0, *torch.tensor(lengths).cumsum(0).tolist()], dtype=torch.int32, device="cuda")


class Pages:
    """Page table and lengths that both layers share."""

    def __init__(self, batch, page_rows, max_pages):
        self.batch, self.page_rows, self.max_pages, self.n_pages = batch, page_rows, max_pages, batch * max_pages
        self.table = torch.randperm(self.n_pages, device="cuda").to(torch.int32).view(batch, max_pages)
        self.rows = page_rows * max_pages


class DenseLayer:
    """x -> attention output of a layer with plain keys and values."""

    def __init__(self, pages, d_model, q_heads, kv_heads, d):
        self.pages, self.hq, self.hkv, self.d = pages, q_heads, kv_heads, d
        self.w_qkv = randn(d_model, (q_heads + 2 * kv_heads) * d, scale=d_model ** -0.5)
        self.inv_freq = 10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64, device="cuda") / d)
        self.desc = W.dense_desc(pages.batch, q_heads, kv_heads, d, "bf16")
        self.ctx = W.wsvd_create(0)
        self.workspace = torch.empty(W.wsvd_dense_workspace_bytes(self.desc), dtype=torch.uint8, device="cuda")
        W.wsvd_set_workspace(self.ctx, self.workspace)
        self.k, self.v = (torch.zeros(pages.n_pages, kv_heads, pages.page_rows, d, dtype=BF16, device="cuda") for _ in range(2))
        self.lens = torch.zeros(pages.batch, dtype=torch.int32, device="cuda")
        self.cache = W.make_paged_cache(self.k, self.v, None, None, self.lens, pages.table, pages.page_rows, pages.max_pages, pages.n_pages)

    def append(self, x, cu, stream=None, keep_keys=False):
        """Queries, rotated; with keep_keys the rotated keys and the values too.  The lengths count the new tokens already."""
        wq, wkv = self.hq * self.d, self.hkv * self.d
        y, n = x @ self.w_qkv, x.shape[0]
        k_out = y[:, wq:] if keep_keys else None                       # in place
        W.wsvd_dense_append_paged(self.ctx, self.desc, y, wq + 2 * wkv, y[:, wq:], wq + 2 * wkv, y[:, wq + wkv:], wq + 2 * wkv, n, cu, None,
                                  self.inv_freq, y, wq + 2 * wkv, k_out, wq + 2 * wkv, self.cache, stream)
        return y

    def prompt(self, x, lengths):
        """Whole prompts, packed, into empty sequences."""
        cu, wq, wkv = prefix(lengths), self.hq * self.d, self.hkv * self.d
        self.lens.copy_(cu[1:] - cu[:-1])
        y, out, ld = self.append(x, cu, keep_keys=True), torch.empty(x.shape[0], wq, dtype=BF16, device="cuda"), wq + 2 * wkv
        W.wsvd_dense_prefill_attn(self.ctx, self.desc, y, ld, y[:, wq:], ld, y[:, wq + wkv:], ld, x.shape[0], x.shape[0], cu, None, 1, out, wq)
        return out

    def more(self, x, lengths):
        """The next tokens of every sequence, behind what its pages hold."""
        cu, wq = prefix(lengths), self.hq * self.d
        self.lens += cu[1:] - cu[:-1]
        y, out = self.append(x, cu), torch.empty(x.shape[0], wq, dtype=BF16, device="cuda")
        W.wsvd_dense_prefill_attn_paged(self.ctx, self.desc, y, y.shape[1], x.shape[0], cu, self.cache, out, wq)
        return out

    def step(self, x, out, stream=None):
        """One token of every sequence."""
        self.lens += 1
        y = self.append(x, None, stream)
        W.wsvd_dense_decode_attn_paged(self.ctx, self.desc, y, y.shape[1], self.cache, self.pages.rows, out, stream)


class LatentLayer:
    """The same with int8 latents of rank r per head in place of keys and values."""

    def __init__(self, pages, d_model, q_heads, kv_heads, d, rank):
        self.pages, self.hq, self.hkv, self.d = pages, q_heads, kv_heads, d
        self.w_q = randn(d_model, q_heads * d, scale=d_model ** -0.5)
        self.desc = W.layer_desc(pages.batch, q_heads, kv_heads, d, d_model, rank, pages.rows, "i8", "bf16", "bf16", "bf16")
        self.ctx = W.wsvd_create(0)
        self.workspace = torch.empty(W.wsvd_workspace_bytes(self.desc), dtype=torch.uint8, device="cuda")
        W.wsvd_set_workspace(self.ctx, self.workspace)
        self.a = []
        for _ in range(2):
            packed = torch.empty(W.wsvd_factor_a_bytes(self.desc), dtype=torch.uint8, device="cuda")
            W.wsvd_pack_factor_a(self.ctx, self.desc, randn(kv_heads, d_model, rank, scale=d_model ** -0.5), packed)
            self.a.append(packed)
        self.b = [randn(kv_heads, rank, d, scale=rank ** -0.5) for _ in range(2)]
        codes, meta = W.wsvd_paged_cache_bytes(self.desc, pages.page_rows, pages.n_pages)
        self.pools = [torch.zeros(n, dtype=torch.uint8, device="cuda") for n in (codes, codes, meta, meta)]
        self.lens = torch.zeros(pages.batch, dtype=torch.int32, device="cuda")
        self.cache = W.make_paged_cache(*self.pools, self.lens, pages.table, pages.page_rows, pages.max_pages, pages.n_pages)

    def fill(self, x, lengths):
        """The next tokens of every sequence into the pools, the lengths advance."""
        at = 0
        for b, n in enumerate(lengths):
            W.wsvd_prefill_append_paged(self.ctx, self.desc, x[at:at + n].contiguous(), n, b, *self.a, self.cache)
            at += n

    def step(self, x, out, stream=None):
        q = (x @ self.w_q).view(self.pages.batch, self.hq, self.d)
        W.wsvd_latent_append_paged(self.ctx, self.desc, x, None, *self.a, self.cache, stream)
        W.wsvd_decode_attn_paged(self.ctx, self.desc, q, None, *self.b, self.cache, self.pages.rows, out, stream)


def run(steps=6, seed=0):
    """Serves the prompts; returns what a check needs: the layers, the hidden states in order and the outputs."""
    torch.manual_seed(seed)
    d_model, hq, hkv, d, rank, first, second = 512, 8, 2, 128, 32, [70, 5, 200, 33], [30, 61, 1, 90]
    pages = Pages(len(first), 64, 8)
    dense, latent = DenseLayer(pages, d_model, hq, hkv, d), LatentLayer(pages, d_model, hq, hkv, d, rank)
    x1, x2 = randn(sum(first), d_model), randn(sum(second), d_model)
    prompt_out, more_out = dense.prompt(x1, first), dense.more(x2, second)
    latent.fill(x1, first)
    latent.fill(x2, second)
    assert torch.equal(dense.lens, latent.lens)

    # one step of both layers as a graph: the dense layer's lengths advance with a torch addition, the latent layer's with its append
    x, dense_out = torch.zeros(pages.batch, d_model, dtype=BF16, device="cuda"), torch.empty(pages.batch, hq, d, dtype=BF16, device="cuda")
    latent_out = torch.empty(pages.batch, hq, d, dtype=torch.float32, device="cuda")
    x @ dense.w_qkv, x @ latent.w_q                                     # the library products' own set-up stays out of the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        stream = torch.cuda.current_stream()
        dense.step(x, dense_out, stream)
        latent.step(x, latent_out, stream)
    tokens, dense_outs, latent_outs = [], [], []
    for _ in range(steps):
        tokens.append(randn(pages.batch, d_model))
        x.copy_(tokens[-1])
        graph.replay()
        dense_outs.append(dense_out.clone())
        latent_outs.append(latent_out.clone())
    for layer in (dense, latent):
        status = W.wsvd_check(layer.ctx)
        assert status == W.OK, W.status_str(status)
    assert torch.equal(dense.lens, latent.lens)
    return dict(dense=dense, latent=latent, first=first, second=second, x1=x1, x2=x2, tokens=tokens, prompt=prompt_out, more=more_out,
                dense_outs=dense_outs, latent_outs=latent_outs)


def close(result):
    torch.cuda.synchronize()
    for layer in (result["dense"], result["latent"]):
        W.wsvd_destroy(layer.ctx)


if __name__ == "__main__":
    r = run()
    print("rows per sequence:", r["dense"].lens.tolist())
    print("bytes of a cached token: dense %d, latent %d" % (2 * r["dense"].hkv * r["dense"].d * 2, 2 * r["latent"].hkv * (32 + 2)))
    print("prompt", tuple(r["prompt"].shape), "continuation", tuple(r["more"].shape), "step", tuple(r["dense_outs"][-1].shape),
          "all finite:", all(bool(torch.isfinite(t).all()) for t in (r["prompt"], r["more"], *r["dense_outs"], *r["latent_outs"])))
    close(r)
