"""Inputs and plain 64-bit forms of the dense-layer operators (rotary append, decode and prompt attention over plain keys and
values) for the tests.  Everything on the CPU, with loops over sequences and heads and no code of the library."""
from __future__ import annotations

import math

import torch

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
F64 = torch.float64
SMALLEST = {"bf16": 0.0, "f16": 2.0 ** -25}           # half a step of the type's subnormal numbers


def half_step(dtype):
    return torch.finfo(DTYPES[dtype]).eps / 2


def randn(g, dtype, *shape, scale=1.0):
    return (torch.randn(shape, generator=g, dtype=torch.float32) * scale).to(DTYPES[dtype])


def prefix(n):
    return torch.tensor([0] + list(torch.tensor(n).cumsum(0)), dtype=torch.int32)


class Pool:
    """A page pool with its table: pages dealt out in a random order, everything that no row owns is NaN."""

    def __init__(self, g, lens, hkv, d, page_rows, dtype, max_pages=None, fill_rows=True):
        self.lens, self.R, self.hkv, self.d = list(lens), page_rows, hkv, d
        used = [-(-n // page_rows) for n in lens]
        self.max_pages = max_pages or max(1, max(used))
        self.n_pages = sum(used) + 3
        order = torch.randperm(self.n_pages, generator=g).tolist()
        self.table = torch.full((len(lens), self.max_pages), -7, dtype=torch.int32)        # never to be looked at
        for b, n in enumerate(used):
            for i in range(n):
                self.table[b, i] = order.pop()
        self.k = torch.full((self.n_pages, hkv, page_rows, d), math.nan, dtype=DTYPES[dtype])
        self.v = self.k.clone()
        if fill_rows:
            for b, n in enumerate(lens):
                self.put(b, 0, randn(g, dtype, n, hkv, d), randn(g, dtype, n, hkv, d))

    def put(self, b, row, k, v):
        for i in range(k.shape[0]):
            page, at = int(self.table[b, (row + i) // self.R]), (row + i) % self.R
            self.k[page, :, at], self.v[page, :, at] = k[i], v[i]

    def rows(self, b, n=None):
        """[n, hkv, d] keys and values of sequence b."""
        n = self.lens[b] if n is None else n
        if n == 0:
            z = self.k.new_zeros(0, self.hkv, self.d)
            return z, z
        pages = self.table[b, : -(-n // self.R)].long()
        take = lambda x: x[pages].transpose(1, 2).reshape(-1, self.hkv, self.d)[:n]
        return take(self.k), take(self.v)


def rotate(x, pos, inv_freq):
    """[n, heads, d] turned by pos * inv_freq as complex numbers."""
    h = x.shape[-1] // 2
    z = torch.complex(x[..., :h].to(F64), x[..., h:].to(F64)) * torch.polar(torch.ones(1, dtype=F64), pos.to(F64)[:, None] * inv_freq)[:, None]
    return torch.cat([z.real, z.imag], -1)


def attend(q, k, v, last, scale):
    """One sequence: q [n, Hq, d], k and v [t, Hkv, d], query i sees the keys up to last[i].  Returns the output and the
    weighted mean of |v| (what a relative error of the weights is multiplied with), [n, Hq, d]."""
    n, hq, d = q.shape
    g = hq // k.shape[1]
    out, size = torch.zeros(n, hq, d, dtype=F64), torch.zeros(n, hq, d, dtype=F64)
    for i in range(n):
        t = int(last[i]) + 1
        if t <= 0:
            continue
        for h in range(hq):
            w = torch.softmax(k[:t, h // g].to(F64) @ q[i, h].to(F64) * scale, 0)
            out[i, h] = w @ v[:t, h // g].to(F64)
            size[i, h] = w @ v[:t, h // g].to(F64).abs()
    return out, size


def attend_fast(q, k, v, last, scale):
    """attend with the queries of a head together."""
    n, hq, d = q.shape
    g = hq // k.shape[1]
    out, size = torch.zeros(n, hq, d, dtype=F64), torch.zeros(n, hq, d, dtype=F64)
    hidden = torch.arange(k.shape[0])[None, :] > torch.as_tensor(last)[:, None]
    some = ~hidden.all(1)
    if not some.any():
        return out, size
    for h in range(hq):
        w = torch.softmax((q[some, h].to(F64) @ k[:, h // g].to(F64).t() * scale).masked_fill(hidden[some], -math.inf), 1)
        out[some, h] = w @ v[:, h // g].to(F64)
        size[some, h] = w @ v[:, h // g].to(F64).abs()
    return out, size


def check(got, want, size, dtype, weights_rounded):
    """Element by element: the output's rounding (half a step of the value), the weights' (half a step each, where they are
    rounded to the type: a mean of |v| carries it), and fp32 scores and sums: 2^-12 of that mean covers products of up to
    2^8 terms at 2^-24 each with scores up to 2^4."""
    h = half_step(dtype)
    err = (got.to(F64) - want).abs()
    tol = h * want.abs() + ((h if weights_rounded else 0.0) * (1 + h) + 2.0 ** -12) * size + SMALLEST[dtype]
    assert torch.isfinite(got).all(), "not finite"
    worst = (err / tol.clamp(min=1e-30)).max().item()
    assert worst <= 1.0, f"{worst:.3f} of the tolerance"
    return worst
