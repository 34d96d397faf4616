"""The 8-bit pages of dense layers for the tests, from their definition: E4M3 in 64 bits, blocks of 16 rows with a power of two for a
scale, where a block's bytes lie, and page tables from a free list.  On the CPU, with loops, and no code of the library."""
from __future__ import annotations

import math

import torch

from dense_ref import DTYPES, F64

MOST, LEAST, BIAS = 448.0, -100, 127
TOP = {"bf16": 120, "f16": 8}                    # the exponent at which 256 scales pass the type


def number(code):
    """What a byte stands for."""
    x, m = (code >> 3) & 15, code & 7
    v = math.nan if code & 127 == 127 else (1 + m / 8) * 2.0 ** (x - 7) if x else m * 2.0 ** -9
    return -v if code >> 7 else v


NUMBERS = torch.tensor([number(c) for c in range(256)], dtype=F64)
SCALES = torch.tensor([2.0 ** (b - BIAS) for b in range(256)], dtype=F64)


def exponent(x):
    """The least e from LEAST on with max|finite x| <= 448 * 2^e."""
    x = x.to(F64).abs()
    most = x[torch.isfinite(x)].max().item() if torch.isfinite(x).any() else 0.0
    e = LEAST
    if most > MOST * 2.0 ** LEAST:
        e = math.frexp(most / MOST)[1] - 1
        while most > MOST * 2.0 ** e:
            e += 1
    return e


def rounded(y):
    """To the nearest E4M3, ties to even, in 64 bits; 448 above, NaN where there is none."""
    a = y.abs().clamp(max=MOST)
    step = SCALES[torch.frexp(a.nan_to_num(1).clamp(min=2.0 ** -6))[1] - 1 - 3 + BIAS]
    return torch.copysign(torch.round(a / step) * step, y)


def quantised(x, e, dtype):
    """Numbers that the codes of x under 2^e stand for, over the scale."""
    y = x.to(F64) / 2.0 ** e
    y = torch.where(torch.isfinite(x), y, math.nan)
    return rounded(y.clamp(-240, 240) if e >= TOP[dtype] else y)


def place(d, row, dim, keys):
    return dim // 16 * 256 + row * 16 + dim % 16 if keys else dim // 64 * 1024 + row // 4 * 256 + dim % 64 * 4 + row % 4


def places(d, keys):
    return torch.tensor([[place(d, r, x, keys) for x in range(d)] for r in range(16)])


def bytes_of(numbers):
    """Numbers of E4M3 as bytes."""
    table = {}
    for c in range(256):
        v = number(c)
        table[("nan",) if v != v else (v, math.copysign(1, v))] = c
    return torch.tensor([table[("nan",) if v != v else (v, math.copysign(1, v))] for v in numbers.flatten().tolist()], dtype=torch.uint8).view(numbers.shape)


class F8Pool:
    """A page pool with its table, pages dealt out in a random order.  Bytes that no row has written are `fill`, NaN codes unless told."""

    def __init__(self, g, lens, hkv, d, page_rows, dtype, max_pages=None, fill=0x7F, spare=3):
        self.lens, self.R, self.hkv, self.d, self.dtype = list(lens), page_rows, hkv, d, dtype
        used = [-(-n // page_rows) for n in lens]
        self.max_pages = max_pages or max(1, max(used))
        self.n_pages = sum(used) + spare
        order = torch.randperm(self.n_pages, generator=g).tolist()
        self.table = torch.full((len(lens), self.max_pages), -7, dtype=torch.int32)        # never to be looked at
        for b, n in enumerate(used):
            for i in range(n):
                self.table[b, i] = order.pop()
        blocks = (self.n_pages, hkv, page_rows // 16)
        self.codes = {x: torch.full((*blocks, 16 * d), fill, dtype=torch.uint8) for x in "kv"}
        self.scales = {x: torch.full(blocks, 200, dtype=torch.uint8) for x in "kv"}
        self.at = {"k": places(d, True), "v": places(d, False)}

    def where(self, b, row):
        return int(self.table[b, row // self.R]), row % self.R // 16

    def append(self, b, row, k, v):
        """Rows [row, row + n) of sequence b, k and v [n, hkv, d] of the type, by the rule of the append."""
        at, n = 0, k.shape[0]
        while at < n:
            r0 = (row + at) % 16
            m = min(16 - r0, n - at)
            page, block = self.where(b, row + at)
            for x, new in (("k", k[at:at + m]), ("v", v[at:at + m])):
                for h in range(self.hkv):
                    codes, scale = self.codes[x][page, h, block], self.scales[x][page, h]
                    e = exponent(new[:, h])
                    if r0 > 0:
                        old = int(scale[block]) - BIAS
                        if e > old:
                            spots = self.at[x][:r0].flatten()
                            codes[spots] = bytes_of(rounded(NUMBERS[codes[spots].long()] * 2.0 ** (old - e)))
                        e = max(e, old)
                    codes[self.at[x][r0:r0 + m]] = bytes_of(quantised(new[:, h], e, self.dtype))
                    scale[block] = e + BIAS
            at += m

    def random(self, g, spread=3):
        """Every sequence full of rows: finite codes, scales around 2^-7 so that values are about 1 and less."""
        for b, n in enumerate(self.lens):
            for r in range(0, n, 16):
                page, block = self.where(b, r)
                m = min(16, n - r)
                for x in "kv":
                    spots = self.at[x][:m].flatten()
                    for h in range(self.hkv):
                        y = (torch.randn(len(spots), generator=g, dtype=F64) * 100).clamp(-MOST, MOST)
                        self.codes[x][page, h, block][spots] = y.to(torch.float32).to(torch.float8_e4m3fn).view(torch.uint8)
                        self.scales[x][page, h, block] = BIAS - 7 - int(torch.randint(0, spread, (1,), generator=g)) if spread else BIAS - 7
        return self

    def set(self, x, b, row, h, dim, code):
        page, block = self.where(b, row)
        self.codes[x][page, h, block, self.at[x][row % 16, dim]] = code

    def rows(self, b, n=None):
        """[n, hkv, d] keys and values of sequence b, in 64 bits."""
        n = self.lens[b] if n is None else n
        out = []
        for x in "kv":
            y = torch.zeros(n, self.hkv, self.d, dtype=F64)
            for r in range(0, n, 16):
                page, block = self.where(b, r)
                m = min(16, n - r)
                z = NUMBERS[self.codes[x][page, :, block][:, self.at[x][:m].flatten()].long()].view(self.hkv, m, self.d)
                y[r:r + m] = (z * SCALES[self.scales[x][page, :, block].long()][:, None, None]).transpose(0, 1)
            out.append(y)
        return out


class Tables:
    """Page table, lengths and free list on the host, by the rules of the two calls."""

    def __init__(self, batch, page_rows, max_pages, n_pages, order):
        self.R, self.max_pages, self.n_pages = page_rows, max_pages, n_pages
        self.table = [[-9] * max_pages for _ in range(batch)]
        self.lens, self.free, self.n_free = [0] * batch, list(order), len(order)
        self.free += [-5] * (n_pages - len(order))

    def grow(self, new):
        cu, positions, slots, short = [0], [], [], False
        for b, n in enumerate(new):
            for r in range(self.lens[b], self.lens[b] + n):
                pg = r // self.R
                if r % self.R == 0 and pg < self.max_pages:
                    if self.n_free:
                        self.n_free -= 1
                        self.table[b][pg] = self.free[self.n_free]
                    else:
                        self.table[b][pg] = -1
                page = self.table[b][pg] if pg < self.max_pages else -1
                short = short or page < 0
                positions.append(r)
                slots.append(page * self.R + r % self.R if page >= 0 else -1)
            self.lens[b] += n
            cu.append(cu[-1] + n)
        return cu, positions, slots, short

    def release(self, done):
        for b, end in enumerate(done):
            if end:
                for i in range(-(-min(self.lens[b], self.max_pages * self.R) // self.R)):
                    if 0 <= self.table[b][i] < self.n_pages:
                        self.free[self.n_free] = self.table[b][i]
                        self.n_free += 1
                self.lens[b] = 0
