"""Measured calls of the 8-bit cache of the dense layers: pages of E4M3 codes with a scale for each block of 16 rows and kv head, and
the page tables kept on the GPU.

Four operators, in the order in which a serving step calls them:

* ``pages``   pages of finished sequences back to the free list, pages for the new tokens, their positions and slots;
* ``append``  rotary embedding of the new tokens' queries and keys, keys and values quantised into the pages of their sequences;
* ``decode``  attention of one new token per sequence over its pages;
* ``chunk``   causal attention of packed tokens that continue sequences (a prompt's next piece, draft tokens) over the pages.

``own`` chooses between the plain form (elementary torch operations in 32 bits) and the library's entry points.

A page holds page_rows rows of every kv head, in blocks of 16 rows.  Keys of a block lie as [d / 16][16 rows][16 dims], values as
[d / 64][4 groups of rows][64 dims][4 rows], a byte each.  A block has one scale for its keys and one for its values, a byte b that
stands for 2^(b - 127).
"""
from __future__ import annotations

import math
import random

import torch

own = False

F32, F64, I32, U8 = torch.float32, torch.float64, torch.int32, torch.uint8
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
ROPE_BASE = 10000.0
WIDE_SHARE, WIDE_GAIN = 0.02, 4.0            # key channels that are wider than the others
MOST, LEAST_EXPONENT, BIAS = 448.0, -100, 127
TOP_EXPONENT = {"bf16": 120, "f16": 8}       # where 256 times the scale passes the type: codes up to 240


# ------------------------------------------------------------------------------------------------ the cases
def _case(kind, batch, q_heads, kv_heads, d_head, rows, tokens, dtype="bf16", page_rows=64, **more):
    """rows: cached rows before the call, tokens: new ones (of the longest sequence each, where ragged)."""
    c = dict(kind=kind, batch=batch, q_heads=q_heads, kv_heads=kv_heads, d_head=d_head, rows=rows, tokens=tokens, dtype=dtype,
             page_rows=page_rows, ragged=False, shifted=False)
    c.update(more)
    return c


def _pages(batch, rows, tokens, page_rows, prompts, done):
    """prompts, done: percent of the slots whose sequence begins with a prompt, and has ended; the others go on by one token."""
    return dict(kind="pages", batch=batch, rows=rows, tokens=tokens, page_rows=page_rows, prompts=prompts, done=done)


def listed():
    return [
        # the smallest call: a few sequences go on by a token each, a latency floor
        dict(_pages(8, 1000, 1, 64, 0, 0), name="pages_8seq"),
        # a busy step of continuous batching: requests end, others begin with prompts, most go on
        dict(_pages(1024, 8192, 2048, 16, 12, 10), name="pages_1024seq_prompts"),
        # one token of one sequence of a small model
        dict(_case("append", 1, 8, 8, 64, 256, 1, "f16"), name="append_1seq"),
        # a decode step of continuous batching: one token of each of 32 sequences of any length, grouped heads
        dict(_case("append", 32, 28, 4, 128, 8191, 1, ragged=True), name="append_gqa_32seq"),
        # prompts of a batch: every token's queries and keys rotated, image tokens dropped before (positions are not row numbers)
        dict(_case("append", 16, 32, 32, 128, 0, 2048, ragged=True, shifted=True, page_rows=128), name="append_prompts_16x2048"),
        # interactive use: one sequence of a 7B-class vision-language model, image prefix plus text
        dict(_case("decode", 1, 32, 32, 128, 640, 1), name="decode_1seq_640"),
        # one long document, few heads: only a split over its length fills the chip
        dict(_case("decode", 1, 16, 2, 64, 65001, 1, "f16", page_rows=16), name="decode_1seq_65001_d64"),
        # continuous batching, sequences of any length in small shuffled pages
        dict(_case("decode", 23, 32, 8, 128, 3001, 1, ragged=True, page_rows=16), name="decode_ragged_23x3001"),
        # grouped-query attention over long contexts, the serving batch
        dict(_case("decode", 32, 28, 4, 128, 8192, 1, page_rows=128), name="decode_gqa_32x8192"),
        # a few draft tokens of several sequences to be looked at together
        dict(_case("chunk", 4, 8, 8, 64, 700, 5, "f16"), name="chunk_4x5_after_700_d64"),
        # the next piece of a few prompts behind what their pages hold
        dict(_case("chunk", 3, 32, 8, 128, 1501, 333, page_rows=16), name="chunk_3x333_after_1501"),
        # the last piece of a long prompt
        dict(_case("chunk", 1, 28, 4, 128, 6144, 2048, "f16", page_rows=128), name="chunk_2048_after_6144"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the same ranges: head layouts, types, page sizes, batches and lengths spread over their logarithm, no
    more rows, tokens or (query, key) pairs than the largest listed case of the kind has."""
    kind = rng.choice(["pages", "append", "append", "decode", "decode", "chunk", "chunk"])
    page_rows = rng.choice([16, 32, 64, 112, 128, 256])
    if kind == "pages":
        batch, prompts = _log(rng, 1, 1024), rng.choice([0, 5, 30])
        tokens = _log(rng, 2, max(3, min(8192, 100 * 122 * 2048 // batch // max(prompts, 1)))) if prompts else 1
        return _pages(batch, _log(rng, 1, 8192), tokens, page_rows, prompts, rng.choice([0, 10, 50]))
    hq, hkv, d = rng.choice([(8, 8, 64), (16, 2, 64), (32, 32, 128), (28, 4, 128), (32, 8, 128), (16, 1, 128), (12, 4, 64)])
    c = _case(kind, _log(rng, 1, 64), hq, hkv, d, 0, 1, rng.choice(["bf16", "bf16", "f16"]), page_rows, ragged=rng.random() < 0.6)
    width = hkv * d
    if kind == "append":
        c["shifted"] = rng.random() < 0.3
        c["tokens"] = 1 if rng.random() < 0.4 else _log(rng, 2, max(2, 16 * 2048 * 32 * 128 // ((hq + 2 * hkv) // 3 * d) // c["batch"] // 2))
        c["rows"] = rng.choice([0, _log(rng, 1, 2048)])
        c["tokens"] = min(c["tokens"], 4096)
    elif kind == "decode":
        c["rows"] = _log(rng, 1, max(2, min(65001, 32 * 8192 * 4 * 128 // width // c["batch"])))
    else:
        c["batch"] = _log(rng, 1, 16)
        pairs = 28 * 2048 * 7168 // (hq * c["batch"])
        c["tokens"] = _log(rng, 2, min(4096, max(2, math.isqrt(pairs))))
        c["rows"] = rng.choice([0, _log(rng, 1, max(2, min(8192, pairs // c["tokens"] - c["tokens"])))])
    return c


def _lengths(c):
    """(cached rows before, new tokens) of every sequence: part of the case, the same for every seed."""
    rng = random.Random(repr(sorted((k, v) for k, v in c.items() if k != "name")))
    if c["kind"] == "pages":
        before, new, done = [], [], []
        for b in range(c["batch"]):
            x = rng.randrange(100)
            begins, ends = x < c["prompts"], c["prompts"] <= x < c["prompts"] + c["done"]
            before.append(0 if begins else rng.randint(max(1, c["rows"] // 8), c["rows"]))
            new.append(rng.randint(max(1, c["tokens"] // 8), c["tokens"]) if begins else 0 if ends else 1)
            done.append(int(ends))
        return before, new, done
    some = lambda n: n if not c["ragged"] or n < 2 else rng.randint(max(1, n // 8), n)
    before = [c["rows"]] + [some(c["rows"]) for _ in range(c["batch"] - 1)]
    new = [c["tokens"]] + [some(c["tokens"]) for _ in range(c["batch"] - 1)]
    if c["kind"] == "decode":
        new = [0] * c["batch"]             # the row of the new token is counted in rows
    return before, new


def work(case):
    c = case
    if c["kind"] == "pages":
        before, new, done = _lengths(c)
        n, R = sum(new), c["page_rows"]
        moved = sum(-(-b // R) if e else -(-(b + m) // R) - -(-b // R) for b, m, e in zip(before, new, done))
        return {"bytes": 20 * c["batch"] + 8 * n + 8 * moved, "flops": 0}
    before, new = _lengths(c)
    n, heads = sum(new), c["kv_heads"]
    width_q, width_kv = c["q_heads"] * c["d_head"], heads * c["d_head"]
    if c["kind"] == "append":
        # queries, keys and values in; rotated queries, codes and scales, and for prompts the rotated keys out
        blocks = sum((b + m - 1) // 16 - b // 16 + 1 for b, m in zip(before, new) if m)
        return {"bytes": 2 * n * (2 * width_q + 3 * width_kv + (width_kv if c["tokens"] > 1 else 0)) + 2 * blocks * heads, "flops": 3 * n * (width_q + width_kv)}
    rows = sum(before) + (n if c["kind"] == "chunk" else 0)
    held = 2 * rows * width_kv + rows * heads // 8
    if c["kind"] == "decode":
        return {"bytes": held + 4 * c["batch"] * width_q, "flops": 4 * rows * width_q}
    pairs = sum(m * (m + 1) // 2 + m * b for b, m in zip(before, new))
    return {"bytes": held + 4 * n * width_q, "flops": 4 * pairs * width_q}


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + 37)
    return g


def _randn(g, dtype, *shape, wide=0):
    """Unit Gaussians; `wide` = d_head: a few channels of every head WIDE_GAIN times wider, as keys have them."""
    x = torch.randn(shape, device="cuda", generator=g, dtype=dtype if math.prod(shape) > 1 << 24 else F32)
    if wide:
        x = x * torch.where(torch.rand(wide, device="cuda", generator=g) < WIDE_SHARE, WIDE_GAIN, 1.0).to(x.dtype)
    return x.to(dtype)


def _ints(v):
    return torch.tensor(v, dtype=I32, device="cuda")


def _prefix(n):
    total, out = 0, [0]
    for x in n:
        total += x
        out.append(total)
    return out


def _pool(g, dtype, n_pages, heads, R, d, keys):
    """Codes and scales of pages full of rows: keys with wide channels, values of a size of their head's own."""
    codes = torch.empty(n_pages, heads, R * d, dtype=U8, device="cuda")
    scales = torch.empty(n_pages, heads, R // 16, dtype=U8, device="cuda")
    size = torch.ones(heads, device="cuda") if keys else torch.exp2(torch.rand(heads, device="cuda", generator=g) * 6 - 4)
    step = max(1, (1 << 25) // (heads * R * d))
    for p in range(0, n_pages, step):
        n = min(step, n_pages - p)
        x = (_randn(g, dtype, n, heads, R, d, wide=d if keys else 0) * size.to(dtype)[:, None, None]).float().view(n, heads, R // 16, 16, d)
        e = _exponent(x.abs().amax((-1, -2)))
        y = _code(x, e[..., None, None], None)
        y = y.view(n, heads, R // 16, 16, d // 16, 16).transpose(3, 4) if keys else y.view(n, heads, R // 16, 4, 4, d // 64, 64).permute(0, 1, 2, 5, 3, 6, 4)
        codes[p:p + n] = y.reshape(n, heads, -1)
        scales[p:p + n] = (e + BIAS).to(U8)
    return codes, scales


def _paged(s, g, lens):
    """A table over shuffled pages, with some pages of nobody."""
    R = s["case"]["page_rows"]
    max_pages = max(1, -(-max(lens) // R))
    used = [-(-x // R) for x in lens]
    n_pages = sum(used) + max(1, sum(used) // 16)
    free = torch.randperm(n_pages, device="cuda", generator=g, dtype=I32)
    at, start = torch.arange(max_pages, device="cuda"), _ints(_prefix(used)[:-1])
    table = torch.where(at < _ints(used)[:, None], free[(start[:, None] + at).clamp(max=n_pages - 1)], 0)
    s.update(lens=_ints(lens), max_pages=max_pages, n_pages=n_pages, table=table.contiguous(), max_len=max(lens))


def prepare(case, seed):
    c, g = dict(case), _gen(seed)
    B, R = c["batch"], c["page_rows"]
    if c["kind"] == "pages":
        before, new, done = _lengths(c)
        s = dict(case=c, n=sum(new))
        used = [-(-x // R) for x in before]
        most = max(-(-(b + m) // R) for b, m in zip(before, new))
        n_pages = sum(used) + sum(-(-m // R) + 1 for m in new) + 7
        order = torch.randperm(n_pages, device="cuda", generator=g, dtype=I32)
        at, start = torch.arange(most, device="cuda"), _ints(_prefix(used)[:-1])
        free = torch.zeros(n_pages, dtype=I32, device="cuda")
        free[: n_pages - sum(used)] = order[sum(used):]
        s.update(lens=_ints(before), new=_ints(new), done=_ints(done), max_pages=most, n_pages=n_pages, free=free, n_free=_ints([n_pages - sum(used)]),
                 table=torch.where(at < _ints(used)[:, None], order[(start[:, None] + at).clamp(max=n_pages - 1)], 0).contiguous(),
                 lens_kept=_ints([0] * B), n_free_kept=_ints([0]), lens_out=_ints([0] * B), n_free_out=_ints([0]), cu=_ints([0] * (B + 1)),
                 positions=_ints([0] * s["n"]), slots=_ints([0] * s["n"]))
        if own:
            _handle(s)
        return s
    dt, Hq, Hkv, d = DTYPES[c["dtype"]], c["q_heads"], c["kv_heads"], c["d_head"]
    before, new = _lengths(c)
    n = sum(new)
    s = dict(case=c, before=before, new=new, n=n, scale=1.0 / math.sqrt(d), cu=_ints(_prefix(new)), longest=max(new))
    _paged(s, g, [x + y for x, y in zip(before, new)])
    s["k_pool"], s["k_scale"] = _pool(g, dt, s["n_pages"], Hkv, R, d, True)
    s["v_pool"], s["v_scale"] = _pool(g, dt, s["n_pages"], Hkv, R, d, False)
    if c["kind"] == "append":
        # one projection's output: queries, keys and values of a token side by side
        s["qkv"] = _randn(g, dt, n, (Hq + 2 * Hkv) * d)
        s["inv_freq"] = ROPE_BASE ** (-torch.arange(0, d, 2, device="cuda", dtype=F64) / d)
        s["q_out"] = torch.empty(n, Hq * d, dtype=dt, device="cuda")
        s["k_out"] = torch.empty(n, Hkv * d, dtype=dt, device="cuda") if c["tokens"] > 1 else None
        s["positions"] = None
        if c["shifted"]:
            dropped = torch.repeat_interleave(_ints([577 + 31 * b for b in range(B)]), _ints(new).long())
            s["positions"] = dropped + _ints([b + i for b, m in zip(before, new) for i in range(m)])
    else:
        s["q"] = 1.5 * _randn(g, dt, B if c["kind"] == "decode" else n, Hq * d)
        s["out"] = torch.empty_like(s["q"])
    if own:
        _handle(s)
    return s


# ------------------------------------------------------------------------------------------------ the library's calls
_kept = {}


def _handle(s):
    """What a serving program sets up once: page pool or descriptor and cache view, context with its workspace."""
    import paper_2604_02570_amd as W
    c = s["case"]
    s["W"], s["stream"] = W, torch.cuda.current_stream().cuda_stream
    if "ctx" not in _kept:
        _kept["ctx"] = W.wsvd_create(0)
    s["ctx"] = _kept["ctx"]
    if c["kind"] == "pages":
        s["pool"] = W.make_page_pool(s["table"], s["free"], c["batch"], c["page_rows"], s["max_pages"], s["n_pages"])
        return
    s["desc"] = W.dense_desc(c["batch"], c["q_heads"], c["kv_heads"], c["d_head"], c["dtype"], s["scale"])
    s["cache"] = W.make_paged_cache(s["k_pool"], s["v_pool"], s["k_scale"], s["v_scale"], s["lens"], s["table"], c["page_rows"], s["max_pages"],
                                    s["n_pages"])
    need = W.wsvd_dense_workspace_bytes(s["desc"])
    if "ws" not in _kept or _kept["ws"].numel() < need:
        _kept["ws"] = torch.empty(need, dtype=U8, device="cuda")
        W.wsvd_set_workspace(_kept["ctx"], _kept["ws"])


def _held(s):
    """The cache as the numbers that its bytes stand for."""
    return [s["k_pool"].view(E4M3), s["v_pool"].view(E4M3), s["k_scale"].view(E8M0), s["v_scale"].view(E8M0)]


def _run_own(s):
    c, W = s["case"], s["W"]
    if c["kind"] == "pages":
        W.wsvd_pages_release(s["ctx"], s["pool"], s["done"], s["lens"], s["n_free"], s["lens_kept"], s["n_free_kept"], s["stream"])
        W.wsvd_pages_grow(s["ctx"], s["pool"], s["new"], s["n"], s["lens_kept"], s["n_free_kept"], s["lens_out"], s["n_free_out"], s["cu"],
                          s["positions"], s["slots"], s["stream"])
        return [s["lens_out"], s["n_free_out"], s["cu"], s["positions"], s["slots"], s["table"], s["free"]]
    wq, wkv = c["q_heads"] * c["d_head"], c["kv_heads"] * c["d_head"]
    if c["kind"] == "append":
        x, ld = s["qkv"], wq + 2 * wkv
        W.wsvd_dense_append_paged_f8(s["ctx"], s["desc"], x, ld, x[:, wq:], ld, x[:, wq + wkv:], ld, s["n"], s["cu"], s["positions"],
                                     s["inv_freq"], s["q_out"], wq, s["k_out"], wkv, s["cache"], s["stream"])
        return [t for t in (s["q_out"], s["k_out"]) if t is not None] + _held(s)
    if c["kind"] == "decode":
        W.wsvd_dense_decode_attn_paged_f8(s["ctx"], s["desc"], s["q"], wq, s["cache"], s["max_len"], s["out"], s["stream"])
    else:
        W.wsvd_dense_prefill_attn_paged_f8(s["ctx"], s["desc"], s["q"], wq, s["n"], s["cu"], s["cache"], s["out"], wq, s["stream"])
    return s["out"]


# ------------------------------------------------------------------------------------------------ the plain forms
def _pages_plain(s):
    c = s["case"]
    R, at = c["page_rows"], torch.arange(s["max_pages"], device="cuda", dtype=I32)
    # pages of sequences that have ended go behind the free list's last
    gone = (at < ((s["lens"] + R - 1) // R)[:, None]) & (s["done"] != 0)[:, None]
    place = torch.where(gone, s["n_free"] + (torch.cumsum(gone.flatten(), 0) - 1).view_as(gone), s["n_pages"])
    free = torch.cat([s["free"], s["free"][:1]]).scatter_(0, place.flatten(), s["table"].flatten())[:-1]
    s["free"].copy_(free)
    lens, n_free = torch.where(s["done"] != 0, 0, s["lens"]), s["n_free"] + gone.sum(dtype=I32)
    # and come off its end for the new tokens
    after = lens + s["new"]
    have = (lens + R - 1) // R
    need = ((after + R - 1) // R).clamp(max=s["max_pages"]) - have
    j = at - have[:, None]
    which = n_free - 1 - (torch.cumsum(need, 0) - need)[:, None] - j
    page = torch.where(which >= 0, free[which.clamp(0, s["n_pages"] - 1).long()], -1)
    s["table"].copy_(torch.where((j >= 0) & (j < need[:, None]), page, s["table"]))
    s["lens_out"].copy_(after)
    s["n_free_out"].copy_((n_free - need.sum()).clamp(min=0))
    s["cu"][1:] = torch.cumsum(s["new"], 0)
    t = torch.arange(s["n"], device="cuda", dtype=I32)
    b = torch.searchsorted(s["cu"][1:].contiguous(), t, right=True)
    row = lens[b] + t - s["cu"][b]
    s["positions"].copy_(row)
    page = s["table"][b, (row // R).long()]
    s["slots"].copy_(torch.where(page >= 0, page * R + row % R, -1))
    return [s["lens_out"], s["n_free_out"], s["cu"], s["positions"], s["slots"], s["table"], s["free"]]


def _exponent(a):
    """The least e from LEAST_EXPONENT on with a <= 448 * 2^e: 448 is 0.875 * 2^9."""
    m, e = torch.frexp(a)
    return (e - 9 + (m > 0.875)).clamp(min=LEAST_EXPONENT)


def _code(x, e, dtype):
    """x / 2^e as E4M3, to nearest even; not finite: NaN; no code whose value passes the type."""
    y = x * torch.exp2(-e.float())
    if dtype is not None:
        top = torch.where(e >= TOP_EXPONENT[dtype], 240.0, MOST)
        y = torch.minimum(torch.maximum(y, -top), top)
    return torch.where(torch.isfinite(x), y, math.nan).to(E4M3).view(U8)


def _key_rows(pool, R, d):
    """Codes of keys by row: a view [pages, heads, blocks, 16, d / 16, 16] of them as they lie."""
    return pool.view(*pool.shape[:2], R // 16, d // 16, 16, 16).transpose(3, 4)


def _value_rows(pool, R, d):
    """Codes of values by row: a view [pages, heads, blocks, 4, 4, d / 64, 64]."""
    return pool.view(*pool.shape[:2], R // 16, d // 64, 4, 64, 4).permute(0, 1, 2, 4, 6, 3, 5)


def _rotate(x, cos, sin):
    """Dims (i, i + d/2) of [n, heads, d] turned by their angle, in 32 bits."""
    a, b = x.float().chunk(2, -1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _tokens(s):
    """Sequence and row of every new token."""
    t, cu = torch.arange(s["n"], device="cuda"), s["cu"].long()
    b = torch.searchsorted(cu[1:].contiguous(), t, right=True)
    return b, t - cu[b]


def _append_plain(s):
    c = s["case"]
    Hq, Hkv, d, R = c["q_heads"], c["kv_heads"], c["d_head"], c["page_rows"]
    b, i = _tokens(s)
    row = s["lens"].long()[b] - (s["cu"][1:] - s["cu"][:-1]).long()[b] + i
    pos = row if s["positions"] is None else s["positions"]
    angle = pos.double()[:, None] * s["inv_freq"]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    x = s["qkv"].view(s["n"], Hq + 2 * Hkv, d)
    s["q_out"].copy_(_rotate(x[:, :Hq], cos, sin).view(s["n"], -1))
    k = _rotate(x[:, Hq:Hq + Hkv], cos, sin).to(x.dtype)
    if s["k_out"] is not None:
        s["k_out"].copy_(k.view(s["n"], -1))
    page, block, at = s["table"].long()[b, row // R], row % R // 16, row % 16
    # the blocks that get rows, in the tokens' order; a token that begins one stands for it
    begins = (i == 0) | (at == 0)
    unit = torch.cumsum(begins, 0) - 1
    most_units = min(s["n"], s["n"] // 16 + 2 * c["batch"])
    some = torch.arange(most_units, device="cuda") <= unit[-1]
    first = torch.zeros(most_units, dtype=torch.int64, device="cuda")
    first.scatter_reduce_(0, unit, torch.arange(s["n"], device="cuda"), "amin", include_self=False)
    first = torch.where(some, first, first[0])                                                       # (of no block: the first one again)
    upage, ublock, uat = page[first], block[first], at[first]
    for rows, pool, scale, view, shape in ((k, s["k_pool"], s["k_scale"], _key_rows, (16, d // 16, 16)),
                                           (x[:, Hq + Hkv:], s["v_pool"], s["v_scale"], _value_rows, (4, 4, d // 64, 64))):
        y = rows.float()
        most = torch.where(torch.isfinite(y), y.abs(), 0.0).amax(-1)
        e = _exponent(torch.zeros(most_units, Hkv, device="cuda").index_reduce_(0, unit, most, "amax"))
        e = torch.where(some[:, None], e, e[0])
        was = scale[upage, :, ublock].int() - BIAS
        e = torch.where((uat > 0)[:, None], torch.maximum(e, was), e)
        # rows that the block held before move to its new scale, the new ones join them
        codes = view(pool, R, d)
        held = codes[upage, :, ublock].reshape(-1, Hkv, 16, d)
        moved = _code(held.view(E4M3).float(), (e - was)[..., None, None], None)
        before = torch.arange(16, device="cuda") < uat[:, None]
        codes[upage, :, ublock] = torch.where(before[:, None, :, None], moved, held).view(-1, Hkv, *shape)
        scale[upage, :, ublock] = (e + BIAS).to(U8)
        new = _code(y, e[unit][..., None], c["dtype"])
        if view is _key_rows:
            codes[page, :, block, at] = new.view(-1, Hkv, d // 16, 16)
        else:
            codes[page, :, block, at // 4, at % 4] = new.view(-1, Hkv, d // 64, 64)
    return [t for t in (s["q_out"], s["k_out"]) if t is not None] + _held(s)


def _gathered(s, name):
    """A pool's rows by sequence, [B, Hkv, rows, d] in 32 bits."""
    c = s["case"]
    codes = (_key_rows if name == "k" else _value_rows)(s[name + "_pool"], c["page_rows"], c["d_head"])[s["table"].long()]
    x = codes.reshape(*codes.shape[:4], -1).view(E4M3).float() * torch.exp2(s[name + "_scale"][s["table"].long()].float() - BIAS)[..., None]
    x = x.transpose(1, 2)
    return x.reshape(x.shape[0], x.shape[1], -1, c["d_head"])


def _attend(q, k, v, seen, scale):
    """softmax(scale q k^T) v over the keys that are seen; q [B, Hkv, n, d], k and v [B, Hkv, t, d], seen broadcast to [B, Hkv, n, t].
    A query that sees nothing gets zeros."""
    w = torch.matmul(q * scale, k.transpose(-1, -2).contiguous())
    w = torch.where(seen, w, -math.inf)
    most = w.amax(-1, keepdim=True)
    w = torch.exp(w - torch.where(most == -math.inf, 0.0, most))
    total = w.sum(-1, keepdim=True)
    return torch.matmul(w, v) / torch.where(total == 0, 1.0, total)


def _decode_plain(s):
    c = s["case"]
    q = s["q"].float().view(c["batch"], c["kv_heads"], -1, c["d_head"])
    k, v = _gathered(s, "k"), _gathered(s, "v")
    seen = (torch.arange(k.shape[2], device="cuda") < s["lens"][:, None])[:, None, None]
    return _attend(q, k, v, seen, s["scale"]).to(s["q"].dtype).view(c["batch"], -1)


def _chunk_plain(s):
    c = s["case"]
    B, Hq, Hkv, d, n = c["batch"], c["q_heads"], c["kv_heads"], c["d_head"], s["longest"]
    at = (s["cu"][:-1].long()[:, None] + torch.arange(n, device="cuda")).clamp(max=s["n"] - 1)       # packed -> [B, longest]
    q = s["q"].view(s["n"], Hkv, Hq // Hkv, d)[at].float().permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, d)
    new, lens = (s["cu"][1:] - s["cu"][:-1]).long(), s["lens"].long()
    k, v = _gathered(s, "k"), _gathered(s, "v")
    last = (lens - new)[:, None] + torch.arange(n, device="cuda")
    key = torch.arange(k.shape[2], device="cuda")
    seen = (key <= last[..., None]) & (key < lens[:, None, None])                                     # [B, n, t]
    o = _attend(q, k, v, seen[:, None, None].expand(B, 1, Hq // Hkv, n, -1).reshape(B, 1, -1, k.shape[2]), s["scale"]).to(s["q"].dtype)
    b, i = _tokens(s)
    return o.view(B, Hkv, Hq // Hkv, n, d)[b, :, :, i].reshape(s["n"], -1)


def run(state):
    if own:
        return _run_own(state)
    return {"pages": _pages_plain, "append": _append_plain, "decode": _decode_plain, "chunk": _chunk_plain}[state["case"]["kind"]](state)


# ------------------------------------------------------------------------------------------------ from the definition, in 64 bits
def _table64():
    """The 256 numbers of E4M3 from their bits: sign, four of exponent with a bias of 7, three of mantissa."""
    out = []
    for b in range(256):
        x, m = (b >> 3) & 15, b & 7
        v = math.nan if b & 127 == 127 else (1 + m / 8) * 2.0 ** (x - 7) if x else m / 8 * 2.0 ** -6
        out.append(-v if b >> 7 else v)
    return torch.tensor(out, dtype=F64, device="cuda")


def _places(c, keys):
    """Where row r, dim x of a block lies in its bytes, [16, d]."""
    r, x = torch.arange(16, device="cuda")[:, None], torch.arange(c["d_head"], device="cuda")
    return x // 16 * 256 + r * 16 + x % 16 if keys else x // 64 * 1024 + r // 4 * 256 + x % 64 * 4 + r % 4


def _exact_pages(s):
    R = s["case"]["page_rows"]
    table, free, lens = s["table"].tolist(), s["free"].tolist(), s["lens"].tolist()
    new, done, top = s["new"].tolist(), s["done"].tolist(), int(s["n_free"])
    for b, e in enumerate(done):
        if e:
            for i in range(-(-lens[b] // R)):
                free[top] = table[b][i]
                top += 1
            lens[b] = 0
    cu, positions, slots = [0], [], []
    for b, n in enumerate(new):
        for r in range(lens[b], lens[b] + n):
            if r % R == 0:
                top -= 1
                table[b][r // R] = free[top]
            positions.append(r)
            slots.append(table[b][r // R] * R + r % R)
        lens[b] += n
        cu.append(cu[-1] + n)
    return [_ints(lens), _ints([top]), _ints(cu), _ints(positions), _ints(slots), _ints(table), _ints(free)]


def exact(case, seed):
    """The same outputs in 64 bits, sequence by sequence and head by head; codes before their rounding to 8 bits."""
    s = prepare(case, seed)
    c = s["case"]
    if c["kind"] == "pages":
        return _exact_pages(s)
    B, Hq, Hkv, d, R = c["batch"], c["q_heads"], c["kv_heads"], c["d_head"], c["page_rows"]
    G, cu, number = Hq // Hkv, _prefix(s["new"]), _table64()
    key_at, value_at = _places(c, True), _places(c, False)
    if c["kind"] == "append":
        x = s["qkv"].double().view(-1, Hq + 2 * Hkv, d)
        q_out, k_out = torch.empty(s["n"], Hq, d, dtype=F64, device="cuda"), torch.empty(s["n"], Hkv, d, dtype=F64, device="cuda")
        held = {n: number[s[n + "_pool"].long()].view(s["n_pages"], Hkv, R // 16, 16 * d) for n in "kv"}
        scales = {n: torch.ldexp(torch.ones((), dtype=F64, device="cuda"), s[n + "_scale"].int() - BIAS) for n in "kv"}
        for b in range(B):
            n, t, r0 = s["new"][b], slice(cu[b], cu[b + 1]), s["before"][b]
            p = torch.arange(r0, r0 + n, device="cuda").double() if s["positions"] is None else s["positions"][t].double()
            turn = torch.polar(torch.ones((), dtype=F64, device="cuda"), p[:, None] * s["inv_freq"][None, :])[:, None, :]
            for src, dst in ((x[t, :Hq], q_out), (x[t, Hq:Hq + Hkv], k_out)):
                z = torch.complex(src[..., : d // 2], src[..., d // 2:]) * turn
                dst[t] = torch.cat([z.real, z.imag], -1)
            pages, b0 = s["table"][b].long(), r0 // 16
            blocks = torch.arange(b0, (r0 + n - 1) // 16 + 1, device="cuda")
            where, inside = pages[blocks * 16 // R], blocks * 16 % R // 16
            for name, rows, at in (("k", k_out[t], key_at), ("v", x[t, Hq + Hkv:], value_at)):
                y = torch.zeros(len(blocks) * 16, Hkv, d, dtype=F64, device="cuda")
                y[r0 - 16 * b0: r0 - 16 * b0 + n] = rows
                y = y.view(-1, 16, Hkv, d).transpose(1, 2)
                most = y.to(s["qkv"].dtype).double().abs().amax((2, 3))
                step = torch.exp2(torch.ceil(torch.log2(most / MOST)).clamp(min=LEAST_EXPONENT))
                was = scales[name][where, :, inside]
                if r0 % 16:
                    step[0] = torch.maximum(step[0], was[0])
                old = held[name][where, :, inside][..., at.flatten()].view(-1, Hkv, 16, d)
                row = blocks[:, None] * 16 + torch.arange(16, device="cuda")
                fresh, kept = ((row >= r0) & (row < r0 + n))[:, None, :, None], (row < r0)[:, None, :, None]
                z = torch.where(fresh, y / step[..., None, None], torch.where(kept, old * (was / step)[..., None, None], old))
                back = torch.empty(len(blocks), Hkv, 16 * d, dtype=F64, device="cuda")
                back[..., at.flatten()] = z.reshape(len(blocks), Hkv, 16 * d)
                held[name][where, :, inside] = back
                scales[name][where, :, inside] = step
        out = [q_out.view(s["n"], -1)] + ([k_out.view(s["n"], -1)] if s["k_out"] is not None else [])
        return out + [held["k"].view_as(s["k_pool"]), held["v"].view_as(s["v_pool"]), scales["k"], scales["v"]]
    out = torch.zeros(B if c["kind"] == "decode" else s["n"], Hq, d, dtype=F64, device="cuda")
    for b in range(B):
        t = slice(b, b + 1) if c["kind"] == "decode" else slice(cu[b], cu[b + 1])
        n, total, pages = t.stop - t.start, s["before"][b] + s["new"][b], s["table"][b].long()
        at = torch.arange(total, device="cuda")
        hidden = at[None, :] > at[total - n:, None] if c["kind"] == "chunk" else None
        for h in range(Hkv):
            k, v = ((number[s[x + "_pool"].view(s["n_pages"], Hkv, R // 16, -1)[pages, h][..., place.flatten()].long()].view(-1, R // 16, 16, d) *
                     torch.exp2(s[x + "_scale"][pages, h].double() - BIAS)[..., None, None]).reshape(-1, d)[:total] for x, place in (("k", key_at), ("v", value_at)))
            for i in range(G):
                w = s["q"].view(-1, Hq, d)[t, h * G + i].double() @ k.t().contiguous() * s["scale"]
                out[t, h * G + i] = torch.softmax(w if hidden is None else w.masked_fill(hidden, -math.inf), -1) @ v
    return out.view(out.shape[0], -1)
