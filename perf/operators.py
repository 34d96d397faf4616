"""Measured calls of the dense-layer operators: attention layers whose keys and values are kept uncompressed in a paged
cache, next to the layers whose cache is the low-rank latent.

Four operators, in the order in which a layer calls them:

* ``append``  rotary embedding of the new tokens' queries and keys, keys and values stored in the pages of their sequences;
* ``decode``  attention of one new token per sequence over its pages;
* ``prompt``  causal attention of whole prompts packed one behind another, lengths given by their prefix sums;
* ``chunk``   the same for tokens that continue sequences whose earlier rows are in the pages.

``own`` chooses between the plain form (elementary torch operations in 32 bits) and the library's entry points.
"""
from __future__ import annotations

import math
import random

import torch

own = False

F32, F64 = torch.float32, torch.float64
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
ROPE_BASE = 10000.0
WIDE_SHARE, WIDE_GAIN = 0.02, 4.0            # key channels that are wider than the others


# ------------------------------------------------------------------------------------------------ the cases
def _case(kind, batch, q_heads, kv_heads, d_head, rows, tokens, dtype="bf16", page_rows=64, **more):
    """rows: cached rows before the call, tokens: new ones (of the longest sequence each, where ragged)."""
    c = dict(kind=kind, batch=batch, q_heads=q_heads, kv_heads=kv_heads, d_head=d_head, rows=rows, tokens=tokens, dtype=dtype,
             page_rows=page_rows, ragged=False, causal=True, shifted=False)
    c.update(more)
    return c


def listed():
    return [
        # the smallest call: one token of one sequence of a small model, a latency floor
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
        # two short questions
        dict(_case("prompt", 2, 8, 8, 64, 0, 35, "f16"), name="prompt_2x35_d64"),
        # a mixed batch of prompts, odd lengths, grouped heads
        dict(_case("prompt", 6, 28, 4, 128, 0, 1501, ragged=True), name="prompt_gqa_ragged_6x1501"),
        # a full batch of prompts, one query head per kv head
        dict(_case("prompt", 16, 32, 32, 128, 0, 2048), name="prompt_16x2048"),
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
    kind = rng.choice(["append", "decode", "decode", "prompt", "prompt", "chunk"])
    hq, hkv, d = rng.choice([(8, 8, 64), (16, 2, 64), (32, 32, 128), (28, 4, 128), (32, 8, 128), (16, 1, 128), (12, 4, 64)])
    c = _case(kind, _log(rng, 1, 64), hq, hkv, d, 0, 1, rng.choice(["bf16", "bf16", "f16"]), rng.choice([16, 32, 64, 112, 128, 256]),
              ragged=rng.random() < 0.6)
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
        pairs = 16 * 32 * 2048 * 2048 // 2 // (hq * c["batch"])
        c["tokens"] = _log(rng, 2, min(4096, max(2, math.isqrt(pairs))))
        if kind == "chunk":
            pairs = 28 * 2048 * 8192 // (hq * c["batch"])
            c["tokens"] = min(c["tokens"], max(2, math.isqrt(pairs // 2)))
            c["rows"] = _log(rng, 1, max(2, min(8192, pairs // c["tokens"] - c["tokens"])))
        else:
            c["causal"] = rng.random() < 0.85
    return c


def _lengths(c):
    """(cached rows before, new tokens) of every sequence: part of the case, the same for every seed."""
    rng = random.Random(repr(sorted((k, v) for k, v in c.items() if k != "name")))
    some = lambda n: n if not c["ragged"] or n < 2 else rng.randint(max(1, n // 8), n)
    before = [c["rows"]] + [some(c["rows"]) for _ in range(c["batch"] - 1)]
    new = [c["tokens"]] + [some(c["tokens"]) for _ in range(c["batch"] - 1)]
    if c["kind"] == "decode":
        new = [0] * c["batch"]             # the row of the new token is counted in rows
    return before, new


def work(case):
    c = case
    before, new = _lengths(c)
    n, width_q, width_kv = sum(new), c["q_heads"] * c["d_head"], c["kv_heads"] * c["d_head"]
    if c["kind"] == "append":
        # queries, keys and values in; rotated queries, pages, and for prompts the rotated keys out
        return {"bytes": 2 * n * (2 * width_q + 4 * width_kv + (width_kv if c["tokens"] > 1 else 0)), "flops": 3 * n * (width_q + width_kv)}
    if c["kind"] == "decode":
        return {"bytes": 4 * sum(before) * width_kv + 4 * c["batch"] * width_q, "flops": 4 * sum(before) * width_q}
    pairs = sum((n * (n + 1) // 2 if c["causal"] else n * n) + n * b for b, n in zip(before, new))
    return {"bytes": 4 * n * width_q + 4 * (n + sum(before)) * width_kv, "flops": 4 * pairs * width_q}


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + 29)
    return g


def _randn(g, dtype, *shape, wide=0):
    """Unit Gaussians; `wide` = d_head: a few channels of every head WIDE_GAIN times wider, as keys have them."""
    x = torch.randn(shape, device="cuda", generator=g, dtype=dtype if math.prod(shape) > 1 << 24 else F32)
    if wide:
        x = x * torch.where(torch.rand(wide, device="cuda", generator=g) < WIDE_SHARE, WIDE_GAIN, 1.0).to(x.dtype)
    return x.to(dtype)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _prefix(n):
    total, out = 0, [0]
    for x in n:
        total += x
        out.append(total)
    return out


def prepare(case, seed):
    c, g, dt = dict(case), _gen(seed), DTYPES[case["dtype"]]
    B, Hq, Hkv, d, R = c["batch"], c["q_heads"], c["kv_heads"], c["d_head"], c["page_rows"]
    before, new = _lengths(c)
    n = sum(new)
    s = dict(case=c, before=before, new=new, n=n, scale=1.0 / math.sqrt(d), cu=_ints(_prefix(new)), longest=max(new))
    if c["kind"] != "prompt":
        lens = [x + y for x, y in zip(before, new)]
        max_pages = -(-max(lens) // R)
        used = [-(-x // R) for x in lens]
        n_pages = sum(used) + max(1, sum(used) // 16)               # a pool with some pages of nobody
        free = torch.randperm(n_pages, device="cuda", generator=g, dtype=torch.int32)
        at, start = torch.arange(max_pages, device="cuda"), _ints(_prefix(used)[:-1])
        table = torch.where(at < _ints(used)[:, None], free[(start[:, None] + at).clamp(max=n_pages - 1)], 0)
        s.update(lens=_ints(lens), max_pages=max_pages, n_pages=n_pages, table=table.contiguous(), max_len=max(lens),
                 k_pool=_randn(g, dt, n_pages, Hkv, R, d, wide=d), v_pool=_randn(g, dt, n_pages, Hkv, R, d))
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
    elif c["kind"] == "decode":
        s["q"] = 1.5 * _randn(g, dt, B, Hq * d)
        s["out"] = torch.empty(B, Hq * d, dtype=dt, device="cuda")
    else:
        s["q"] = 1.5 * _randn(g, dt, n, Hq * d)
        s["out"] = torch.empty(n, Hq * d, dtype=dt, device="cuda")
        if c["kind"] == "prompt":
            s["k"], s["v"] = _randn(g, dt, n, Hkv, d, wide=d).view(n, -1), _randn(g, dt, n, Hkv * d)
    if own:
        _handle(s)
    return s


# ------------------------------------------------------------------------------------------------ the library's calls
_kept = {}


def _handle(s):
    """What a serving program sets up once per layer: descriptor, cache view, context with its workspace."""
    import paper_2604_02570_amd as W
    c = s["case"]
    s["W"], s["stream"] = W, torch.cuda.current_stream().cuda_stream
    s["desc"] = W.dense_desc(c["batch"], c["q_heads"], c["kv_heads"], c["d_head"], c["dtype"], s["scale"])
    if "table" in s:
        s["cache"] = W.make_paged_cache(s["k_pool"], s["v_pool"], None, None, s["lens"], s["table"], c["page_rows"], s["max_pages"], s["n_pages"])
    need = W.wsvd_dense_workspace_bytes(s["desc"])
    if "ctx" not in _kept:
        _kept["ctx"] = W.wsvd_create(0)
    if "ws" not in _kept or _kept["ws"].numel() < need:
        _kept["ws"] = torch.empty(need, dtype=torch.uint8, device="cuda")
        W.wsvd_set_workspace(_kept["ctx"], _kept["ws"])
    s["ctx"] = _kept["ctx"]


def _run_own(s):
    c, W = s["case"], s["W"]
    wq, wkv = c["q_heads"] * c["d_head"], c["kv_heads"] * c["d_head"]
    if c["kind"] == "append":
        x, ld = s["qkv"], wq + 2 * wkv
        W.wsvd_dense_append_paged(s["ctx"], s["desc"], x, ld, x[:, wq:], ld, x[:, wq + wkv:], ld, s["n"], s["cu"], s["positions"],
                                  s["inv_freq"], s["q_out"], wq, s["k_out"], wkv, s["cache"], s["stream"])
        return [t for t in (s["q_out"], s["k_out"], s["k_pool"], s["v_pool"]) if t is not None]
    if c["kind"] == "decode":
        W.wsvd_dense_decode_attn_paged(s["ctx"], s["desc"], s["q"], wq, s["cache"], s["max_len"], s["out"], s["stream"])
    elif c["kind"] == "prompt":
        W.wsvd_dense_prefill_attn(s["ctx"], s["desc"], s["q"], wq, s["k"], wkv, s["v"], wkv, s["n"], s["n"], s["cu"], None, c["causal"],
                                  s["out"], wq, s["stream"])
    else:
        W.wsvd_dense_prefill_attn_paged(s["ctx"], s["desc"], s["q"], wq, s["n"], s["cu"], s["cache"], s["out"], wq, s["stream"])
    return s["out"]


# ------------------------------------------------------------------------------------------------ the plain forms
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
    page = s["table"].long()[b, row // R]
    s["k_pool"][page, :, row % R] = k
    s["v_pool"][page, :, row % R] = x[:, Hq + Hkv:]
    return [t for t in (s["q_out"], s["k_out"], s["k_pool"], s["v_pool"]) if t is not None]


def _gathered(s, pool):
    """A pool's rows by sequence, [B, Hkv, rows, d] in 32 bits."""
    x = pool[s["table"].long()].transpose(1, 2)
    return x.reshape(x.shape[0], x.shape[1], -1, x.shape[-1]).float()


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
    k, v = _gathered(s, s["k_pool"]), _gathered(s, s["v_pool"])
    seen = (torch.arange(k.shape[2], device="cuda") < s["lens"][:, None])[:, None, None]
    return _attend(q, k, v, seen, s["scale"]).to(s["q"].dtype).view(c["batch"], -1)


def _prompt_plain(s):
    c = s["case"]
    B, Hq, Hkv, d, n = c["batch"], c["q_heads"], c["kv_heads"], c["d_head"], s["longest"]
    at = (s["cu"][:-1].long()[:, None] + torch.arange(n, device="cuda")).clamp(max=s["n"] - 1)       # packed -> [B, longest]
    q = s["q"].view(s["n"], Hkv, Hq // Hkv, d)[at].float().permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, d)
    new = (s["cu"][1:] - s["cu"][:-1]).long()
    if c["kind"] == "prompt":
        k, v = (s[x].view(s["n"], Hkv, d)[at].float().transpose(1, 2).contiguous() for x in "kv")
        lens = new
    else:
        k, v = _gathered(s, s["k_pool"]), _gathered(s, s["v_pool"])
        lens = s["lens"].long()
    key = torch.arange(k.shape[2], device="cuda")
    last = (lens - new)[:, None] + torch.arange(n, device="cuda") if c["causal"] else (lens - 1)[:, None].expand(B, n)
    seen = (key <= last[..., None]) & (key < lens[:, None, None])                                     # [B, n, t]
    o = _attend(q, k, v, seen[:, None, None].expand(B, 1, Hq // Hkv, n, -1).reshape(B, 1, -1, k.shape[2]), s["scale"]).to(s["q"].dtype)
    b, i = _tokens(s)
    return o.view(B, Hkv, Hq // Hkv, n, d)[b, :, :, i].reshape(s["n"], -1)


def run(state):
    if own:
        return _run_own(state)
    return {"append": _append_plain, "decode": _decode_plain, "prompt": _prompt_plain, "chunk": _prompt_plain}[state["case"]["kind"]](state)


# ------------------------------------------------------------------------------------------------ from the definition, in 64 bits
def exact(case, seed):
    """The same outputs in 64 bits, sequence by sequence and head by head."""
    s = prepare(case, seed)
    c = s["case"]
    B, Hq, Hkv, d, R = c["batch"], c["q_heads"], c["kv_heads"], c["d_head"], c["page_rows"]
    G, cu = Hq // Hkv, _prefix(s["new"])
    if c["kind"] == "append":
        x = s["qkv"].double().view(-1, Hq + 2 * Hkv, d)
        q_out, k_out = torch.empty(s["n"], Hq, d, dtype=F64, device="cuda"), torch.empty(s["n"], Hkv, d, dtype=F64, device="cuda")
        K, V = s["k_pool"].double(), s["v_pool"].double()
        for b in range(B):
            n, t = s["new"][b], slice(cu[b], cu[b + 1])
            rows = torch.arange(s["before"][b], s["before"][b] + n, device="cuda")
            p = rows.double() if s["positions"] is None else s["positions"][t].double()
            turn = torch.polar(torch.ones((), dtype=F64, device="cuda"), p[:, None] * s["inv_freq"][None, :])[:, None, :]
            for src, dst in ((x[t, :Hq], q_out), (x[t, Hq:Hq + Hkv], k_out)):
                z = torch.complex(src[..., : d // 2], src[..., d // 2:]) * turn
                dst[t] = torch.cat([z.real, z.imag], -1)
            pages = s["table"][b].long()
            K[pages[rows // R], :, rows % R] = k_out[t]
            V[pages[rows // R], :, rows % R] = x[t, Hq + Hkv:]
        out = [q_out.view(s["n"], -1)] + ([k_out.view(s["n"], -1)] if s["k_out"] is not None else [])
        return out + [K, V]
    out = torch.zeros(B if c["kind"] == "decode" else s["n"], Hq, d, dtype=F64, device="cuda")
    for b in range(B):
        t = slice(b, b + 1) if c["kind"] == "decode" else slice(cu[b], cu[b + 1])
        n, total = t.stop - t.start, s["before"][b] + s["new"][b]
        for h in range(Hkv):
            if c["kind"] == "prompt":
                k, v = (s[x].view(-1, Hkv, d)[t, h].double() for x in "kv")
            else:
                k, v = (s[x][s["table"][b].long(), h].reshape(-1, d)[:total].double() for x in ("k_pool", "v_pool"))
            hidden = None
            if c["causal"] and c["kind"] != "decode":
                at = torch.arange(total, device="cuda")
                hidden = at[None, :] > at[total - n:, None]
            for i in range(G):
                w = s["q"].view(-1, Hq, d)[t, h * G + i].double() @ k.t().contiguous() * s["scale"]
                out[t, h * G + i] = torch.softmax(w if hidden is None else w.masked_fill(hidden, -math.inf), -1) @ v
    return out.view(out.shape[0], -1)
