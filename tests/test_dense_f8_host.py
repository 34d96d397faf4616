"""Entry points of the 8-bit pages and of the page tables without a GPU: what they refuse, and the reference that the GPU tests use against
torch's own E4M3."""
import ctypes
import math
import os
import subprocess

import pytest
import torch

import paper_2604_02570_amd as W
from dense_ref import F64
from f8_ref import MOST, NUMBERS, bytes_of, exponent, place, quantised, rounded
from test_dense_host import A, BAD_CACHE, BAD_DESC, CSRC, ctx, desc, refuses  # noqa: F401


def cache(**kw):
    a = {**dict(k=A, v=A, ks=A, vs=A, lens=A, table=A, page_rows=16, max_pages=4, n_pages=9), **kw}
    return W.make_paged_cache(a["k"], a["v"], a["ks"], a["vs"], a["lens"], a["table"], a["page_rows"], a["max_pages"], a["n_pages"])


def append(ctx, d=None, c=None, **kw):
    a = {**dict(q=A, q_ld=1024, k=A, k_ld=256, v=A, v_ld=256, n=3, cu=None, pos=None, inv=A, q_out=A, q_out_ld=1024, k_out=A, k_out_ld=256), **kw}
    W.wsvd_dense_append_paged_f8(ctx, d or desc(), a["q"], a["q_ld"], a["k"], a["k_ld"], a["v"], a["v_ld"], a["n"], a["cu"], a["pos"], a["inv"],
                                 a["q_out"], a["q_out_ld"], a["k_out"], a["k_out_ld"], c or cache(), 0)


def decode(ctx, d=None, c=None, **kw):
    a = {**dict(q=A, q_ld=1024, most=64, out=A), **kw}
    W.wsvd_dense_decode_attn_paged_f8(ctx, d or desc(), a["q"], a["q_ld"], c or cache(), a["most"], a["out"], 0)


def chunk(ctx, d=None, c=None, **kw):
    a = {**dict(q=A, q_ld=1024, n_q=9, cu_q=A, out=A, out_ld=1024), **kw}
    W.wsvd_dense_prefill_attn_paged_f8(ctx, d or desc(), a["q"], a["q_ld"], a["n_q"], a["cu_q"], c or cache(), a["out"], a["out_ld"], 0)


def pool(**kw):
    a = {**dict(table=A, free=A, batch=3, page_rows=16, max_pages=4, n_pages=9), **kw}
    return W.make_page_pool(a["table"], a["free"], a["batch"], a["page_rows"], a["max_pages"], a["n_pages"])


def grow(ctx, p=None, **kw):
    a = {**dict(new=A, n=5, lens=A, n_free=A, lens_out=A, n_free_out=A, cu=A, positions=A, slots=A), **kw}
    W.wsvd_pages_grow(ctx, p or pool(), a["new"], a["n"], a["lens"], a["n_free"], a["lens_out"], a["n_free_out"], a["cu"], a["positions"], a["slots"], 0)


def release(ctx, p=None, **kw):
    a = {**dict(done=A, lens=A, n_free=A, lens_out=A, n_free_out=A), **kw}
    W.wsvd_pages_release(ctx, p or pool(), a["done"], a["lens"], a["n_free"], a["lens_out"], a["n_free_out"], 0)


@pytest.mark.parametrize("kw,status", BAD_DESC)
def test_descriptors_refused(ctx, kw, status):
    for f in (append, decode, chunk):
        refuses(status, f, ctx, desc(**kw))
    with pytest.raises(W.WsvdError) as e:
        W.wsvd_dense_f8_cache_bytes(desc(**kw), 16, 4)
    assert e.value.status == status


@pytest.mark.parametrize("kw,status", BAD_CACHE + [(dict(ks=None), W.E_NULL), (dict(vs=None), W.E_NULL)])
def test_caches_refused(ctx, kw, status):
    for f in (append, decode, chunk):
        refuses(status, f, ctx, None, cache(**kw))


def test_context_refused():
    for f in (append, decode, chunk, grow, release):
        refuses(W.E_NULL, f, None)


def test_calls_refused(ctx):
    for kw, status in ((dict(q=None), W.E_NULL), (dict(k=None), W.E_NULL), (dict(q=A + 8), W.E_ALIGN), (dict(v_ld=248), W.E_SHAPE), (dict(n=4), W.E_SHAPE),
                       (dict(n=(1 << 24) + 1, cu=A), W.E_SHAPE), (dict(inv=A + 4), W.E_ALIGN), (dict(k_ld=512), W.E_SHAPE)):
        refuses(status, append, ctx, **kw)
    for kw, status in ((dict(q=None), W.E_NULL), (dict(out=A + 8), W.E_ALIGN), (dict(most=65), W.E_CAPACITY), (dict(most=-1), W.E_SHAPE), (dict(), W.E_WORKSPACE)):
        refuses(status, decode, ctx, **kw)
    for kw, status in ((dict(cu_q=None), W.E_NULL), (dict(n_q=-1), W.E_SHAPE), (dict(out_ld=1028), W.E_ALIGN), (dict(), W.E_WORKSPACE)):
        refuses(status, chunk, ctx, **kw)
    append(ctx, n=0, cu=A, q=0, k=0, v=0, q_out=0, k_out=0)            # nothing to do
    chunk(ctx, n_q=0, q=0, out=0)


def test_page_tables_refused(ctx):
    for kw, status in ((dict(table=None), W.E_NULL), (dict(free=None), W.E_NULL), (dict(batch=0), W.E_SHAPE), (dict(batch=65537), W.E_SHAPE),
                       (dict(page_rows=24), W.E_SHAPE), (dict(page_rows=8), W.E_SHAPE), (dict(page_rows=4112), W.E_SHAPE), (dict(max_pages=0), W.E_SHAPE),
                       (dict(n_pages=0), W.E_SHAPE), (dict(n_pages=1 << 27), W.E_SHAPE), (dict(n_pages=(1 << 24) + 1), W.E_SHAPE),
                       (dict(n_pages=1 << 24, page_rows=128), W.E_SHAPE), (dict(page_rows=4096, max_pages=1 << 16), W.E_SHAPE),
                       (dict(table=A + 2), W.E_ALIGN), (dict(free=A + 1), W.E_ALIGN)):
        for f in (grow, release):
            refuses(status, f, ctx, pool(**kw))
    for kw, status in ((dict(lens=None), W.E_NULL), (dict(n_free=None), W.E_NULL), (dict(lens_out=None), W.E_NULL), (dict(n_free_out=None), W.E_NULL),
                       (dict(n=-1), W.E_SHAPE), (dict(n=(1 << 24) + 1), W.E_SHAPE), (dict(new=None), W.E_SHAPE), (dict(new=A + 2), W.E_ALIGN),
                       (dict(lens=A + 1), W.E_ALIGN), (dict(cu=A + 2), W.E_ALIGN), (dict(positions=A + 2), W.E_ALIGN), (dict(slots=A + 2), W.E_ALIGN),
                       (dict(n_free_out=A + 2), W.E_ALIGN)):
        refuses(status, grow, ctx, **kw)
    for kw, status in ((dict(done=None), W.E_NULL), (dict(lens=None), W.E_NULL), (dict(n_free_out=None), W.E_NULL), (dict(done=A + 2), W.E_ALIGN)):
        refuses(status, release, ctx, **kw)


def test_pool_sizes():
    assert W.wsvd_dense_f8_cache_bytes(desc(n_q_heads=8, n_kv_heads=2, d_head=128), 48, 5) == (5 * 2 * 48 * 128, 5 * 2 * 3)
    for rows, pages in ((0, 5), (24, 5), (4112, 5), (16, 0)):
        with pytest.raises(W.WsvdError):
            W.wsvd_dense_f8_cache_bytes(desc(), rows, pages)


def test_struct_size():
    assert ctypes.sizeof(W.PagePool) == 2 * ctypes.sizeof(ctypes.c_void_p) + 4 * 4


# ------------------------------------------------------------------------------------------------ the reference
def test_numbers_and_their_rounding_are_those_of_torch():
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).to(F64)
    assert torch.equal(torch.isnan(want), torch.isnan(NUMBERS)) and torch.equal(want.nan_to_num(7), NUMBERS.nan_to_num(7))
    x = torch.cat([torch.linspace(-MOST, MOST, 40001, dtype=F64), torch.linspace(-0.1, 0.1, 4001, dtype=F64)]).float()
    assert torch.equal(rounded(x.to(F64)).float(), x.to(torch.float8_e4m3fn).float())
    some = NUMBERS[~torch.isnan(NUMBERS)]
    assert torch.equal(NUMBERS[bytes_of(some).long()], some)


def test_exponents():
    for e in range(-100, 121):
        assert exponent(torch.tensor([MOST * 2.0 ** e, 0.0], dtype=F64)) == e
        if e < 120:
            assert exponent(torch.tensor([-MOST * 2.0 ** e * (1 + 2.0 ** -8)], dtype=F64)) == e + 1
    assert exponent(torch.zeros(3)) == -100 and exponent(torch.tensor([math.inf, math.nan, 449.0])) == 1
    # nothing that is stored passes the type
    for dtype, t in (("bf16", torch.bfloat16), ("f16", torch.float16)):
        x = torch.tensor([torch.finfo(t).max, torch.finfo(t).tiny, -torch.finfo(t).max]).to(t)
        e = exponent(x)
        assert torch.isfinite((quantised(x, e, dtype) * 2.0 ** e).to(t)).all()


def test_places_are_a_block():
    for d in (64, 128):
        for keys in (True, False):
            assert sorted(place(d, r, x, keys) for r in range(16) for x in range(d)) == list(range(16 * d))


PROGRAM = r"""
#include "wsvd_dense_plan.h"
#include <cstdio>
#include <initializer_list>
#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)
int main() {
  for (int64_t n = 1; n <= 1 << 24; n = n < 3000 ? n + 1 : n + n / 3 < 1 << 24 ? n + n / 3 : n < 1 << 24 ? 1 << 24 : n + 1)
    for (int batch : {1, 7, 64, 300, 65536})
      for (int heads : {3, 12, 96, 1026, 2900})
        for (bool packed : {false, true}) {
          if (!packed && n != batch) continue;
          const DenseF8Append a = dense_f8_append(n, batch, heads, packed);
          CHECK(a.units >= 1 && a.units <= n && a.splits >= 1 && a.splits <= (heads + 3) / 4);
          CHECK(dense_launchable(a.units * a.splits, 256));
        }
  // a few tokens a sequence as columns: a tile for every 16 or 32 pairs of every sequence, and words for their parts in the workspace's 512 parts of 128 rows
  for (int seed = 1; seed < 20000; seed++) {
    unsigned x = (unsigned)seed * 2654435761u;
    auto next = [&](unsigned most) { x = x * 1664525u + 1013904223u; return (int)((x >> 8) % most); };
    const int batch = 1 + next(seed % 2 ? 8 : 300), group = 1 + next(16), Hkv = 1 << next(11);
    int64_t n = 0, tiles[3] = {};
    for (int b = 0; b < batch; b++) {
      const int len = next(7) ? next(seed % 5 ? 4 : 90) : 0;
      n += len; tiles[1] += (len * group + 15) / 16; tiles[2] += (len * group + 31) / 32;
    }
    if (n == 0) continue;
    const DenseF8Columns c = dense_f8_columns(n, batch, Hkv, group);
    CHECK((c.sets == 1 || c.sets == 2) && c.tiles >= tiles[c.sets] && c.splits >= 1 && c.splits <= (c.joins ? kDenseFold * kDenseFold : kDenseFold));
    CHECK(!c.joins || (c.sets == 1 && n * group * Hkv <= 128));
    if (c.taken) CHECK(dense_launchable(c.tiles * c.splits * Hkv, 512) && (c.splits == 1 || c.tiles * c.splits * Hkv * c.sets * 16 * 8 <= (int64_t)kDensePromptParts * kDensePromptRows * 4));
  }
  CHECK(dense_f8_columns(1, 65536, 1024, 1).tiles == 1 && !dense_f8_columns(1 << 24, 1, 1, 16).taken && dense_f8_columns(20, 4, 8, 1).taken);
  CHECK(dense_f8_columns(256, 32, 8, 4).taken && dense_f8_columns(256, 32, 8, 4).sets == 2 && dense_f8_columns(20, 4, 8, 1).sets == 1);
  // a unit for every block that a call writes to, however its tokens are spread and wherever its sequences stand
  for (int seed = 1; seed < 3000; seed++) {
    unsigned x = (unsigned)seed * 2654435761u;
    auto next = [&](unsigned most) { x = x * 1664525u + 1013904223u; return (int)((x >> 8) % most); };
    const int batch = 1 + next(70);
    int64_t n = 0, units = 0;
    for (int b = 0; b < batch; b++) {
      const int row = next(50), len = next(seed % 3 ? 4 : 200);
      n += len;
      if (len > 0) units += (row + len - 1) / 16 - row / 16 + 1;
    }
    if (n > 0) CHECK(dense_f8_append(n, batch, 12, true).units >= units);
  }
  // workgroups that join chunks: of every sequence of a wave's lanes, or none
  for (int Hkv = 1; Hkv <= 1024; Hkv++)
    for (int batch : {1, 2, 3, 4, 7, 8, 16, 31, 32, 33, 64, 65, 65536})
      for (int most : {100, 1024, 1025, 100000}) {
        const int waves = dense_waves(batch, Hkv, most), joins = dense_f8_joins(batch, dense_target(waves, Hkv), waves);
        CHECK(joins == 0 || (joins == batch && batch <= 32 && waves == 8));
        CHECK(dense_launchable(dense_decode_workgroups(batch, Hkv, dense_target(waves, Hkv), false) + (int64_t)joins * 16 * Hkv, 512) || joins == 0);
      }
  for (int batch : {1, 64, 65, 256, 257, 65536})
    for (int64_t n : {0, 1, 256, 257, 1024, 1025, 1 << 20, 1 << 24}) {
      const PagesLaunch l = pages_launch(batch, n);
      CHECK(l.workgroups >= 1 && l.workgroups <= 128 && l.threads % 64 == 0 && l.threads >= 64 && l.threads <= (unsigned)kPagesThreads);
    }
  return 0;
}
"""


def test_launches_hold_their_work(tmp_path):
    source, program = tmp_path / "f8.cpp", tmp_path / "f8"
    source.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-I", CSRC, str(source), "-o", str(program)], check=True)
    r = subprocess.run([str(program)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


def test_calls_of_more_threads_than_a_launch_has_are_refused(ctx):
    many, longer = dict(batch=65536, n_q_heads=128, n_kv_heads=128, d_head=64), dict(max_pages=200)
    refuses(W.E_SHAPE, decode, ctx, desc(**many), cache(**longer), q_ld=8192, most=2000)
    refuses(W.E_WORKSPACE, decode, ctx, desc(**many), cache(**longer), q_ld=8192, most=64)
    refuses(W.E_SHAPE, chunk, ctx, desc(n_q_heads=1024, n_kv_heads=64, d_head=64), q_ld=65536, out_ld=65536, n_q=1 << 24)
