"""Dense-layer entry points without a GPU: what they refuse, and the arithmetic of pages and work division that the kernels share
with the host (compiled here for the CPU)."""
import ctypes
import os
import subprocess

import pytest

import paper_2604_02570_amd as W

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2604_02570_amd", "csrc")
A = 1 << 20                                     # an address that is aligned and never followed


@pytest.fixture
def ctx():
    """A context's memory, all zeros: one without a workspace.  A refused call follows nothing in it but that."""
    memory = ctypes.create_string_buffer(1 << 14)
    yield ctypes.c_void_p(ctypes.addressof(memory))


def desc(**kw):
    return W.dense_desc(**{**dict(batch=3, n_q_heads=8, n_kv_heads=2, d_head=128, dtype="bf16"), **kw})


def cache(**kw):
    a = {**dict(k=A, v=A, lens=A, table=A, page_rows=16, max_pages=4, n_pages=9), **kw}
    return W.make_paged_cache(a["k"], a["v"], None, None, a["lens"], a["table"], a["page_rows"], a["max_pages"], a["n_pages"])


def append(ctx, d=None, c=None, **kw):
    a = {**dict(q=A, q_ld=1024, k=A, k_ld=256, v=A, v_ld=256, n=3, cu=None, pos=None, inv=A, q_out=A, q_out_ld=1024, k_out=A, k_out_ld=256), **kw}
    W.wsvd_dense_append_paged(ctx, d or desc(), a["q"], a["q_ld"], a["k"], a["k_ld"], a["v"], a["v_ld"], a["n"], a["cu"], a["pos"], a["inv"],
                              a["q_out"], a["q_out_ld"], a["k_out"], a["k_out_ld"], c or cache(), 0)


def decode(ctx, d=None, c=None, **kw):
    a = {**dict(q=A, q_ld=1024, most=64, out=A), **kw}
    W.wsvd_dense_decode_attn_paged(ctx, d or desc(), a["q"], a["q_ld"], c or cache(), a["most"], a["out"], 0)


def prompt(ctx, d=None, **kw):
    a = {**dict(q=A, q_ld=1024, k=A, k_ld=256, v=A, v_ld=256, n_q=9, n_kv=9, cu_q=A, cu_kv=None, causal=1, out=A, out_ld=1024), **kw}
    W.wsvd_dense_prefill_attn(ctx, d or desc(), a["q"], a["q_ld"], a["k"], a["k_ld"], a["v"], a["v_ld"], a["n_q"], a["n_kv"], a["cu_q"], a["cu_kv"],
                              a["causal"], a["out"], a["out_ld"], 0)


def chunk(ctx, d=None, c=None, **kw):
    a = {**dict(q=A, q_ld=1024, n_q=9, cu_q=A, out=A, out_ld=1024), **kw}
    W.wsvd_dense_prefill_attn_paged(ctx, d or desc(), a["q"], a["q_ld"], a["n_q"], a["cu_q"], c or cache(), a["out"], a["out_ld"], 0)


def refuses(status, f, *args, **kw):
    with pytest.raises(W.WsvdError) as e:
        f(*args, **kw)
    assert e.value.status == status, (W.STATUS_NAMES[e.value.status], kw)


BAD_DESC = [(dict(batch=0), W.E_SHAPE), (dict(batch=65537), W.E_SHAPE), (dict(n_q_heads=7), W.E_SHAPE), (dict(n_kv_heads=0), W.E_SHAPE),
            (dict(n_q_heads=34, n_kv_heads=2), W.E_SHAPE), (dict(n_q_heads=2048, n_kv_heads=256), W.E_SHAPE), (dict(d_head=96), W.E_SHAPE),
            (dict(d_head=256), W.E_SHAPE), (dict(dtype="f32"), W.E_DTYPE), (dict(dtype="i8"), W.E_DTYPE), (dict(sm_scale=-1.0), W.E_SHAPE),
            (dict(sm_scale=float("nan")), W.E_SHAPE), (dict(sm_scale=float("inf")), W.E_SHAPE)]
BAD_CACHE = [(dict(k=None), W.E_NULL), (dict(v=None), W.E_NULL), (dict(lens=None), W.E_NULL), (dict(table=None), W.E_NULL), (dict(k=A + 8), W.E_ALIGN),
             (dict(v=A + 2), W.E_ALIGN), (dict(lens=A + 2), W.E_ALIGN), (dict(table=A + 1), W.E_ALIGN), (dict(page_rows=8), W.E_SHAPE),
             (dict(page_rows=24), W.E_SHAPE), (dict(page_rows=4112), W.E_SHAPE), (dict(max_pages=0), W.E_SHAPE), (dict(n_pages=0), W.E_SHAPE),
             (dict(page_rows=4096, max_pages=1 << 16), W.E_SHAPE)]


@pytest.mark.parametrize("kw,status", BAD_DESC)
def test_descriptors_refused(ctx, kw, status):
    for f in (append, decode, prompt, chunk):
        refuses(status, f, ctx, desc(**kw))
    with pytest.raises(W.WsvdError) as e:
        W.wsvd_dense_workspace_bytes(desc(**kw))
    assert e.value.status == status


@pytest.mark.parametrize("kw,status", BAD_CACHE)
def test_caches_refused(ctx, kw, status):
    for f in (append, decode, chunk):
        refuses(status, f, ctx, None, cache(**kw))


def test_context_refused():
    for f in (append, decode, prompt, chunk):
        refuses(W.E_NULL, f, None)


def test_append_refuses(ctx):
    for kw, status in ((dict(q=None), W.E_NULL), (dict(q_out=None), W.E_NULL), (dict(k=None), W.E_NULL), (dict(v=None), W.E_NULL),
                       (dict(q=A + 8), W.E_ALIGN), (dict(k_ld=260), W.E_ALIGN), (dict(v_ld=248), W.E_SHAPE), (dict(q_ld=1016), W.E_SHAPE),
                       (dict(k_out_ld=(1 << 24) + 8), W.E_SHAPE), (dict(q_ld=2048, q_out_ld=1024), W.E_SHAPE), (dict(k_ld=512), W.E_SHAPE),
                       (dict(inv=A + 4), W.E_ALIGN), (dict(cu=A + 2), W.E_ALIGN), (dict(pos=A + 2), W.E_ALIGN), (dict(n=-1, cu=A), W.E_SHAPE),
                       (dict(n=4), W.E_SHAPE), (dict(n=(1 << 24) + 1, cu=A), W.E_SHAPE)):
        refuses(status, append, ctx, **kw)
    append(ctx, n=0, cu=A)                      # nothing to do
    append(ctx, n=0, cu=A, q=None, q_out=None, k_out=None)


def test_decode_refuses(ctx):
    for kw, status in ((dict(q=None), W.E_NULL), (dict(out=None), W.E_NULL), (dict(q=A + 2), W.E_ALIGN), (dict(out=A + 8), W.E_ALIGN),
                       (dict(q_ld=1020), W.E_SHAPE), (dict(q_ld=1028), W.E_ALIGN), (dict(most=-1), W.E_SHAPE), (dict(most=65), W.E_CAPACITY),
                       (dict(), W.E_WORKSPACE)):
        refuses(status, decode, ctx, **kw)


def test_prompts_refuse(ctx):
    for kw, status in ((dict(q=None), W.E_NULL), (dict(k=None), W.E_NULL), (dict(v=None), W.E_NULL), (dict(out=None), W.E_NULL), (dict(cu_q=None), W.E_NULL),
                       (dict(q=A + 2), W.E_ALIGN), (dict(k_ld=252), W.E_SHAPE), (dict(out_ld=1028), W.E_ALIGN), (dict(cu_q=A + 1), W.E_ALIGN),
                       (dict(cu_kv=A + 1), W.E_ALIGN), (dict(n_q=-1), W.E_SHAPE), (dict(n_kv=8), W.E_SHAPE), (dict(n_kv=-1, cu_kv=A), W.E_SHAPE),
                       (dict(causal=2), W.E_SHAPE), (dict(), W.E_WORKSPACE), (dict(k=None, v=None, n_kv=0, cu_kv=A), W.E_WORKSPACE)):
        refuses(status, prompt, ctx, **kw)
    for kw, status in ((dict(q=None), W.E_NULL), (dict(out=None), W.E_NULL), (dict(cu_q=None), W.E_NULL), (dict(cu_q=A + 2), W.E_ALIGN),
                       (dict(n_q=-1), W.E_SHAPE), (dict(out_ld=1000), W.E_SHAPE), (dict(), W.E_WORKSPACE)):
        refuses(status, chunk, ctx, **kw)
    prompt(ctx, n_q=0, n_kv=0)
    chunk(ctx, n_q=0)


def test_workspace_holds_what_the_kernels_put_there():
    for batch, hq, hkv, d in ((1, 8, 8, 64), (1, 16, 1, 128), (32, 28, 4, 128), (4096, 32, 8, 128), (3, 1024, 1024, 64)):
        target = max(1, (1024 if batch * hkv >= 1024 else 512 if batch * hkv >= 512 else 256) // hkv)
        need = W.wsvd_dense_workspace_bytes(desc(batch=batch, n_q_heads=hq, n_kv_heads=hkv, d_head=d)) - 65536
        assert need >= (target + batch) * hq * (d + 2) * 8          # one word per value of every chunk
        assert need >= 512 * 128 * (d + 2) * 4                      # 512 parts of 128 rows


PROGRAM = r"""
#include "wsvd_dense_plan.h"
#include <cstdio>
#include <cstdlib>
#include <vector>
#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)
int main() {
  // pages: the product is the division, for every granule a cache can have and every page size
  for (int rows = 16; rows <= 4096; rows += 16) {
    const uint32_t magic = dense_page_magic(rows);
    const int n = rows / 16, last = (1 << 23) - 1;
    for (int g = 0; g < 3000; g++) CHECK(dense_page_index(g, magic) == g / n);
    for (int i = 0; i < 3000; i++) { const int g = last - i; CHECK(dense_page_index(g, magic) == g / n); }
    for (int k = 1; k <= last / n; k += 1 + last / n / 500) CHECK(dense_page_index(k * n, magic) == k && dense_page_index(k * n - 1, magic) == k - 1);
  }
  // bad entries are reported and read as page 0
  for (int e : {-1, -2147483647 - 1, 9, 10, 2147483647}) { bool bad = false; CHECK(dense_page(e, 9, bad) == 0 && bad); }
  for (int e = 0; e < 9; e++) { bool bad = false; CHECK(dense_page(e, 9, bad) == e && !bad); bad = true; dense_page(e, 9, bad); CHECK(bad); }
  // rows: past 32 bits, and always inside the pool
  CHECK(dense_pool_row(1 << 20, 5, 1, 7, 8, 64) == ((uint64_t)(1 << 20) * 8 + 7) * 64 + 16);
  for (int rows : {16, 48, 112, 4096})
    for (int g = 0; g < 700; g++) {
      const int pg = dense_page_index(g, dense_page_magic(rows));
      const uint64_t at = dense_pool_row(4, g, pg, 2, 3, rows);
      CHECK(at % 16 == 0 && at + 16 <= (uint64_t)5 * 3 * rows && at >= (uint64_t)(4 * 3 + 2) * rows);
    }
  // chunks of the decode attention
  std::srand(7);
  for (int round = 0; round < 40000; round++) {
    const int Hkv = 1 << (std::rand() % 11), B = 1 + std::rand() % (round % 3 ? 70 : 700), target = dense_target(dense_waves(B, Hkv, round % 2 ? 1000 : 5000), Hkv);
    CHECK(target <= dense_target(dense_waves(B, Hkv, 0), Hkv));          // the workspace's
    const int alone = 1 + std::rand() % 12, least = 1 + std::rand() % 6;
    std::vector<int> u(B);
    int total = 0, most = 0;
    for (int& x : u) {
      x = dense_units_of(std::rand() % 5 ? std::rand() % (1 << (std::rand() % 21)) : 0);
      total += x; most = x > most ? x : most;
    }
    auto count = [&](int units) { int n = 0; for (int x : u) n += dense_chunks(x, units); return n; };
    const int units = dense_units(total, most, B, target, alone, least, count);
    const int n = count(units);
    CHECK(units >= 1 && n >= B && n <= target + B);                  // the grid and the workspace are for target + B
    if (B <= 64 && B <= target) CHECK(n <= target);
    for (int x : u) {
      const int c = dense_chunks(x, units);
      CHECK(c >= 1 && c <= kDenseFold * kDenseFold);
      const int each = (x + c - 1) / c;                              // every row in exactly one chunk (the last may be short or empty)
      CHECK(each <= units && (long long)each * c >= x);
    }
  }
  CHECK(dense_units_of(0) == 0 && dense_units_of(1) == 1 && dense_units_of(128) == 1 && dense_units_of(129) == 2);
  // a tile's blocks over its workgroups
  for (int n = 1; n < 3000; n += 7)
    for (int s = 1; s <= 32; s++) {
      CHECK(dense_share(0, n, s) == 0 && dense_share(s, n, s) == n);
      for (int k = 0; k < s; k++) CHECK(dense_share(k + 1, n, s) >= dense_share(k, n, s) + n / s);
    }
  return 0;
}
"""


def test_pages_and_work_division(tmp_path):
    source, program = tmp_path / "plan.cpp", tmp_path / "plan"
    source.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-I", CSRC, str(source), "-o", str(program)], check=True)
    r = subprocess.run([str(program)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


def test_tags_of_words_are_no_sum():
    """Plain fp32 sums of other calls lie where a call waits for tagged words: a tag is a signalling NaN, which arithmetic never makes,
    with low bits set, which a NaN that came from 16 bits has not."""
    import re
    tags = []
    for name, constant in (("wsvd_attn_common.h", "kSplitTag"), ("wsvd_append_split.h", "kLLTag")):
        with open(os.path.join(CSRC, name)) as f:
            tags.append(int(re.search(r"constexpr uint32_t %s = (0x[0-9A-Fa-f]+)u" % constant, f.read()).group(1), 16))
    assert len(set(tags)) == 2
    for tag in tags:
        assert tag >> 23 & 0xFF == 0xFF and not tag >> 22 & 1 and tag & 0x1FFF


def test_calls_of_more_threads_than_a_launch_has_are_refused(ctx):
    """2^32 threads: WSVD_E_SHAPE, not an error of the launch (and what fits gets as far as the workspace)."""
    many, longer = dict(batch=65536, n_q_heads=128, n_kv_heads=128, d_head=64), dict(max_pages=200)
    refuses(W.E_SHAPE, decode, ctx, desc(**many), cache(**longer), q_ld=8192, most=2000)
    refuses(W.E_WORKSPACE, decode, ctx, desc(**many), cache(**longer), q_ld=8192, most=64)
    refuses(W.E_WORKSPACE, decode, ctx, desc(**{**many, "n_q_heads": 64, "n_kv_heads": 64}), cache(**longer), q_ld=8192, most=2000)
    refuses(W.E_SHAPE, decode, ctx, desc(**{**many, "n_q_heads": 1024, "n_kv_heads": 1024}), cache(), q_ld=65536, most=64)
    wide = dict(n_q_heads=1024, n_kv_heads=64, d_head=64)
    for f, kw in ((prompt, dict(k_ld=4096, v_ld=4096, n_kv=1 << 24)), (prompt, dict(k_ld=4096, v_ld=4096, n_kv=1 << 24, causal=0)), (chunk, {})):
        refuses(W.E_SHAPE, f, ctx, desc(**wide), q_ld=65536, out_ld=65536, n_q=1 << 24, **kw)
        refuses(W.E_WORKSPACE, f, ctx, desc(**wide), q_ld=65536, out_ld=65536, n_q=1 << 20, **{**kw, **({"n_kv": 1 << 20} if kw else {})})


LAUNCHES = r"""
#include "wsvd_dense_plan.h"
#include <cstdio>
#include <initializer_list>
#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)
int main() {
  CHECK(dense_launchable((1 << 24) - 1, 256) && !dense_launchable(1 << 24, 256) && dense_launchable((1 << 23) - 1, 512));
  // appends of every size are a launch, and every token is in it
  for (int64_t n = 1; n <= 1 << 24; n = n < 5000 ? n + 1 : n + n / 3 < 1 << 24 ? n + n / 3 : n < 1 << 24 ? 1 << 24 : n + 1)
    for (int items : {12, 64, 127, 128, 255, 256, 400, 5000}) {
      const int t = dense_append_tokens(n, items);
      CHECK((t == 1 || t == 2 || t == 4) && dense_launchable((n + t - 1) / t, 256));
      CHECK(n >= (1 << 24) || t == (n < 2048 || items >= 256 ? 1 : items >= 128 ? 2 : 4));
    }
  // what the interface promises to take
  for (int Hkv = 1; Hkv <= 1024; Hkv *= 2)
    for (int B = 1; B <= 65536 && (int64_t)B * Hkv <= 1 << 22; B = 2 * B + (B & 2)) {
      for (int len : {0, 1024, 1025, 1 << 27}) {
        const int waves = dense_waves(B, Hkv, len);
        for (bool alone : {false, true}) CHECK(dense_launchable(dense_decode_workgroups(B, Hkv, dense_target(waves, Hkv), alone), 64 * waves));
      }
      for (int G = 1; G <= 16; G++)
        if (G * Hkv <= 1024)
          for (bool causal : {false, true}) {
            const int64_t most = ((int64_t)1 << 30) / (G * Hkv), n = most < 1 << 24 ? most : 1 << 24;
            CHECK(dense_launchable(dense_prompt_grid(n, B, Hkv, G, causal).workgroups, 256));
          }
    }
  // enough workgroups for every division of the tokens among the sequences: two tiles a workgroup, or one
  for (int B : {1, 2, 7, 300})
    for (int G : {1, 3, 7, 16})
      for (int Hkv : {1, 8})
        for (int seed = 1; seed < 400; seed++) {
          int64_t n = 0, one = 0, two = 0;
          unsigned x = (unsigned)seed * 2654435761u;
          for (int b = 0; b < B; b++) {
            x = x * 1664525u + 1013904223u;
            const int64_t len = (x >> 8) % (seed % 3 ? 40 : 3000), tiles = (len * G + 127) / 128;
            n += len; one += tiles; two += (tiles + 1) / 2;
          }
          for (bool causal : {false, true}) {
            const DensePromptGrid g = dense_prompt_grid(n, B, Hkv, G, causal);
            CHECK(g.workgroups >= (g.pairs ? two : one) * Hkv);
          }
        }
  return 0;
}
"""


def test_launches_hold_their_work(tmp_path):
    source, program = tmp_path / "launches.cpp", tmp_path / "launches"
    source.write_text(LAUNCHES)
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-I", CSRC, str(source), "-o", str(program)], check=True)
    r = subprocess.run([str(program)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


def test_calls_without_tokens_take_tensors_without_memory(ctx):
    """An empty tensor has no address: such calls have nothing to do, as with any other address."""
    append(ctx, n=0, cu=A, q=0, k=0, v=0, q_out=0, k_out=0)
    append(ctx, n=0, cu=A, q=None, k=None, v=None, q_out=None, k_out=None)
    append(ctx, n=0, cu=A, q=0, k=0, v=0, q_out=A, k_out=A)
    prompt(ctx, n_q=0, n_kv=0, q=0, k=0, v=0, out=0)
    prompt(ctx, n_q=0, n_kv=7, q=0, out=0, cu_kv=A)
    chunk(ctx, n_q=0, q=0, out=0)
    refuses(W.E_NULL, prompt, ctx, n_q=0, n_kv=7, q=0, out=0, k=0, cu_kv=A)
    for f, kw in ((append, dict(n=0, cu=A, k=A + 8)), (prompt, dict(n_q=0, n_kv=0, q=A + 2)), (chunk, dict(n_q=0, out=A + 8))):
        refuses(W.E_ALIGN, f, ctx, **kw)
    for f in (prompt, chunk):
        refuses(W.E_NULL, f, ctx, n_q=0, cu_q=None, **({"n_kv": 0} if f is prompt else {}))
