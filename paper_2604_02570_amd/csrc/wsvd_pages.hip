// Page tables kept on the GPU: the pages of finished sequences, and of rows that are taken back, to a free list, and pages from it for the new
// tokens of a step, with the tokens' prefix sums, positions and slots.  Latency is what counts: a step's tables are a few KB to a MB.
#include "wsvd_dense.h"

namespace {

constexpr int kSeqs = kPagesThreads;                 // sequences at a time, at most: one a thread

struct PagesParams {
  int *table, *free_pages;
  const int *lens, *n_free, *what;                   // what: new tokens, which sequences are done, or the rows they keep
  int *lens_out, *n_free_out;
  int *cu, *positions, *slots;
  int B, R, max_pages, n_pages, n_tokens;
  int* err_word;
  int* counter;                                      // of workgroups, zero between launches
  int apart;                                         // what is written is not what is read
  int keeps;                                         // `what` is rows that are kept
};

// Exclusive prefix sum of one number a thread over the workgroup, and the sum of all.  Numbers are at most 2^24, and no more than that many
// tokens or pages are dealt with.  Sums within a wave that pass 2^25 are taken as that, so that nothing overflows: what begins behind such
// a one begins at 2^24 or later, and what begins before has its place.
struct Scan { int wave[kSeqs / 64]; };
WSVD_DEV int scan_exclusive(Scan& sh, int x, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = blockDim.x >> 6;
  const int incl = min(wave_prefix_int(x), 1 << 25);
  __syncthreads();                                   // (the sums of the call before have been read)
  if (lane == 63) sh.wave[wave] = incl;
  __syncthreads();
  const int sums = wave_prefix_int(lane < n ? sh.wave[lane] : 0);
  total = __builtin_amdgcn_readlane(sums, 63);
  return incl - x + (wave > 0 ? __shfl(sums, wave - 1) : 0);
}
// An entry of the free list: written through, since another workgroup may write it again.
WSVD_DEV void put_page(int* to, int page) { __hip_atomic_store(to, page, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
// The last i in [0, n) with first[i] <= x, where first[0] <= x.
WSVD_DEV int last_at_most(const int* first, int n, int x) {
  int i = 0;
  for (int step = kSeqs / 2; step > 0; step >>= 1)
    if (i + step < n && first[i + step] <= x) i += step;
  return i;
}

// Every workgroup finds all sequences' first tokens and pages from the lengths, in one pass; table entries and tokens are dealt out.  A new
// page is the free list's, not the table's: nobody reads what another workgroup writes.  Lengths and the free list's length may be
// updated in place: then the last workgroup to come writes them, when all have read them.
__global__ __launch_bounds__(kSeqs) void k_pages_grow(PagesParams p) {
  __shared__ Scan scan;
  __shared__ int cu_sh[kSeqs], page_sh[kSeqs], len_sh[kSeqs];
  __shared__ int last_sh;
  const int tid = threadIdx.x, wg = blockIdx.x, wgs = gridDim.x;
  const int R = p.R, cap = p.max_pages * R;
  const int listed = *p.n_free, n_free = min(max(listed, 0), p.n_pages);
  int err = listed != n_free ? (int)WSVD_E_SHAPE : 0;
  auto free_page = [&](int i) {
    if (i >= n_free) { err = err ? err : (int)WSVD_E_CAPACITY; return -1; }
    const int page = p.free_pages[n_free - 1 - i];
    if (page < 0 || page >= p.n_pages) { err = WSVD_E_SHAPE; return -1; }
    return page;
  };
  // a thread's sequence: rows before, new ones, pages before, new ones, the first token and the first new page's number in the step
  int len, add, have, need, t0, p0;
  int tokens = 0, pages = 0;                         // of the sequences before
  auto place = [&](int base) {
    const int b = base + tid, old = b < p.B ? p.lens[b] : 0, more = b >= p.B ? 0 : p.what ? p.what[b] : 1;
    len = min(max(old, 0), cap);
    add = min(max(more, 0), 1 << 24);
    int total;
    t0 = tokens + scan_exclusive(scan, add, total);
    add = max(min(add, p.n_tokens - t0), 0);
    t0 = min(t0, p.n_tokens);
    tokens = min(tokens + total, p.n_tokens);
    if (len != old || add != more) err = WSVD_E_SHAPE;
    else if (add > cap - len) err = err ? err : (int)WSVD_E_CAPACITY;
    have = (len + R - 1) / R;
    need = min((len + add + R - 1) / R, p.max_pages) - have;
    p0 = pages + scan_exclusive(scan, need, total);
    pages += total;
  };
  auto commit = [&](int base) { if (base + tid < p.B) p.lens_out[base + tid] = len + add; };
  for (int base = 0; base < p.B; base += (int)blockDim.x) {
    const int b = base + tid, n_here = min(p.B - base, (int)blockDim.x), first_token = tokens, first_page = pages;
    place(base);
    cu_sh[tid] = t0; page_sh[tid] = p0; len_sh[tid] = len;
    if (wg == 0 && p.cu && b < p.B) p.cu[b] = t0;
    __syncthreads();
    for (int i = first_page + wg * (int)blockDim.x + tid; i < pages; i += wgs * (int)blockDim.x) {
      const int s = last_at_most(page_sh, n_here, i);
      p.table[(size_t)(base + s) * p.max_pages + (len_sh[s] + R - 1) / R + i - page_sh[s]] = free_page(i);
    }
    if (p.positions || p.slots)
      for (int t = first_token + wg * (int)blockDim.x + tid; t < tokens; t += wgs * (int)blockDim.x) {
        const int s = last_at_most(cu_sh, n_here, t), row = len_sh[s] + t - cu_sh[s];
        if (p.positions) p.positions[t] = row;
        if (p.slots) {
          const int pg = row / R, had = (len_sh[s] + R - 1) / R;
          int page = -1;
          if (pg < had) {
            page = p.table[(size_t)(base + s) * p.max_pages + pg];
            if (page < 0 || page >= p.n_pages) { page = -1; err = WSVD_E_SHAPE; }
          } else if (pg < p.max_pages) {
            page = free_page(page_sh[s] + pg - had);
          }
          p.slots[t] = page < 0 ? -1 : page * R + row - pg * R;
        }
      }
    if (wgs == 1 || (p.apart && wg == 0)) commit(base);              // (what is read of the lengths later is other sequences')
  }
  if (err) atomicExch(p.err_word, err);
  if (p.apart && wg > 0) return;
  if (wgs > 1 && !p.apart) {
    __syncthreads();
    if (tid == 0) {
      last_sh = atomicAdd(p.counter, 1) == wgs - 1;
      if (last_sh) atomicExch(p.counter, 0);
    }
    __syncthreads();
    if (!last_sh) return;
    const int all_tokens = tokens, all_pages = pages;
    if (p.B > (int)blockDim.x) tokens = pages = 0;
    for (int base = 0; base < p.B; base += (int)blockDim.x) {
      if (p.B > (int)blockDim.x) place(base);
      commit(base);
    }
    tokens = all_tokens; pages = all_pages;
  }
  if (tid == 0) {
    *p.n_free_out = max(n_free - pages, 0);
    if (p.cu) p.cu[p.B] = tokens;
  }
}

// The table entries of sequence b whose pages go: first, and how many.  Of a sequence that is done all, of one that keeps rows those that only
// later rows reach.
struct Gone { int first, n; };
WSVD_DEV Gone pages_gone(const PagesParams& p, int b) {
  if (b >= p.B) return {0, 0};
  const int len = min(max(p.lens[b], 0), p.max_pages * p.R), what = p.what[b];
  const int kept = !p.keeps ? (what != 0 ? 0 : len) : min(max(what, 0), len), first = (kept + p.R - 1) / p.R;
  return {first, (len + p.R - 1) / p.R - first};
}
// Pages that go, in the order of sequences and rows, behind the free list's last.  An entry's place is its number
// among those that go, as long as all are pages; that some are not (a free list that ended left -1) is rare, and then the last
// workgroup to come does it all once more, leaving those out.  (1024 sequences, 99 of them done with 26661 pages: 32 us as one workgroup that
// counts the pages first.)
WSVD_DEV void pages_left_out(const PagesParams& p, int n_free, int& end, int* first_sh, int* from_sh, int* count_sh, Scan& scan) {
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  end = n_free;
  for (int base = 0; base < p.B; base += (int)blockDim.x) {
    const int n_here = min(p.B - base, (int)blockDim.x);
    const Gone gone = pages_gone(p, base + tid);
    __syncthreads();
    from_sh[tid] = gone.first; count_sh[tid] = gone.n;
    __syncthreads();
    // a wave a sequence: its pages counted, and written once it is known where they begin
    auto each = [&](int s, auto put) {
      const int n = __builtin_amdgcn_readfirstlane(count_sh[s]), from = __builtin_amdgcn_readfirstlane(from_sh[s]);
      int before = 0;
      for (int i0 = 0; i0 < n; i0 += 64) {
        const int i = i0 + lane, page = i < n ? p.table[(size_t)(base + s) * p.max_pages + from + i] : -1;
        const bool valid = page >= 0 && page < p.n_pages;
        const unsigned long long m = __ballot(valid);
        if (valid) put(before + __builtin_popcountll(m & ((1ull << lane) - 1)), page);
        before += __builtin_popcountll(m);
      }
      return before;
    };
    for (int s = wave; s < n_here; s += (int)blockDim.x / 64) {
      const int n = each(s, [](int, int) {});
      if (lane == 0) first_sh[s] = n;
    }
    __syncthreads();
    int total;
    const int first = end + scan_exclusive(scan, tid < n_here ? first_sh[tid] : 0, total);
    first_sh[tid] = first;
    __syncthreads();
    for (int s = wave; s < n_here; s += (int)blockDim.x / 64)
      each(s, [&](int i, int page) {
        if (first_sh[s] + i < p.n_pages) put_page(p.free_pages + first_sh[s] + i, page);
      });
    end = min(end + total, p.n_pages + 1);
  }
}
__global__ __launch_bounds__(kSeqs) void k_pages_release(PagesParams p) {
  __shared__ Scan scan;
  __shared__ int first_sh[kSeqs], from_sh[kSeqs], count_sh[kSeqs];
  __shared__ int last_sh, none_sh;
  const int tid = threadIdx.x, wg = blockIdx.x, wgs = gridDim.x;
  const int listed = *p.n_free, n_free = min(max(listed, 0), p.n_pages);
  int end = n_free, none = 0;
  if (tid == 0) none_sh = 0;
  for (int base = 0; base < p.B; base += (int)blockDim.x) {
    const int n_here = min(p.B - base, (int)blockDim.x);
    const Gone gone = pages_gone(p, base + tid);
    int total;
    const int first = end + scan_exclusive(scan, gone.n, total);
    first_sh[tid] = first; from_sh[tid] = gone.first;
    __syncthreads();
    for (int i = end + wg * (int)blockDim.x + tid; i < min(end + total, p.n_pages); i += wgs * (int)blockDim.x) {
      const int s = last_at_most(first_sh, n_here, i);
      const int page = p.table[(size_t)(base + s) * p.max_pages + from_sh[s] + i - first_sh[s]];
      if (page < 0 || page >= p.n_pages) none = 1; else put_page(p.free_pages + i, page);
    }
    end = min(end + total, p.n_pages + 1);           // (that many, or too many)
  }
  __syncthreads();
  if (none) none_sh = 1;
  if (wgs > 1) {
    wait_vmem_done();                                // (what is written once more comes behind what all have written)
    __syncthreads();
    if (tid == 0) {
      if (none_sh) atomicExch(p.counter + 32, 1);
      wait_vmem_done();
      last_sh = atomicAdd(p.counter, 1) == wgs - 1;
      if (last_sh) {
        none_sh = atomicExch(p.counter + 32, 0);
        atomicExch(p.counter, 0);
      }
    }
    __syncthreads();
    if (!last_sh) return;
  }
  __syncthreads();
  if (none_sh) {
    wait_vmem_done();
    pages_left_out(p, n_free, end, first_sh, from_sh, count_sh, scan);
  }
  bool err = end > p.n_pages || listed != n_free;
  for (int b = tid; b < p.B; b += (int)blockDim.x) {
    const int len = p.lens[b], what = p.what[b];
    err = err || (p.keeps && what < 0);
    p.lens_out[b] = p.keeps ? min(max(what, 0), len) : what != 0 ? 0 : len;
  }
  if (err) atomicExch(p.err_word, (int)WSVD_E_SHAPE);
  if (tid == 0) *p.n_free_out = min(end, p.n_pages);
}

bool aligned4(const void* p) { return ((uintptr_t)p & 3u) == 0; }
wsvd_status check_pool(const wsvd_page_pool* c) {
  if (!c || !c->block_table || !c->free_pages) return WSVD_E_NULL;
  if (c->batch < 1 || c->batch > 65536 || c->page_rows < 16 || c->page_rows % 16 != 0 || c->page_rows > 4096 || c->max_pages < 1 || c->n_pages < 1) return WSVD_E_SHAPE;
  if ((int64_t)c->max_pages * c->page_rows > ((int64_t)1 << 27) || c->n_pages > 1 << 24 || (int64_t)c->n_pages * c->page_rows > 0x7FFFFFFF) return WSVD_E_SHAPE;
  if (!aligned4(c->block_table) || !aligned4(c->free_pages)) return WSVD_E_ALIGN;
  return WSVD_OK;
}
PagesParams params_of(const wsvd_ctx* ctx, const wsvd_page_pool* c) {
  PagesParams p = {};
  p.table = c->block_table; p.free_pages = c->free_pages;
  p.B = c->batch; p.R = c->page_rows; p.max_pages = c->max_pages; p.n_pages = c->n_pages;
  p.err_word = ctx->err_word; p.counter = ctx->readers;
  return p;
}

}  // namespace

extern "C" {

wsvd_status wsvd_pages_grow(wsvd_ctx* ctx, const wsvd_page_pool* pool, const int32_t* new_lens, int64_t n_tokens, const int32_t* seq_lens,
                            const int32_t* n_free, int32_t* seq_lens_out, int32_t* n_free_out, int32_t* cu_tokens, int32_t* positions,
                            int32_t* slots, void* hip_stream) {
  if (!ctx || !seq_lens || !n_free || !seq_lens_out || !n_free_out) return WSVD_E_NULL;
  const wsvd_status st = check_pool(pool);
  if (st != WSVD_OK) return st;
  for (const void* x : {(const void*)new_lens, (const void*)seq_lens, (const void*)n_free, (const void*)seq_lens_out, (const void*)n_free_out,
                        (const void*)cu_tokens, (const void*)positions, (const void*)slots})
    if (!aligned4(x)) return WSVD_E_ALIGN;
  if (n_tokens < 0 || n_tokens > ((int64_t)1 << 24) || (!new_lens && n_tokens != pool->batch)) return WSVD_E_SHAPE;
  PagesParams p = params_of(ctx, pool);
  p.lens = seq_lens; p.n_free = n_free; p.what = new_lens; p.lens_out = seq_lens_out; p.n_free_out = n_free_out;
  p.cu = cu_tokens; p.positions = positions; p.slots = slots; p.n_tokens = (int)n_tokens;
  p.apart = seq_lens != seq_lens_out && n_free != n_free_out;
  const PagesLaunch l = pages_launch(pool->batch, n_tokens);
  k_pages_grow<<<l.workgroups, l.threads, 0, (hipStream_t)hip_stream>>>(p);
  return hipGetLastError() == hipSuccess ? WSVD_OK : WSVD_E_HIP;
}

static wsvd_status give_back(wsvd_ctx* ctx, const wsvd_page_pool* pool, const int32_t* what, bool keeps, const int32_t* seq_lens, const int32_t* n_free,
                             int32_t* seq_lens_out, int32_t* n_free_out, void* hip_stream) {
  if (!ctx || !what || !seq_lens || !n_free || !seq_lens_out || !n_free_out) return WSVD_E_NULL;
  const wsvd_status st = check_pool(pool);
  if (st != WSVD_OK) return st;
  for (const void* x : {(const void*)what, (const void*)seq_lens, (const void*)n_free, (const void*)seq_lens_out, (const void*)n_free_out})
    if (!aligned4(x)) return WSVD_E_ALIGN;
  PagesParams p = params_of(ctx, pool);
  p.lens = seq_lens; p.n_free = n_free; p.what = what; p.keeps = keeps; p.lens_out = seq_lens_out; p.n_free_out = n_free_out;
  const PagesLaunch l = pages_launch(pool->batch, (int64_t)pool->batch * pool->max_pages / 16);
  k_pages_release<<<l.workgroups, l.threads, 0, (hipStream_t)hip_stream>>>(p);
  return hipGetLastError() == hipSuccess ? WSVD_OK : WSVD_E_HIP;
}
wsvd_status wsvd_pages_release(wsvd_ctx* ctx, const wsvd_page_pool* pool, const int32_t* done, const int32_t* seq_lens, const int32_t* n_free,
                               int32_t* seq_lens_out, int32_t* n_free_out, void* hip_stream) {
  return give_back(ctx, pool, done, false, seq_lens, n_free, seq_lens_out, n_free_out, hip_stream);
}
wsvd_status wsvd_pages_keep(wsvd_ctx* ctx, const wsvd_page_pool* pool, const int32_t* kept_lens, const int32_t* seq_lens, const int32_t* n_free,
                            int32_t* seq_lens_out, int32_t* n_free_out, void* hip_stream) {
  return give_back(ctx, pool, kept_lens, true, seq_lens, n_free, seq_lens_out, n_free_out, hip_stream);
}

}  // extern "C"
