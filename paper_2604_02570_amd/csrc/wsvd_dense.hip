// Dense layers next to latent ones: rotary embedding with the append to a paged cache of plain keys and values, and the
// attention of one new token per sequence over it.
#include <type_traits>
#include "wsvd_attn_common.h"
#include "wsvd_dense.h"

namespace {

// ONCE: data that is read or written once and need not stay in the caches
template <bool ONCE, class V>
WSVD_DEV V load_row(const V* p) { return ONCE ? __builtin_nontemporal_load(p) : *p; }
template <bool ONCE, class V>
WSVD_DEV void store_row(V* p, V v) { if (ONCE) __builtin_nontemporal_store(v, p); else *p = v; }

// ---------------------------------------------------------------- append
// Rotation of the new tokens' queries and keys (dims i and i + d/2 turned by position * inv_freq[i]) and their keys and values
// stored in the pages.  Bound: memory, every element read and written once (16 prompts of 2048 tokens and less, 32 heads of 128:
// 1.03 GB in 183 us, 5.6 TB/s, where a copy of 1 GiB reaches 4.9 to 5.2); few tokens: three dependent loads (32 tokens of 28 / 4
// heads: 3.7 us on the GPU).
//   A wave finds its token's sequence, row and page, and its lanes the token's d / 2 angles, once for all heads: in 64 bits as
// far as whole turns go (an fp32 product of a position of 1e5 would be off by 6e-3 radians), the sine and cosine of what is
// left in 32.  Then the workgroup goes over the (token, head) pairs, 16 bytes of each half per thread.
// ONCE: nothing of it need stay in the caches.
template <class T, int D, int TOK, bool ONCE>
__global__ __launch_bounds__(256) void k_dense_append(DenseAppendParams p) {
  constexpr int HALF = D / 2, PER = D / 16;          // threads per (token, head)
  __shared__ float cs[TOK][2][HALF];
  __shared__ int64_t slot_sh[TOK];                   // row in the pools of head 0, in rows; -1: nothing is stored
  __shared__ int live_sh[TOK];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t t0 = (int64_t)blockIdx.x * TOK;
  if (wave < TOK) {
    const int t = (int)t0 + wave;
    int b = p.B, row = 0;
    if (t < p.n_tokens) {
      b = p.cu ? dense_sequence_of(p.cu, p.B, t, lane) : t;
      b = __builtin_amdgcn_readfirstlane(b);
    }
    const bool live = b < p.B && (!p.cu || t >= p.cu[b]);
    int64_t slot = -1;
    if (live) {
      row = p.pages.seq_lens[b] - 1 - (p.cu ? p.cu[b + 1] - 1 - t : 0);
      const int pos = p.positions ? p.positions[t] : row;
      if (row < 0 || row >= (int64_t)p.pages.max_pages * p.pages.page_rows) {
        if (lane == 0) atomicExch(p.err_word, (int)(row < 0 ? WSVD_E_SHAPE : WSVD_E_CAPACITY));
      } else {
        const int page = p.pages.block_table[(size_t)b * p.pages.max_pages + row / p.pages.page_rows];
        if (page < 0 || page >= p.pages.n_pages) {
          if (lane == 0) atomicExch(p.err_word, (int)WSVD_E_SHAPE);
        } else {
          slot = (int64_t)page * p.Hkv * p.pages.page_rows + row % p.pages.page_rows;
        }
      }
      if (p.inv_freq && lane < HALF) {
        const double turns = (double)pos * p.inv_freq[lane] * 0.15915494309189533576888376337251;   // / 2 pi
        const float x = (float)(turns - __builtin_rint(turns));
        float sn, co;
        sincospif(2.f * x, &sn, &co);
        cs[wave][0][lane] = co;
        cs[wave][1][lane] = sn;
      }
    }
    if (lane == 0) { slot_sh[wave] = slot; live_sh[wave] = live; }
  }
  __syncthreads();
  const int heads = p.Hq + 2 * p.Hkv, n = heads * PER;
  for (int e = tid; e < TOK * n; e += 256) {
    const int w = TOK > 1 ? e / n : 0, i = TOK > 1 ? e - w * n : e;
    const int h = i / PER, part = i % PER;
    if (!live_sh[w]) continue;
    const int64_t t = t0 + w;
    const int kind = h < p.Hq ? 0 : h < p.Hq + p.Hkv ? 1 : 2;
    const int hh = kind == 0 ? h : kind == 1 ? h - p.Hq : h - p.Hq - p.Hkv;
    const uint16_t* src = kind == 0 ? p.q + t * p.q_ld : kind == 1 ? p.k + t * p.k_ld : p.v + t * p.v_ld;
    if (kind == 0 && !p.q_out) continue;
    src += hh * D + part * 8;
    v4i a = load_row<ONCE>((const v4i*)src), b = load_row<ONCE>((const v4i*)(src + HALF));
    if (p.inv_freq && kind < 2) {
      v4i ra, rb;
#pragma unroll
      for (int x = 0; x < 4; x++) {
        const int c = part * 8 + 2 * x;
        const float c0 = cs[w][0][c], c1 = cs[w][0][c + 1], s0 = cs[w][1][c], s1 = cs[w][1][c + 1];
        const float a0 = dense_low<T>(a[x]), a1 = dense_high<T>(a[x]), b0 = dense_low<T>(b[x]), b1 = dense_high<T>(b[x]);
        ra[x] = (int)dense_pack<T>(a0 * c0 - b0 * s0, a1 * c1 - b1 * s1);
        rb[x] = (int)dense_pack<T>(b0 * c0 + a0 * s0, b1 * c1 + a1 * s1);
      }
      a = ra; b = rb;
    }
    if (kind == 0) {
      uint16_t* dst = p.q_out + t * p.q_out_ld + hh * D + part * 8;
      store_row<ONCE>((v4i*)dst, a); store_row<ONCE>((v4i*)(dst + HALF), b);
      continue;
    }
    if (kind == 1 && p.k_out) {
      uint16_t* dst = p.k_out + t * p.k_out_ld + hh * D + part * 8;
      store_row<ONCE>((v4i*)dst, a); store_row<ONCE>((v4i*)(dst + HALF), b);
    }
    if (slot_sh[w] >= 0) {
      uint16_t* dst = (kind == 1 ? p.pages.k : p.pages.v) + (slot_sh[w] + (int64_t)hh * p.pages.page_rows) * D + part * 8;
      store_row<ONCE>((v4i*)dst, a); store_row<ONCE>((v4i*)(dst + HALF), b);
    }
  }
}

// ---------------------------------------------------------------- decode attention
// One new token per sequence over its pages: per (sequence, kv head) one pass over its rows with the running maximum and sum of the
// softmax, for all heads of the group at once.
//   S^T [16 rows x heads] = K q^T, O^T [d x heads] += V^T P^T on 16x16x32 products.  The heads are the 16 columns, so a lane owns one
// head and 4 of 16 rows; its 8 weights of 32 rows are, as they lie, its part of the second product's operand (the contraction over
// rows may run in any order, V is taken in that one).  V's operand is made in registers: a lane loads 8 rows' same dims in whole
// lines and pairs them up with one byte permute per two elements.
// Bound: HBM.  32 x 8192 rows of 4 heads of 128 (537 MB): 86.8 us, 6.2 TB/s (a kernel that only reads them: 81 us); 640 rows of 32
// heads (10.5 MB): 7.8 us, of which 3.3 are a launch that finds no row, and the rest a CU's stream of 74 GB/s.
// A workgroup's place: sequence, chunk of it, chunks it has, its length, the rows of a chunk; false for a workgroup that has none.
struct DensePlace { int b, chunk, n_chunks, len, rows; };

WSVD_DEV int dense_length(const DenseDecodeParams& p, int b) { return b < p.B ? min(max(p.pages.seq_lens[b], 0), p.max_len) : 0; }

// Every wave finds its workgroup's place from the lengths of all sequences: the most units a chunk may take (dense_units), the
// sequences' chunks, and their prefix sums.  Where no sequence can be long enough to be cut, that is its number (1024 sequences of up to
// 100 rows, 8 heads of 64: 92 -> 37 us).
WSVD_DEV bool dense_place(const DenseDecodeParams& p, int idx, int lane, DensePlace& at) {
  if (p.alone) {
    at = {idx, 0, 1, __builtin_amdgcn_readfirstlane(dense_length(p, idx)), p.max_len};
    return true;
  }
  const int mine = dense_length(p, lane);            // (the first 64 sequences' lengths are read once)
  auto length = [&](int base) { return base == 0 ? mine : dense_length(p, base + lane); };
  int total = 0, most = 0;
  for (int base = 0; base < p.B; base += 64) {
    const int u = dense_units_of(length(base));
    total += wave_sum_int(u);
    most = max(most, wave_max_int(u));
  }
  const int units = dense_units(total, most, p.B, p.target, p.alone_units, p.min_units, [&](int units) {
    return wave_sum_int(lane < p.B ? dense_chunks(dense_units_of(mine), units) : 0);
  });
  int first = 0;
  for (int base = 0; base < p.B; base += 64) {
    const int len = length(base), u = dense_units_of(len), n = base + lane < p.B ? dense_chunks(u, units) : 0;
    const int end = first + wave_prefix_int(n);
    const unsigned long long m = __ballot(end > idx);
    if (m) {
      const int l = __builtin_ctzll(m);
      at.b = base + l;
      at.n_chunks = __builtin_amdgcn_readlane(n, l);
      at.chunk = idx - (__builtin_amdgcn_readlane(end, l) - at.n_chunks);
      at.len = __builtin_amdgcn_readlane(len, l);
      at.rows = (__builtin_amdgcn_readlane(u, l) + at.n_chunks - 1) / at.n_chunks * kDenseUnit;
      return true;
    }
    first = __builtin_amdgcn_readlane(end, 63);
  }
  return false;
}

WSVD_DEV float quarters_max(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return halves_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
WSVD_DEV float quarters_sum(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return halves_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// ---------------------------------------------------------------- joining the chunks of a sequence
// A chunk's partial results (maximum, sum and un-normalised row of every head of the group) go to the workgroup of the last chunk
// of its group of kDenseFold, and where there are several groups, their results to the workgroup of the sequence's last chunk: as
// words {value, tag}, as the latent attention's splits hand theirs over (attn_merge_splits: who waits has a higher workgroup
// number than those it waits for, and the wait is bounded).  The fold is in the order of the chunks.  Words are cleared
// where they are read.  (A join by a second launch: 3.4 us more for 2 chunks of 32 heads; by the workgroup that draws the last
// ticket: 2.9.)
WSVD_DEV unsigned long long* dense_part(const DenseDecodeParams& p, int chunk, int kv, int d) {
  return p.parts + ((size_t)chunk * p.Hkv + kv) * p.G * (d + 2);
}
WSVD_DEV void dense_push(unsigned long long* to, float v) { __hip_atomic_store(to, split_word(v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

WSVD_DEV unsigned long long dense_word(const unsigned long long* at) { return __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
WSVD_DEV void dense_clear(unsigned long long* at) { __hip_atomic_store(at, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// What a workgroup holds of its chunk, or of its group's chunks: by output e = head * D + dim, as many as a thread has.
template <int D, int NW>
struct DensePartial {
  static constexpr int N = 16 * D / (64 * NW);
  float M[N], L[N], U[N];
};

// Takes the partial results of n < kDenseFold chunks, `step` apart from `chunk` on, in front of its own.
template <int D, int NW>
WSVD_DEV void dense_fold(const DenseDecodeParams& p, int chunk, int step, int n, int kv, DensePartial<D, NW>& own, float* sh /* [2][kDenseFold][16] */) {
  constexpr int N = DensePartial<D, NW>::N, AT_ONCE = N < 4 ? N : 4, NF = kDenseFold - 1;
  static_assert(NF * 16 <= 64 * NW, "a thread for every chunk's maxima");
  const int tid = threadIdx.x, G = p.G;
  unsigned long long* const part = dense_part(p, chunk, kv, D);
  const size_t stride = (size_t)step * p.Hkv * G * (D + 2);
  float *m_sh = sh, *l_sh = sh + kDenseFold * 16;
  // All words of a thread are asked for at once, and again until all have come: its outputs' rows (four outputs at a time), and for
  // n * G threads a chunk's maximum and sum.  (One output after the other: 8 us more for 60 chunks of 16 heads of 128; a
  // look at the sums alone first, so that the others are asked for once: 1.1 us more for 8 chunks of them.)
  bool has = tid < n * G, came = true;
  const int mk = has ? tid / G : 0, mg = has ? tid - mk * G : 0;
  const unsigned long long none = split_word(0.f);
#pragma unroll
  for (int i0 = 0; i0 < N; i0 += AT_ONCE) {
    if (i0 > 0 && i0 * 64 * NW >= G * D) break;
    unsigned long long* const ml = part + mk * stride + mg * (D + 2);
    unsigned long long w[AT_ONCE][NF], wm = none, wl = none;
    bool all = false;
    for (int budget = 1 << 14; budget && !all; budget--) {
      if (i0 == 0 && has) { wm = dense_word(ml); wl = dense_word(ml + 1); }
#pragma unroll
      for (int i = 0; i < AT_ONCE; i++) {
        const uint32_t e = tid + (i0 + i) * 64 * NW, off = e / D * (D + 2) + 2 + e % D;
#pragma unroll
        for (int k = 0; k < NF; k++) w[i][k] = k < n && (int)e < G * D ? dense_word(part + k * stride + off) : none;
      }
      all = (uint32_t)(wm >> 32) == kSplitTag && (uint32_t)(wl >> 32) == kSplitTag;
#pragma unroll
      for (int i = 0; i < AT_ONCE; i++)
#pragma unroll
        for (int k = 0; k < NF; k++) all = all && (uint32_t)(w[i][k] >> 32) == kSplitTag;
      if (!all) __builtin_amdgcn_s_sleep(1);
    }
    came = came && all;
    if (i0 == 0) {
      if (has) {
        m_sh[mk * 16 + mg] = __uint_as_float((uint32_t)wm);
        l_sh[mk * 16 + mg] = __uint_as_float((uint32_t)wl);
        dense_clear(ml);
        dense_clear(ml + 1);
      }
      __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < AT_ONCE; i++) {
      const int e = tid + (i0 + i) * 64 * NW, g = e / D;
      if (e < G * D) {
        const uint32_t off = g * (D + 2) + 2 + e % D;
        float M = own.M[i0 + i], L = 0.f, U = 0.f;
        for (int k = 0; k < n; k++) M = fmaxf(M, m_sh[k * 16 + g]);
#pragma unroll
        for (int k = 0; k < NF; k++)
          if (k < n) {
            const float m = m_sh[k * 16 + g], f = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - M);  // (nothing seen: l and u are 0, or NaN)
            L += l_sh[k * 16 + g] * f;
            U += dense_scaled(__uint_as_float((uint32_t)w[i][k]), f);
            dense_clear(part + k * stride + off);
          }
        const float f = own.M[i0 + i] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(own.M[i0 + i] - M);
        own.L[i0 + i] = L + own.L[i0 + i] * f;
        own.U[i0 + i] = U + dense_scaled(own.U[i0 + i], f);
        own.M[i0 + i] = M;
      }
    }
  }
  if (!came) atomicExch(p.err_word, (int)WSVD_E_HIP);              // never seen; keeps the wait finite
  __syncthreads();
}

template <int D>
struct DenseTile {
  v4i k[2][D / 32];                                  // 16 rows each, as they lie in memory
  typedef int Piece __attribute__((ext_vector_type(D / 32)));
  Piece v[8];                                        // row 4 quarter + i of either half, D / 16 dims
};

// ONCE: the rows are asked for as data that is read once and need not stay in the caches.
template <class T, int D, int NW, bool ONCE>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_dense_decode(DenseDecodeParams p) {
  constexpr int NK = D / 32, NJ = D / 16;
  extern __shared__ __attribute__((aligned(256))) float o_sh[];      // a granule pair's keys for each wave; at the end [NW][G][D]
  __shared__ float m_sh[NW][16], l_sh[NW][16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, qd = lane >> 4;
  const int kv = blockIdx.x % p.Hkv, idx = blockIdx.x / p.Hkv;
  DensePlace at;
  if (!dense_place(p, idx, lane, at)) return;
  if (at.chunk == 0 && kv == 0 && threadIdx.x == 0 && p.pages.seq_lens[at.b] > p.max_len) atomicExch(p.err_word, (int)WSVD_E_SHAPE);
  const int G = p.G;
  const int first = at.chunk * at.rows, end = min(at.len, first + at.rows);
  const int n_tiles = (max(end - first, 0) + 31) >> 5;

  // queries as the second operand: column c = head of the group
  v4i q[NK];
  {
    const uint16_t* qp = p.q + (int64_t)at.b * p.q_ld + (kv * G + min(c, G - 1)) * D + qd * 8;
#pragma unroll
    for (int j = 0; j < NK; j++) {
      const v4i x = *(const v4i*)(qp + j * 32);
#pragma unroll
      for (int i = 0; i < 4; i++) q[j][i] = c < G ? x[i] : 0;
    }
  }
  // Where the wave's next 32 tiles lie, a lane for each half of one: its pages are looked up side by side, and what a tile's
  // requests wait for is two lane reads.
  const int* table = p.pages.block_table + (size_t)at.b * p.pages.max_pages;
  const int last_granule = (at.len - 1) >> 4;
  bool bad = false;
  uint32_t at_low = 0, at_high = 0;
  auto look_up = [&](int t) {
    const int granule = min((first >> 4) + 2 * (t + NW * (lane >> 1)) + (lane & 1), last_granule);
    const int pg = dense_page_index(granule, p.pages.page_magic);
    const int page = dense_page(table[pg], p.pages.n_pages, bad);
    const uint64_t at = dense_pool_row(page, granule, pg, kv, p.Hkv, p.pages.page_rows) * D;
    at_low = (uint32_t)at; at_high = (uint32_t)(at >> 32);
  };
  auto load = [&](DenseTile<D>& tile, int i) {       // i: the tile's number among those looked up
#pragma unroll
    for (int g = 0; g < 2; g++) {
      const uint64_t base = (uint64_t)(uint32_t)__builtin_amdgcn_readlane(at_low, 2 * i + g) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane(at_high, 2 * i + g) << 32;
      const uint16_t *kp = p.pages.k + base, *vp = p.pages.v + base;
#pragma unroll
      for (int j = 0; j < NK; j++) tile.k[g][j] = load_row<ONCE>((const v4i*)(kp + j * 512 + lane * 8));
#pragma unroll
      for (int i2 = 0; i2 < 4; i2++)
        tile.v[4 * g + i2] = load_row<ONCE>((const typename DenseTile<D>::Piece*)(vp + (4 * qd + i2) * D + c * NJ));
    }
  };
  // A wave's keys go through LDS of its own: requested in whole lines (asked for as the product's operand, 16 rows of 64 bytes per
  // request, they cost the CU's address pipeline four times as much: 640 rows in two chunks 14.3 us against 11.8, when it was tried)
  // and read back by key, the 16-byte pieces of a row permuted so that neither side meets a bank twice.
  const uint32_t k_lds = lds_address(o_sh) + wave * (64 * D);
  uint32_t k_put[NK], k_get[NK];
#pragma unroll
  for (int j = 0; j < NK; j++) {
    const int row = (j * 64 + lane) / (D / 8), piece = lane % (D / 8);
    k_put[j] = k_lds + row * 2 * D + (piece ^ (D == 128 ? row : row >> 1)) * 16;
    k_get[j] = k_lds + c * 2 * D + ((4 * j + qd) ^ (D == 128 ? c : c >> 1)) * 16;
  }
  typedef __attribute__((address_space(3))) v4i lds_v4i;
  float m = -INFINITY, l = 0.f;
  v4f o[NJ];
#pragma unroll
  for (int j = 0; j < NJ; j++) o[j] = v4f{0.f, 0.f, 0.f, 0.f};

  bool odd = false;                                  // careful: infinite values and NaN alone, or all but those (see below)
  auto attend = [&](DenseTile<D>& tile, int t, auto careful) {
#pragma clang fp contract(off)                       // (a score is the same number against the limit and in its weight)
    constexpr bool CAREFUL = decltype(careful)::value;
    const int r0 = first + t * 32;
    float s[8];
#pragma unroll
    for (int g = 0; g < 2; g++)
#pragma unroll
      for (int j = 0; j < NK; j++) *(lds_v4i*)(uintptr_t)(k_put[j] + g * 32 * D) = tile.k[g][j];
#pragma unroll
    for (int g = 0; g < 2; g++) {
      v4f x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < NK; j++) x = T::mfma16(*(const lds_v4i*)(uintptr_t)(k_get[j] + g * 32 * D), q[j], x);
#pragma unroll
      for (int i = 0; i < 4; i++) s[4 * g + i] = x[i] * p.c_scale;
    }
    if (r0 + 32 > end) {                             // rows behind the sequence's end: no weight, and no value that could be NaN
#pragma unroll
      for (int i = 0; i < 8; i++) {
        const bool out = r0 + 16 * (i >> 2) + 4 * qd + (i & 3) >= end;
        s[i] = out ? -INFINITY : s[i];
#pragma unroll
        for (int j = 0; j < NK; j++) tile.v[i][j] = out ? 0 : tile.v[i][j];
      }
    }
    float most = s[0];
#pragma unroll
    for (int i = 1; i < 8; i++) most = fmaxf(most, s[i]);
    if (__ballot(most - m > T::kTop)) {              // (see the element types)
      const float top = quarters_max(most), low = top - T::kRaise;
      const float mn = fmaxf(m, top - low > T::kTop ? top : low);    // (steps of 16, between scores of 2^27 and 2^28)
      const float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
      l *= keep;
#pragma unroll
      for (int j = 0; j < NJ; j++)
#pragma unroll
        for (int i = 0; i < 4; i++) o[j][i] = CAREFUL ? dense_scaled(o[j][i], keep) : o[j][i] * keep;
      m = mn;
    }
    if (CAREFUL) {
#pragma unroll
      for (int i = 0; i < 8; i++)
#pragma unroll
        for (int j = 0; j < NK; j++) tile.v[i][j] &= (int)(odd ? dense_odd<T>((uint32_t)tile.v[i][j]) : ~dense_odd<T>((uint32_t)tile.v[i][j]));
    }
    const float ref = m == -INFINITY ? 0.f : m;
    float w[8];
#pragma unroll
    for (int i = 0; i < 8; i++) { w[i] = __builtin_amdgcn_exp2f(s[i] - ref); l += w[i]; }
    if (CAREFUL && odd) {
#pragma unroll
      for (int i = 0; i < 8; i++) w[i] = s[i] == -INFINITY ? 0.f : 1.f;
    }
    // weights as a pair of 16-bit numbers (bf16: off by at most 2^-17 of the weight; f16: by 2^-23 of it or 2^-36 of the reference's)
    v4i hi, lo;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const uint32_t h = dense_pack<T>(w[2 * i], w[2 * i + 1]), rest = dense_pack<T>(w[2 * i] - dense_low<T>(h), w[2 * i + 1] - dense_high<T>(h));
      hi[i] = (int)h;
      lo[i] = (int)(CAREFUL && odd ? h : rest);
    }
#pragma unroll
    for (int j = 0; j < NJ; j++) {
      v4i a;
#pragma unroll
      for (int i = 0; i < 4; i++)
        a[i] = (int)__builtin_amdgcn_perm((uint32_t)tile.v[2 * i + 1][j >> 1], (uint32_t)tile.v[2 * i][j >> 1], (j & 1) ? 0x07060302u : 0x05040100u);
      o[j] = T::mfma16(a, hi, o[j]);
      o[j] = T::mfma16(a, lo, o[j]);
    }
  };
  constexpr std::true_type yes{};
  constexpr std::false_type no{};
  for (int t = wave; t < n_tiles; t += 32 * NW) {    // 32 tiles of the wave
    look_up(t);
    const int n = min(32, (n_tiles - t + NW - 1) / NW);
    DenseTile<D> t0, t1;
    load(t0, 0);
    int i = 0;
    for (; i + 2 < n; i += 2) {
      load(t1, i + 1);
      attend(t0, t + NW * i, no);
      load(t0, i + 2);
      attend(t1, t + NW * (i + 1), no);
    }
    if (i + 1 < n) load(t1, i + 1);
    attend(t0, t + NW * i, no);
    if (i + 1 < n) attend(t1, t + NW * (i + 1), no);
  }
  // A value that is infinite meets the low part of its weight too, which may be 0 or less and makes it no number, and a weight that the
  // type or 32 bits round to 0.  Where something is none, all once more, a tile at a time: first such values alone, with 1 for every
  // weight (any weight leaves infinite what is infinite) but 0 under a score of -inf, then the others, as exactly as ever.
  float zero = 0.f;                                  // NaN where a value is infinite or none
#pragma unroll
  for (int j = 0; j < NJ; j++)
#pragma unroll
    for (int i = 0; i < 4; i++) zero = fmaf(o[j][i], 0.f, zero);
  if (__ballot(zero != 0.f && c < G)) {              // (columns without a head may hold anything)
#pragma unroll
    for (int j = 0; j < NJ; j++) o[j] = v4f{0.f, 0.f, 0.f, 0.f};
    odd = true;
#pragma unroll 1
    for (int pass = 0; pass < 2; pass++, odd = false) {
      m = -INFINITY; l = 0.f;
#pragma unroll 1
      for (int t = wave; t < n_tiles; t += NW) {
        DenseTile<D> tile;
        look_up(t);
        load(tile, 0);
        attend(tile, t, yes);
      }
    }
  }
  if (__ballot(bad) && lane == 0) atomicExch(p.err_word, (int)WSVD_E_SHAPE);
  l = quarters_sum(l);
  __syncthreads();                                   // (the keys' LDS becomes the accumulators')
  if (c < G) {
    if (qd == 0) { m_sh[wave][c] = m; l_sh[wave][c] = l; }
    // (A head's dims start 4 c further on in its row, since the heads' rows begin at one bank: one row of 16 heads 7.1 -> 5.8 us, 640
    // rows 10.1 -> 8.7, 15127 rows 21.7 -> 20.5.)
#pragma unroll
    for (int i = 0; i < 4; i++)
#pragma unroll
      for (int j = 0; j < NJ; j += 4)
        *(v4f*)(o_sh + (wave * G + c) * D + ((NJ * (4 * qd + i) + j + 4 * c) & (D - 1))) = v4f{o[j][i], o[j + 1][i], o[j + 2][i], o[j + 3][i]};
  }
  __syncthreads();
  DensePartial<D, NW> r;
#pragma unroll
  for (int i = 0; i < DensePartial<D, NW>::N; i++) {
    const int e = threadIdx.x + i * 64 * NW, g = e / D, x = e % D;
    r.M[i] = -INFINITY; r.L[i] = r.U[i] = 0.f;
    if (e < G * D) {
#pragma unroll
      for (int w = 0; w < NW; w++) r.M[i] = fmaxf(r.M[i], m_sh[w][g]);
#pragma unroll
      for (int w = 0; w < NW; w++) {
        const float k = m_sh[w][g] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_sh[w][g] - r.M[i]);
        r.L[i] += l_sh[w][g] * k;
        r.U[i] += dense_scaled(o_sh[(w * G + g) * D + ((x + 4 * g) & (D - 1))], k);
      }
    }
  }
  if (at.n_chunks > 1) {
    const int c0 = idx - at.chunk, group = at.chunk / kDenseFold, n_groups = (at.n_chunks + kDenseFold - 1) / kDenseFold;
    const bool last = at.chunk == at.n_chunks - 1, ends = last || at.chunk % kDenseFold == kDenseFold - 1;
    __syncthreads();
    const int folds = !ends ? 0 : last && n_groups > 1 ? 2 : 1;
#pragma unroll 1
    for (int i = 0; i < folds; i++)                  // the group's chunks, then the groups' results
      dense_fold<D, NW>(p, i == 0 ? c0 + group * kDenseFold : c0 + kDenseFold - 1, i == 0 ? 1 : kDenseFold,
                    i == 0 ? at.chunk % kDenseFold : n_groups - 1, kv, r, o_sh);
    if (!last) {
      unsigned long long* const part = dense_part(p, idx, kv, D);
#pragma unroll
      for (int i = 0; i < DensePartial<D, NW>::N; i++) {
        const int e = threadIdx.x + i * 64 * NW, g = e / D, x = e % D;
        if (e < G * D) {
          dense_push(part + g * (D + 2) + 2 + x, r.U[i]);
          if (x == 0) { dense_push(part + g * (D + 2), r.M[i]); dense_push(part + g * (D + 2) + 1, r.L[i]); }
        }
      }
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < DensePartial<D, NW>::N; i++) {
    const int e = threadIdx.x + i * 64 * NW;
    if (e < G * D) p.out[((int64_t)at.b * p.Hkv * G + kv * G) * D + e] = (uint16_t)dense_pack<T>(r.L[i] == 0.f ? 0.f : r.U[i] / r.L[i], 0.f);
  }
}

template <class T, int D, int TOK>
hipError_t launch_append_form(const DenseAppendParams& p, hipStream_t s) {
  const int wgs = (p.n_tokens + TOK - 1) / TOK;
  // Calls that move 100 MB and more do not leave their rows in the last-level cache for whoever reads them next: 16 x ~1150 tokens of
  // 32 heads (1.03 GB) 205 -> 179 us; 4 x 300 of 32 / 8 (17 MB) 8.0 -> 8.3 the other way.
  if ((int64_t)p.n_tokens * (2 * p.Hq + 4 * p.Hkv) * D * 2 >= 100000000) k_dense_append<T, D, TOK, true><<<wgs, 256, 0, s>>>(p);
  else k_dense_append<T, D, TOK, false><<<wgs, 256, 0, s>>>(p);
  return hipGetLastError();
}
template <class T, int D>
hipError_t launch_append(const DenseAppendParams& p, hipStream_t s) {
  const int tokens = dense_append_tokens(p.n_tokens, (p.Hq + 2 * p.Hkv) * (D / 16));
  return tokens == 1 ? launch_append_form<T, D, 1>(p, s) : tokens == 2 ? launch_append_form<T, D, 2>(p, s) : launch_append_form<T, D, 4>(p, s);
}
template <class T, int D, int NW, bool ONCE>
hipError_t launch_decode_form(const DenseDecodeParams& p, hipStream_t s) {
  constexpr int LDS = NW * D * 4 * 16;               // 32 keys a wave, and later 16 rows of fp32
  static LdsLimit limit;
  if (LDS + NW * 16 * 8 > 65536) {
    const hipError_t e = wsvd_raise_lds(limit, (const void*)k_dense_decode<T, D, NW, ONCE>, LDS);
    if (e != hipSuccess) return e;
  }
  k_dense_decode<T, D, NW, ONCE><<<(unsigned)dense_decode_workgroups(p.B, p.Hkv, p.target, p.alone != 0), 64 * NW, LDS, s>>>(p);
  return hipGetLastError();
}
template <class T, int D, bool ONCE>
hipError_t launch_decode_waves(const DenseDecodeParams& p, hipStream_t s) {
  return p.waves == 8 ? launch_decode_form<T, D, 8, ONCE>(p, s) : p.waves == 4 ? launch_decode_form<T, D, 4, ONCE>(p, s) : launch_decode_form<T, D, 2, ONCE>(p, s);
}
template <class T, int D>
hipError_t launch_decode(const DenseDecodeParams& p, hipStream_t s) {
  // Rows of 100 MB and more do not stay in the last-level cache (256 MB) until they are read again, and reading them as data that
  // does is slower: 32 x 8192 rows of 4 heads (537 MB) 100 us against 90, 8 x 1000 of 32 (131 MB) 27.8 against 25.3; 74 MB over and
  // over out of that cache 17.9 against 20.
  const bool once = (int64_t)p.B * p.max_len * p.Hkv * D * 4 >= 100000000;
  return once ? launch_decode_waves<T, D, true>(p, s) : launch_decode_waves<T, D, false>(p, s);
}

}  // namespace

hipError_t wsvd_launch_dense_append(const DenseAppendParams& p, int dtype, int d, hipStream_t s) {
  if (dtype == WSVD_BF16) return d == 128 ? launch_append<DenseBf16, 128>(p, s) : launch_append<DenseBf16, 64>(p, s);
  return d == 128 ? launch_append<DenseF16, 128>(p, s) : launch_append<DenseF16, 64>(p, s);
}
hipError_t wsvd_launch_dense_decode(const DenseDecodeParams& p, int dtype, int d, hipStream_t s) {
  if (dtype == WSVD_BF16) return d == 128 ? launch_decode<DenseBf16, 128>(p, s) : launch_decode<DenseBf16, 64>(p, s);
  return d == 128 ? launch_decode<DenseF16, 128>(p, s) : launch_decode<DenseF16, 64>(p, s);
}
