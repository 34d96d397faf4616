// Shared by the decode attentions of dense layers, over 16-bit pages and over 8-bit ones: a workgroup's part of the sequences, found
// from lengths that only the device knows, and the join of the parts of a sequence.
#pragma once
#include "wsvd_attn_common.h"
#include "wsvd_dense.h"

namespace {

// ONCE: data that is read or written once and need not stay in the caches
template <bool ONCE, class V>
WSVD_DEV V load_row(const V* p) { return ONCE ? __builtin_nontemporal_load(p) : *p; }
template <bool ONCE, class V>
WSVD_DEV void store_row(V* p, V v) { if (ONCE) __builtin_nontemporal_store(v, p); else *p = v; }

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
  at.chunk = idx - first; at.rows = units;           // behind the last chunk, and the units of one
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
// Of a sequence whose chunks others join (dense_finish): the rows of all its n chunks, and behind them a head's maxima and its sums, chunk by
// chunk, so that lanes read them side by side (with all in a chunk's words, as above, 64 chunks of 8 heads of 64: 10.9 us in place of 10.4).
struct DensePartWords { unsigned long long *row, *max; };            // max: and n further on the sum
WSVD_DEV DensePartWords dense_many(const DenseDecodeParams& p, int c0, int n, int chunk, int kv, int g, int d) {
  unsigned long long* const first = p.parts + (size_t)c0 * p.Hkv * p.G * (d + 2);
  return {first + (((size_t)chunk * p.Hkv + kv) * p.G + g) * d, first + (size_t)n * p.Hkv * p.G * d + (size_t)(kv * p.G + g) * 2 * n + chunk};
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

// The waves' results in LDS ([NW][G][D], a head's dims 4 of its number further on in their row) joined, and with those of the other chunks
// of the sequence; the last chunk's workgroup writes the output: to(e) is where output e = head * D + dim goes.  WHOLE, where not
// 0: the chunks of sequences of more than so many are all handed over, for others to join.
template <class T, int D, int NW, int WHOLE = 0, class To>
WSVD_DEV void dense_finish(const DenseDecodeParams& p, const DensePlace& at, int idx, int kv, float* o_sh, const float (*m_sh)[16], const float (*l_sh)[16], To to) {
  const int G = p.G;
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
  const bool apart = WHOLE && at.n_chunks > WHOLE;
  if (at.n_chunks > 1) {
    const int c0 = idx - at.chunk, group = at.chunk / kDenseFold, n_groups = (at.n_chunks + kDenseFold - 1) / kDenseFold;
    const bool last = at.chunk == at.n_chunks - 1, ends = last || at.chunk % kDenseFold == kDenseFold - 1;
    __syncthreads();
    const int folds = !ends || apart ? 0 : last && n_groups > 1 ? 2 : 1;
#pragma unroll 1
    for (int i = 0; i < folds; i++)                  // the group's chunks, then the groups' results
      dense_fold<D, NW>(p, i == 0 ? c0 + group * kDenseFold : c0 + kDenseFold - 1, i == 0 ? 1 : kDenseFold,
                    i == 0 ? at.chunk % kDenseFold : n_groups - 1, kv, r, o_sh);
    if (!last || apart) {
      const DensePartWords at_part = apart ? dense_many(p, c0, at.n_chunks, at.chunk, kv, 0, D) : DensePartWords{};
      unsigned long long* const part = dense_part(p, idx, kv, D);
#pragma unroll
      for (int i = 0; i < DensePartial<D, NW>::N; i++) {
        const int e = threadIdx.x + i * 64 * NW, g = e / D, x = e % D;
        if (e < G * D) {
          dense_push(apart ? at_part.row + e : part + g * (D + 2) + 2 + x, r.U[i]);
          if (x == 0) {
            dense_push(apart ? at_part.max + 2 * g * at.n_chunks : part + g * (D + 2), r.M[i]);
            dense_push(apart ? at_part.max + (2 * g + 1) * at.n_chunks : part + g * (D + 2) + 1, r.L[i]);
          }
        }
      }
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < DensePartial<D, NW>::N; i++) {
    const int e = threadIdx.x + i * 64 * NW;
    if (e < G * D) *to(e) = (uint16_t)dense_pack<T>(r.L[i] == 0.f ? 0.f : r.U[i] / r.L[i], 0.f);
  }
}

}  // namespace
