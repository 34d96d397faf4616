// Dense layers next to latent ones: rotary embedding with the append to a paged cache of plain keys and values, and the
// attention of one new token per sequence over it.
#include "wsvd_dense.h"

namespace {

// ---------------------------------------------------------------- append
// Rotation of the new tokens' queries and keys (dims i and i + d/2 turned by position * inv_freq[i]) and their keys and values
// stored in the pages.  Bound: memory, every element read and written once; few tokens: two dependent loads.
//   A wave finds its token's sequence, row and page, and its lanes the token's d / 2 angles, once for all heads: in 64 bits as
// far as whole turns go (an fp32 product of a position of 1e5 would be off by 6e-3 radians), the sine and cosine of what is
// left in 32.  Then the workgroup goes over the (token, head) pairs, 16 bytes of each half per thread.
template <class T, int D, int TOK>
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
    v4i a = *(const v4i*)src, b = *(const v4i*)(src + HALF);
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
      *(v4i*)dst = a; *(v4i*)(dst + HALF) = b;
      continue;
    }
    if (kind == 1 && p.k_out) {
      uint16_t* dst = p.k_out + t * p.k_out_ld + hh * D + part * 8;
      *(v4i*)dst = a; *(v4i*)(dst + HALF) = b;
    }
    if (slot_sh[w] >= 0) {
      uint16_t* dst = (kind == 1 ? p.pages.k : p.pages.v) + (slot_sh[w] + (int64_t)hh * p.pages.page_rows) * D + part * 8;
      *(v4i*)dst = a; *(v4i*)(dst + HALF) = b;
    }
  }
}

// ---------------------------------------------------------------- decode attention
// A chunk's place: sequence, chunk of it, chunks it has; false for a workgroup that has none.
struct DensePlace { int b, chunk, n_chunks, len, rows; };

// units a chunk takes, from the lengths of all sequences
WSVD_DEV int dense_chunk_units(const DenseDecodeParams& p, int lane) {
  int total = 0;
  for (int base = 0; base < p.B; base += 64) {
    const int i = base + lane;
    const int len = i < p.B ? min(max(p.pages.seq_lens[i], 0), p.max_len) : 0;
    total += wave_sum_int((len + kDenseUnit - 1) / kDenseUnit);
  }
  return max(p.min_units, (total + p.target - 1) / p.target);
}
WSVD_DEV int dense_chunks(const DenseDecodeParams& p, int b, int units, int& len) {
  len = b < p.B ? min(max(p.pages.seq_lens[b], 0), p.max_len) : 0;
  const int u = (len + kDenseUnit - 1) / kDenseUnit;
  return b < p.B ? max(1, (u + units - 1) / units) : 0;
}
WSVD_DEV bool dense_place(const DenseDecodeParams& p, int idx, int lane, DensePlace& at) {
  const int units = dense_chunk_units(p, lane);
  int first = 0;
  for (int base = 0; base < p.B; base += 64) {
    int len;
    const int n = dense_chunks(p, base + lane, units, len);
    const int end = first + wave_prefix_int(n, lane);
    const unsigned long long m = __ballot(end > idx);
    if (m) {
      const int l = __builtin_ctzll(m);
      at.b = base + l;
      at.n_chunks = __builtin_amdgcn_readlane(n, l);
      at.chunk = idx - (__builtin_amdgcn_readlane(end, l) - at.n_chunks);
      at.len = __builtin_amdgcn_readlane(len, l);
      at.rows = units * kDenseUnit;
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

template <int D>
struct DenseTile {
  v4i k[2][D / 32];                                  // 16 rows each, operand of the score product
  uint32_t v[8][D / 32];                             // row 4 quarter + i of either half, D / 16 dims
};

template <class T, int D>
__global__ __launch_bounds__(256) void k_dense_decode(DenseDecodeParams p) {
  constexpr int NK = D / 32, NJ = D / 16;
  __shared__ float o_sh[4][16][D], m_sh[4][16], l_sh[4][16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, qd = lane >> 4;
  const int kv = blockIdx.x % p.Hkv, idx = blockIdx.x / p.Hkv;
  DensePlace at;
  if (!dense_place(p, idx, lane, at)) return;
  if (at.chunk == 0 && kv == 0 && threadIdx.x == 0 && p.pages.seq_lens[at.b] > p.max_len) atomicExch(p.err_word, (int)WSVD_E_SHAPE);
  const int G = p.G;
  const int first = at.chunk * at.rows, end = min(at.len, first + at.rows);
  const int n_tiles = (end - first + 31) >> 5;

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
  const int* table = p.pages.block_table + (size_t)at.b * p.pages.max_pages;
  const int per_page = p.pages.page_rows >> 4, last_granule = (at.len - 1) >> 4;
  bool bad = false;
  auto load = [&](DenseTile<D>& tile, int t) {
#pragma unroll
    for (int g = 0; g < 2; g++) {
      const int granule = min((first >> 4) + 2 * t + g, last_granule);
      const int pg = granule / per_page;
      int page = __builtin_amdgcn_readfirstlane(table[pg]);
      bad |= page < 0 || page >= p.pages.n_pages;
      page = page < 0 || page >= p.pages.n_pages ? 0 : page;
      const size_t base = (((size_t)page * p.Hkv + kv) * p.pages.page_rows + (granule - pg * per_page) * 16) * D;
      const uint16_t *kp = p.pages.k + base, *vp = p.pages.v + base;
#pragma unroll
      for (int j = 0; j < NK; j++) tile.k[g][j] = *(const v4i*)(kp + c * D + j * 32 + qd * 8);
#pragma unroll
      for (int i = 0; i < 4; i++)
        __builtin_memcpy(tile.v[4 * g + i], __builtin_assume_aligned(vp + (4 * qd + i) * D + c * NJ, D / 8), NJ * 2);
    }
  };
  float m = -INFINITY, l = 0.f;
  v4f o[NJ];
#pragma unroll
  for (int j = 0; j < NJ; j++) o[j] = v4f{0.f, 0.f, 0.f, 0.f};

  auto attend = [&](DenseTile<D>& tile, int t) {
    const int r0 = first + t * 32;
    float s[8];
#pragma unroll
    for (int g = 0; g < 2; g++) {
      v4f x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < NK; j++) x = T::mfma16(tile.k[g][j], q[j], x);
#pragma unroll
      for (int i = 0; i < 4; i++) s[4 * g + i] = x[i] * p.c_scale;
    }
    if (r0 + 32 > end) {                             // rows behind the sequence's end: no weight, and no value that could be NaN
#pragma unroll
      for (int i = 0; i < 8; i++) {
        const bool out = r0 + 16 * (i >> 2) + 4 * qd + (i & 3) >= end;
        s[i] = out ? -INFINITY : s[i];
#pragma unroll
        for (int j = 0; j < NK; j++) tile.v[i][j] = out ? 0u : tile.v[i][j];
      }
    }
    float most = s[0];
#pragma unroll
    for (int i = 1; i < 8; i++) most = fmaxf(most, s[i]);
    if (__ballot(most > m + 8.f)) {                  // the reference moves only when a weight would pass 2^8
      const float mn = fmaxf(m, quarters_max(most));
      const float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
      l *= keep;
#pragma unroll
      for (int j = 0; j < NJ; j++)
#pragma unroll
        for (int i = 0; i < 4; i++) o[j][i] *= keep;
      m = mn;
    }
    const float ref = m == -INFINITY ? 0.f : m;
    float w[8];
#pragma unroll
    for (int i = 0; i < 8; i++) { w[i] = __builtin_amdgcn_exp2f(s[i] - ref); l += w[i]; }
    v4i hi, lo;                                      // weights as a pair of 16-bit numbers: what is lost is below fp32's own rounding of the sum
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const uint32_t h = dense_pack<T>(w[2 * i], w[2 * i + 1]);
      hi[i] = (int)h;
      lo[i] = (int)dense_pack<T>(w[2 * i] - dense_low<T>(h), w[2 * i + 1] - dense_high<T>(h));
    }
#pragma unroll
    for (int j = 0; j < NJ; j++) {
      v4i a;
#pragma unroll
      for (int i = 0; i < 4; i++)
        a[i] = (int)__builtin_amdgcn_perm(tile.v[2 * i + 1][j >> 1], tile.v[2 * i][j >> 1], (j & 1) ? 0x07060302u : 0x05040100u);
      o[j] = T::mfma16(a, hi, o[j]);
      o[j] = T::mfma16(a, lo, o[j]);
    }
  };
  if (wave < n_tiles) {
    DenseTile<D> t0, t1;
    load(t0, wave);
    int t = wave;
    for (; t + 4 < n_tiles; t += 8) {
      load(t1, t + 4);
      attend(t0, t);
      load(t0, t + 8);                               // (past the end: the last rows once more)
      attend(t1, t + 4);
    }
    if (t < n_tiles) attend(t0, t);
  }
  if (bad && lane == 0) atomicExch(p.err_word, (int)WSVD_E_SHAPE);
  l = quarters_sum(l);
  if (c < G) {
    if (qd == 0) { m_sh[wave][c] = m; l_sh[wave][c] = l; }
#pragma unroll
    for (int j = 0; j < NJ; j++)
#pragma unroll
      for (int i = 0; i < 4; i++) o_sh[wave][c][NJ * (4 * qd + i) + j] = o[j][i];
  }
  __syncthreads();
  for (int e = threadIdx.x; e < G * D; e += 256) {
    const int g = e / D, x = e % D;
    float M = m_sh[0][g];
#pragma unroll
    for (int w = 1; w < 4; w++) M = fmaxf(M, m_sh[w][g]);
    float L = 0.f, U = 0.f;
#pragma unroll
    for (int w = 0; w < 4; w++) {
      const float k = m_sh[w][g] == -INFINITY ? (l_sh[w][g] == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(m_sh[w][g] - M);
      L += l_sh[w][g] * k;
      U += o_sh[w][g][x] * k;
    }
    if (at.n_chunks == 1) {
      const float r = L == 0.f ? 0.f : U / L;
      p.out[((int64_t)at.b * p.Hkv * G + kv * G + g) * D + x] = (uint16_t)dense_pack<T>(r, 0.f);
    } else {
      float* part = p.parts + (((size_t)idx * p.Hkv + kv) * G + g) * (D + 2);
      part[2 + x] = U;
      if (x == 0) { part[0] = M; part[1] = L; }
    }
  }
}

// The chunks of a sequence folded in their order, one workgroup per (sequence, head).
template <class T, int D>
__global__ __launch_bounds__(D) void k_dense_join(DenseDecodeParams p) {
  const int lane = threadIdx.x & 63, Hq = p.Hkv * p.G, b = blockIdx.x / Hq, h = blockIdx.x % Hq;
  const int units = dense_chunk_units(p, lane);
  int first = 0, n = 0;
  for (int base = 0; base <= b; base += 64) {
    int len;
    const int k = dense_chunks(p, base + lane, units, len);
    const int end = wave_prefix_int(k, lane);
    if (b - base < 64) { n = __builtin_amdgcn_readlane(k, b - base); first += __builtin_amdgcn_readlane(end, b - base) - n; }
    else first += __builtin_amdgcn_readlane(end, 63);
  }
  if (n <= 1) return;
  const size_t step = (size_t)p.Hkv * p.G * (D + 2);
  const float* part = p.parts + (size_t)first * step + (size_t)h * (D + 2);
  float M = -INFINITY, L = 0.f, U = 0.f;
  for (int i = 0; i < n; i++, part += step) {
    const float m = part[0], l = part[1], u = part[2 + threadIdx.x];
    const float mn = fmaxf(M, m);
    const float keep = M == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(M - mn), e = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
    L = L * keep + l * e;                            // (nothing seen yet: L and U are 0, or NaN)
    U = U * keep + u * e;
    M = mn;
  }
  p.out[((int64_t)b * Hq + h) * D + threadIdx.x] = (uint16_t)dense_pack<T>(L == 0.f ? 0.f : U / L, 0.f);
}

template <class T, int D>
hipError_t launch_append(const DenseAppendParams& p, hipStream_t s) {
  if (p.n_tokens >= 2048) k_dense_append<T, D, 4><<<(p.n_tokens + 3) / 4, 256, 0, s>>>(p);
  else k_dense_append<T, D, 1><<<p.n_tokens, 256, 0, s>>>(p);
  return hipGetLastError();
}
template <class T, int D>
hipError_t launch_decode(const DenseDecodeParams& p, hipStream_t s) {
  k_dense_decode<T, D><<<(p.target + p.B) * p.Hkv, 256, 0, s>>>(p);
  if (p.max_len > p.min_units * kDenseUnit) k_dense_join<T, D><<<p.B * p.Hkv * p.G, D, 0, s>>>(p);
  return hipGetLastError();
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
