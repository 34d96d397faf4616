// Dense layers over 8-bit pages: rotary embedding with the append that quantises, and the attention of one new token per sequence.
#include "wsvd_dense_f8.h"
#include "wsvd_dense_join.h"

namespace {

// ---------------------------------------------------------------- append
// Rotation of the new tokens' queries and keys, keys and values quantised into the blocks of their sequences.  A unit is the new rows of one
// block (1 to 16 of them): who has a unit has all that the block's scales depend on, so that no two workgroups write to one block and
// nothing is handed over.  A workgroup has the units that begin with its TOK tokens.
//   The new rows' largest magnitude gives the scale that they need; a block that held rows keeps the larger of its scale and that one, and
// where its own was the smaller one its codes move (rarely: their exponents shift).  A key is quantised as the 16-bit number that k_out has.
template <class T, int D, int TOK>
__global__ __launch_bounds__(256) void k_dense_append_f8(DenseAppendParams p) {
  constexpr int HALF = D / 2, PER = D / 8, ND = D / 64;
  struct Unit { int t, n, row; int64_t block; };     // first token, tokens, the first one's row; block in the pools, -1: nothing is stored
  __shared__ Unit unit_sh[TOK];
  __shared__ float cs[kF8Rows][2][HALF];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t t0 = (int64_t)blockIdx.x * TOK;
  for (int i = wave; i < TOK; i += 4) {
    const int t = (int)t0 + i;
    Unit u = {t, 0, 0, -1};
    int b = p.B;
    if (t < p.n_tokens) b = __builtin_amdgcn_readfirstlane(p.cu ? dense_sequence_of(p.cu, p.B, t, lane) : t);
    const int from = b < p.B && p.cu ? p.cu[b] : t;
    if (b < p.B && t >= from) {
      const int end = p.cu ? min(p.cu[b + 1], p.n_tokens) : t + 1;
      u.row = p.pages.seq_lens[b] - 1 - (p.cu ? p.cu[b + 1] - 1 - t : 0);
      if (u.row < 0 || t == from || u.row % kF8Rows == 0) {
        u.n = u.row < 0 ? 1 : min(kF8Rows - u.row % kF8Rows, end - t);
        if (u.row < 0 || u.row >= (int64_t)p.pages.max_pages * p.pages.page_rows) {
          if (lane == 0) atomicExch(p.err_word, (int)(u.row < 0 ? WSVD_E_SHAPE : WSVD_E_CAPACITY));
        } else {
          const int pg = u.row / p.pages.page_rows, page = p.pages.block_table[(size_t)b * p.pages.max_pages + pg];
          if (page < 0 || page >= p.pages.n_pages) {
            if (lane == 0) atomicExch(p.err_word, (int)WSVD_E_SHAPE);
          } else {
            u.block = (int64_t)f8_block(page, u.row / kF8Rows, pg, 0, p.Hkv, p.pages.page_rows);
          }
        }
      }
    }
    if (lane == 0) unit_sh[i] = u;
  }
  __syncthreads();
  const int blocks = p.pages.page_rows / kF8Rows;    // of a kv head in a page
  const int r = lane & 15, qd = lane >> 4;
  for (int i = 0; i < TOK; i++) {
    const Unit u = unit_sh[i];
    if (u.n <= 0) continue;
    if (p.inv_freq) {
      for (int e = tid; e < u.n * HALF; e += 256) {  // (whole turns in 64 bits, the sine and cosine of what is left in 32)
        const int j = e / HALF, x = e % HALF, pos = p.positions ? p.positions[u.t + j] : u.row + j;
        const double turns = (double)pos * p.inv_freq[x] * 0.15915494309189533576888376337251;   // / 2 pi
        const float f = (float)(turns - __builtin_rint(turns));
        sincospif(2.f * f, &cs[j][1][x], &cs[j][0][x]);
      }
      __syncthreads();
    }
    const int r0 = u.row & (kF8Rows - 1), new_end = r0 + u.n;        // the block's rows that are new: r0 .. new_end - 1
    const bool stored = u.block >= 0;
    for (int h = blockIdx.y * 4 + wave; h < p.Hq + 2 * p.Hkv; h += gridDim.y * 4) {
      if (h < p.Hq + p.Hkv) {                        // a query or key head: a lane has PER dims of either half of a row
        const bool key = h >= p.Hq;
        const int hh = key ? h - p.Hq : h;
        if (!key && !p.q_out) continue;
        float most = 0.f;
        uint32_t w[2][PER / 2];
        if (r < u.n) {
          const uint16_t* src = key ? p.k + (int64_t)(u.t + r) * p.k_ld : p.q + (int64_t)(u.t + r) * p.q_ld;
          src += hh * D + qd * PER;
#pragma unroll
          for (int x = 0; x < PER / 8; x++)
#pragma unroll
            for (int y = 0; y < 2; y++) {
              const v4i a = *(const v4i*)(src + y * HALF + x * 8);
#pragma unroll
              for (int z = 0; z < 4; z++) w[y][4 * x + z] = (uint32_t)a[z];
            }
          if (p.inv_freq) {
#pragma unroll
            for (int x = 0; x < PER / 2; x++) {
              const int c = qd * PER + 2 * x;
              const float c0 = cs[r][0][c], c1 = cs[r][0][c + 1], s0 = cs[r][1][c], s1 = cs[r][1][c + 1];
              const float a0 = dense_low<T>(w[0][x]), a1 = dense_high<T>(w[0][x]), b0 = dense_low<T>(w[1][x]), b1 = dense_high<T>(w[1][x]);
              w[0][x] = dense_pack<T>(a0 * c0 - b0 * s0, a1 * c1 - b1 * s1);
              w[1][x] = dense_pack<T>(b0 * c0 + a0 * s0, b1 * c1 + a1 * s1);
            }
          }
          uint16_t* out = key ? p.k_out : p.q_out;
          if (out) {
            out += (int64_t)(u.t + r) * (key ? p.k_out_ld : p.q_out_ld) + hh * D + qd * PER;
#pragma unroll
            for (int x = 0; x < PER / 8; x++)
#pragma unroll
              for (int y = 0; y < 2; y++)
                *(v4i*)(out + y * HALF + x * 8) = v4i{(int)w[y][4 * x], (int)w[y][4 * x + 1], (int)w[y][4 * x + 2], (int)w[y][4 * x + 3]};
          }
          if (key) {
#pragma unroll
            for (int y = 0; y < 2; y++)
#pragma unroll
              for (int x = 0; x < PER / 2; x++) {
                const float a = __builtin_fabsf(dense_low<T>(w[y][x])), b = __builtin_fabsf(dense_high<T>(w[y][x]));
                most = fmaxf(most, fmaxf(f8_finite(a) ? a : 0.f, f8_finite(b) ? b : 0.f));
              }
          }
        }
        if (!key || !stored) continue;
        const int64_t block = u.block + (int64_t)hh * blocks;
        uint8_t* const codes = (uint8_t*)p.pages.k + block * (kF8Rows * D);
        uint8_t* const scale = p.scales.k + block;
        const int old = r0 > 0 ? (int)*scale - kF8Bias : kF8Least;
        const int e = max(f8_exponent(wave_max(most)), old);
        // 16 dims of a row lie together: at d_head 64 a lane has half of them
        auto at = [&](int y, int row) {
          const int dim = y * HALF + qd * PER;
          return codes + ((dim >> 4) * kF8Rows + row) * 16 + (dim & 15);
        };
        if (r < u.n) {
          const float inverse = f8_power(-e), top = f8_top<T>(e);
#pragma unroll
          for (int y = 0; y < 2; y++) {
            uint32_t c[PER / 4];
#pragma unroll
            for (int x = 0; x < PER / 4; x++)
              c[x] = f8_codes(f8_scaled<T>(dense_low<T>(w[y][2 * x]), inverse, top), f8_scaled<T>(dense_high<T>(w[y][2 * x]), inverse, top),
                              f8_scaled<T>(dense_low<T>(w[y][2 * x + 1]), inverse, top), f8_scaled<T>(dense_high<T>(w[y][2 * x + 1]), inverse, top));
            __builtin_memcpy(__builtin_assume_aligned(at(y, r0 + r), PER), c, PER);
          }
        }
        if (r0 > 0 && e > old && r < r0) {           // rows that the block held before
          const float by = f8_power(max(old - e, -40));
#pragma unroll
          for (int y = 0; y < 2; y++) {
            uint32_t c[PER / 4];
            __builtin_memcpy(c, __builtin_assume_aligned(at(y, r), PER), PER);
#pragma unroll
            for (int x = 0; x < PER / 4; x++) c[x] = f8_moved(c[x], by);
            __builtin_memcpy(__builtin_assume_aligned(at(y, r), PER), c, PER);
          }
        }
        if (lane == 0) *scale = (uint8_t)(e + kF8Bias);
      } else if (stored) {                           // a value head: a lane has 4 dims of 4 rows, in every 64 dims
        const int hh = h - p.Hq - p.Hkv, x0 = 4 * r;
        const int64_t block = u.block + (int64_t)hh * blocks;
        uint8_t* const codes = (uint8_t*)p.pages.v + block * (kF8Rows * D);
        uint8_t* const scale = p.scales.v + block;
        const int old = r0 > 0 ? (int)*scale - kF8Bias : kF8Least;
        uint32_t fresh = 0, before = 0;              // bytes of a dword whose rows are new, or were there
        v2i w[4][ND];
        float most = 0.f;
#pragma unroll
        for (int j = 0; j < 4; j++) {
          const int row = 4 * qd + j;
          if (row >= r0 && row < new_end) fresh |= 0xFFu << (8 * j);
          if (row < r0) before |= 0xFFu << (8 * j);
#pragma unroll
          for (int c = 0; c < ND; c++) {
            w[j][c] = v2i{0, 0};
            if (row >= r0 && row < new_end) w[j][c] = *(const v2i*)(p.v + (int64_t)(u.t + row - r0) * p.v_ld + hh * D + c * 64 + x0);
#pragma unroll
            for (int y = 0; y < 2; y++) {
              const float a = __builtin_fabsf(dense_low<T>((uint32_t)w[j][c][y])), b = __builtin_fabsf(dense_high<T>((uint32_t)w[j][c][y]));
              most = fmaxf(most, fmaxf(f8_finite(a) ? a : 0.f, f8_finite(b) ? b : 0.f));
            }
          }
        }
        const int e = max(f8_exponent(wave_max(most)), old);
        const bool moves = r0 > 0 && e > old;
        const float inverse = f8_power(-e), top = f8_top<T>(e), by = f8_power(max(old - e, -40));
        if (fresh || (moves && before)) {
#pragma unroll
          for (int c = 0; c < ND; c++) {
            v4i* const to = (v4i*)(codes + c * 1024 + qd * 256 + x0 * 4);
            v4i was = {0, 0, 0, 0};
            if (fresh != ~0u) was = *to;             // (rows that are not the call's stay as they are)
#pragma unroll
            for (int x = 0; x < 4; x++) {
              float y[4];
#pragma unroll
              for (int j = 0; j < 4; j++) {
                const uint32_t z = (uint32_t)w[j][c][x >> 1];
                y[j] = f8_scaled<T>(x & 1 ? dense_high<T>(z) : dense_low<T>(z), inverse, top);
              }
              const uint32_t made = f8_codes(y[0], y[1], y[2], y[3]);
              uint32_t kept = (uint32_t)was[x];
              if (moves) kept = (f8_moved(kept, by) & before) | (kept & ~before);
              was[x] = (int)((made & fresh) | (kept & ~fresh));
            }
            *to = was;
          }
        }
        if (lane == 0) *scale = (uint8_t)(e + kF8Bias);
      }
    }
    if (TOK > 1) __syncthreads();                    // (the next unit's angles go where this one's are)
  }
}

// ---------------------------------------------------------------- decode attention
// k_dense_decode's mathematics (wsvd_dense.hip) over codes: 16x16x32 products with the heads as the 16 columns, a lane owns one head and 4
// of 16 rows.  Both operands are made from the codes as they lie, a conversion of two with their block's scale each.
template <int D>
struct F8Tile {
  v4i k[2][D / 64], v[2][D / 64];                    // two blocks
};

template <class T, int D, int NW, bool ONCE>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_dense_decode_f8(DenseDecodeParams p) {
  constexpr int ND = D / 64, NK = D / 32, NJ = D / 16;
  extern __shared__ __attribute__((aligned(256))) float o_sh[];      // [NW][G][D]
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

  // queries as the second operand: column c = head of the group, dims in the order in which a lane has a key's
  v4i q[NK];
  {
    const uint16_t* qp = p.q + (int64_t)at.b * p.q_ld + (kv * G + min(c, G - 1)) * D + qd * 16;
#pragma unroll
    for (int j = 0; j < NK; j++) {
      const v4i x = *(const v4i*)(qp + (j >> 1) * 64 + (j & 1) * 8);
#pragma unroll
      for (int i = 0; i < 4; i++) q[j][i] = c < G ? x[i] : 0;
    }
  }
  // Where the wave's next 32 tiles lie, a lane for each of a tile's blocks.
  const int* table = p.pages.block_table + (size_t)at.b * p.pages.max_pages;
  const int last_granule = (at.len - 1) >> 4;
  bool bad = false;
  uint32_t at_low = 0, at_high = 0, k_scale = 0, v_scale = 0;
  auto look_up = [&](int t) {
    const int granule = min((first >> 4) + 2 * (t + NW * (lane >> 1)) + (lane & 1), last_granule);
    const int pg = dense_page_index(granule, p.pages.page_magic);
    const int page = dense_page(table[pg], p.pages.n_pages, bad);
    const uint64_t block = f8_block(page, granule, pg, kv, p.Hkv, p.pages.page_rows), at = block * (kF8Rows * D);
    at_low = (uint32_t)at; at_high = (uint32_t)(at >> 32);
    k_scale = (uint32_t)p.scales.k[block] << 23; v_scale = (uint32_t)p.scales.v[block] << 23;
  };
  auto load = [&](F8Tile<D>& tile, int i) {          // i: the tile's number among those looked up
#pragma unroll
    for (int g = 0; g < 2; g++) {
      const uint64_t base = (uint64_t)(uint32_t)__builtin_amdgcn_readlane(at_low, 2 * i + g) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane(at_high, 2 * i + g) << 32;
      const uint8_t *kp = (const uint8_t*)p.pages.k + base, *vp = (const uint8_t*)p.pages.v + base;
#pragma unroll
      for (int j = 0; j < ND; j++) tile.k[g][j] = load_row<ONCE>((const v4i*)(kp + j * 1024 + lane * 16));
#pragma unroll
      for (int j = 0; j < ND; j++) tile.v[g][j] = load_row<ONCE>((const v4i*)(vp + j * 1024 + lane * 16));
    }
  };
  float m = -INFINITY, l = 0.f;
  v4f o[NJ];                                         // [64 dims][one of 4]: row 4 qd + i is dim 64 (j / 4) + 16 qd + 4 i + j % 4
#pragma unroll
  for (int j = 0; j < NJ; j++) o[j] = v4f{0.f, 0.f, 0.f, 0.f};

  auto attend = [&](F8Tile<D>& tile, int t, int i) {
#pragma clang fp contract(off)                       // (a score is the same number against the limit and in its weight)
    const int r0 = first + t * 32;
    float s[8];
#pragma unroll
    for (int g = 0; g < 2; g++) {
      const float scale = __uint_as_float((uint32_t)__builtin_amdgcn_readlane(k_scale, 2 * i + g));
      v4f x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < NK; j++) {
        const uint32_t c0 = (uint32_t)tile.k[g][j >> 1][2 * (j & 1)], c1 = (uint32_t)tile.k[g][j >> 1][2 * (j & 1) + 1];
        x = T::mfma16(v4i{f8_pair<T, false>(c0, scale), f8_pair<T, true>(c0, scale), f8_pair<T, false>(c1, scale), f8_pair<T, true>(c1, scale)}, q[j], x);
      }
#pragma unroll
      for (int y = 0; y < 4; y++) s[4 * g + y] = x[y] * p.c_scale;
    }
    if (r0 + 32 > end) {                             // rows behind the sequence's end: no weight, and no value that could be NaN
#pragma unroll
      for (int g = 0; g < 2; g++) {
        const int n = min(max(end - (r0 + 16 * g + 4 * qd), 0), 4);
        const uint32_t seen = n == 4 ? ~0u : (1u << (8 * n)) - 1u;
#pragma unroll
        for (int y = 0; y < 4; y++) s[4 * g + y] = y < n ? s[4 * g + y] : -INFINITY;
#pragma unroll
        for (int j = 0; j < ND; j++)
#pragma unroll
          for (int y = 0; y < 4; y++) tile.v[g][j][y] &= (int)seen;
      }
    }
    float most = s[0];
#pragma unroll
    for (int y = 1; y < 8; y++) most = fmaxf(most, s[y]);
    if (__ballot(most - m > T::kTop)) {              // (see the element types)
      const float top = quarters_max(most), low = top - T::kRaise;
      const float mn = fmaxf(m, top - low > T::kTop ? top : low);    // (steps of 16, between scores of 2^27 and 2^28)
      const float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
      l *= keep;
#pragma unroll
      for (int j = 0; j < NJ; j++)
#pragma unroll
        for (int y = 0; y < 4; y++) o[j][y] *= keep;
      m = mn;
    }
    const float ref = m == -INFINITY ? 0.f : m;
    float w[8];
#pragma unroll
    for (int y = 0; y < 8; y++) { w[y] = __builtin_amdgcn_exp2f(s[y] - ref); l += w[y]; }
    // weights as a pair of 16-bit numbers (bf16: off by at most 2^-17 of the weight; f16: by 2^-23 of it or 2^-36 of the reference's)
    v4i hi, lo;
#pragma unroll
    for (int y = 0; y < 4; y++) {
      const uint32_t h = dense_pack<T>(w[2 * y], w[2 * y + 1]);
      hi[y] = (int)h;
      lo[y] = (int)dense_pack<T>(w[2 * y] - dense_low<T>(h), w[2 * y + 1] - dense_high<T>(h));
    }
    const float s0 = __uint_as_float((uint32_t)__builtin_amdgcn_readlane(v_scale, 2 * i)), s1 = __uint_as_float((uint32_t)__builtin_amdgcn_readlane(v_scale, 2 * i + 1));
#pragma unroll
    for (int j = 0; j < NJ; j++) {
      const uint32_t c0 = (uint32_t)tile.v[0][j >> 2][j & 3], c1 = (uint32_t)tile.v[1][j >> 2][j & 3];
      const v4i a = {f8_pair<T, false>(c0, s0), f8_pair<T, true>(c0, s0), f8_pair<T, false>(c1, s1), f8_pair<T, true>(c1, s1)};
      o[j] = T::mfma16(a, hi, o[j]);
      o[j] = T::mfma16(a, lo, o[j]);
    }
  };
  for (int t = wave; t < n_tiles; t += 32 * NW) {    // 32 tiles of the wave
    look_up(t);
    const int n = min(32, (n_tiles - t + NW - 1) / NW);
    F8Tile<D> t0, t1;
    load(t0, 0);
    int i = 0;
    for (; i + 2 < n; i += 2) {
      load(t1, i + 1);
      attend(t0, t + NW * i, i);
      load(t0, i + 2);
      attend(t1, t + NW * (i + 1), i + 1);
    }
    if (i + 1 < n) load(t1, i + 1);
    attend(t0, t + NW * i, i);
    if (i + 1 < n) attend(t1, t + NW * (i + 1), i + 1);
  }
  if (__ballot(bad) && lane == 0) atomicExch(p.err_word, (int)WSVD_E_SHAPE);
  l = quarters_sum(l);
  __syncthreads();
  if (c < G) {
    if (qd == 0) { m_sh[wave][c] = m; l_sh[wave][c] = l; }
    // (A head's dims start 4 c further on in its row, since the heads' rows begin at one bank.)
#pragma unroll
    for (int y = 0; y < 4; y++)
#pragma unroll
      for (int j = 0; j < NJ; j += 4)
        *(v4f*)(o_sh + (wave * G + c) * D + ((16 * j + 16 * qd + 4 * y + 4 * c) & (D - 1))) = v4f{o[j][y], o[j + 1][y], o[j + 2][y], o[j + 3][y]};
  }
  __syncthreads();
  dense_finish<T, D, NW>(p, at, idx, kv, o_sh, m_sh, l_sh);
}

template <class T, int D, int TOK>
hipError_t launch_append_form(const DenseAppendParams& p, int splits, hipStream_t s) {
  k_dense_append_f8<T, D, TOK><<<dim3((unsigned)((p.n_tokens + TOK - 1) / TOK), (unsigned)splits), 256, 0, s>>>(p);
  return hipGetLastError();
}
template <class T, int D>
hipError_t launch_append(const DenseAppendParams& p, hipStream_t s) {
  const DenseF8Append a = dense_f8_append(p.n_tokens, p.B, p.Hq + 2 * p.Hkv, p.cu != nullptr);
  return a.tokens == 1 ? launch_append_form<T, D, 1>(p, a.splits, s) : launch_append_form<T, D, 16>(p, a.splits, s);
}
template <class T, int D, int NW, bool ONCE>
hipError_t launch_decode_form(const DenseDecodeParams& p, hipStream_t s) {
  constexpr int LDS = NW * D * 4 * 16;
  static LdsLimit limit;
  if (LDS + NW * 16 * 8 > 65536) {
    const hipError_t e = wsvd_raise_lds(limit, (const void*)k_dense_decode_f8<T, D, NW, ONCE>, LDS);
    if (e != hipSuccess) return e;
  }
  k_dense_decode_f8<T, D, NW, ONCE><<<(unsigned)dense_decode_workgroups(p.B, p.Hkv, p.target, p.alone != 0), 64 * NW, LDS, s>>>(p);
  return hipGetLastError();
}
template <class T, int D, bool ONCE>
hipError_t launch_decode_waves(const DenseDecodeParams& p, hipStream_t s) {
  return p.waves == 8 ? launch_decode_form<T, D, 8, ONCE>(p, s) : p.waves == 4 ? launch_decode_form<T, D, 4, ONCE>(p, s) : launch_decode_form<T, D, 2, ONCE>(p, s);
}
template <class T, int D>
hipError_t launch_decode(const DenseDecodeParams& p, hipStream_t s) {
  const bool once = (int64_t)p.B * p.max_len * p.Hkv * D * 2 >= 100000000;      // (as k_dense_decode's)
  return once ? launch_decode_waves<T, D, true>(p, s) : launch_decode_waves<T, D, false>(p, s);
}

}  // namespace

hipError_t wsvd_launch_dense_append_f8(const DenseAppendParams& p, int dtype, int d, hipStream_t s) {
  if (dtype == WSVD_BF16) return d == 128 ? launch_append<DenseBf16, 128>(p, s) : launch_append<DenseBf16, 64>(p, s);
  return d == 128 ? launch_append<DenseF16, 128>(p, s) : launch_append<DenseF16, 64>(p, s);
}
hipError_t wsvd_launch_dense_decode_f8(const DenseDecodeParams& p, int dtype, int d, hipStream_t s) {
  if (dtype == WSVD_BF16) return d == 128 ? launch_decode<DenseBf16, 128>(p, s) : launch_decode<DenseBf16, 64>(p, s);
  return d == 128 ? launch_decode<DenseF16, 128>(p, s) : launch_decode<DenseF16, 64>(p, s);
}
