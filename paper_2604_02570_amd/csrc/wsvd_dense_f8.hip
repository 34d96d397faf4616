// Dense layers over 8-bit pages: rotary embedding with the append that quantises, and the attention of one new token per sequence.
#include <type_traits>
#include "wsvd_dense_f8.h"
#include "wsvd_dense_join.h"

namespace {

// ---------------------------------------------------------------- append
// Rotation of the new tokens' queries and keys, keys and values quantised into the blocks of their sequences.  A unit is the new rows of one
// block (1 to 16 of them): who has a head of a unit has all that the block's scale depends on, so that no two waves write to one block and
// nothing is handed over.  A workgroup has one unit, or a share of its heads.
//   The new rows' largest magnitude gives the scale that they need; a block that held rows keeps the larger of its scale and that one, and
// where its own was the smaller one its codes move (rarely: their exponents shift).  A key is quantised as the 16-bit number that k_out has.
//   Bound: memory, every element read once, 16-bit ones and codes written once.  19029 tokens of 32 heads of 128 (936 MB): 171 us, 5.5 TB/s, where a
// copy of 1 GiB reaches 5.1.  Loads and stores go in whole lines (a lane with 16 dims of a row, two requests that share lines: 271 us, with 8 dims of
// two rows 244); rows as data that is used once (208 of 219 us with two workgroups a unit); the workgroups of a unit side by side (205 -> 197 with
// three); four waves a SIMD (three, with the next head asked for ahead: 196); units found from the lengths (by workgroups of 16 tokens each: 181; of
// one, most of which have none: 4 x 300 tokens of 32 / 8 heads 25.9 us, now 11.7).  32 tokens of 28 / 4 heads: 6.4 us on the GPU, five dependent
// steps: lengths, page, scale and rows, the wave's maximum, the store.
struct F8Unit { int t, n, row; int64_t block; };     // first token, tokens, the first one's row; block in the pools, -1: nothing is stored
// The call's unit number idx, in the tokens' order; n = 0 where there is none.  A wave's work: 256 sequences' borders and lengths are asked for at
// once, a lane for each of 64.
WSVD_DEV F8Unit f8_unit(const DenseAppendParams& p, int idx, int lane) {
  F8Unit u = {idx, 0, 0, -1};
  int b = idx;
  if (p.cu) {
    b = -1;
    int before = 0;
    auto look = [&](int base, auto groups) {
      constexpr int N = decltype(groups)::value;
      int from[N], row[N], n[N], units[N];
#pragma unroll
      for (int i = 0; i < N; i++) {
        const int s = min(base + 64 * i + lane, p.B - 1), to = p.cu[s + 1];
        from[i] = p.cu[s];
        row[i] = p.pages.seq_lens[s] - (to - from[i]);
        // (tokens that are not there, and borders that are none: no unit)
        n[i] = base + 64 * i + lane < p.B && from[i] >= 0 ? min(to, p.n_tokens) - from[i] : 0;
        units[i] = n[i] > 0 ? ((row[i] + n[i] - 1) >> 4) - (row[i] >> 4) + 1 : 0;
      }
#pragma unroll
      for (int i = 0; i < N; i++) {
        const int end = before + wave_prefix_int(units[i]);
        const unsigned long long m = __ballot(end > idx);
        if (m && b < 0) {
          const int at = __builtin_ctzll(m), f = __builtin_amdgcn_readlane(from[i], at), r = __builtin_amdgcn_readlane(row[i], at), k = __builtin_amdgcn_readlane(n[i], at);
          const int nth = idx - (__builtin_amdgcn_readlane(end, at) - __builtin_amdgcn_readlane(units[i], at));
          b = base + 64 * i + at;
          u.row = nth == 0 ? r : ((r >> 4) + nth) * kF8Rows;
          u.t = f + (u.row - r);
          u.n = min(kF8Rows - (u.row & (kF8Rows - 1)), k - (u.row - r));
        }
        before = __builtin_amdgcn_readlane(end, 63);
      }
    };
    if (p.B <= 64) look(0, std::integral_constant<int, 1>{});
    else for (int base = 0; base < p.B && b < 0; base += 256) look(base, std::integral_constant<int, 4>{});
    if (b < 0) return u;
  } else {
    u.row = p.pages.seq_lens[b] - 1;
    u.n = 1;
  }
  if (u.row < 0 || u.row >= (int64_t)p.pages.max_pages * p.pages.page_rows) {
    if (lane == 0) atomicExch(p.err_word, (int)(u.row < 0 ? WSVD_E_SHAPE : WSVD_E_CAPACITY));
    return u;
  }
  const int granule = u.row / kF8Rows, pg = dense_page_index(granule, p.pages.page_magic);
  const int page = p.pages.block_table[(size_t)b * p.pages.max_pages + pg];
  if (page < 0 || page >= p.pages.n_pages) {
    if (lane == 0) atomicExch(p.err_word, (int)WSVD_E_SHAPE);
  } else {
    u.block = (int64_t)f8_block(page, granule, pg, 0, p.Hkv, p.pages.page_rows);
  }
  return u;
}

template <class T, int D, bool ONCE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(4))) void k_dense_append_f8(DenseAppendParams p, int splits) {
  constexpr int HALF = D / 2, ND = D / 64, PER_ROUND = 1024 / D, ROUNDS = kF8Rows / PER_ROUND;     // rows at a time: in whole lines
  constexpr int N = D / 16;
  __shared__ float cs[kF8Rows][2][HALF];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int split = (int)(blockIdx.x % (unsigned)splits), step = splits * 4, heads = p.Hq + 2 * p.Hkv;
  const double freq = p.inv_freq ? p.inv_freq[tid % HALF] : 0.;      // (asked for before anything is known of the tokens)
  const int blocks = p.pages.page_rows / kF8Rows;    // of a kv head in a page
  const int r = lane / (D / 16), x8 = lane % (D / 16) * 8;            // of queries and keys: row of a round, dims of either half
  const int qd = lane >> 4, x4 = lane % 16 * 4;      // of values: group of rows, dims of every 64
  const F8Unit u = f8_unit(p, (int)(blockIdx.x / (unsigned)splits), lane);
  if (u.n <= 0) return;
  const int r0 = u.row & (kF8Rows - 1), new_end = r0 + u.n;          // the block's rows that are new: r0 .. new_end - 1
  const bool stored = u.block >= 0;
  // what a lane has of a head: of queries and keys [round][half of the dims] of 8, of values [row of 4][64 dims] of 4
  auto fetch = [&](int h, v2i (&w)[N]) {
    if (h < p.Hq + p.Hkv) {
      const bool key = h >= p.Hq;
      if (!key && !p.q_out) return;
      const uint16_t* const src = (key ? p.k + (h - p.Hq) * D : p.q + h * D) + x8;
      const int64_t ld = key ? p.k_ld : p.q_ld;
#pragma unroll
      for (int y = 0; y < ROUNDS; y++)
#pragma unroll
        for (int z = 0; z < 2; z++) {
          const int t = y * PER_ROUND + r;
          v4i x = {0, 0, 0, 0};
          if (t < u.n) x = load_row<ONCE>((const v4i*)(src + (int64_t)(u.t + t) * ld + z * HALF));
          w[4 * y + 2 * z] = v2i{x[0], x[1]};
          w[4 * y + 2 * z + 1] = v2i{x[2], x[3]};
        }
    } else {
      const uint16_t* const src = p.v + (h - p.Hq - p.Hkv) * D + x4;
#pragma unroll
      for (int j = 0; j < 4; j++)
#pragma unroll
        for (int c = 0; c < ND; c++) {
          const int row = 4 * qd + j;
          w[j * ND + c] = v2i{0, 0};
          if (row >= r0 && row < new_end) w[j * ND + c] = load_row<ONCE>((const v2i*)(src + (int64_t)(u.t + row - r0) * p.v_ld + c * 64));
        }
    }
  };
  int h = split * 4 + wave;
  v2i w[N];
  if (h < heads) fetch(h, w);                      // (under the angles)
  if (p.inv_freq) {
    for (int e = tid; e < u.n * HALF; e += 256) {  // (whole turns in 64 bits, the sine and cosine of what is left in 32)
      const int j = e / HALF, x = e % HALF, pos = p.positions ? p.positions[u.t + j] : u.row + j;
      const double turns = (double)pos * freq * 0.15915494309189533576888376337251;   // / 2 pi
      const float f = (float)(turns - __builtin_rint(turns));
      sincospif(2.f * f, &cs[j][1][x], &cs[j][0][x]);
    }
    __syncthreads();
  }
  for (; h < heads; h += step) {
    const bool value = h >= p.Hq + p.Hkv, key = !value && h >= p.Hq;
    const int hh = value ? h - p.Hq - p.Hkv : key ? h - p.Hq : h;
    const int64_t block = u.block + (int64_t)hh * blocks;
    uint8_t* const codes = (uint8_t*)(value ? p.pages.v : p.pages.k) + block * (kF8Rows * D);
    uint8_t* const scale = (value ? p.scales.v : p.scales.k) + block;
    const int old = (key || value) && stored && r0 > 0 ? (int)*scale - kF8Bias : kF8Least;
    // bytes of a value dword whose rows are new, or were there
    const uint32_t fresh = f8_bytes(new_end - 4 * qd) & ~f8_bytes(r0 - 4 * qd), before = f8_bytes(r0 - 4 * qd);
    v4i was[ND];
    if (value && stored && fresh != ~0u) {         // (rows that are not the call's stay as they are)
#pragma unroll
      for (int c = 0; c < ND; c++) was[c] = *(const v4i*)(codes + c * 1024 + qd * 256 + x4 * 4);
    }
    float most = 0.f;
    if (!value) {
      uint16_t* const out = key ? p.k_out : p.q_out;
#pragma unroll
      for (int y = 0; y < ROUNDS; y++) {
        const int t = y * PER_ROUND + r;
        if (t < u.n && (key || out)) {
          if (p.inv_freq) {
#pragma unroll
            for (int x = 0; x < 4; x++) {
              const int c = x8 + 2 * x;
              const float c0 = cs[t][0][c], c1 = cs[t][0][c + 1], s0 = cs[t][1][c], s1 = cs[t][1][c + 1];
              const uint32_t a = (uint32_t)w[4 * y + (x >> 1)][x & 1], b = (uint32_t)w[4 * y + 2 + (x >> 1)][x & 1];
              const float a0 = dense_low<T>(a), a1 = dense_high<T>(a), b0 = dense_low<T>(b), b1 = dense_high<T>(b);
              w[4 * y + (x >> 1)][x & 1] = (int)dense_pack<T>(a0 * c0 - b0 * s0, a1 * c1 - b1 * s1);
              w[4 * y + 2 + (x >> 1)][x & 1] = (int)dense_pack<T>(b0 * c0 + a0 * s0, b1 * c1 + a1 * s1);
            }
          }
          if (out) {
            uint16_t* const to = out + (int64_t)(u.t + t) * (key ? p.k_out_ld : p.q_out_ld) + hh * D + x8;
#pragma unroll
            for (int z = 0; z < 2; z++)
              store_row<ONCE>((v4i*)(to + z * HALF), v4i{w[4 * y + 2 * z][0], w[4 * y + 2 * z][1], w[4 * y + 2 * z + 1][0], w[4 * y + 2 * z + 1][1]});
          }
        }
      }
    }
    if ((key || value) && stored) {
#pragma unroll
      for (int x = 0; x < 2 * N; x++) most = f8_most<T>(most, (uint32_t)w[x >> 1][x & 1]);       // (what a lane has none of is 0)
      const int e = max(f8_exponent(wave_max(most)), old);
      const bool moves = r0 > 0 && e > old;
      const float inverse = f8_power(-e), top = f8_top<T>(e), by = f8_power(max(old - e, -40));
      if (key) {
        auto at = [&](int z, int row) {            // 16 dims of a row lie together
          const int dim = z * HALF + x8;
          return (v2i*)(codes + ((dim >> 4) * kF8Rows + row) * 16 + (dim & 8));
        };
#pragma unroll
        for (int y = 0; y < ROUNDS; y++) {
          const int t = y * PER_ROUND + r;
          if (t < u.n) {
#pragma unroll
            for (int z = 0; z < 2; z++) {
              v2i c;
#pragma unroll
              for (int x = 0; x < 2; x++) {
                const uint32_t a = (uint32_t)w[4 * y + 2 * z + x][0], b = (uint32_t)w[4 * y + 2 * z + x][1];
                c[x] = (int)f8_codes(f8_scaled(dense_low<T>(a), inverse, top), f8_scaled(dense_high<T>(a), inverse, top),
                                     f8_scaled(dense_low<T>(b), inverse, top), f8_scaled(dense_high<T>(b), inverse, top));
              }
              store_row<ONCE>(at(z, r0 + t), c);
            }
          }
          if (moves && t < r0) {                   // row t, which the block held before
#pragma unroll
            for (int z = 0; z < 2; z++) {
              v2i c = *at(z, t);
              c[0] = (int)f8_moved((uint32_t)c[0], by); c[1] = (int)f8_moved((uint32_t)c[1], by);
              *at(z, t) = c;
            }
          }
        }
      } else if (fresh || (moves && before)) {
#pragma unroll
        for (int c = 0; c < ND; c++) {
          v4i to;
#pragma unroll
          for (int x = 0; x < 4; x++) {
            float y[4];
#pragma unroll
            for (int j = 0; j < 4; j++) {
              const uint32_t z = (uint32_t)w[j * ND + c][x >> 1];
              y[j] = f8_scaled(x & 1 ? dense_high<T>(z) : dense_low<T>(z), inverse, top);
            }
            to[x] = (int)f8_codes(y[0], y[1], y[2], y[3]);
            if (fresh != ~0u) {
              uint32_t kept = (uint32_t)was[c][x];
              if (moves) kept = (f8_moved(kept, by) & before) | (kept & ~before);
              to[x] = (int)(((uint32_t)to[x] & fresh) | (kept & ~fresh));
            }
          }
          store_row<ONCE>((v4i*)(codes + c * 1024 + qd * 256 + x4 * 4), to);
        }
      }
      if (lane == 0) *scale = (uint8_t)(e + kF8Bias);
    }
    if (h + step < heads) fetch(h + step, w);
  }
}

// ---------------------------------------------------------------- decode attention
// k_dense_decode's mathematics (wsvd_dense.hip) over codes: 16x16x32 products with the heads as the 16 columns, a lane owns one head and 4
// of 16 rows.  Both operands are made from the codes as they lie, a conversion of two with their block's scale each (at full rate).
// Bound: HBM.  32 x 8192 rows of 4 heads of 128 (270 MB): 47.4 us, 5.7 TB/s; the same launches and requests without the arithmetic 46.2, a kernel
// that only reads so many bytes 41.1.  640 rows of 32 heads (5.3 MB): 6.5 us, without arithmetic 4.7, of which 3.3 are a launch that finds no row.
// (Tiles of 64 rows, so that twice as much is asked for ahead: 48.1 us and 6.9; workgroups of 4 waves, two to a CU: 51.2 and 7.0; one chunk a
// sequence, on half of the CUs: 52.8.)
constexpr int kF8Tile = 2;
template <int D>
struct F8Tile {
  v4i k[kF8Tile][D / 64], v[kF8Tile][D / 64];        // two blocks
};

// Several tokens a sequence (where dense_f8_columns says so): the columns are 16 of a sequence's (token, head) pairs, token-major, or two sets of 16 that
// share the rows' codes and their conversion (which costs as much as one set's products).  A column sees the rows up to its own.
// The sequence's first query, pairs before, columns; the last row that the first one sees; the tile's number, and of one column that in the tile.
struct F8Columns { int q_start, row0, n, first_limit, tile, column; };
// A workgroup's sequence, columns (of WIDTH) and chunk: tile number idx of the call, share `split` of its rows; or (one) the tile of pair number idx.
template <int WIDTH>
WSVD_DEV bool f8_columns(const DenseDecodeParams& p, int idx, int split, int lane, DensePlace& at, F8Columns& col, bool one = false) {
  const int most = p.pages.max_pages * p.pages.page_rows;
  for (int base = 0, before = 0, tiles_before = 0; base < p.B; base += 64) {
    const int i = base + lane;
    int qs = 0, n = 0, len = 0;
    if (i < p.B) {
      qs = min(max(p.cu_q[i], 0), p.n_q);
      n = min(max(p.cu_q[i + 1], qs), p.n_q) - qs;
      len = p.pages.seq_lens[i];
    }
    const int tiles = (n * p.group + WIDTH - 1) / WIDTH, tiles_end = tiles_before + wave_prefix_int(tiles);
    const int mine = one ? n * p.group : tiles, end = one ? before + wave_prefix_int(mine) : tiles_end;
    const unsigned long long m = __ballot(end > idx);
    before = __builtin_amdgcn_readlane(end, 63); tiles_before = __builtin_amdgcn_readlane(tiles_end, 63);
    if (!m) continue;
    const int l = __builtin_ctzll(m);
    at.b = base + l;
    n = __builtin_amdgcn_readlane(n, l); len = __builtin_amdgcn_readlane(len, l);
    if (len > most && threadIdx.x == 0) atomicExch(p.err_word, (int)WSVD_E_SHAPE);
    len = min(max(len, 0), most);
    col.q_start = __builtin_amdgcn_readlane(qs, l);
    const int number = idx - (__builtin_amdgcn_readlane(end, l) - __builtin_amdgcn_readlane(mine, l)), tile = one ? number / WIDTH : number;
    col.column = number - tile * WIDTH;
    col.tile = __builtin_amdgcn_readlane(tiles_end, l) - __builtin_amdgcn_readlane(tiles, l) + tile;
    col.row0 = WIDTH * tile;
    col.n = min(WIDTH, n * p.group - col.row0);
    col.first_limit = len - n + col.row0 / p.group;
    at.len = max(len - n + (col.row0 + col.n - 1) / p.group + 1, 0);
    const int units = dense_units_of(at.len);
    at.n_chunks = units <= p.alone_units ? 1 : min(p.splits, (units + p.min_units - 1) / p.min_units);
    at.chunk = split;
    at.rows = (units + at.n_chunks - 1) / at.n_chunks * kDenseUnit;
    return split < at.n_chunks;
  }
  return false;
}

// The join of many chunks, a workgroup a head or pair (g of p.G): dims in lanes, an eighth of the n chunks from c0 on a wave, all words of a thread asked
// for at once.  The workgroup has a higher number than those it waits for, and the wait is bounded.  Words are cleared where they are read.
template <class T, int D>
WSVD_DEV void f8_join(const DenseDecodeParams& p, int c0, int n, int kv, int g, int lane, int wave, float* sh, uint16_t* out) {
  constexpr int ND = D / 64, CHUNKS = kDenseFold * kDenseFold / 8;   // a wave's chunks
  const DensePartWords part = dense_many(p, c0, n, 0, kv, g, D);
  const size_t stride = (size_t)p.Hkv * p.G * D;
  const unsigned long long none = split_word(0.f);
  auto come = [&](unsigned long long x) { return (uint32_t)(x >> 32) == kSplitTag; };
  unsigned long long w[ND][CHUNKS], wm = none, wl = none;          // (maxima and sums: the first wave's, a lane a chunk)
  float *const f_sh = sh, *const l_sh = sh + 64, *const u_sh = sh + 128;       // [chunk], [1], [wave][D]
  const bool has = wave == 0 && lane < n;
  bool all = false;
  for (int budget = 1 << 20; budget && !all; budget--) {
    if (has) { wm = dense_word(part.max + lane); wl = dense_word(part.max + n + lane); }
#pragma unroll
    for (int x = 0; x < ND; x++)
#pragma unroll
      for (int k = 0; k < CHUNKS; k++) w[x][k] = wave + 8 * k < n ? dense_word(part.row + (wave + 8 * k) * stride + x * 64 + lane) : none;
    all = come(wm) && come(wl);
#pragma unroll
    for (int x = 0; x < ND; x++)
#pragma unroll
      for (int k = 0; k < CHUNKS; k++) all = all && come(w[x][k]);
    if (!all) __builtin_amdgcn_s_sleep(1);
  }
  if (!all) atomicExch(p.err_word, (int)WSVD_E_HIP);               // never seen; keeps the wait finite
  if (wave == 0) {
    const float m = has ? __uint_as_float((uint32_t)wm) : -INFINITY, M = wave_max(m);
    const float f = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - M);      // (nothing seen: l and u are 0, or NaN)
    const float L = wave_sum(__uint_as_float((uint32_t)wl) * f);
    f_sh[lane] = f;
    if (lane == 0) *l_sh = L;
    if (has) { dense_clear(part.max + lane); dense_clear(part.max + n + lane); }
  }
  __syncthreads();
#pragma unroll
  for (int x = 0; x < ND; x++) {
    float U = 0.f;
#pragma unroll
    for (int k = 0; k < CHUNKS; k++)
      if (wave + 8 * k < n) {
        U += dense_scaled(__uint_as_float((uint32_t)w[x][k]), f_sh[wave + 8 * k]);
        dense_clear(part.row + (wave + 8 * k) * stride + x * 64 + lane);
      }
    u_sh[wave * D + x * 64 + lane] = U;
  }
  __syncthreads();
  const int x = threadIdx.x;
  if (x < D) {
    const float L = *l_sh;
    float U = 0.f;
#pragma unroll
    for (int k = 0; k < 8; k++) U += u_sh[k * D + x];
    out[x] = (uint16_t)dense_pack<T>(L == 0.f ? 0.f : U / L, 0.f);
  }
}

// The sequence and head of joining workgroup idx, where chunks have `units`.
template <class T, int D>
WSVD_DEV void f8_join_sequence(const DenseDecodeParams& p, int idx, int units, int kv, int lane, int wave, float* sh) {
  const int n_mine = lane < p.B ? dense_chunks(dense_units_of(dense_length(p, lane)), units) : 0;
  const unsigned long long many = __ballot(n_mine > kF8Whole);
  const int which = idx / p.G, g = idx - which * p.G;
  const unsigned long long sel = __ballot((many >> lane & 1) && __builtin_popcountll(many & ((1ull << lane) - 1)) == which);
  if (!sel) return;
  const int b = __builtin_ctzll(sel), n = __builtin_amdgcn_readlane(n_mine, b), c0 = __builtin_amdgcn_readlane(wave_prefix_int(n_mine), b) - n;
  f8_join<T, D>(p, c0, n, kv, g, lane, wave, sh, p.out + (((int64_t)b * p.Hkv + kv) * p.G + g) * D);
}

// SETS: of 16 columns of several tokens; 0: one token a sequence, its heads.  JOINS: with workgroups that join chunks (a form of its own: 1 x 7 tokens
// behind 3000 rows without them as part of the same form 15.9 us in place of 14.2).
template <class T, int D, int NW, bool ONCE, int SETS, bool JOINS>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_dense_decode_f8(DenseDecodeParams p) {
  constexpr int ND = D / 64, NK = D / 32, NJ = D / 16, NB = kF8Tile, ROWS = 16 * NB, AHEAD = 64 / NB;        // rows of a tile; tiles looked up at a time
  extern __shared__ __attribute__((aligned(256))) float o_sh[];      // [NW][G][D]
  __shared__ float m_sh[NW][16], l_sh[NW][16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, qd = lane >> 4;
  constexpr bool TOKENS = SETS > 0;
  constexpr int C = TOKENS ? SETS : 1;
  const int kv = blockIdx.x % p.Hkv;
  int idx = blockIdx.x / p.Hkv;
  DensePlace at;
  F8Columns col = {};
  if constexpr (TOKENS) {
    const int tile = idx / p.splits, pair = idx - p.tiles * p.splits;
    const bool joins = JOINS && pair >= 0;
    if (!f8_columns<16 * C>(p, joins ? pair : tile, joins ? 0 : idx - tile * p.splits, lane, at, col, joins)) return;
    p.parts += (size_t)col.tile * p.splits * p.Hkv * (16 * C) * (D + 2);       // (a tile's chunks are among themselves)
    if (joins) {
      if (at.n_chunks <= kF8Whole) return;
      const int set = col.column / 16, row = col.row0 + col.column, token = row / p.group;
      p.parts += (size_t)set * p.splits * p.Hkv * 16 * (D + 2);
      p.G = min(col.n - 16 * set, 16);
      f8_join<T, D>(p, 0, at.n_chunks, kv, col.column - 16 * set, lane, wave, o_sh,
                    p.out + (int64_t)(col.q_start + token) * p.out_ld + (kv * p.group + row - token * p.group) * D);
      return;
    }
    idx = at.chunk;
  } else {
    if (!dense_place(p, idx, lane, at)) {
      if constexpr (JOINS) f8_join_sequence<T, D>(p, at.chunk, at.rows, kv, lane, wave, o_sh);
      return;
    }
    if (at.chunk == 0 && kv == 0 && threadIdx.x == 0 && p.pages.seq_lens[at.b] > p.max_len) atomicExch(p.err_word, (int)WSVD_E_SHAPE);
    col.n = p.G;
  }
  const int first = at.chunk * at.rows, end = min(at.len, first + at.rows);
  const int n_tiles = (max(end - first, 0) + ROWS - 1) / ROWS;

  // queries as the second operand: column c of a set = head of the group, or pair, dims in the order in which a lane has a key's
  v4i q[C][NK];
  int limit[C];                                      // the last row that the column sees
#pragma unroll
  for (int x = 0; x < C; x++) {
    const int pair = col.row0 + min(16 * x + c, col.n - 1), token = TOKENS ? pair / p.group : 0;
    limit[x] = col.first_limit + token - (TOKENS ? col.row0 / p.group : 0);
    const uint16_t* qp = TOKENS ? p.q + (int64_t)(col.q_start + token) * p.q_ld + (kv * p.group + pair - token * p.group) * D + qd * 16
                                : p.q + (int64_t)at.b * p.q_ld + (kv * p.G + pair) * D + qd * 16;
#pragma unroll
    for (int j = 0; j < NK; j++) {
      const v4i y = *(const v4i*)(qp + (j >> 1) * 64 + (j & 1) * 8);
#pragma unroll
      for (int i = 0; i < 4; i++) q[x][j][i] = 16 * x + c < col.n ? y[i] : 0;
    }
  }
  // Where the wave's next AHEAD tiles lie, a lane for each of a tile's blocks.
  const int* table = p.pages.block_table + (size_t)at.b * p.pages.max_pages;
  const int last_granule = (at.len - 1) >> 4;
  bool bad = false;
  uint32_t at_low = 0, at_high = 0, k_scale = 0, v_scale = 0;
  auto look_up = [&](int t) {
    const int granule = min((first >> 4) + NB * (t + NW * (lane / NB)) + lane % NB, last_granule);
    const int pg = dense_page_index(granule, p.pages.page_magic);
    const int page = dense_page(table[pg], p.pages.n_pages, bad);
    const uint64_t block = f8_block(page, granule, pg, kv, p.Hkv, p.pages.page_rows), at = block * (kF8Rows * D);
    at_low = (uint32_t)at; at_high = (uint32_t)(at >> 32);
    k_scale = (uint32_t)p.scales.k[block] << 23; v_scale = (uint32_t)p.scales.v[block] << 23;
  };
  auto load = [&](F8Tile<D>& tile, int i) {      // i: the tile's number among those looked up
#pragma unroll
    for (int g = 0; g < NB; g++) {
      const uint64_t base = (uint64_t)(uint32_t)__builtin_amdgcn_readlane(at_low, NB * i + g) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane(at_high, NB * i + g) << 32;
      const uint8_t *kp = (const uint8_t*)p.pages.k + base, *vp = (const uint8_t*)p.pages.v + base;
#pragma unroll
      for (int j = 0; j < ND; j++) tile.k[g][j] = load_row<ONCE>((const v4i*)(kp + j * 1024 + lane * 16));
#pragma unroll
      for (int j = 0; j < ND; j++) tile.v[g][j] = load_row<ONCE>((const v4i*)(vp + j * 1024 + lane * 16));
    }
  };
  float m[C], l[C];
  v4f o[C][NJ];                                      // [64 dims][one of 4]: row 4 qd + i is dim 64 (j / 4) + 16 qd + 4 i + j % 4
#pragma unroll
  for (int x = 0; x < C; x++) {
    m[x] = -INFINITY; l[x] = 0.f;
#pragma unroll
    for (int j = 0; j < NJ; j++) o[x][j] = v4f{0.f, 0.f, 0.f, 0.f};
  }

  auto attend = [&](F8Tile<D>& tile, int t, int i) {
#pragma clang fp contract(off)                       // (a score is the same number against the limit and in its weight)
    const int r0 = first + t * ROWS;
    float s[C][4 * NB];
#pragma unroll
    for (int g = 0; g < NB; g++) {
      const float scale = __uint_as_float((uint32_t)__builtin_amdgcn_readlane(k_scale, NB * i + g));
      v4f y[C];
#pragma unroll
      for (int x = 0; x < C; x++) y[x] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < NK; j++) {
        const uint32_t c0 = (uint32_t)tile.k[g][j >> 1][2 * (j & 1)], c1 = (uint32_t)tile.k[g][j >> 1][2 * (j & 1) + 1];
        const v4i a = {f8_pair<T, false>(c0, scale), f8_pair<T, true>(c0, scale), f8_pair<T, false>(c1, scale), f8_pair<T, true>(c1, scale)};
#pragma unroll
        for (int x = 0; x < C; x++) y[x] = T::mfma16(a, q[x][j], y[x]);
      }
#pragma unroll
      for (int x = 0; x < C; x++)
#pragma unroll
        for (int z = 0; z < 4; z++) s[x][4 * g + z] = y[x][z] * p.c_scale;
    }
    // Values that are none, of rows that some columns see and others do not (TOKENS): apart, as ones, and what sees one is none.
    v4i none[TOKENS ? NB : 1][TOKENS ? ND : 1];
    bool apart = false;
    if (r0 + ROWS > (TOKENS ? min(end, col.first_limit + 1) : end)) {  // rows behind the sequence's end: no weight, and no value that could be NaN
      uint32_t found = 0;
#pragma unroll
      for (int g = 0; g < NB; g++) {
        const int at = r0 + 16 * g + 4 * qd, n = end - at;
#pragma unroll
        for (int x = 0; x < C; x++)
#pragma unroll
          for (int y = 0; y < 4; y++) s[x][4 * g + y] = y < n && (!TOKENS || at + y <= limit[x]) ? s[x][4 * g + y] : -INFINITY;
#pragma unroll
        for (int j = 0; j < ND; j++)
#pragma unroll
          for (int y = 0; y < 4; y++) {
            tile.v[g][j][y] &= (int)f8_bytes(n);
            if constexpr (TOKENS) {
              const uint32_t flags = (((uint32_t)tile.v[g][j][y] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u, all = flags | (flags - (flags >> 7));
              found |= flags;
              none[g][j][y] = (int)(all & 0x38383838u);
              tile.v[g][j][y] &= (int)~all;
            }
          }
      }
      apart = __ballot(found != 0) != 0;
    }
    // weights as a pair of 16-bit numbers (bf16: off by at most 2^-17 of the weight; f16: by 2^-23 of it or 2^-36 of the reference's)
    v4i hi[C], lo[C];
#pragma unroll
    for (int x = 0; x < C; x++) {
      float most = s[x][0];
#pragma unroll
      for (int y = 1; y < 4 * NB; y++) most = fmaxf(most, s[x][y]);
      if (__ballot(most - m[x] > T::kTop)) {         // (see the element types)
        const float top = quarters_max(most), low = top - T::kRaise;
        const float mn = fmaxf(m[x], top - low > T::kTop ? top : low);       // (steps of 16, between scores of 2^27 and 2^28)
        const float keep = m[x] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[x] - mn);
        l[x] *= keep;
#pragma unroll
        for (int j = 0; j < NJ; j++)
#pragma unroll
          for (int y = 0; y < 4; y++) o[x][j][y] *= keep;
        m[x] = mn;
      }
      const float ref = m[x] == -INFINITY ? 0.f : m[x];
      float w[8];
#pragma unroll
      for (int y = 0; y < 8; y++) { w[y] = __builtin_amdgcn_exp2f(s[x][y] - ref); l[x] += w[y]; }
#pragma unroll
      for (int y = 0; y < 4; y++) {
        const uint32_t h = dense_pack<T>(w[2 * y], w[2 * y + 1]);
        hi[x][y] = (int)h;
        lo[x][y] = (int)dense_pack<T>(w[2 * y] - dense_low<T>(h), w[2 * y + 1] - dense_high<T>(h));
      }
    }
    const float s0 = __uint_as_float((uint32_t)__builtin_amdgcn_readlane(v_scale, NB * i)), s1 = __uint_as_float((uint32_t)__builtin_amdgcn_readlane(v_scale, NB * i + 1));
#pragma unroll
    for (int j = 0; j < NJ; j++) {
      const uint32_t c0 = (uint32_t)tile.v[0][j >> 2][j & 3], c1 = (uint32_t)tile.v[1][j >> 2][j & 3];
      const v4i a = {f8_pair<T, false>(c0, s0), f8_pair<T, true>(c0, s0), f8_pair<T, false>(c1, s1), f8_pair<T, true>(c1, s1)};
#pragma unroll
      for (int x = 0; x < C; x++) {
        o[x][j] = T::mfma16(a, hi[x], o[x][j]);
        o[x][j] = T::mfma16(a, lo[x], o[x][j]);
      }
    }
    if constexpr (TOKENS) {
      if (apart) {
#pragma unroll
        for (int x = 0; x < C; x++) {
          v4i sees;
#pragma unroll
          for (int y = 0; y < 4; y++) {
            const int at = r0 + 16 * (y >> 1) + 4 * qd + 2 * (y & 1);
            sees[y] = (int)dense_pack<T>(at <= limit[x] ? 1.f : 0.f, at + 1 <= limit[x] ? 1.f : 0.f);
          }
#pragma unroll
          for (int j = 0; j < NJ; j++) {
            const uint32_t c0 = (uint32_t)none[0][j >> 2][j & 3], c1 = (uint32_t)none[1][j >> 2][j & 3];
            const v4f n = T::mfma16(v4i{f8_pair<T, false>(c0, 1.f), f8_pair<T, true>(c0, 1.f), f8_pair<T, false>(c1, 1.f), f8_pair<T, true>(c1, 1.f)}, sees, v4f{0.f, 0.f, 0.f, 0.f});
#pragma unroll
            for (int y = 0; y < 4; y++) o[x][j][y] = n[y] > 0.f ? __builtin_nanf("") : o[x][j][y];
          }
        }
      }
    }
  };
  for (int t = wave; t < n_tiles; t += AHEAD * NW) {
    look_up(t);
    const int n = min(AHEAD, (n_tiles - t + NW - 1) / NW);
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
#pragma unroll
  for (int x = 0; x < C; x++) {
    const int G = min(col.n - 16 * x, 16);           // the set's columns
    if (G <= 0) break;
    const float sum = quarters_sum(l[x]);
    __syncthreads();
    if (c < G) {
      if (qd == 0) { m_sh[wave][c] = m[x]; l_sh[wave][c] = sum; }
      // (A head's dims start 4 c further on in its row, since the heads' rows begin at one bank.)
#pragma unroll
      for (int y = 0; y < 4; y++)
#pragma unroll
        for (int j = 0; j < NJ; j += 4)
          *(v4f*)(o_sh + (wave * G + c) * D + ((16 * j + 16 * qd + 4 * y + 4 * c) & (D - 1))) = v4f{o[x][j][y], o[x][j + 1][y], o[x][j + 2][y], o[x][j + 3][y]};
    }
    __syncthreads();
    p.G = G;
    dense_finish<T, D, NW, JOINS ? kF8Whole : 0>(p, at, idx, kv, o_sh, m_sh, l_sh, [&](int e) {
      if constexpr (TOKENS) {
        const int pair = col.row0 + 16 * x + e / D, token = pair / p.group;
        return p.out + (int64_t)(col.q_start + token) * p.out_ld + (kv * p.group + pair - token * p.group) * D + e % D;
      } else {
        return p.out + ((int64_t)at.b * p.Hkv * G + kv * G) * D + e;
      }
    });
    p.parts += (size_t)p.splits * p.Hkv * 16 * (D + 2);              // (of several tokens: the next set's words)
  }
}

template <class T, int D>
hipError_t launch_append(const DenseAppendParams& p, hipStream_t s) {
  const DenseF8Append a = dense_f8_append(p.n_tokens, p.B, p.Hq + 2 * p.Hkv, p.cu != nullptr);
  const bool once = (int64_t)p.n_tokens * (2 * p.Hq + 4 * p.Hkv) * D * 2 >= 100000000;
  const unsigned grid = (unsigned)(a.units * a.splits);
  if (once) k_dense_append_f8<T, D, true><<<grid, 256, 0, s>>>(p, a.splits);
  else k_dense_append_f8<T, D, false><<<grid, 256, 0, s>>>(p, a.splits);
  return hipGetLastError();
}
template <class T, int D, int NW, bool ONCE, int SETS, bool JOINS>
hipError_t launch_decode_form(const DenseDecodeParams& p, int64_t workgroups, hipStream_t s) {
  constexpr int LDS = NW * D * 4 * 16;
  static LdsLimit limit;
  if (LDS + NW * 16 * 8 > 65536) {
    const hipError_t e = wsvd_raise_lds(limit, (const void*)k_dense_decode_f8<T, D, NW, ONCE, SETS, JOINS>, LDS);
    if (e != hipSuccess) return e;
  }
  k_dense_decode_f8<T, D, NW, ONCE, SETS, JOINS><<<(unsigned)workgroups, 64 * NW, LDS, s>>>(p);
  return hipGetLastError();
}
template <class T, int D, bool ONCE>
hipError_t launch_decode_waves(const DenseDecodeParams& p, hipStream_t s) {
  const int64_t n = dense_decode_workgroups(p.B, p.Hkv, p.target, p.alone != 0), joins = p.alone ? 0 : dense_f8_joins(p.B, p.target, p.waves);
  if (joins) return launch_decode_form<T, D, 8, ONCE, 0, true>(p, n + joins * p.G * p.Hkv, s);
  return p.waves == 8 ? launch_decode_form<T, D, 8, ONCE, 0, false>(p, n, s) : p.waves == 4 ? launch_decode_form<T, D, 4, ONCE, 0, false>(p, n, s)
                                                                                 : launch_decode_form<T, D, 2, ONCE, 0, false>(p, n, s);
}
template <class T, int D>
hipError_t launch_decode(DenseDecodeParams p, hipStream_t s) {
  if (p.cu_q) {
    const DenseF8Columns c = dense_f8_columns(p.n_q, p.B, p.Hkv, p.group);
    p.tiles = (int)c.tiles;
    const int64_t n = c.tiles * p.splits * p.Hkv;
    if (c.joins) return launch_decode_form<T, D, 8, false, 1, true>(p, n + (int64_t)p.n_q * p.group * p.Hkv, s);
    return c.sets == 2 ? launch_decode_form<T, D, 8, false, 2, false>(p, n, s) : launch_decode_form<T, D, 8, false, 1, false>(p, n, s);
  }
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
