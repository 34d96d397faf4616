// Dense layers: attention of many query tokens per sequence (prompts packed one behind another, or the next tokens of
// sequences whose earlier rows are in a paged cache), tiled for the matrix cores.
//
//   S^T [64 keys x 32 queries] = K Q^T              keys from LDS, queries in registers
//   softmax down the columns                        a lane owns one query and half of a block's keys
//   O^T [d x 32 queries] += V^T P^T                 values read transposed from LDS (ds_read_b64_tr_b16)
//
// The order of the contraction over keys is free: the lane that ends up with a weight is the lane whose operand slot takes
// it, so P never leaves the registers and the transposed reads of V pick the keys in that order.  A query row is a (token,
// head) pair, token-major, so the G heads of a kv head share every staged key block, and a tile covers few tokens: less of
// the causal triangle is computed for nothing.
//
// Weights are fp32 up to the second product and in the sum, and rounded once to the 16 bits of its operand (off by at most 2^-8 of a
// weight in bf16, 2^-11 in f16).  Outputs are then off from 64 bits by 2.1e-3 to 2.3e-3 in bf16 and 2.2e-4 to 2.8e-4 in f16, where the output's own
// rounding makes 1.6e-3 to 1.7e-3 and 2.0e-4 to 2.1e-4: a pair of words a weight, as in the decode attention, would be half as many matrix
// products again in a loop that they bind.
//
// A workgroup is 4 waves of 32 query rows; two workgroups share a CU, so that one multiplies while the other starts, waits or ends.
// Blocks of 64 keys go straight from memory to LDS, two stages deep.  A wave runs one block's softmax under the next block's score
// products and its own first value products, and the next block's maximum under the other value products; what it costs is then
//   * matrix products: 1024 cycles per block and wave at d 128,
//   * vector instructions: about 120 and 32 exponentials, about as long, spread evenly over the products,
//   * power: at full load the chip runs at 1.9 GHz instead of 2.4 (the same call on zeros takes 0.84 of the time).
// Counted at 16 x 2048 tokens, of a SIMD's time: matrix cores 53 %, vector instructions 50 %, LDS instructions 40 % of a CU's, no bank
// conflicts.  Matrix and vector instructions of a SIMD's two waves hardly overlap.
// 1 x 8192 tokens, 32 heads of 128: 1.13 PFLOP/s without a mask, 1.08 causal (products of 16384^2 matrices on that card: 1.35); 16 x 2048
// tokens: 0.89, with 1.07 GB of queries, keys, values and outputs.  d 64: 0.97 without a mask, 0.90 causal.
// Tried and not faster: 8 waves to a workgroup (0.86 where 4 have 0.90 at 16 x 2048); 64 rows a wave, one wave a SIMD (0.71: the
// accumulators no longer fit the vector registers); the weights' sum by the matrix cores; the longest tiles of all sequences first
// (16 x 2048: 0.57, keys and values no longer stay in the L2); lines of later blocks fetched to the L2 ahead.
#include <algorithm>
#include <type_traits>
#include "wsvd_attn_common.h"
#include "wsvd_dense.h"

namespace {

constexpr int kKeys = 64;                            // keys of a staged block
// Blocks that a workgroup of several for one tile has at least: the join is a second launch of 4 to 5 us, a block takes 1 to 1.5.
constexpr int kLeastBlocks = 6;

// lds_copy16 without the compiler's knowledge: it would let every later read of LDS wait for the copy (the next block's, while
// this one is worked on: 16 x 2048 tokens 1124 us, with the loops' other waits gone 763).  The copies are waited for by
// lds_copy_wait_barrier alone.  (M0 is a reserved register: the compiler gives it to no value, writes it right before an instruction of its
// own that reads it, of which there is none here, and takes no clobber of it: it warns that one has no defined effect.)
WSVD_DEV void copy16(uint32_t lds, const uint8_t* base, uint32_t offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "memory");
}

// The same number, as one that the compiler knows nothing of: what is made of it is made where it is needed, and not kept in a register
// over the loops between.
WSVD_DEV int anew(int x) {
  asm volatile("" : "+v"(x));
  return x;
}
WSVD_DEV int anew_scalar(int x) {
  asm volatile("" : "+s"(x));
  return x;
}

// A workgroup's sequence and tile (a sequence's last tiles, which see the most keys, first), from one read of the lengths.  Where
// workgroups take two tiles (p.pairs), the second is as far from the sequence's first as the first is from its last, so that all
// pairs of a sequence cost the same; the tile in the middle of an odd number stays alone.
struct PromptPlace {
  int b, q_start, nq, kv_start, nk;
  int tile, second;                                  // second: -1 where there is none
  int ahead;                                         // query token i sees the keys up to i + ahead
  int splits;                                        // workgroups that share the tile's keys
};
// blocks of keys that a tile's last row sees
template <int ROWS>
WSVD_DEV int prompt_blocks(const DensePromptParams& p, const PromptPlace& at, int tile) {
  const int seen = p.causal ? min(at.nk, (min((tile + 1) * ROWS, at.nq * p.G) - 1) / p.G + at.ahead + 1) : at.nk;
  return seen > 0 ? (seen + kKeys - 1) / kKeys : 0;
}
template <bool PAGED, int ROWS>
WSVD_DEV bool prompt_place(const DensePromptParams& p, int idx, int lane, PromptPlace& at) {
  const int most = PAGED ? p.pages.max_pages * p.pages.page_rows : p.n_kv;
  for (int base = 0, before = 0; base < p.B; base += 64) {
    const int i = base + lane;
    int qs = 0, n_q = 0, ks = 0, n_k = 0;
    if (i < p.B) {
      const int q0 = p.cu_q[i], q1 = p.cu_q[i + 1];
      if (PAGED) {
        n_k = p.pages.seq_lens[i];
      } else {
        const int k0 = p.cu_kv[i], k1 = p.cu_kv[i + 1];
        ks = min(max(k0, 0), most);
        n_k = min(max(k1, ks), most) - ks;
      }
      qs = min(max(q0, 0), p.n_q);
      n_q = min(max(q1, qs), p.n_q) - qs;
    }
    const int tiles = (n_q * p.G + ROWS - 1) / ROWS, k = p.pairs ? (tiles + 1) / 2 : tiles, end = before + wave_prefix_int(k);
    const unsigned long long m = __ballot(end > idx);
    before = __builtin_amdgcn_readlane(end, 63);
    if (!m) continue;
    const int l = __builtin_ctzll(m);
    at.b = base + l;
    const int from_end = idx - (__builtin_amdgcn_readlane(end, l) - __builtin_amdgcn_readlane(k, l));
    at.tile = __builtin_amdgcn_readlane(tiles, l) - 1 - from_end;
    at.second = p.pairs && from_end < at.tile ? from_end : -1;
    at.q_start = __builtin_amdgcn_readlane(qs, l); at.nq = __builtin_amdgcn_readlane(n_q, l);
    at.kv_start = __builtin_amdgcn_readlane(ks, l); at.nk = __builtin_amdgcn_readlane(n_k, l);
    if (PAGED) {
      if (at.nk > most && threadIdx.x == 0) atomicExch(p.err_word, (int)WSVD_E_SHAPE);
      at.nk = min(max(at.nk, 0), most);
    }
    at.ahead = at.nk - at.nq;
    at.splits = max(1, min(p.splits, prompt_blocks<ROWS>(p, at, at.tile) / kLeastBlocks));
    return true;
  }
  return false;
}
WSVD_DEV float* prompt_part(const DensePromptParams& p, int idx, int kv, int split, int rows, int d) {
  return p.parts + (((size_t)idx * p.Hkv + kv) * p.splits + split) * rows * (d + 2);
}

template <class T, int D, bool PAGED, int NW>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(D == 128 ? 2 : 3, D == 128 ? 2 : 3))) void k_dense_prompt(DensePromptParams p) {
  constexpr int ROWS = 32 * NW;                      // query rows of a workgroup
  constexpr int PIECES = D / 8, RPI = 64 / PIECES;   // 16-byte pieces of a row; rows that one copy of a wave brings
  constexpr int COPIES = kKeys / NW / RPI;
  constexpr int ROW_BYTES = 2 * D, PLANE = kKeys * ROW_BYTES, STAGE = 2 * PLANE;
  constexpr int ND = D / 32, NS = D / 16;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[2 * STAGE];
  __shared__ int odd_sh[NW];                         // a wave's results that are no numbers
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 31, half = lane >> 5;
  const int kv = blockIdx.x % p.Hkv, split = blockIdx.x / p.Hkv % p.splits, idx = blockIdx.x / p.Hkv / p.splits;
  PromptPlace at;
  if (!prompt_place<PAGED, ROWS>(p, idx, lane, at) || split >= at.splits) return;
  // A workgroup of several for a tile has a part of the tile's blocks: key0 on, everything below counts from there.
  int tile = at.tile, n_blocks = prompt_blocks<ROWS>(p, at, tile);
  const int block0 = dense_share(split, n_blocks, at.splits), key0 = block0 * kKeys;
  n_blocks = dense_share(split + 1, n_blocks, at.splits) - block0;
  const int b = at.b, q_start = at.q_start, NR = at.nq * p.G, ahead = at.ahead - key0, nk = at.nk - key0;
  // this lane's query: operand of the score product
  v4i q[NS];
  auto load_q = [&](int tile) {
    const int i = anew(lane), row = min(tile * ROWS + 32 * wave + (i & 31), NR - 1), tok = row / p.G, head = kv * p.G + row - tok * p.G;
    const uint16_t* qp = p.q + (int64_t)(q_start + tok) * p.q_ld + head * D + (i >> 5) * 8;
#pragma unroll
    for (int s = 0; s < NS; s++) q[s] = *(const v4i*)(qp + s * 16);
  };
  load_q(tile);

  // staging: a wave's share of a block's rows, the 16-byte pieces of a row permuted so that the reads below meet no bank twice
  const uint32_t lds0 = lds_address(lds);
  const int my_row = lane / PIECES, my_piece = lane % PIECES;
  static_assert(kKeys / NW == 16 && COPIES * RPI == 16, "");
  const uint32_t k_stride = PAGED ? ROW_BYTES : (uint32_t)p.k_ld * 2u, v_stride = PAGED ? ROW_BYTES : (uint32_t)p.v_ld * 2u;
  const uint32_t k_piece = (my_piece ^ (D == 128 ? my_row : my_row >> 1)) * 16, v_piece = (my_piece ^ (D == 128 ? my_row << 2 : (my_row & 2) << 1)) * 16;
  // Paged: a wave's rows of a block lie in one granule of 16.  Where they lie is looked up for 64 blocks at a time, a lane for each.
  static_assert(16 % (kKeys / NW) == 0, "");
  bool bad = false;
  uint32_t at_low = 0, at_high = 0;
  int looked_up = 0;                                 // the first of those blocks
  auto look_up = [&](int kb) {
    looked_up = kb;
    const int granule = min((key0 + (kb + lane) * kKeys + wave * (kKeys / NW)) >> 4, (at.nk - 1) >> 4), pg = dense_page_index(granule, p.pages.page_magic);
    const int page = dense_page(p.pages.block_table[(size_t)b * p.pages.max_pages + pg], p.pages.n_pages, bad);
    const uint64_t bytes = dense_pool_row(page, granule, pg, kv, p.Hkv, p.pages.page_rows) * ROW_BYTES;
    at_low = (uint32_t)bytes; at_high = (uint32_t)(bytes >> 32);
  };
  // (rows of a copy are a scalar's distance apart: what a lane adds is the same for every block)
  auto stage = [&](int kb, int buf, bool keys) {
    const uint32_t to = lds0 + buf * STAGE + (keys ? 0 : PLANE) + wave * (16 * ROW_BYTES);
    const uint32_t stride = keys ? k_stride : v_stride;
    if (!PAGED && (kb + 1) * kKeys > nk) {           // a block that ends before its last row: that one in the place of those behind it
      const uint8_t* from = (const uint8_t*)((keys ? p.k : p.v) + ((int64_t)at.kv_start + key0 + kb * kKeys) * (keys ? p.k_ld : p.v_ld) + kv * D);
      const int row = wave * 16 + anew(my_row);
#pragma unroll 1
      for (int i = 0; i < COPIES; i++)               // (rarely: small rather than fast)
        copy16(to + i * 1024, from, (uint32_t)min(row + i * RPI, nk - 1 - kb * kKeys) * stride + (keys ? k_piece ^ (i << 6) : v_piece));
      return;
    }
    const uint8_t* from;
    if (PAGED) {
      const int i = kb - looked_up;
      from = (const uint8_t*)(keys ? p.pages.k : p.pages.v) +
             ((uint64_t)(uint32_t)__builtin_amdgcn_readlane(at_low, i) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane(at_high, i) << 32);
    } else {
      from = (const uint8_t*)((keys ? p.k : p.v) + ((int64_t)at.kv_start + key0 + kb * kKeys + wave * 16) * (keys ? p.k_ld : p.v_ld) + kv * D);
    }
#pragma unroll
    for (int i = 0; i < COPIES; i++)
      copy16(to + i * 1024, from + (uint64_t)(i * RPI) * stride, my_row * stride + (keys ? k_piece ^ (i << 6) : v_piece));
  };

  // addresses of the operands in a stage
  uint32_t k_at[NS], v_at[ND];
  {
    const int sw = D == 128 ? n & 15 : (n >> 1) & 7;
#pragma unroll
    for (int s = 0; s < NS; s++) k_at[s] = lds0 + n * ROW_BYTES + ((2 * s + half) ^ sw) * 16;
    const int i = lane & 15, key = 4 * half + (i >> 2);
#pragma unroll
    for (int d = 0; d < ND; d++) {
      const int chunk = D == 128 ? d ^ (i >> 2) : d ^ (i >> 3);
      v_at[d] = lds0 + PLANE + key * ROW_BYTES + chunk * 64 + ((lane >> 4) & 1) * 32 + (i & 3) * 8;
    }
  }
  typedef short v4s __attribute__((ext_vector_type(4)));
  auto read_k = [&](uint32_t stage, int kb, int s) {
    return *(const __attribute__((address_space(3))) v4i*)(uintptr_t)(k_at[s] + stage + kb * 32 * ROW_BYTES);
  };
  auto read_v = [&](uint32_t stage, int d, int s) {  // 16 keys from 16 s, 32 dims from 32 d
    const uint32_t at = v_at[d] + stage + s * 16 * ROW_BYTES;
    const v2i lo = __builtin_bit_cast(v2i, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(uintptr_t)at));
    const v2i hi = __builtin_bit_cast(v2i, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(uintptr_t)(at + 8 * ROW_BYTES)));
    return v4i{lo[0], lo[1], hi[0], hi[1]};
  };

  struct Scores { v16f s[2]; };
  int limit = 0;                                     // the last key that this lane's query sees
  float m, l[2];                                     // maximum; sums of every other weight
  v16f o[ND];
  auto clear = [&] {
    m = -INFINITY; l[0] = l[1] = 0.f;
#pragma unroll
    for (int d = 0; d < ND; d++)
#pragma unroll
      for (int i = 0; i < 16; i++) o[d][i] = 0.f;
  };

  auto multiply = [&](Scores& r, uint32_t stage) {   // a block's scores
#pragma unroll
    for (int h = 0; h < 2; h++)
#pragma unroll
      for (int i = 0; i < 16; i++) r.s[h][i] = 0.f;
#pragma unroll
    for (int x = 0; x < NS; x++)
#pragma unroll
      for (int h = 0; h < 2; h++) r.s[h] = T::mfma32(read_k(stage, h, x), q[x], r.s[h]);
  };
  // keys that this lane's query does not see
  auto last_seen = [&](int kb) { return limit - kb * kKeys - 4 * half; };
  auto hide = [&](Scores& r, int at, int rel) { r.s[at >> 4][at & 15] = 32 * (at >> 4) + 8 * ((at & 15) >> 2) + (at & 3) > rel ? -INFINITY : r.s[at >> 4][at & 15]; };
  auto hide_all = [&](Scores& r, int kb) {
    const int rel = last_seen(kb);
#pragma unroll
    for (int i = 0; i < 32; i++) hide(r, i, rel);
  };
  auto largest = [&](const Scores& r) {
    float most = r.s[0][0];
#pragma unroll
    for (int h = 0; h < 2; h++)
#pragma unroll
      for (int i = 0; i < 16; i++) most = fmaxf(most, r.s[h][i]);
    return most;
  };
  auto refer = [&](float most, auto careful) {       // (see the element types; the difference is formed as the weights' are, without rounding)
    if (__ballot(fmaf(most, p.c_scale, -m) > T::kTop)) {
      const float top = halves_max(most), low = fmaf(top, p.c_scale, -T::kRaise);
      const float mn = fmaxf(m, fmaf(top, p.c_scale, -low) > T::kTop ? top * p.c_scale : low);     // (steps of 16, between scores of 2^27 and 2^28)
      const float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
      l[0] *= keep; l[1] *= keep;
#pragma unroll
      for (int d = 0; d < ND; d++)
#pragma unroll
        for (int i = 0; i < 16; i++) o[d][i] = decltype(careful)::value ? dense_scaled(o[d][i], keep) : o[d][i] * keep;
      m = mn;
    }
  };
  struct Weights { uint32_t w[4][4]; };             // a quarter of the keys: 16, 4 words of which are this lane's
  auto weigh = [&](const Scores& r, Weights& w, int j) {           // two weights, one of 16 words
    const float ref = m == -INFINITY ? 0.f : m;
    const int at = 2 * (j & 7);
    const float a = __builtin_amdgcn_exp2f(fmaf(r.s[j >> 3][at], p.c_scale, -ref)), c = __builtin_amdgcn_exp2f(fmaf(r.s[j >> 3][at + 1], p.c_scale, -ref));
    l[0] += a; l[1] += c;
    w.w[j >> 2][j & 3] = dense_pack<T>(a, c);
  };
  auto operand = [&](const Weights& w, int x) { return v4i{(int)w.w[x][0], (int)w.w[x][1], (int)w.w[x][2], (int)w.w[x][3]}; };

  // One block's weights under the next block's score products (where there is a next one), then its value products under the next
  // block's maximum.  V0, K1: the stages they lie in; hidden: whether a query may not see all of the next block.
  auto step = [&](const Scores& r, Scores& next, uint32_t V0, uint32_t K1, int kb_next, auto more, auto hidden) {
    constexpr bool MORE = decltype(more)::value, HIDDEN = decltype(hidden)::value;
    Weights w;
    v4i v[2][ND];
    // Everything in the order in which it is to run: operands are asked for AHEAD products before they are needed, and a product is
    // followed by the vector instructions that run beside it (the compiler, left to itself, asks and waits for each operand).  The
    // weights of EARLY quarters of the keys come beside the next block's score products, those of the others beside the value products of
    // the first quarters, the next block's maxima beside the last (all weights beside the scores: 3 x 333 tokens behind 1501 rows
    // 51.6 us, two quarters 48.2, three 48.5; 16 x 2048 tokens 647, 632, 631).  AHEAD 4 at d_head 64 takes registers that three waves a
    // SIMD do not have (2048 tokens behind 8000, 16 / 2 heads: 150 us, 134 with 2).
    constexpr int AHEAD = D == 128 ? 4 : 2, NP = 2 * NS, EARLY = 2, FREE = 4 - EARLY;
    if (MORE) {
      v4i k[AHEAD];
#pragma unroll
      for (int i = 0; i < AHEAD; i++) k[i] = read_k(K1, i & 1, i >> 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < NP; i++) {
        next.s[i & 1] = T::mfma32(k[i % AHEAD], q[i >> 1], i < 2 ? v16f{} : next.s[i & 1]);
        if (i + AHEAD < NP) k[i % AHEAD] = read_k(K1, i & 1, (i + AHEAD) >> 1);
        else {
#pragma unroll
          for (int d = (i + AHEAD - NP) * ND / AHEAD; d < (i + AHEAD - NP + 1) * ND / AHEAD; d++) v[0][d] = read_v(V0, d, 0);
        }
#pragma unroll
        for (int j = i * 4 * EARLY / NP; j < (i + 1) * 4 * EARLY / NP; j++) weigh(r, w, j);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
#pragma unroll
      for (int d = 0; d < ND; d++) v[0][d] = read_v(V0, d, 0);
#pragma unroll
      for (int j = 0; j < 4 * EARLY; j++) weigh(r, w, j);
    }
    const int rel = HIDDEN ? last_seen(kb_next) : 0;
    float most[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int x = 0; x < 4; x++) {
      const v4i pw = operand(w, x);
#pragma unroll
      for (int d = 0; d < ND; d++) {
        o[d] = T::mfma32(v[x & 1][d], pw, o[d]);
        if (x < 3) v[(x + 1) & 1][d] = read_v(V0, d, x + 1);
        if (x < FREE) {
#pragma unroll
          for (int j = d * 4 / ND; j < (d + 1) * 4 / ND; j++) weigh(r, w, 4 * (x + EARLY) + j);
        } else if (MORE) {
          constexpr int N = 32 / ((4 - FREE) * ND);
#pragma unroll
          for (int i = 0; i < N; i++) {
            const int at = ((x - FREE) * ND + d) * N + i;
            if (HIDDEN) hide(next, at, rel);
            most[i & 1] = fmaxf(most[i & 1], next.s[at >> 4][at & 15]);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if (MORE) refer(fmaxf(most[0], most[1]), std::false_type{});
  };
  // A block whose values may be no numbers: those must not meet the weight 0 of a query that does not see them, or one that is only
  // rounded to 0.  The products leave them out, and the queries that do see them get them added (NaN where the score is -inf).
  auto careful = [&](int kb) {
    const uint32_t at = (kb & 1) * STAGE;
    Scores r;
    Weights w;
    multiply(r, at);
    hide_all(r, kb);
    refer(largest(r), std::true_type{});
    for (int j = 0; j < 16; j++) weigh(r, w, j);
    uint32_t odd = 0;
#pragma unroll
    for (int x = 0; x < 4; x++) {
      const v4i pw = operand(w, x);
#pragma unroll
      for (int d = 0; d < ND; d++) {
        v4i a = read_v(at, d, x);
#pragma unroll
        for (int y = 0; y < 4; y++) {
          const uint32_t t = dense_odd<T>((uint32_t)a[y]);
          odd |= t;
          a[y] &= (int)~t;
        }
        o[d] = T::mfma32(a, pw, o[d]);
      }
    }
    if (__ballot(odd != 0)) {
      const int rel = limit - kb * kKeys, half = anew(lane) >> 5;
      uint32_t none = 0;                             // of this lane's keys, those with a score of -inf
#pragma unroll 1
      for (int h = 1; h >= 0; h--) {                 // (scored again: nothing of them is kept over the products)
        v16f x = {};
#pragma unroll
        for (int s = 0; s < NS; s++) x = T::mfma32(read_k(anew_scalar(at), anew_scalar(h), s), q[s], x);
#pragma unroll
        for (int i = 15; i >= 0; i--) none = 2 * none + (x[i] == -INFINITY);
      }
      const uint32_t other = (uint32_t)__shfl_xor((int)none, 32);
#pragma unroll 1
      for (int key = 0; key < kKeys; key++) {
        const bool sees = key <= rel;
        const uint32_t theirs = (key >> 2 & 1) == half ? none : other;
        const float weight = (float)(~theirs >> (16 * (key >> 5) + 4 * (key >> 3 & 3) + (key & 3)) & 1u);
        const uint32_t row_at = lds0 + at + PLANE + key * ROW_BYTES;
        const int sw = D == 128 ? (key & 3) << 2 : ((key >> 1) & 1) << 2;
#pragma unroll
        for (int d = 0; d < ND; d++)
#pragma unroll
          for (int g = 0; g < 4; g++) {
            const int dim = 32 * d + 8 * g + 4 * half;
            const v2i x = *(const __attribute__((address_space(3))) v2i*)(uintptr_t)(row_at + ((dim >> 3) ^ sw) * 16 + (dim & 7) * 2);
            const uint32_t t0 = dense_odd<T>((uint32_t)x[0]), t1 = dense_odd<T>((uint32_t)x[1]);
            if (sees && (t0 & 0x8000u)) o[d][4 * g] = fmaf(dense_low<T>((uint32_t)x[0]), weight, o[d][4 * g]);
            if (sees && (t0 >> 31)) o[d][4 * g + 1] = fmaf(dense_high<T>((uint32_t)x[0]), weight, o[d][4 * g + 1]);
            if (sees && (t1 & 0x8000u)) o[d][4 * g + 2] = fmaf(dense_low<T>((uint32_t)x[1]), weight, o[d][4 * g + 2]);
            if (sees && (t1 >> 31)) o[d][4 * g + 3] = fmaf(dense_high<T>((uint32_t)x[1]), weight, o[d][4 * g + 3]);
          }
      }
    }
  };

  // Block kb + 1's keys and block kb's values are there, and nobody reads the stages any more that the next copies go to.  Behind
  // the last block come the first keys of the workgroup's second tile.
  int next_blocks = at.second >= 0 ? prompt_blocks<ROWS>(p, at, at.second) : 0;
  auto sync = [&](int kb) {
    lds_copy_wait_barrier<0>();
    if (PAGED && kb + 2 >= looked_up + 64) look_up(anew_scalar(kb + 1));
    if (kb + 2 < n_blocks) stage(kb + 2, kb & 1, true);
    if (kb + 1 < n_blocks) stage(kb + 1, (kb + 1) & 1, false);
    else if (next_blocks > 0) {
      if (PAGED && looked_up != 0) look_up(anew_scalar(0));
      stage(anew_scalar(0), 0, true);
      if (next_blocks > 1) stage(anew_scalar(1), 1, true);
    }
  };
  auto queries_there = [&] {                         // no wait for them in the loops, which would be one for the copies too
#pragma unroll
    for (int s = 0; s < NS; s++) asm volatile("" : "+v"(q[s]));
  };
  if (n_blocks > 0) {
    if (PAGED) look_up(0);
    stage(0, 0, true);
    if (n_blocks > 1) stage(1, 1, true);
    stage(0, 0, false);
  }
  queries_there();
  if (n_blocks > 0) lds_copy_wait_barrier<0>();
  constexpr std::true_type yes{};
  constexpr std::false_type no{};
#pragma unroll 1
  for (;;) {
    // a wave's 32 rows: the keys that its last one sees, and those that all of them see
    const int row0 = tile * ROWS, wrow = row0 + 32 * wave, wlast = min(wrow + 31, NR - 1), here = min(nk, n_blocks * kKeys);
    const int wseen = wrow >= NR ? 0 : p.causal ? min(here, wlast / p.G + ahead + 1) : here;
    const int wall = p.causal ? wrow / p.G + ahead + 1 : here;
    const int n_mine = (max(wseen, 0) + kKeys - 1) / kKeys;
    const int n_whole = max(0, min(wseen, wall)) / kKeys;            // blocks that all of the wave's queries see whole
    limit = p.causal ? min(wrow + n, NR - 1) / p.G + ahead : nk - 1;
    clear();
    if (n_blocks > 0) {
      Scores r0, r1;
      int kb = 0;
      if (n_mine > 0) {
        multiply(r0, 0);
        if (n_whole == 0) hide_all(r0, 0);
        refer(largest(r0), no);
      }
      sync(0);                                       // (the third block's keys go where the first one's were)
      if (n_mine > 0) {
        for (; kb + 2 < n_whole; kb += 2) {
          __builtin_amdgcn_s_setprio(1);             // (the wave that multiplies goes before the one that copies or waits: 4 % at 8192 tokens)
          step(r0, r1, 0, STAGE, 0, yes, no);
          __builtin_amdgcn_s_setprio(0);
          sync(kb + 1);
          __builtin_amdgcn_s_setprio(1);
          step(r1, r0, STAGE, 0, 0, yes, no);
          __builtin_amdgcn_s_setprio(0);
          sync(kb + 2);
        }
        for (; kb + 1 < n_mine; kb++) {
          __builtin_amdgcn_s_setprio(1);
          step(r0, r1, (kb & 1) * STAGE, STAGE - (kb & 1) * STAGE, kb + 1, yes, yes);
          __builtin_amdgcn_s_setprio(0);
          r0 = r1;
          sync(kb + 1);
        }
      }
      if (next_blocks > 0) load_q(at.second);        // (the last scores are there)
      if (n_mine > 0) step(r0, r1, (kb & 1) * STAGE, 0, 0, no, no);
      for (; kb + 1 < n_blocks; kb++) sync(kb + 1);  // (waves whose queries see no more of the keys still copy)

      // Something is no number: it may be a value that met a weight of 0.  All once more, carefully (results that should be no
      // numbers come out the same).
      float zero = 0.f;                              // NaN where a value is infinite or none
#pragma unroll
      for (int d = 0; d < ND; d++)
#pragma unroll
        for (int i = 0; i < 16; i++) zero = fmaf(o[d][i], 0.f, zero);
      odd_sh[wave] = __ballot(zero != 0.f) != 0;
      queries_there();
      lds_copy_wait_barrier<0>();                    // (the second tile's keys are there, and nobody reads this one's any more)
      bool odd = false;
#pragma unroll
      for (int w = 0; w < NW; w++) odd = odd || odd_sh[w] != 0;
      if (odd) {
        clear();
        if (next_blocks > 0) { load_q(tile); queries_there(); }
        for (kb = 0; kb < n_blocks; kb++) {
          if (PAGED && kb % 64 == 0) look_up(anew_scalar(kb));
          stage(kb, kb & 1, true);
          stage(kb, kb & 1, false);
          lds_copy_wait_barrier<0>();
          if (kb < n_mine) careful(kb);
        }
        if (next_blocks > 0) {
          load_q(at.second);
          queries_there();
          if (PAGED) look_up(anew_scalar(0));
          __syncthreads();
          stage(anew_scalar(0), 0, true);
          if (next_blocks > 1) stage(anew_scalar(1), 1, true);
          lds_copy_wait_barrier<0>();
        }
      }
    }
    if (next_blocks > 0) stage(anew_scalar(0), 0, false);
    if (at.splits > 1) {                             // a part: as it is, for k_dense_prompt_join
      float* const part = prompt_part(p, idx, kv, split, ROWS, D);
      const int i0 = anew(lane), half = i0 >> 5, r = 32 * wave + (i0 & 31);
      const float sum = halves_sum(l[0] + l[1]);
      if (half == 0) { part[2 * r] = m; part[2 * r + 1] = sum; }
#pragma unroll
      for (int d = 0; d < ND; d++)
#pragma unroll
        for (int g = 0; g < 4; g++)
          *(v4f*)(part + 2 * ROWS + r * D + 32 * d + 8 * g + 4 * half) =
              v4f{o[d][4 * g], o[d][4 * g + 1], o[d][4 * g + 2], o[d][4 * g + 3]};
      break;
    }
    // The output from the accumulators, 16 bytes a lane: the halves of a wave have 4 of 8 dims each, and swap so that the first half
    // stores the even pieces and the second the odd ones.
    const float sum = halves_sum(l[0] + l[1]), inv = sum == 0.f ? 0.f : 1.f / sum;
    if (__ballot(sum == 0.f)) {                      // zeros, whatever the values are that scores of -inf met
#pragma unroll
      for (int d = 0; d < ND; d++)
#pragma unroll
        for (int i = 0; i < 16; i++) o[d][i] = sum == 0.f ? 0.f : o[d][i];
    }
    const int i0 = anew(lane), row = wrow + (i0 & 31);
    if (row < NR) {
      const int tok = row / p.G;
      uint16_t* const to = p.out + (int64_t)(q_start + tok) * p.out_ld + (kv * p.G + row - tok * p.G) * D + (i0 >> 5) * 8;
#pragma unroll
      for (int d = 0; d < ND; d++)
#pragma unroll
        for (int g = 0; g < 4; g += 2) {
          v4i x;
#pragma unroll
          for (int i = 0; i < 2; i++) {
            const uint32_t even = dense_pack<T>(o[d][4 * g + 2 * i] * inv, o[d][4 * g + 2 * i + 1] * inv);
            const uint32_t odd = dense_pack<T>(o[d][4 * g + 4 + 2 * i] * inv, o[d][4 * g + 4 + 2 * i + 1] * inv);
            const auto r = __builtin_amdgcn_permlane32_swap(even, odd, false, false);
            x[i] = (int)r[0]; x[2 + i] = (int)r[1];
          }
          *(v4i*)(to + 32 * d + 8 * g) = x;
        }
    }
    if (next_blocks == 0 && (at.second < 0 || tile == at.second)) break;
    tile = at.second;
    n_blocks = next_blocks;
    next_blocks = 0;
  }
  if (__ballot(bad) && lane == 0) atomicExch(p.err_word, (int)WSVD_E_SHAPE);
}

// The parts of the tiles that several workgroups share, joined in their order: 16 rows of a tile per workgroup, 8 or 4 dims of a
// row per thread.
template <class T, int D, bool PAGED, int ROWS>
__global__ __launch_bounds__(256) void k_dense_prompt_join(DensePromptParams p) {
  constexpr int N = D / 16;
  const int lane = threadIdx.x & 63, kv = blockIdx.x % p.Hkv, idx = blockIdx.x / p.Hkv;
  PromptPlace at;
  if (!prompt_place<PAGED, ROWS>(p, idx, lane, at) || at.splits == 1) return;
  const int r = blockIdx.y * 16 + threadIdx.x / 16, x = threadIdx.x % 16 * N, row = at.tile * ROWS + r;
  if (row >= at.nq * p.G) return;
  float M = -INFINITY, L = 0.f, O[N];
#pragma unroll
  for (int i = 0; i < N; i++) O[i] = 0.f;
  const float* const parts = prompt_part(p, idx, kv, 0, ROWS, D);
  for (int s0 = 0; s0 < at.splits; s0 += 4) {        // four in flight
    float m[4], l[4], mn = M;
    v4f o[4][N / 4];
#pragma unroll
    for (int k = 0; k < 4; k++) {
      const float* const part = parts + (size_t)min(s0 + k, at.splits - 1) * ROWS * (D + 2);
      m[k] = part[2 * r]; l[k] = part[2 * r + 1];
#pragma unroll
      for (int i = 0; i < N / 4; i++) o[k][i] = *(const v4f*)(part + 2 * ROWS + r * D + x + 4 * i);
    }
#pragma unroll
    for (int k = 0; k < 4; k++) mn = fmaxf(mn, m[k]);
    const float keep = M == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(M - mn);
    L *= keep;                                       // (nothing seen: the sum and the row are 0, or NaN)
#pragma unroll
    for (int i = 0; i < N; i++) O[i] = dense_scaled(O[i], keep);
#pragma unroll
    for (int k = 0; k < 4; k++)
      if (s0 + k < at.splits) {
        const float add = m[k] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[k] - mn);
        L += l[k] * add;
#pragma unroll
        for (int i = 0; i < N; i++) O[i] += dense_scaled(o[k][i / 4][i % 4], add);
      }
    M = mn;
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
  const int t = row / p.G;
  uint32_t out[N / 2];
#pragma unroll
  for (int i = 0; i < N / 2; i++) out[i] = L == 0.f ? 0 : dense_pack<T>(O[2 * i] * inv, O[2 * i + 1] * inv);
  __builtin_memcpy(__builtin_assume_aligned(p.out + (int64_t)(at.q_start + t) * p.out_ld + (kv * p.G + row - t * p.G) * D + x, N * 2), out, N * 2);
}

template <class T, int D, bool PAGED>
hipError_t launch(DensePromptParams& p, hipStream_t s) {
  constexpr int NW = 4, ROWS = 32 * NW;
  static_assert(ROWS == kDensePromptRows, "");
  const DensePromptGrid grid = dense_prompt_grid(p.n_q, p.B, p.Hkv, p.G, p.causal != 0);
  const int64_t wgs = grid.workgroups;
  p.pairs = grid.pairs;
  // no sequence has more keys than there are, and no workgroup of several fewer than kLeastBlocks blocks of them
  const int64_t keys = PAGED ? (int64_t)p.pages.max_pages * p.pages.page_rows : p.n_kv;
  const int64_t most = std::min<int64_t>({32, kDensePromptParts / wgs, (keys + kKeys - 1) / kKeys / kLeastBlocks});
  p.splits = p.pairs ? 1 : (int)std::max<int64_t>(most, 1);
  k_dense_prompt<T, D, PAGED, NW><<<dim3((unsigned)(wgs * p.splits)), 64 * NW, 0, s>>>(p);
  if (p.splits > 1) k_dense_prompt_join<T, D, PAGED, ROWS><<<dim3((unsigned)wgs, ROWS / 16), 256, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t wsvd_launch_dense_prompt(DensePromptParams& p, int dtype, int d, bool paged, hipStream_t s) {
  if (dtype == WSVD_BF16) {
    if (d == 128) return paged ? launch<DenseBf16, 128, true>(p, s) : launch<DenseBf16, 128, false>(p, s);
    return paged ? launch<DenseBf16, 64, true>(p, s) : launch<DenseBf16, 64, false>(p, s);
  }
  if (d == 128) return paged ? launch<DenseF16, 128, true>(p, s) : launch<DenseF16, 128, false>(p, s);
  return paged ? launch<DenseF16, 64, true>(p, s) : launch<DenseF16, 64, false>(p, s);
}
