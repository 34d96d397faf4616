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
#include <type_traits>
#include "wsvd_dense.h"

namespace {

constexpr int kKeys = 64;                            // keys of a staged block

// lds_copy16 without the compiler's knowledge: it would let every later read of LDS wait for the copy (the next block's, while
// this one is worked on).  The copies are waited for by lds_copy_wait_barrier alone.
WSVD_DEV void copy16(uint32_t lds, const uint8_t* base, uint32_t offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "memory");
}

template <class T, int D, bool PAGED, int NW>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_dense_prompt(DensePromptParams p) {
  constexpr int ROWS = 32 * NW;                      // query rows of a workgroup
  constexpr int PIECES = D / 8, RPI = 64 / PIECES;   // 16-byte pieces of a row; rows that one copy of a wave brings
  constexpr int COPIES = kKeys / NW / RPI;
  constexpr int ROW_BYTES = 2 * D, PLANE = kKeys * ROW_BYTES, STAGE = 2 * PLANE;
  constexpr int ND = D / 32, NS = D / 16;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[2 * STAGE];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 31, half = lane >> 5;
  const int kv = blockIdx.x % p.Hkv;

  // this workgroup's sequence and tile: the last tiles, which see the most keys, first
  auto bounds = [&](const int* cu, int b, int most, int& start) {
    start = min(max(cu[b], 0), most);
    return min(max(cu[b + 1], start), most) - start;
  };
  int b = -1, tile = 0;
  {
    int total = 0;
    for (int base = 0; base < p.B; base += 64) {
      int start, k = 0;
      if (base + lane < p.B) k = (bounds(p.cu_q, base + lane, p.n_q, start) * p.G + ROWS - 1) / ROWS;
      total += wave_sum_int(k);
    }
    const int idx = total - 1 - (int)(blockIdx.x / p.Hkv);
    if (idx < 0) return;
    int before = 0;
    for (int base = 0; base < p.B; base += 64) {
      int start, k = 0;
      if (base + lane < p.B) k = (bounds(p.cu_q, base + lane, p.n_q, start) * p.G + ROWS - 1) / ROWS;
      const int end = before + wave_prefix_int(k);
      const unsigned long long m = __ballot(end > idx);
      if (m) {
        const int l = __builtin_ctzll(m);
        b = base + l;
        tile = idx - (__builtin_amdgcn_readlane(end, l) - __builtin_amdgcn_readlane(k, l));
        break;
      }
      before = __builtin_amdgcn_readlane(end, 63);
    }
  }
  int q_start, kv_start = 0;
  const int nq = bounds(p.cu_q, b, p.n_q, q_start);
  int nk;
  if (PAGED) {
    const int len = p.pages.seq_lens[b], most = p.pages.max_pages * p.pages.page_rows;
    nk = min(max(len, 0), most);
    if (len > most && tile == 0 && kv == 0 && threadIdx.x == 0) atomicExch(p.err_word, (int)WSVD_E_SHAPE);
  } else {
    nk = bounds(p.cu_kv, b, p.n_kv, kv_start);
  }
  q_start = __builtin_amdgcn_readfirstlane(q_start); kv_start = __builtin_amdgcn_readfirstlane(kv_start);
  nk = __builtin_amdgcn_readfirstlane(nk);
  const int NR = nq * p.G, row0 = tile * ROWS;
  const int ahead = nk - nq;                         // query token i sees the keys up to i + ahead
  const int last_row = min(row0 + ROWS, NR) - 1;
  const int seen = p.causal ? min(nk, last_row / p.G + ahead + 1) : nk;
  const int n_blocks = seen > 0 ? (seen + kKeys - 1) / kKeys : 0;
  // a wave's 32 rows: the keys that its last one sees, and those that all of them see
  const int wrow = row0 + 32 * wave, wlast = min(wrow + 31, NR - 1);
  const int wseen = wrow >= NR ? 0 : p.causal ? min(nk, wlast / p.G + ahead + 1) : nk;
  const int wall = p.causal ? wrow / p.G + ahead + 1 : nk;

  // this lane's query: operand of the score product, and the last key it sees
  const int row = min(wrow + n, NR - 1), tok = row / p.G, head = kv * p.G + row - tok * p.G;
  const int limit = p.causal ? tok + ahead : nk - 1;
  v4i q[NS];
  {
    const uint16_t* qp = p.q + (int64_t)(q_start + tok) * p.q_ld + head * D + half * 8;
#pragma unroll
    for (int s = 0; s < NS; s++) q[s] = *(const v4i*)(qp + s * 16);
  }

  // staging: a wave's share of a block's rows, the 16-byte pieces of a row permuted so that the reads below meet no bank twice
  const uint32_t lds0 = lds_address(lds);
  const int my_row = lane / PIECES, my_piece = lane % PIECES;
  bool bad = false;
  const int* table = PAGED ? p.pages.block_table + (size_t)b * p.pages.max_pages : nullptr;
  auto stage = [&](int kb, int buf) {
#pragma unroll
    for (int i = 0; i < COPIES; i++) {
      const int r0 = (wave * COPIES + i) * RPI, r = r0 + my_row;
      const int kp = my_piece ^ (D == 128 ? r & 15 : (r >> 1) & 7), vp = my_piece ^ (D == 128 ? (r & 3) << 2 : ((r >> 1) & 1) << 2);
      const uint8_t *ks, *vs;
      uint32_t ko, vo;
      if (PAGED) {
        const int granule = min((kb * kKeys + r0) >> 4, (nk - 1) >> 4), pg = dense_page_index(granule, p.pages.page_magic);
        int page = __builtin_amdgcn_readfirstlane(table[pg]);
        bad |= page < 0 || page >= p.pages.n_pages;
        page = page < 0 || page >= p.pages.n_pages ? 0 : page;
        const size_t base = (((size_t)page * p.Hkv + kv) * p.pages.page_rows + (granule * 16 - pg * p.pages.page_rows)) * ROW_BYTES;
        ks = (const uint8_t*)p.pages.k + base; vs = (const uint8_t*)p.pages.v + base;
        ko = vo = (uint32_t)((r & 15) * ROW_BYTES);
      } else {
        const int64_t first = (int64_t)kv_start + kb * kKeys;
        const int rr = min(r, nk - 1 - kb * kKeys);
        ks = (const uint8_t*)(p.k + first * p.k_ld + kv * D); vs = (const uint8_t*)(p.v + first * p.v_ld + kv * D);
        ko = (uint32_t)rr * (uint32_t)p.k_ld * 2u; vo = (uint32_t)rr * (uint32_t)p.v_ld * 2u;
      }
      copy16(lds0 + buf * STAGE + r0 * ROW_BYTES, ks, ko + kp * 16);
      copy16(lds0 + buf * STAGE + PLANE + r0 * ROW_BYTES, vs, vo + vp * 16);
    }
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
  auto read_k = [&](int kb, int s) { return *(const __attribute__((address_space(3))) v4i*)(uintptr_t)(k_at[s] + kb * 32 * ROW_BYTES); };
  auto read_v = [&](int d, int s) {                  // 16 keys from 16 s, 32 dims from 32 d
    const uint32_t at = v_at[d] + s * 16 * ROW_BYTES;
    const v2i lo = __builtin_bit_cast(v2i, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(uintptr_t)at));
    const v2i hi = __builtin_bit_cast(v2i, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(uintptr_t)(at + 8 * ROW_BYTES)));
    return v4i{lo[0], lo[1], hi[0], hi[1]};
  };

  float m = -INFINITY, l = 0.f;
  v16f o[ND];
#pragma unroll
  for (int d = 0; d < ND; d++)
#pragma unroll
    for (int i = 0; i < 16; i++) o[d][i] = 0.f;

  auto attend = [&](int kb, auto masked) {
    constexpr bool MASKED = decltype(masked)::value;
    v16f s[2];
#pragma unroll
    for (int h = 0; h < 2; h++)
#pragma unroll
      for (int i = 0; i < 16; i++) s[h][i] = 0.f;
#pragma unroll
    for (int x = 0; x < NS; x++)
#pragma unroll
      for (int h = 0; h < 2; h++) s[h] = T::mfma32(read_k(h, x), q[x], s[h]);
    v4i v0[ND];                                      // the first values' operands come in under the softmax
#pragma unroll
    for (int d = 0; d < ND; d++) v0[d] = read_v(d, 0);
    // operands are asked for AHEAD products before they are needed: left to itself the compiler asks and waits for each
    constexpr int AHEAD = 4;
    __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
    for (int i = 0; i < 2 * NS - AHEAD; i++) { __builtin_amdgcn_sched_group_barrier(0x008, 1, 0); __builtin_amdgcn_sched_group_barrier(0x100, 1, 0); }
#pragma unroll
    for (int i = 0; i < AHEAD; i++) { __builtin_amdgcn_sched_group_barrier(0x008, 1, 0); __builtin_amdgcn_sched_group_barrier(0x100, ND / 2, 0); }
    __builtin_amdgcn_sched_barrier(0);
    const int rel = limit - kb * kKeys - 4 * half;
    if (MASKED) {
#pragma unroll
      for (int h = 0; h < 2; h++)
#pragma unroll
        for (int i = 0; i < 16; i++) s[h][i] = 32 * h + 8 * (i >> 2) + (i & 3) > rel ? -INFINITY : s[h][i];
    }
    float most = s[0][0];
#pragma unroll
    for (int h = 0; h < 2; h++)
#pragma unroll
      for (int i = 0; i < 16; i++) most = fmaxf(most, s[h][i]);
    most *= p.c_scale;
    if (__ballot(most > m + 8.f)) {                  // the reference moves only when a weight would pass 2^8
      const float mn = fmaxf(m, halves_max(most));
      const float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
      l *= keep;
#pragma unroll
      for (int d = 0; d < ND; d++)
#pragma unroll
        for (int i = 0; i < 16; i++) o[d][i] *= keep;
      m = mn;
    }
    const float ref = m == -INFINITY ? 0.f : m;
    uint32_t w[2][8];
#pragma unroll
    for (int h = 0; h < 2; h++)
#pragma unroll
      for (int i = 0; i < 8; i++) {
        const float a = __builtin_amdgcn_exp2f(fmaf(s[h][2 * i], p.c_scale, -ref)), c = __builtin_amdgcn_exp2f(fmaf(s[h][2 * i + 1], p.c_scale, -ref));
        l += a; l += c;
        w[h][i] = dense_pack<T>(a, c);
      }
    __builtin_amdgcn_sched_barrier(0);
    uint32_t odd = 0;
#pragma unroll
    for (int x = 0; x < 4; x++) {
      const int h = x >> 1, i = 4 * (x & 1);
      const v4i pw = {(int)w[h][i], (int)w[h][i + 1], (int)w[h][i + 2], (int)w[h][i + 3]};
#pragma unroll
      for (int d = 0; d < ND; d++) {
        v4i a = x == 0 ? v0[d] : read_v(d, x);
        if (MASKED) {                                // a value that is no number must not meet the weight 0 of a query that does not see it
#pragma unroll
          for (int y = 0; y < 4; y++) {
            const uint32_t t = (((uint32_t)a[y] & T::kExponent) + T::kExponentUlp) & 0x80008000u;
            odd |= t;
            a[y] &= (int)~(t | (t - (t >> 15)));
          }
        }
        o[d] = T::mfma32(a, pw, o[d]);
      }
    }
    if (!MASKED) {
#pragma unroll
      for (int i = 0; i < 3 * ND; i++) { __builtin_amdgcn_sched_group_barrier(0x100, 2, 0); __builtin_amdgcn_sched_group_barrier(0x008, 1, 0); }
      __builtin_amdgcn_sched_group_barrier(0x008, ND, 0);
    }
    if (MASKED && __ballot(odd != 0)) {              // such values, for the queries that do see them
      for (int key = 0; key < kKeys; key++) {
        const bool sees = key - 4 * half <= rel;
        const uint32_t at = lds0 + (kb & 1) * STAGE + PLANE + key * ROW_BYTES;
        const int sw = D == 128 ? (key & 3) << 2 : ((key >> 1) & 1) << 2;
#pragma unroll
        for (int d = 0; d < ND; d++)
#pragma unroll
          for (int g = 0; g < 4; g++) {
            const int dim = 32 * d + 8 * g + 4 * half;
            const v2i x = *(const __attribute__((address_space(3))) v2i*)(uintptr_t)(at + ((dim >> 3) ^ sw) * 16 + (dim & 7) * 2);
            const uint32_t t0 = (((uint32_t)x[0] & T::kExponent) + T::kExponentUlp) & 0x80008000u;
            const uint32_t t1 = (((uint32_t)x[1] & T::kExponent) + T::kExponentUlp) & 0x80008000u;
            if (sees && (t0 & 0x8000u)) o[d][4 * g] += dense_low<T>((uint32_t)x[0]);
            if (sees && (t0 >> 31)) o[d][4 * g + 1] += dense_high<T>((uint32_t)x[0]);
            if (sees && (t1 & 0x8000u)) o[d][4 * g + 2] += dense_low<T>((uint32_t)x[1]);
            if (sees && (t1 >> 31)) o[d][4 * g + 3] += dense_high<T>((uint32_t)x[1]);
          }
      }
    }
  };

  // Blocks that all of the wave's queries see whole, then the others: two loops, since one with both forms copies the
  // accumulators in every block.
  const int n_whole = max(0, min(wseen, wall)) / kKeys;
  auto next = [&](int kb) {
    lds_copy_wait_barrier<0>();                      // this block is there, and nobody reads the other stage any more
    if (kb + 1 < n_blocks) stage(kb + 1, (kb + 1) & 1);
  };
  auto turn = [&] {                                  // the operands' addresses to the other stage
#pragma unroll
    for (int s = 0; s < NS; s++) k_at[s] ^= STAGE;
#pragma unroll
    for (int d = 0; d < ND; d++) v_at[d] ^= STAGE;
  };
  if (n_blocks > 0) stage(0, 0);
#pragma unroll
  for (int s = 0; s < NS; s++) asm volatile("" : "+v"(q[s]));      // the queries are there: no wait for them in the loops, which would be one for the copies too
  int kb = 0;
  for (; kb < n_whole; kb++) {
    next(kb);
    attend(kb, std::false_type{});
    turn();
  }
  for (; kb < n_blocks; kb++) {
    next(kb);
    if (kb * kKeys < wseen) attend(kb, std::true_type{});
    turn();
  }
  if (bad && lane == 0) atomicExch(p.err_word, (int)WSVD_E_SHAPE);
  l = halves_sum(l);
  const float inv = l == 0.f ? 0.f : 1.f / l;
  if (wrow + n < NR) {
    uint16_t* op = p.out + (int64_t)(q_start + tok) * p.out_ld + head * D + 4 * half;
#pragma unroll
    for (int d = 0; d < ND; d++)
#pragma unroll
      for (int g = 0; g < 4; g++) {
        v2i r;
        r[0] = (int)dense_pack<T>(o[d][4 * g] * inv, o[d][4 * g + 1] * inv);
        r[1] = (int)dense_pack<T>(o[d][4 * g + 2] * inv, o[d][4 * g + 3] * inv);
        *(v2i*)(op + 32 * d + 8 * g) = r;
      }
  }
}

template <class T, int D, bool PAGED>
hipError_t launch(DensePromptParams& p, hipStream_t s) {
  constexpr int NW = 4;
  p.tiles = (int)(((int64_t)p.n_q * p.G) / (32 * NW)) + p.B;       // at most: every sequence ends inside a tile
  k_dense_prompt<T, D, PAGED, NW><<<dim3((unsigned)(p.tiles * p.Hkv)), 64 * NW, 0, s>>>(p);
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
