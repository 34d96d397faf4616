// Shared by the dense-layer kernels (uncompressed keys and values in a paged cache): parameters, 16-bit element types, and
// the wave-wide searches that find a workgroup's sequence from lengths only the device knows.
#pragma once
#include "wsvd_dev.h"
#include "wsvd_internal.h"

// ---------------------------------------------------------------- element types
// BF16 and F16 operands of the matrix cores, 8 per lane and 4 dwords.  kNonFinite: the exponent bits of both halves of a dword.
struct DenseBf16 {
  using Elem = __bf16;
  using V8 = v8bf16;
  static constexpr uint32_t kExponent = 0x7F807F80u, kExponentUlp = 0x00800080u;
  static WSVD_DEV v4f mfma16(v4i a, v4i b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(V8, a), __builtin_bit_cast(V8, b), c, 0, 0, 0); }
  static WSVD_DEV v16f mfma32(v4i a, v4i b, v16f c) { return mfma_bf16(__builtin_bit_cast(V8, a), __builtin_bit_cast(V8, b), c); }
};
struct DenseF16 {
  using Elem = _Float16;
  using V8 = v8f16;
  static constexpr uint32_t kExponent = 0x7C007C00u, kExponentUlp = 0x04000400u;
  static WSVD_DEV v4f mfma16(v4i a, v4i b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(V8, a), __builtin_bit_cast(V8, b), c, 0, 0, 0); }
  static WSVD_DEV v16f mfma32(v4i a, v4i b, v16f c) { return mfma_f16(__builtin_bit_cast(V8, a), __builtin_bit_cast(V8, b), c); }
};
// two values rounded to nearest even, the first in the low half
template <class T>
WSVD_DEV uint32_t dense_pack(float a, float b) {
  typedef typename T::Elem V2 __attribute__((ext_vector_type(2)));
  V2 r;
  r[0] = (typename T::Elem)a; r[1] = (typename T::Elem)b;
  return __builtin_bit_cast(uint32_t, r);
}
template <class T>
WSVD_DEV float dense_low(uint32_t x) { return (float)__builtin_bit_cast(typename T::Elem, (uint16_t)x); }
template <class T>
WSVD_DEV float dense_high(uint32_t x) { return (float)__builtin_bit_cast(typename T::Elem, (uint16_t)(x >> 16)); }

// ---------------------------------------------------------------- wave-wide integer helpers
// Inclusive prefix sum over the wave: within rows of 16 lanes by shifts, then the last lanes' sums onto the rows behind.
WSVD_DEV int wave_prefix_int(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, true);       // row_shr 1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);      // row_bcast 15 into rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);      // row_bcast 31 into rows 2 and 3
  return x;
}
WSVD_DEV int wave_max_int(int x) { return (int)wave_max((float)x); }     // for numbers below 2^24
WSVD_DEV int wave_sum_int(int x) { return __builtin_amdgcn_readlane(wave_prefix_int(x), 63); }

// The sequence that packed token t belongs to: the number of sequences that end at or before it (B where none is left).
WSVD_DEV int dense_sequence_of(const int* cu, int B, int t, int lane) {
  int b = 0;
  for (int base = 0; base < B; base += 64) {
    const int i = base + lane;
    const int end = cu[min(i, B - 1) + 1];
    b += __builtin_popcountll(__ballot(i < B && end <= t));
  }
  return b;
}

// ---------------------------------------------------------------- pages
struct DensePages {
  uint16_t* k;                  // [n_pages][Hkv][page_rows][d]
  uint16_t* v;
  const int* seq_lens;          // [B]
  const int* block_table;       // [B][max_pages]
  int page_rows, max_pages, n_pages;
  uint32_t page_magic;          // dense_page_magic
};
// The page of a sequence's granule of 16 rows (granule / (page_rows / 16)) by a product: exact for granules below 2^23 and up to
// 2^8 granules in a page, since granule * (magic * n - 2^32) < 2^31.  A page of one granule has a magic of 2^32, kept as 0.
inline __host__ __device__ uint32_t dense_page_magic(int page_rows) {
  const uint64_t n = (uint64_t)page_rows / 16;
  return (uint32_t)((((uint64_t)1 << 32) + n - 1) / n);
}
inline __host__ __device__ int dense_page_index(int granule, uint32_t magic) {
  return magic == 0 ? granule : (int)(((uint64_t)(uint32_t)granule * magic) >> 32);
}

// ---------------------------------------------------------------- how the decode attention divides its work
// A CU holds one workgroup of kDenseWaves waves.  Sequences are cut into chunks of whole units (kDenseUnit rows), all of one
// sequence about equal, none with more than dense_units: no more than `target` chunks per kv head in all, where there are fewer
// sequences than that, and at most target + B in any case (u / units + 1 chunks for a sequence of u units, total / units <= target).
constexpr int kDenseWaves = 8, kDenseUnit = 128, kDenseWorkgroups = 256;
inline __host__ __device__ int dense_target(int Hkv) { return kDenseWorkgroups / Hkv > 1 ? kDenseWorkgroups / Hkv : 1; }
inline __host__ __device__ int dense_units_of(int len) { return (int)(((unsigned)len + kDenseUnit - 1) / kDenseUnit); }
inline __host__ __device__ int dense_chunks(int u, int units) { return u > units ? (u + units - 1) / units : 1; }
// The most units of a chunk: all, where the longest sequence has no more than alone_units (one CU streams 74 GB/s, so that 330 KB
// take as long as the hand-over that a cut costs); else at least min_units, and for up to 64 sequences the least at which there
// are at most `target` chunks (a chunk too many is a second round of workgroups: 23 ragged sequences of up to 3001 rows, 8 kv
// heads: 43.8 -> 36.5 us).  count(units): the chunks of all sequences.
template <class Count>
inline __host__ __device__ int dense_units(int total, int most, int B, int target, int alone_units, int min_units, Count count) {
  if (most <= alone_units) return alone_units;
  int units = (int)(((int64_t)total + target - 1) / target);
  units = units > min_units ? units : min_units;
  if (B > 64 || B > target || units >= most || count(units) <= target) return units;
  int low = units, high = most;                      // at `most` there are B chunks
  while (high - low > 1) {
    const int mid = (low + high) / 2;
    if (count(mid) <= target) high = mid; else low = mid;
  }
  return high;
}
// Partial results are folded by groups of kDenseFold chunks and then by groups of those: kDenseFold^2 chunks at most, which no
// sequence exceeds (of total / target units or more a chunk, it has at most `target`).
constexpr int kDenseFold = 16;
static_assert(kDenseWorkgroups <= kDenseFold * kDenseFold, "");

// A prompt of few tiles shares their keys out among several workgroups a tile: as many as fill the chip's two a CU.
constexpr int kDensePromptParts = 512, kDensePromptRows = 128;

struct DenseAppendParams {
  const uint16_t *q, *k, *v;
  uint16_t *q_out, *k_out;
  int64_t q_ld, k_ld, v_ld, q_out_ld, k_out_ld;
  const int *cu, *positions;
  const double* inv_freq;
  DensePages pages;
  int n_tokens, B, Hq, Hkv;
  int* err_word;
};
struct DenseDecodeParams {
  const uint16_t* q;
  int64_t q_ld;
  uint16_t* out;
  DensePages pages;
  unsigned long long* parts;    // words {value, tag} [chunk][Hkv][G][d + 2]: maximum, sum, row
  int B, Hkv, G, max_len, target, alone_units, min_units;
  float c_scale;                // sm_scale * log2(e)
  int* err_word;
};
struct DensePromptParams {
  const uint16_t *q, *k, *v;    // k, v: packed rows (not paged)
  int64_t q_ld, k_ld, v_ld, out_ld;
  uint16_t* out;
  const int *cu_q, *cu_kv;
  DensePages pages;
  float* parts;                 // of tiles that several workgroups share: [tile][Hkv][split] of 128 x {maximum, sum}, 128 rows
  int B, Hkv, G, causal, n_q, n_kv, splits;
  float c_scale;
  int* err_word;
};

hipError_t wsvd_launch_dense_append(const DenseAppendParams& p, int dtype, int d, hipStream_t s);
hipError_t wsvd_launch_dense_decode(const DenseDecodeParams& p, int dtype, int d, hipStream_t s);
hipError_t wsvd_launch_dense_prompt(DensePromptParams& p, int dtype, int d, bool paged, hipStream_t s);
