// Shared by the dense-layer kernels (uncompressed keys and values in a paged cache): parameters, 16-bit element types, and
// the wave-wide searches that find a workgroup's sequence from lengths only the device knows.
#pragma once
#include "wsvd_dense_plan.h"
#include "wsvd_dev.h"
#include "wsvd_internal.h"

// ---------------------------------------------------------------- element types
// BF16 and F16 operands of the matrix cores, 8 per lane and 4 dwords.  kExponent: the exponent bits of both halves of a dword.
//   The softmax's weights are operands too, 2^(score - reference).  The reference is set kRaise below the largest score so far, and set anew when
// a weight would pass 2^kTop.  A bf16 weight can be as small as an fp32 one.  An f16 one has all its bits down to 2^-14 and is gone below
// 2^-25, where the sum of the weights, in fp32, still counts it (65001 rows 26 powers of two below one whose value is 0: output 9 % off).
// So the largest f16 weights are 2^11 to 2^15.9 (the type ends at 65504, 2^15.999): full relative precision 25 powers of two below the largest
// score, and no weight off by more than 2^-36 of the largest.  (Anew at 4.9 more: scores of a later block rarely pass the first one's by more;
// 2048 tokens behind 6144, f16: 217.7 us, at 4 more 219.5, 2^7 to 2^15 218.3.)
struct DenseBf16 {
  using Elem = __bf16;
  using V8 = v8bf16;
  static constexpr uint32_t kExponent = 0x7F807F80u, kExponentUlp = 0x00800080u;
  static constexpr float kRaise = 0.f, kTop = 8.f;
  static WSVD_DEV v4f mfma16(v4i a, v4i b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(V8, a), __builtin_bit_cast(V8, b), c, 0, 0, 0); }
  static WSVD_DEV v16f mfma32(v4i a, v4i b, v16f c) { return mfma_bf16(__builtin_bit_cast(V8, a), __builtin_bit_cast(V8, b), c); }
};
struct DenseF16 {
  using Elem = _Float16;
  using V8 = v8f16;
  static constexpr uint32_t kExponent = 0x7C007C00u, kExponentUlp = 0x04000400u;
  static constexpr float kRaise = 11.f, kTop = 15.9f;
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
// Ones in the halves of a dword that are infinite or no number.
template <class T>
WSVD_DEV uint32_t dense_odd(uint32_t x) {
  const uint32_t t = ((x & T::kExponent) + T::kExponentUlp) & 0x80008000u;
  return t | (t - (t >> 15));
}
// A partial result under another reference: one that is infinite stays so where the factor is too small for 32 bits.
WSVD_DEV float dense_scaled(float u, float k) { return __builtin_isinf(u) ? u : u * k; }

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
  int B, Hkv, G, max_len, waves, target, alone_units, min_units;
  int alone;                    // no sequence is cut
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
  int B, Hkv, G, causal, n_q, n_kv, splits, pairs;
  float c_scale;
  int* err_word;
};

hipError_t wsvd_launch_dense_append(const DenseAppendParams& p, int dtype, int d, hipStream_t s);
hipError_t wsvd_launch_dense_decode(const DenseDecodeParams& p, int dtype, int d, hipStream_t s);
hipError_t wsvd_launch_dense_prompt(DensePromptParams& p, int dtype, int d, bool paged, hipStream_t s);
