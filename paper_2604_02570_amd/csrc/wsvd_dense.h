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
WSVD_DEV int wave_sum_int(int x) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) x += __shfl_xor(x, d, 64);
  return __builtin_amdgcn_readfirstlane(x);
}
WSVD_DEV int wave_prefix_int(int x, int lane) {      // inclusive
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int y = __shfl_up(x, d, 64);
    x += lane >= d ? y : 0;
  }
  return x;
}

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
};

// ---------------------------------------------------------------- how the decode attention divides its work
// The rows of all sequences are dealt out in chunks of the same number of units (kDenseUnit rows), as many that about `target`
// chunks come of it, none of them across two sequences: at most target + B.
constexpr int kDenseUnit = 128;
constexpr int kDenseWorkgroups = 512;                // two of 4 waves on each of 256 CUs
inline __host__ __device__ int dense_target(int Hkv) { return kDenseWorkgroups / Hkv > 1 ? kDenseWorkgroups / Hkv : 1; }

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
  float* parts;                 // [chunk][Hkv][G][d + 2]
  int B, Hkv, G, max_len, target, min_units;
  float c_scale;                // sm_scale * log2(e)
  int* err_word;
};
struct DensePromptParams {
  const uint16_t *q, *k, *v;    // k, v: packed rows (not paged)
  int64_t q_ld, k_ld, v_ld, out_ld;
  uint16_t* out;
  const int *cu_q, *cu_kv;
  DensePages pages;
  int B, Hkv, G, causal, n_q, n_kv, tiles;
  float c_scale;
  int* err_word;
};

hipError_t wsvd_launch_dense_append(const DenseAppendParams& p, int dtype, int d, hipStream_t s);
hipError_t wsvd_launch_dense_decode(const DenseDecodeParams& p, int dtype, int d, hipStream_t s);
hipError_t wsvd_launch_dense_prompt(DensePromptParams& p, int dtype, int d, bool paged, hipStream_t s);
