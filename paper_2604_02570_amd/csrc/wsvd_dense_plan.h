// Arithmetic of the dense-layer kernels that needs no GPU: where a row lies in the pages, and how the decode attention and the
// prompt attention divide their work.  Host and device run the same code.
#pragma once
#include <cstdint>

#ifdef __HIPCC__
#define WSVD_HD __host__ __device__ inline
#else
#define WSVD_HD inline
#endif

// ---------------------------------------------------------------- pages
// The page of a sequence's granule of 16 rows (granule / (page_rows / 16)) by a product: exact for granules below 2^23 and up to
// 2^8 granules in a page, since granule * (magic * n - 2^32) < 2^31.  A page of one granule has a magic of 2^32, kept as 0.
WSVD_HD uint32_t dense_page_magic(int page_rows) {
  const uint64_t n = (uint64_t)page_rows / 16;
  return (uint32_t)((((uint64_t)1 << 32) + n - 1) / n);
}
WSVD_HD int dense_page_index(int granule, uint32_t magic) {
  return magic == 0 ? granule : (int)(((uint64_t)(uint32_t)granule * magic) >> 32);
}
// A table entry as a page: one outside the pool is `bad`, and page 0 is read in its place.
WSVD_HD int dense_page(int entry, int n_pages, bool& bad) {
  const bool out = entry < 0 || entry >= n_pages;
  bad = bad || out;
  return out ? 0 : entry;
}
// Where row 16 * granule of a kv head lies in the pools [n_pages][Hkv][page_rows], in rows; pg the granule's page in the sequence.
WSVD_HD uint64_t dense_pool_row(int page, int granule, int pg, int kv, int Hkv, int page_rows) {
  return ((uint64_t)page * Hkv + kv) * page_rows + (granule * 16 - pg * page_rows);
}

// ---------------------------------------------------------------- how the decode attention divides its work
// A CU holds 8 waves of it: one workgroup of 8 waves, or, where there are many (sequence, kv head) units and none of more than 1024
// rows, 2 of 4 or 4 of 2, so that units begin side by side (44 sequences of one row, 32 heads: 23.5 -> 11.0 us, 64 ragged of up to
// 500 rows, 8 heads: 20.6 -> 17.4; 32 x 2000 rows of 32 heads with workgroups of 2 waves: 166 -> 172).
constexpr int kDenseWavesPerCu = 8, kDenseCus = 256, kDenseUnit = 128;
WSVD_HD int dense_waves(int B, int Hkv, int max_len) {
  const int64_t units = (int64_t)B * Hkv;
  return max_len > 1024 || units < 2 * kDenseCus ? 8 : units < 4 * kDenseCus ? 4 : 2;
}
// Sequences are cut into chunks of whole units of kDenseUnit rows, all of one sequence about equal, none with more than dense_units:
// no more than `target` chunks per kv head in all, where there are fewer sequences than that, and at most target + B in any case
// (u / units + 1 chunks for a sequence of u units, total / units <= target).
WSVD_HD int dense_target(int waves, int Hkv) {
  const int n = kDenseCus * kDenseWavesPerCu / waves / Hkv;
  return n > 1 ? n : 1;
}
WSVD_HD int dense_units_of(int len) { return (int)(((unsigned)len + kDenseUnit - 1) / kDenseUnit); }
WSVD_HD int dense_chunks(int u, int units) { return u > units ? (u + units - 1) / units : 1; }
// Partial results are folded by groups of kDenseFold chunks and then by groups of those: no sequence has more than kDenseFold^2, which
// leaves CUs without rows where one long sequence has few kv heads (with 2, 128 workgroups have some, with 1, 64).
// (Groups of 16: 1 x 65001 rows of 2 heads 18.7 us, of 8: 15.5.  A group's end takes 7 chunks in 2 us, a second level costs 3: all
// of 16 chunks by the last one's workgroup, 7 at a time, take 15.2 us where two levels take 12.7.)
constexpr int kDenseFold = 8;
// The most units of a chunk: all, where the longest sequence has no more than alone_units (one CU streams 74 GB/s, so that 330 KB
// take as long as the hand-over that a cut costs: one sequence, heads of 128, 32 / 32, 32 / 8 and 28 / 4 of them, 640 rows whole 7.7, 7.3
// and 7.7 us, in two 8.5, 8.7, 9.8, in three 7.9, 8.2, 9.1; 768 rows whole 8.7, 7.9, 8.2, in three 8.7, 8.0, 8.8; 1024 whole 10.7, 9.1, 9.5, in
// four 9.5, 8.1, 9.0); else at least min_units, and for up to 64 sequences the least at which there
// are at most `target` chunks (a chunk too many is a second round of workgroups: 23 ragged sequences of up to 3001 rows, 8 kv
// heads: 43.8 -> 36.5 us).  count(units): the chunks of all sequences.
template <class Count>
WSVD_HD int dense_units(int total, int most, int B, int target, int alone_units, int min_units, Count count) {
  if (most <= alone_units) return alone_units;
  int units = (int)(((int64_t)total + target - 1) / target);
  const int least = (most + kDenseFold * kDenseFold - 1) / (kDenseFold * kDenseFold);
  units = units > min_units ? units : min_units;
  units = units > least ? units : least;
  if (B > 64 || B > target || units >= most || count(units) <= target) return units;
  int low = units, high = most;                      // at `most` there are B chunks
  while (high - low > 1) {
    const int mid = (low + high) / 2;
    if (count(mid) <= target) high = mid; else low = mid;
  }
  return high;
}
// A prompt of few tiles shares their keys out among several workgroups a tile: as many as fill the chip's two a CU.
constexpr int kDensePromptParts = 512, kDensePromptRows = 128;

// ---------------------------------------------------------------- launches
// A launch has fewer than 2^32 threads.
WSVD_HD bool dense_launchable(int64_t workgroups, int threads) { return workgroups < ((int64_t)1 << 32) / threads; }
// Tokens of an append workgroup, `items` = 16-byte pairs of a token: as few as give its 256 threads work, one where there are few (16 x ~1700
// tokens of 16 / 2 heads of 64: 4 tokens 50 us, 1 token 74; 16 x 2048 of 28 / 4 heads of 128: 124 and 104), and two where that many workgroups
// of one are no launch.
WSVD_HD int dense_append_tokens(int64_t n_tokens, int items) {
  if (n_tokens < 2048 || (items >= 256 && dense_launchable(n_tokens, 256))) return 1;
  return items >= 128 ? 2 : 4;
}
WSVD_HD int64_t dense_decode_workgroups(int B, int Hkv, int target, bool alone) { return (alone ? (int64_t)B : (int64_t)target + B) * Hkv; }
// The prompt attention's, at most: every sequence ends inside a tile.  Two tiles a workgroup where there are many and they differ: the second
// one's first keys and queries are asked for under the first one's last products, so that every other tile starts without a wait (16 x 2048
// tokens, 32 heads of 128: 650 -> 632 us, 64 x 300, 32 / 8 heads: 129 -> 121, 4 x 4096 of 16 / 2 heads of 64: 166 -> 158; over 13 causal
// calls of 2048 to 5920 tiles 0.93 to 1.04 of the time, 0.98 on average).  With fewer tiles the last round of workgroups costs more (1283
// ragged tiles: 73 -> 81 us), and without a mask all tiles cost the same already.
struct DensePromptGrid { int64_t workgroups; bool pairs; };
WSVD_HD DensePromptGrid dense_prompt_grid(int64_t n_q, int B, int Hkv, int G, bool causal) {
  const int64_t tiles = n_q * G / kDensePromptRows + B;
  const bool pairs = causal && tiles * Hkv >= 2048;
  return {(pairs ? (tiles + B) / 2 : tiles) * Hkv, pairs};
}

// A workgroup's share of a tile's n blocks, one of `splits`: [dense_share(split), dense_share(split + 1)).
WSVD_HD int dense_share(int split, int n, int splits) { return (int)((int64_t)split * n / splits); }
