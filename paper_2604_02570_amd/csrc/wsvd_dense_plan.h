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
// (16-bit rows; over 8-bit ones, of half the bytes, the same numbers are taken, and set_units' least chunk.)
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
// A long sequence among B - 1 short ones has target - B + 1 chunks then, few where B is near `target` (one of 60000 rows, the others of 500, 32 / 8 heads of
// 128, target 32, 8-bit rows: B 24 48 us, 31 149, 32 281, 33 32).
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
// The append over 8-bit pages: units (the new rows of a block of 16), at most, and workgroups that share a unit's heads, four a round.  A workgroup costs
// its place and its angles, so about as many as the chip holds at once, but several a unit where those have many rows, so that a round's end
// is short (us with 1, 2, 4, 8 and 12 workgroups a unit: 19029 tokens of 16 prompts, 32 heads of 128: 228, 183, 172, 170, 181; 2 x 1000, 32 heads:
// 59, 35, 25, 23, 26; 4 x 300, 32 / 8: 23, 15, 11.9, 12.3, 11.7; 300 x 12, 8 heads: 20, 14, 18, 22, 22; 1000 x 4, 28 / 4: 27, 36, 56, 98, 89; 256 x 1, 32 / 8:
// 18, 12.5, 10.6, 16, 17).
struct DenseF8Append { int64_t units; int splits; };
WSVD_HD DenseF8Append dense_f8_append(int64_t n_tokens, int batch, int heads, bool packed) {
  const int64_t begun = n_tokens / 16 + 2 * (int64_t)batch, units = packed && begun < n_tokens ? begun : n_tokens, rounds = (heads + 3) / 4;
  const int64_t least = n_tokens >= 8 * units ? 4 : n_tokens >= 2 * units ? 2 : 1, fill = (1024 + units / 2) / units, some = fill < least ? least : fill;
  return {units, (int)(some < rounds ? some : rounds)};
}
// Attention of a few tokens a sequence over 8-bit pages: tiles of 16 (token, head) pairs, the columns of the decode attention, where the prompt
// attention's of 128 would be mostly empty.  Taken where the call's tokens, spread evenly, make at most 64 pairs a sequence, and no more tiles in all than
// the chip has CUs (a call whose tokens lie otherwise has up to twice as many): a tile reads its rows for itself, at 70 GB/s a CU, and a workgroup of 8 waves costs about 5 us (us as tiles of 128 and of 16; 32 / 8
// heads of 128 unless told: 4 x 5 tokens behind 700 rows, 8 heads of 64: 12.3 and 6.6; 1 x 7 behind 3000: 18 and 14; 8 x 4 behind 1000: 20 and 14; 32 x 3
// behind 2000: 44 and 30; 20 x 5 behind 1500, 28 / 4 heads: 27 and 17; 2 x 64 behind 3000, 8 heads: 21 and 16; past the limits 32 x 8 behind 2000: 44 and 41;
// 8 x 20 behind 3000: 31 and 37; 64 x 8 behind 300: 16 and 37; 1 x 64 behind 30000: 57 and 112).  Pieces of prompts beside single tokens, behind 1000 rows each:
// 256 + 63 x 1, 12 / 1 heads: 26 and 13; 512 + 63 x 1, 7 / 1: 26 and 20; 128 + 7 x 1, 8 / 8 of 64: 14 and 8; 100 + 31 x 1: 32 and 25; the piece behind 8000: 44
// and 38, 45 and 38, 25 and 19, 144 and 58; 200 tokens of one of 32 slots, 16 / 2 heads of 64, behind 8000: 30 and 26.
//   sets: of 16 pairs that a tile holds: two where tiles of one would be too many and those of two are not (a tile of two takes 1.6 times as long; us as
// tiles of 128 and of two sets: 32 x 8 behind 2000: 44 and 37; 32 x 6 behind 2000, 32 / 8 heads of 64: 29 and 18; 64 x 5 behind 1000, 16 / 2 heads of 64: 19
// and 14; 32 x 5 behind 200: 11.6 and 13.0; two sets where one is few enough, 1 x 7 behind 3000: 22; past 64 pairs 1 x 32 behind 2000: 17 and 23; 8 x 16
// behind 1000, 28 / 4 heads: 19 and 22; past the CUs 64 x 8 behind 1000: 33 and 50).
//   tiles: at most, since every sequence with tokens ends inside one.  splits: workgroups that may share a tile's rows, as many as give every CU one, and
// no more than one fold takes (1 x 7 behind 3000: up to 4 14.2, 8 15.4, 16 18.3; 1 x 4 behind 8000, 28 / 4 heads: 19.0, 18.0, 19.7).  From the host's numbers
// alone: one long sequence among many has a share like theirs (32 x 2 behind 500: 12; one of them behind 8000: 37, behind 60000: 282, as tiles of 128 1012).
//   joins: more may share it, and chunks of more than kF8Whole are joined by workgroups of their own, one a pair (1 x 4 behind 8000, 28 / 4 heads: 17.8 and
// 11.8; 1 x 8 behind 65000, 16 / 2 heads of 64: 30.0 and 14.9; 1 x 5 behind 16000, 16 heads: 19.7 and 18.2), as far as half of the CUs hold those, which they
// take also where there is nothing to join (1 x 2 behind 640, 32 heads: 8.2 without and 8.4; past that 16 x 2 behind 200, 16 / 2 heads of 64: 5.9 and 9.1).
constexpr int kF8Whole = 4;
struct DenseF8Columns { bool taken; int sets; int64_t tiles; int splits; bool joins; };
WSVD_HD DenseF8Columns dense_f8_columns(int64_t n_q, int batch, int Hkv, int group) {
  const int64_t some = batch < n_q ? batch : n_q, pairs = (n_q * group + some - 1) / some;
  const int sets = (pairs + 15) / 16 * some * Hkv <= kDenseCus ? 1 : 2, width = 16 * sets;
  const int64_t even = (pairs + width - 1) / width * some * Hkv, n = even <= kDenseCus ? kDenseCus / even : 1;
  const bool joins = sets == 1 && n > kF8Whole && n_q * group * Hkv <= kDenseCus / 2;
  const int most = joins ? kDenseFold * kDenseFold : kDenseFold;
  return {pairs <= 64 && even <= kDenseCus, sets, n_q * group / width + some, (int)(n > most ? most : n), joins};
}
// The page tables' calls: a thread a sequence at a time, and `items` (tokens or table entries) dealt out.
constexpr int kPagesThreads = 1024;
struct PagesLaunch { unsigned workgroups, threads; };
WSVD_HD PagesLaunch pages_launch(int batch, int64_t items) {
  if (batch <= 64 && items <= 256) return {1, 64};
  if (batch <= 256 && items <= 1024) return {1, 256};
  const int64_t n = (items + kPagesThreads - 1) / kPagesThreads;
  return {(unsigned)(n < 1 ? 1 : n > 128 ? 128 : n), kPagesThreads};
}
WSVD_HD int64_t dense_decode_workgroups(int B, int Hkv, int target, bool alone) { return (alone ? (int64_t)B : (int64_t)target + B) * Hkv; }
// Over 8-bit pages sequences of more than kF8Whole chunks have workgroups of their own to join them, one a head, behind all others: in place of two
// folds by the last chunk's, one join of all (us with the folds and so; bf16, heads of 128 unless told: 1 x 65001 rows, 16 / 2 heads of 64: 13.4 and 10.4,
// of 128: 20.1 and 14.7; 1 x 100000, 16 / 1: 27.7 and 17.1; 1 x 16000, 32 / 8: 16.5 and 14.0; 1 x 2000, 28 / 4, of 8 chunks: 10.3 and 8.6; 4 x up to 9000,
// 28 / 4: 18.2 and 14.2).  They take a CU each for 1.7 us also where nothing is to be joined, so only where the sequences can have 8 chunks on the average
// (23 ragged sequences of up to 3001 rows, 8 kv heads, with them 22.9 and without 20.1; at the limit 16 x 4000, 16 / 2 heads of 64: 11.4 without and
// 11.8, 16 x up to 8000 of 128: 19.1 and 18.4).  How many sequences have them: all or none.
WSVD_HD int dense_f8_joins(int B, int target, int waves) { return waves == 8 && target > 8 && target >= 8 * (int64_t)B ? B : 0; }
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
