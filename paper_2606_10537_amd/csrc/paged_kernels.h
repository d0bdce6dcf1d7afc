// Argument blocks and launchers of the paged-cache kernels (internal to the library).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace pd {

// Division of n < 2^31 by a divisor known on the host: n * mul >> shift with
// shift = 31 + ceil(log2 d) and mul = ceil(2^shift / d), which is too large by less than
// n / 2^shift < 1 / d and so never reaches the next quotient.
struct FastDiv {
  uint32_t mul, shift, d;
#ifdef __HIPCC__
  __device__ __forceinline__ int quot(int n) const { return (int)(((uint64_t)(uint32_t)n * mul) >> shift); }
  __device__ __forceinline__ int rem(int n, int q) const { return n - q * (int)d; }
#endif
};
inline FastDiv fast_div(int d) {
  uint32_t log2 = 0;
  while ((1ll << log2) < d) ++log2;
  return FastDiv{(uint32_t)(((1ull << (31 + log2)) + (uint32_t)d - 1) / (uint32_t)d), 31 + log2, (uint32_t)d};
}

struct NormRopeArgs {
  const void *x[2];      // query rows, key rows
  void *y[2];
  const void *w[2];      // norm weights or nullptr
  long long xs[2], ys[2];  // row strides, elements
  const int32_t* pos;    // nullptr: no rotation
  long long rows;
  int Hq, Hkv, D;
  float eps;
  double log2_step;      // log2(rope_base) * 2 / d: pair i turns by pos * 2^(-i * log2_step)
  bool bf16;
  FastDiv by_groups;     // waves of a row
};
hipError_t launch_qk_norm_rope(const NormRopeArgs& a, hipStream_t s);

// The cache as the kernels see it.
struct PagedArgs {
  void *k_pages, *v_pages;
  uint8_t *k_exp, *v_exp;
  void* k_bounds;
  const int32_t *page_table, *kv_len, *new_rows;
  int B, Ln, Hq, Hkv, G, D, R, log2R, n_pages, max_pages, causal;
  bool bf16, fp8, fp4;   // new rows and outputs in bf16 (else fp32); pages in E4M3, in E2M1
  float scale_log2;      // softmax scale * log2(e)
};

// How the pages hold the elements.
enum { kBf16 = 0, kFp8 = 1, kFp32 = 2, kFp4 = 3 };
inline int cache_type(const PagedArgs& p) { return p.fp8 ? kFp8 : p.fp4 ? kFp4 : p.bf16 ? kBf16 : kFp32; }

struct AppendArgs {
  PagedArgs c;
  const void *k_new, *v_new;
  long long ks, vs;      // row strides, elements
  int pages;             // pages that the new rows of one sequence can touch
  FastDiv by_heads, by_pages;
};
hipError_t launch_paged_append(const AppendArgs& a, hipStream_t s);

// Heads of the query, key and value rows that one workgroup takes, at most.
constexpr int kRopeHeads = 8;
struct AppendRopeArgs {
  PagedArgs c;           // Hq = 0: no query rows
  const void *q, *k, *v;
  long long qs, ks, vs;  // row strides, elements
  const void *w_q, *w_k; // norm weights or nullptr
  void* q_out;
  const int32_t* pos;    // nullptr: the positions in the sequences
  float eps;
  bool rotate, stream;   // stream: query rows past the caches
  double step, step_rest;  // log2(rope_base) * 2 / d in two parts, the first of 24 bits: pair i turns by pos * 2^(-i * step)
  int pages;             // pages that the new rows of one sequence can touch
  int heads;             // of a workgroup
  FastDiv by_chunks, by_pages;
};
hipError_t launch_paged_append_rope(AppendRopeArgs a, hipStream_t s);

struct ReadArgs {
  PagedArgs c;
  void *k_out, *v_out;
  int first, n;
  FastDiv by_heads, by_blocks;   // H_kv, workgroups of a (sequence, head)
};
hipError_t launch_paged_read(const ReadArgs& a, hipStream_t s);

struct PageSelectArgs {
  PagedArgs c;
  const void* q;
  int top_k, n_first, n_last;
  int32_t* page_idx;
  double* score;         // [B][H_kv][shares][max_pages] workspace
  int shares;            // page_score_shares
  FastDiv by_group, by_heads, by_blocks, by_shares;   // G, H_kv, workgroups of a share, shares
};
int page_score_blocks(const PagedArgs& p);   // workgroups that score the pages of one (sequence, head, share)
int page_score_shares(const PagedArgs& p);   // shares of its query rows
hipError_t launch_paged_select(const PageSelectArgs& a, hipStream_t s);

// Rows of one query block: the query rows of a (sequence, KV head) are taken in
// blocks of at most this many.
constexpr int kPagedRows = 32;
// Keys that a block of query rows visits at most within a window: the first positions and the window of its first
// row, each in groups of 16, and what the block's other rows see further (causal = 0: besides the new rows).
inline long long paged_window_keys(long long window, long long n_sinks, long long rows_of_block) {
  return (n_sinks + 15) / 16 * 16 + window + rows_of_block + 31;
}

struct PagedAttnArgs {
  PagedArgs c;
  const void* q;
  const int32_t* page_idx;  // nullptr: all pages
  int top_k;
  int window, n_sinks;   // 0: no window
  int window_keys;       // keys, in groups of 16, that a row block visits at most (causal = 0: and the new rows)
  void* o;
  float* lse;
  float* o_part;         // [slot][part_rows][D] sums of a workgroup whose keys are a part of its rows'
  float* ml_part;        // [slot][part_rows][2] their maximum (log2 domain) and weight sum
  int32_t* unit;         // [B][H_kv][row_blocks][4]: a unit's first part, parts and rows
  int32_t* plan;         // nullptr, or 2 + 2 ceil(B / 64) sums of the batch (paged_plan_kernel)
  int row_blocks, part_rows;
  int max_chunks;        // parts of a unit at most; 1: no parts, no join
  float per_part;        // 1 / paged_parts
  float places;          // workgroups that an even batch is cut for (paged_places)
  long long grid;
  FastDiv by_group, by_heads, by_rows, by_blocks, by_units;  // G, H_kv, G * L_n, row_blocks, H_kv * row_blocks
};
// Parts that the keys of a ragged batch are cut into at most, besides one for every unit, for
// `rows` query rows of a KV head.  How many there are is known on the device alone, so as many
// workgroups are launched, and one that finds no part costs its launch: little where a CU
// holds two or more (64 ragged requests in 8 bits 371 us with 2048, 362 with 3328, 367 with
// 4096), but 4 us for a thousand of those with more than 16 rows, of which it holds one
// (8 rows of 4 heads over 8 x 8K keys 51.2 us with 1024, 54.1 with 2048, 56.5 with 2900).
inline int paged_parts(long long rows) { return rows <= 16 ? 3328 : 1024; }
// Workgroups that an even batch's keys are cut for where each gets 8 blocks or more: one a CU, whose waves have
// enough loads in flight, 16 KB each, with bf16; three in 4 bits, 4 KB a wave (8 x 32 heads x 32K keys 212 us with one, 190
// with three; 2 of them 60.8 and 54.5; 1 sequence of 4 heads, 1.3 blocks each with three, 12.9 and 14.9).
inline int paged_places(bool fp4, long long rows) { return fp4 && rows <= 16 ? 3 * 256 : 256; }
// Blocks up to which no unit's keys are cut, and no join follows: 16 where the units alone fill
// the card (32 ragged sequences of 8 heads, 8 new rows, up to 600 / 2048 keys: cut 26.3 and 44.5 us,
// whole 16.4 and 36.8; 12 of 32 heads up to 4096 keys, cut 85, whole 95), 4 elsewhere (8 heads
// x 256 / 512 keys 9.9 and 10.0, whole 6.6 and 8.4; x 1024 keys 9.9 and 15.6).
inline int paged_whole_blocks(long long units) { return units >= 256 ? 16 : 4; }
// Largest batch whose lengths every wave walks by itself; one launch more does it for larger
// ones (walked and planned, ragged lengths, 8 heads: 128 sequences 110 and 109 us, 512 259 and 197,
// 4096 3830 and 833; 65 sequences 64 and 68).
constexpr int kPlanBatch = 128;
// Keys that one workgroup takes at a time.
int paged_block_keys(bool fp32);
hipError_t launch_paged_attn(const PagedAttnArgs& a, hipStream_t s);
// Query rows of a workgroup of the tile kernel, which takes windows of many rows; 0: the other kernel does, whose blocks
// of 32 rows take a CU each, with the keys cut where there are fewer of them (8 heads x 4 query heads, window 1024: 256
// new rows, 256 blocks of 32, 18 us and 24 as 128 blocks of 64; 272 new rows 33 and 24; window 4096, 240 new rows 61 and
// 64, 272 82 and 64; 24 sequences of 9 new rows 36 and 27).  128 rows where they take fewer rounds of the card (2
// sequences of 512 new rows 41 us, 47 with 64; 8 of them 107 and 183; 12 of 80 new rows, two rounds either way, 53 and
// 50).  Also for up to 64 rows over more than one round, unless the keys are many: the waves without rows rest, and two
// workgroups a CU hide each other's start (64 sequences of 16 new rows, windows of 256 / 1024: 22 / 62 and 31 / 70;
// 128 sequences of 9 new rows, window 4000, in 8 bits: 334 and 315).  `keys`: that 32 rows visit at most.
// It goes by the places of the call, as how many hold rows is known on the device alone.  Where few do, every sequence of
// few rows still walks its window in one workgroup a head, and the other kernel, which cuts the keys, may take less (8 x 4
// heads, window 8192, this and the other: one sequence of 512 new rows and three of one 314 us and 263, two of one row in
// 512 places 228 and 88, eight 246 and 163; but 32 such 311 and 562, 64 in 16 places, four of them full, 358 and 431; with
// windows of 1024 the first is 48 and 51).
inline int paged_tile_rows(bool bf16, long long pairs, long long rows, long long keys) {
  const long long blocks = pairs * ((rows + 31) / 32), small = pairs * ((rows + 63) / 64), large = pairs * ((rows + 127) / 128);
  if (!bf16 || rows <= 32 || blocks <= 256) return 0;
  return (large + 255) / 256 < (small + 255) / 256 || (rows <= 64 && small > 256 && keys <= 2048) ? 128 : 64;
}
hipError_t launch_paged_tile(PagedAttnArgs a, int rows, hipStream_t s);

}  // namespace pd
