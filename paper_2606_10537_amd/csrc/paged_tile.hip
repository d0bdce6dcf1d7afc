// Attention of many new rows over the pages, within a sliding window: chunks of a prompt.
//
// The kernel of paged_attn.hip takes 32 query rows a workgroup, so that every key of a window is read and converted for
// 32 rows, and its 16-row products leave half of the matrix cores' rate.  Here a workgroup takes 64 or 128 rows of
// a KV head; the keys go through LDS in tiles of 128 or 64, as bf16 whatever the pages hold, and a wave multiplies 32 rows with
// v_mfma_f32_32x32x16_bf16.  The next tile is on its way in registers while one is multiplied; one barrier a tile.
//
//   S^T = K Q^T: row = key, column = query row; element e of a lane is key 8 (e / 4) + 4 (lane / 32) + e % 4 of 32.
//   O^T += V^T P^T: elements 8 s .. 8 s + 7 of S^T are the B operand of the keys 16 s .., as they stand; the A operand, eight
//     keys of a channel, comes from the rows of V by ds_read_b64_tr_b16 (among 16 lanes, lane j receives element j % 4 of
//     what lanes j / 4, 4 + j / 4, .. point at).
//
// ROWS: 128 rows, four waves of 32; 64, with four of eight waves on the same 32 rows and a quarter of each tile's keys
// each, joined at the end, where there are few row blocks.
#include <algorithm>

#include "paged_common.h"

namespace pd {

typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef short i16x8 __attribute__((ext_vector_type(8)));
#define PD_LDS __attribute__((address_space(3)))

// Elements: chunk c (8 channels) of row r of a tile of KEYS rows.  64-byte groups of chunks of all rows one after the
// other, chunks swapped by bits 2 and 3 of the row: 16 lanes of a K read (one chunk of 16 rows) or of a V read (four
// chunks of four rows) then cover every bank once.
template <int KEYS>
__device__ __forceinline__ int tile_at(int r, int c) { return (c >> 2) * (KEYS * 32) + r * 32 + 8 * ((c & 3) ^ ((r >> 2) & 3)); }

// Two fp32 as bf16, rounded to nearest even, in one instruction.
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  typedef float f32x2_ __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_{lo, hi}, bf16x2));
}

// Eight elements of a page's row, as bf16.
template <int CT>
struct Raw8 {
  uint32_t w[CT == kBf16 ? 4 : CT == kFp8 ? 2 : 1];
  uint32_t ex;
  // Chunk c of row `slot + row` of the page that begins at row `line` of the pool (of one KV head); line and slot are
  // one for many lanes.
  __device__ __forceinline__ void load(const void* pages, const uint8_t* exps, long long line, int slot, int row, int R, int c, int D) {
    const long long first = line + slot;
    if constexpr (CT == kBf16) {
      *(u32x4*)w = *(const u32x4*)((const char*)pages + first * (2 * D) + (uint32_t)(row * 2 * D + c * 16));
    } else if constexpr (CT == kFp8) {
      *(u32x2*)w = *(const u32x2*)((const char*)pages + first * D + (uint32_t)(row * D + c * 8));
      ex = exps[first + (uint32_t)row];
    } else {
      w[0] = *(const uint32_t*)((const char*)pages + first * (D / 2) + (uint32_t)(row * (D / 2) + c * 4));
      ex = exps[line * (D / 32) + slot + (uint32_t)(c / 4 * R + row)];
    }
  }
  __device__ __forceinline__ u32x4 bf16() const {
    if constexpr (CT == kBf16) {
      return *(const u32x4*)w;
    } else if constexpr (CT == kFp8) {
      const float s = exp_to_scale(ex);
      return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[0], s, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[0], s, true)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[1], s, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[1], s, true))};
    } else {
      return from_fp4(w[0], exp_to_scale(ex));
    }
  }
};

// Bits 15 and 31: whether either half is not a finite bf16.
__device__ __forceinline__ uint32_t not_finite(uint32_t x) { return (x & 0x7f807f80u) + 0x00800080u; }

template <int D, int CT, int ROWS, int KEYS, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void paged_tile_kernel(PagedAttnArgs a, FastDiv by_run) {
  constexpr int CH = D / 8, RP = 64 * WAVES / CH, NP = KEYS / RP;   // chunks of a row, rows of a load, loads of a tile
  constexpr int KP = 32 * WAVES / ROWS;                            // waves that share their rows
  constexpr int NB = KEYS / 32 / KP;                               // blocks of 32 keys of a wave in a tile
  constexpr int KS = D / 16, DB = D / 32, TILE = KEYS * D, GT = KEYS / 16;   // GT: groups of a tile
  constexpr int kFar = 1 << 30;
  static_assert(RP % 16 == 0 && 64 / CH <= 16, "the rows that a wave loads at once lie in one group");
  __shared__ __attribute__((aligned(16))) uint16_t lds[2][2][TILE];   // [buffer][K, V]
  __shared__ int odd_tile[4];                                      // a value of tile t is not finite: word t % 4
  const PagedArgs& p = a.c;
  // Workgroup i runs on XCD i % 8: runs of row blocks, which read the same keys, go to the XCDs in turn.  Runs of even length
  // begin one block later each: an XCD hands its workgroups to its parts in turn too, and in a padded batch the first blocks
  // of the runs, the only ones with rows, would all lie in the same part (32 x 8 heads, 512 places for one new row each,
  // window 8192: 588 us, 312 so).
  const uint32_t i = uniform((int)block_id());
  const int turn = by_run.quot(i / kNumXcd), run = by_run.d;
  int in_run = by_run.rem(i / kNumXcd, turn);
  if (run % 2 == 0) {
    in_run -= by_run.rem(turn, by_run.quot(turn));
    in_run += in_run < 0 ? run : 0;
  }
  const int id = (turn * kNumXcd + i % kNumXcd) * run + in_run;
  if (id >= (int)a.grid) return;
  const int bg = a.by_blocks.quot(id), rb = a.by_blocks.rem(id, bg);
  const int b = a.by_heads.quot(bg), g = a.by_heads.rem(bg, b);
  const int wave = uniform((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, n = lane & 31, hi = lane >> 5;
  const int len = paged_len(p, b), n_new = paged_new(p, b), rows = n_new * p.G, row0 = rb * ROWS;
  if (row0 >= rows) return;
  const int first_row = row0 + wave / KP * 32;                     // of the wave; beyond `rows`: none of them is real

  // This lane's query row; lanes beyond the last repeat it, so that a block of few rows needs no masks for them.
  const int r = first_row + n, rr = min(r, rows - 1), nr = a.by_group.quot(rr);
  const int head = g * p.G + a.by_group.rem(rr, nr);
  const long long q_el = (((long long)b * p.Ln + nr) * p.Hq + head) * D;
  const int own = len - n_new + nr;                                // its position
  const int lim = p.causal ? own + 1 : len, low = max(own - a.window + 1, 0);
  bf16x8 qf[KS];
#pragma unroll
  for (int i = 0; i < KS; ++i) qf[i] = *(const bf16x8*)((const uint16_t*)a.q + q_el + 16 * i + 8 * hi);

  // Positions that some row of the workgroup sees: groups of 16, the first positions' and the windows'.
  auto position = [&](int row) { return len - n_new + a.by_group.quot(min(row, rows - 1)); };
  const int any_low = position(row0) - a.window + 1;
  const int end = p.causal ? min(len, max(position(row0 + ROWS - 1) + 1, 0)) : len;
  const int far = (min(a.n_sinks, end) + 15) / 16, from = max(max(any_low, 0) / 16, far);
  const int groups = far + max(0, (end + 15) / 16 - from), tiles = (groups + GT - 1) / GT;
  // Those that all rows of the wave, and of the workgroup, see.
  const int every = p.causal ? position(first_row) + 1 : len;
  const int all_low = position(first_row + 31) - a.window + 1;
  const int wg_every = p.causal ? position(row0) + 1 : len, wg_low = position(row0 + ROWS - 1) - a.window + 1;

  // Where 64 groups lie, a lane each.
  const int32_t* table = p.page_table + (long long)b * p.max_pages;
  int at_page = 0, at_pos = kFar;
  auto locate = [&](int g0) {
    const int i = g0 + lane;
    at_page = 0;
    at_pos = kFar;
    if (i < groups) {
      at_pos = 16 * (i < far ? i : from + i - far);
      const int page = table[at_pos >> p.log2R];
      at_page = (unsigned)page < (unsigned)p.n_pages ? page : -1;
    }
  };

  // This thread's chunks of a tile: rows row + i RP, which lie in one group for the whole wave.
  const int c = threadIdx.x % CH, row = threadIdx.x / CH, wave_row = uniform(wave * (64 / CH));
  Raw8<CT> kr[NP], vr[NP];
  int first[NP];                     // position of the group's first key
  bool lost[NP];                     // its page lies outside the pool
  int located = -1;
  auto fetch = [&](int tile) {
    if (tile / (64 / GT) != located) {
      located = tile / (64 / GT);
      locate(64 * located);
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int gi = (GT * tile & 63) + (wave_row + i * RP) / 16;
      const int page = __builtin_amdgcn_readlane(at_page, gi);
      first[i] = __builtin_amdgcn_readlane(at_pos, gi);
      lost[i] = page < 0;
      const long long line = ((long long)max(page, 0) * p.Hkv + g) * p.R;
      kr[i].load(p.k_pages, p.k_exp, line, first[i] & (p.R - 1), row % 16, p.R, c, D);
      vr[i].load(p.v_pages, p.v_exp, line, first[i] & (p.R - 1), row % 16, p.R, c, D);
    }
  };
  auto put = [&](int t) {
    uint16_t *kt = lds[t & 1][0], *vt = lds[t & 1][1];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int at = tile_at<KEYS>(row + i * RP, c);
      *(u32x4*)&kt[at] = kr[i].bf16();
      u32x4 v = vr[i].bf16();
      const bool plain = !lost[i] && first[i] + 16 <= wg_every && (first[i] >= wg_low || first[i] + 16 <= a.n_sinks);
      if (!plain) {   // some row does not see some key of the group
        // Zeros where none does; what is not finite is left out too, and added by itself to the rows that see it, as a
        // weight of zero does not cancel it.
        const int pos = first[i] + row % 16;
        const bool seen = (pos < end) & ((pos >= any_low) | (pos < a.n_sinks)) & !lost[i];
        uint32_t odd = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          v[w] = seen ? v[w] : 0u;
          const uint32_t bits = not_finite(v[w]) & 0x80008000u;
          odd |= bits;
          v[w] &= (bits & 0x8000u ? 0xffff0000u : 0xffffffffu) & (bits & 0x80000000u ? 0xffffu : 0xffffffffu);
        }
        if (odd) odd_tile[t & 3] = 1;
      }
      *(u32x4*)&vt[at] = v;
    }
  };

  // Offsets of the fragments: K of block 0, V of keys 0.. and 8.. of block 0.
  const int kq = wave % KP * NB;                                   // the wave's first block of a tile
  int v_at[2];
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int k = lane & 15, key = 8 * x + 4 * hi + (k >> 2), ch = (lane >> 4 & 1) * 2 + ((k & 3) >> 1);
    v_at[x] = tile_at<KEYS>(key, ch) + 4 * (k & 1);
  }

  f32x16 o[DB];
  float m = kNoMax, l = 0.f;
#pragma unroll
  for (int i = 0; i < DB; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[i][e] = 0.f;

  auto multiply = [&](int tile, int t, int pages, int positions) {
    const uint16_t *kt = lds[t & 1][0], *vt = lds[t & 1][1];
#pragma unroll
    for (int kb = 0; kb < NB; ++kb) {
      const int blk = kq + kb;
      f32x16 s;
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
      for (int i = 0; i < KS; ++i)
        s = mfma32x32x16(*(const bf16x8*)&kt[tile_at<KEYS>(32 * blk + n, 2 * i + hi)], qf[i], s);
      // The block's V, on its way during the softmax.  512 rows of 8 x 4 heads behind 7.5K keys, a window of 1024: 25.4 us
      // with V read at its products, 24.3 so; with a window of 4096, 70.8 and 65.9.  At 128 rows a workgroup (8 such
      // sequences) 105.6 and 104.3.
      i16x8 v[DB][2];
#pragma unroll
      for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const i16x4 z = __builtin_amdgcn_ds_read_tr16_b64_v4i16((PD_LDS i16x4*)(vt + v_at[x] + i * (KEYS * 32) + (32 * blk + 16 * h) * 32));
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i][h][4 * x + j] = z[j];
          }
      // The block's two groups: their positions, and whether all rows see them.
      int pos[2];
      bool bad[2], whole = true;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int gi = (GT * tile & 63) + 2 * blk + h;
        pos[h] = __builtin_amdgcn_readlane(positions, gi);
        bad[h] = __builtin_amdgcn_readlane(pages, gi) < 0;
        whole = whole && !bad[h] && pos[h] + 16 <= every && (pos[h] >= all_low || pos[h] + 16 <= a.n_sinks);
      }
      if (!whole) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int at = pos[h] + 4 * hi, below = lim - at, above = low - at, first = a.n_sinks - at;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int k = 8 * (e / 4) + e % 4;   // of the group, from `at` on
            const float x = bad[h] ? NAN : s[8 * h + e];
            s[8 * h + e] = (k < below) & ((k >= above) | (k < first)) ? x : -INFINITY;
          }
        }
      }
      float top = s[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) top = fmaxf(top, s[e]);
      {
        const uint32_t u = __float_as_uint(top);
        const auto x = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        top = fmaxf(m, fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1])) * p.scale_log2);
      }
      // The sums are brought to a new maximum only where it has risen by more than 8, each row by itself: what a row
      // sees does not change the rounding of others.
      const bool up = top > m + 8.f;
      if (__any(up)) {
        top = up ? top : m;
        const float f = fast_exp2(m - top);
        l *= f;
#pragma unroll
        for (int i = 0; i < DB; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) o[i][e] *= f;
        m = top;
      }
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[e] = fast_exp2(fmaf(s[e], p.scale_log2, -m));
        sum[e % 4] += s[e];
      }
      l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
      // Weights of one bf16 term, rounded to nearest; their sum is taken before.
      u32x4 w[2];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < 4; ++j) w[h][j] = bf16_pair(s[8 * h + 2 * j], s[8 * h + 2 * j + 1]);
#pragma unroll
      for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          o[i] = mfma32x32x16(__builtin_bit_cast(bf16x8, v[i][h]), __builtin_bit_cast(bf16x8, w[h]), o[i]);
      if (odd_tile[t & 3]) {
        // Values that are not finite, from the pages, to the rows that see their key: with its weight, so that where this
        // has underflowed an infinity gives NaN.
#pragma unroll 1
        for (int key = 0; key < 32; ++key) {
          float x = s[0];
#pragma unroll
          for (int e = 1; e < 16; ++e) x = 4 * (key / 8) + key % 4 == e ? s[e] : x;
          x = __shfl(x, 32 * (key / 4 % 2) + n);
          const int at = pos[key / 16] + key % 16;
          if (bad[key / 16] || !(at < lim && (at >= low || at < a.n_sinks))) continue;
          const int page = max(__builtin_amdgcn_readlane(pages, (GT * tile & 63) + 2 * blk + key / 16), 0);
          const long long line = ((long long)page * p.Hkv + g) * p.R;
#pragma unroll 1
          for (int ch = 0; ch < CH; ++ch) {
            Raw8<CT> raw;
            raw.load(p.v_pages, p.v_exp, line, at & (p.R - 1), 0, p.R, ch, D);
            const u32x4 y = raw.bf16();
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              // Channels 8 ch + 4 hi + j of this lane: block ch / 4, element 4 (ch % 4) + j.
              const uint32_t u = hi ? y[2 + j / 2] : y[j / 2];
              const float v = __uint_as_float(j % 2 ? u & 0xffff0000u : u << 16);
              if (!(fabsf(v) < INFINITY)) {
#pragma unroll
                for (int i = 0; i < DB; ++i)
#pragma unroll
                  for (int k = 0; k < 4; ++k)
                    if (ch == 4 * i + k) o[i][4 * k + j] += x * v;
              }
            }
          }
        }
      }
    }
  };

  if (threadIdx.x < 4) odd_tile[threadIdx.x] = 0;
  __syncthreads();
  if (tiles > 0) {
    // Row blocks of the same keys start at different tiles, so that all but the first rounds find them in the L2
    // cache instead of missing it together at each tile.
    int tile = rb % tiles;
    fetch(tile);
    put(0);
    __syncthreads();
    for (int t = 0; t < tiles; ++t) {
      const int pages = at_page, positions = at_pos, here = tile;
      const bool more = t + 1 < tiles;
      tile = tile + 1 < tiles ? tile + 1 : 0;
      if (more) fetch(tile);
      if (first_row < rows) multiply(here, t, pages, positions);
      if (more) put(t + 1);
      __syncthreads();
      // Every wave has read the word; it is set for tile t + 4 three barriers on.
      if (threadIdx.x == 0) odd_tile[t & 3] = 0;
    }
  }

  {
    const uint32_t u = __float_as_uint(l);
    const auto x = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    l = __uint_as_float(x[0]) + __uint_as_float(x[1]);
  }
  if constexpr (KP > 1) {
    // The other waves of the same rows hand their sums over.
    __shared__ float ml[WAVES][32][2];
    auto part = [&](int w) { return (float*)&lds[0][0][0] + (w - w / KP - 1) * (64 * 16 * DB); };
    if (wave % KP) {
#pragma unroll
      for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int e = 0; e < 16; e += 4)
          *(f32x4*)&part(wave)[((i * 4 + e / 4) * 64 + lane) * 4] = f32x4{o[i][e], o[i][e + 1], o[i][e + 2], o[i][e + 3]};
      if (hi == 0) {
        ml[wave][n][0] = m;
        ml[wave][n][1] = l;
      }
    }
    __syncthreads();
    if (wave % KP) return;
    float top = m, f[KP];
#pragma unroll
    for (int w = 1; w < KP; ++w) top = fmaxf(top, ml[wave + w][n][0]);
    f[0] = fast_exp2(m - top);
    l *= f[0];
#pragma unroll
    for (int w = 1; w < KP; ++w) {
      f[w] = fast_exp2(ml[wave + w][n][0] - top);
      l += ml[wave + w][n][1] * f[w];
    }
    m = top;
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        f32x4 x = f32x4{o[i][e], o[i][e + 1], o[i][e + 2], o[i][e + 3]} * f[0];
#pragma unroll
        for (int w = 1; w < KP; ++w) x += *(const f32x4*)&part(wave + w)[((i * 4 + e / 4) * 64 + lane) * 4] * f[w];
#pragma unroll
        for (int j = 0; j < 4; ++j) o[i][e + j] = x[j];
      }
  }
  if (r >= rows) return;
  const float inv = 1.0f / l;
#pragma unroll
  for (int i = 0; i < DB; ++i)
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      float y[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) y[j] = l == 0.f ? 0.f : o[i][e + j] * inv;
      *(u32x2*)((uint16_t*)a.o + q_el + 32 * i + 2 * e + 4 * hi) = u32x2{bf16_pair(y[0], y[1]), bf16_pair(y[2], y[3])};
    }
  if (hi == 0 && a.lse) a.lse[((long long)b * p.Hq + head) * p.Ln + nr] = l == 0.f ? -INFINITY : (m + __log2f(l)) * kLn2;
}

template <int D, int CT>
hipError_t paged_tile_of(const PagedAttnArgs& a, int rows, hipStream_t s) {
  // The longest runs that deal every sequence to all XCDs: where few sequences of a batch have many new rows, one
  // range of ids an XCD leaves them to a part of the card.
  int heads = 1;
  while (heads < kNumXcd && a.c.Hkv % (2 * heads) == 0) heads *= 2;
  const int run = std::min(((int)a.row_blocks * heads + kNumXcd - 1) / kNumXcd, 256);
  const long long runs = (a.grid + run - 1) / run, grid = (runs + kNumXcd - 1) / kNumXcd * kNumXcd * run;
  const FastDiv by_run = fast_div(run);
  if (rows == 128) hipLaunchKernelGGL((paged_tile_kernel<D, CT, 128, 64, 4>), grid_xy(grid), dim3(256), 0, s, a, by_run);
  else hipLaunchKernelGGL((paged_tile_kernel<D, CT, 64, 128, 8>), grid_xy(grid), dim3(512), 0, s, a, by_run);
  return hipGetLastError();
}

hipError_t launch_paged_tile(PagedAttnArgs a, int rows, hipStream_t s) {
  a.row_blocks = (a.c.G * a.c.Ln + rows - 1) / rows;
  a.by_blocks = fast_div(a.row_blocks);
  a.grid = (long long)a.c.B * a.c.Hkv * a.row_blocks;
  const bool wide = a.c.D == 128;
  switch (cache_type(a.c)) {
    case kBf16: return wide ? paged_tile_of<128, kBf16>(a, rows, s) : paged_tile_of<64, kBf16>(a, rows, s);
    case kFp8: return wide ? paged_tile_of<128, kFp8>(a, rows, s) : paged_tile_of<64, kFp8>(a, rows, s);
    default: return wide ? paged_tile_of<128, kFp4>(a, rows, s) : paged_tile_of<64, kFp4>(a, rows, s);
  }
}

}  // namespace pd
