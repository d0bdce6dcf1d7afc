// The paged cache but for its attention: head norms with rotary positions, writing
// rows into the pages (quantised to E4M3 where the cache is), reading them back,
// and the choice of pages by a bound on their scores.
#include "paged_common.h"

namespace pd {

// ---------------------------------------------------------------------------
// Head norms and rotary positions.
//
// y = x * w / sqrt(mean x^2 + eps), then (y_i, y_{i+d/2}) turned by pos * base^(-2i/d).
// Every element is read and written once; nothing else is moved, so memory bounds
// it.  A lane holds 16 bytes of a head, d/E lanes a head row, so a wave takes 64 E / d
// heads at a time: the sum of squares is a butterfly over those lanes, and the
// partner of a rotation sits d/2E lanes away.
//
// The angle is taken in turns in double precision (pos * f_i, f_i = base^(-2i/d) /
// 2 pi) and reduced by its nearest integer; sine and cosine are taken in fp32 at the
// nearest fp32 number and turned by what that left over, so that they keep their leading
// bits near zero (fp32 rows' error 7.4e-8 of the 2-norm without, 6.9e-8 with it, in the same
// time).  The angle's error stays below 1e-7 turns up to positions of 2^31, and it costs one
// double product for each pair and wave, not one for each head.  Lanes 0..d/2-1 take a pair each
// and hand the sines and cosines over through LDS.
//
// U: head groups a wave loads before it uses the first.  STREAM: loads and stores past the
// caches, for calls beyond what these hold (32768 rows of 64 heads 178 us, 197 without; a 4096-row
// call of 40 heads 17.3 and 18.2, and there the reader finds the rows in the caches).
template <bool BF16, int D, int U, bool STREAM>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(NormRopeArgs a) {
  constexpr int E = BF16 ? 8 : 4;       // elements of a lane
  constexpr int L = D / E;              // lanes of a head
  constexpr int HP = 64 / L;            // heads of a wave
  __shared__ float2 table[4][D / 2];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, c = lane % L;
  const int item = uniform((int)block_id() * 4 + wave), at = a.by_groups.quot(item);
  const long long row = at;
  if (row >= a.rows) return;
  const int h0 = a.by_groups.rem(item, at) * HP * U + lane / L, H = a.Hq + a.Hkv;
  const char* src[U];
  char* dst[U];
  Row16<BF16> x[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int h = h0 + u * HP;
    const int t = h >= a.Hq ? 1 : 0;
    const long long el = (long long)(t ? h - a.Hq : h) * D + c * E;
    src[u] = (const char*)(t ? a.x[1] : a.x[0]) + (row * (t ? a.xs[1] : a.xs[0]) + el) * (BF16 ? 2 : 4);
    dst[u] = (char*)(t ? a.y[1] : a.y[0]) + (row * (t ? a.ys[1] : a.ys[0]) + el) * (BF16 ? 2 : 4);
    if (h >= H) x[u].zero();
    else if constexpr (STREAM) x[u].load_once(src[u]);
    else x[u].load(src[u]);
  }
  float cs[E], sn[E];
  if (a.pos) {
    // The wave's own part of the table: written and read by one wave, in order.
    if (lane < D / 2) {
      const double f = exp2(-(double)lane * a.log2_step) * 0.15915494309189535;
      const double turn = (double)a.pos[row] * f, part = turn - rint(turn);
      const float near = (float)part, rest = (float)(part - (double)near) * 6.2831855f;
      float s, co;
      sincospif(2.0f * near, &s, &co);
      table[wave][lane] = make_float2(fmaf(-s, rest, co), fmaf(co, rest, s));
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float2 z = table[wave][(c % (L / 2)) * E + e];
      cs[e] = z.x;
      sn[e] = c < L / 2 ? -z.y : z.y;   // out_i = y_i cos - y' sin, out_{i+d/2} = y_{i+d/2} cos + y' sin
    }
  }
  Row16<BF16> wv[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    if (a.w[t]) wv[t].load((const char*)a.w[t] + c * 16);
    else wv[t].zero();
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int h = h0 + u * HP, t = h >= a.Hq ? 1 : 0;
    float y[E];
    x[u].unpack(y);
    if (a.w[0] || a.w[1]) {
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) s = fmaf(y[e], y[e], s);
      const float r = 1.0f / sqrtf(lanes_sum<L>(s) * (1.0f / D) + a.eps);
      float w[E], w1[E];
      wv[0].unpack(w);
      wv[1].unpack(w1);
      const bool norm = t ? a.w[1] != nullptr : a.w[0] != nullptr;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float z = y[e] * r * (t ? w1[e] : w[e]);
        y[e] = norm ? z : y[e];
      }
    }
    if (a.pos) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        y[e] = fmaf(partner<L>(y[e]), sn[e], y[e] * cs[e]);
      }
    }
    x[u].pack(y);
    if (h < H) {
      if constexpr (STREAM) x[u].store_once(dst[u]);
      else x[u].store(dst[u]);
    }
  }
}

template <bool BF16, int D>
hipError_t norm_rope_of(NormRopeArgs a, hipStream_t s) {
  constexpr int HP = 64 / (D / (BF16 ? 8 : 4));
  const int H = a.Hq + a.Hkv, all = (H + HP - 1) / HP;   // head groups of a row
  // Up to five head groups a wave, the row's groups shared evenly among its waves, keep
  // enough loads in flight and compute a row's angles seldom (H = 40, d = 64: 81 us with
  // waves of 32 and 8 heads, 60 with one of 40) where that leaves eight waves for every CU;
  // below that every group is a wave of its own.
  const int waves = (all + 4) / 5;
  const bool wide = a.rows * waves >= 8 * kNumCu;
  const int U = wide ? (all + waves - 1) / waves : 1, groups = (all + U - 1) / U;
  a.by_groups = fast_div(groups);
  const dim3 grid = grid_xy((a.rows * groups + 3) / 4);
  const bool stream = (double)a.rows * H * D * (BF16 ? 4 : 8) >= 256e6;   // what the last cache holds
#define PD_NORM(N)                                                                                                  \
  case N:                                                                                                           \
    if (stream) hipLaunchKernelGGL((qk_norm_rope_kernel<BF16, D, N, true>), grid, dim3(256), 0, s, a);      \
    else hipLaunchKernelGGL((qk_norm_rope_kernel<BF16, D, N, false>), grid, dim3(256), 0, s, a);            \
    break
  switch (U) {
    PD_NORM(1);
    PD_NORM(2);
    PD_NORM(3);
    PD_NORM(4);
    PD_NORM(5);
  }
#undef PD_NORM
  return hipGetLastError();
}

hipError_t launch_qk_norm_rope(const NormRopeArgs& a, hipStream_t s) {
  if (a.bf16) return a.D == 128 ? norm_rope_of<true, 128>(a, s) : norm_rope_of<true, 64>(a, s);
  return a.D == 128 ? norm_rope_of<false, 128>(a, s) : norm_rope_of<false, 64>(a, s);
}

// ---------------------------------------------------------------------------
// Writing rows into the pages.
//
// One workgroup per (sequence, page that new rows fall into, KV head): the bounds of a
// page need all its rows, and so no atomics are needed.  A lane holds 16 bytes
// of a row as in the norm kernel; even waves take the key rows, odd ones the value
// rows.  Memory bounds it: every new row is read once and written once.  A single
// token is one chain of loads: the lengths, then the row and the page's number, then the
// old bounds.
//
// Quantisation: e from the bits of the largest magnitude (448 = 1.75 * 2^8, so e is the
// binary exponent minus 8, or one more where the mantissa exceeds 1.75), the
// product with 2^-e is exact, and the conversion rounds to nearest even.  In 4 bits the largest
// magnitude is that of 32 channels, four lanes in bf16 (6 = 1.5 * 2^2).
//
// NW: waves.  Eight where a page may take more than 64 new rows (pages of 256 rows, one head,
// 4000 rows: 12.5 us, 16.2 with four, 11.9 with sixteen, which take 80 instead of 51 us for
// prompts of four sequences of 32 heads over pages of 128 rows).
template <int CT, int D, int NW>
__global__ __launch_bounds__(NW * 64) void paged_append_kernel(AppendArgs a) {
  constexpr bool BF16 = CT != kFp32;
  constexpr int E = BF16 ? 8 : 4, L = D / E, HP = 64 / L, EB = BF16 ? 2 : 4;
  __shared__ float bound[NW / 2][2][D];
  const PagedArgs& p = a.c;
  const int id = uniform((int)block_id());
  const int bj = a.by_heads.quot(id), h = a.by_heads.rem(id, bj);
  const int b = a.by_pages.quot(bj);
  if (b >= p.B) return;
  const int len = paged_len(p, b), n_new = paged_new(p, b);
  const int start = len - n_new;                       // position of new row 0; below 0: rows that are not written
  const int j = (max(start, 0) >> p.log2R) + a.by_pages.rem(bj, b);
  const int lo = max(max(start, 0), j << p.log2R), hi = min(len, (j + 1) << p.log2R);
  if (lo >= hi) return;
  const int number = p.page_table[(long long)b * p.max_pages + j];
  const bool there = (unsigned)number < (unsigned)p.n_pages;
  const int page = there ? number : 0;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, c = lane % L;
  const int kv = wave & 1;
  const char* src = (const char*)(kv ? a.v_new : a.k_new) + ((long long)h * D + c * E) * EB;
  const long long stride = (kv ? a.vs : a.ks) * EB;
  const long long base = ((long long)page * p.Hkv + h) * p.R;   // row of the pool
  const CacheRow<CT, D> to(p, kv, base, c);
  const bool bounds = p.k_bounds && kv == 0;
  const bool widen = (lo & (p.R - 1)) != 0;            // the page's row 0 is an older one
  // This thread's element of the bounds: the least keys, then the largest.
  const int bi = threadIdx.x;
  const long long bat = ((long long)page * p.Hkv + h) * 2 * D + bi;
  float old = 0.f;
  if (p.k_bounds && widen && bi < 2 * D) {
    if constexpr (BF16) old = bf16_to_f32(((const uint16_t*)p.k_bounds)[bat]);
    else old = ((const float*)p.k_bounds)[bat];
  }
  float least[E], most[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    least[e] = INFINITY;
    most[e] = -INFINITY;
  }
  constexpr int U = 4;   // rows of a lane in flight
  for (int r0 = lo + (wave >> 1) * HP * U; r0 < hi; r0 += NW / 2 * HP * U) {
    Row16<BF16> x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = min(r0 + u * HP + lane / L, hi - 1);
      x[u].load_once(src + ((long long)b * p.Ln + (r - start)) * stride);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = r0 + u * HP + lane / L;
      const bool live = r < hi && there;
      const int slot = r & (p.R - 1);
      float y[E];
      x[u].unpack(y);
      if (bounds && live) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          least[e] = fminf(least[e], y[e]);
          most[e] = fmaxf(most[e], y[e]);
        }
      }
      to.put(x[u], y, slot, live);
    }
  }
  if (!p.k_bounds) return;
  if (bounds) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
#pragma unroll
      for (int k = L; k < 64; k *= 2) {
        least[e] = fminf(least[e], __shfl_xor(least[e], k));
        most[e] = fmaxf(most[e], __shfl_xor(most[e], k));
      }
      if (lane < L) {
        bound[wave >> 1][0][c * E + e] = least[e];
        bound[wave >> 1][1][c * E + e] = most[e];
      }
    }
  }
  __syncthreads();
  if (bi >= 2 * D || !there) return;
  const bool up = bi >= D;
  const int ch = up ? bi - D : bi;
  float x = widen ? old : up ? -INFINITY : INFINITY;
#pragma unroll
  for (int w = 0; w < NW / 2; ++w) x = up ? fmaxf(x, bound[w][1][ch]) : fminf(x, bound[w][0][ch]);
  if constexpr (BF16) ((uint16_t*)p.k_bounds)[bat] = f32_to_bf16(x);
  else ((float*)p.k_bounds)[bat] = x;
}

hipError_t launch_paged_append(const AppendArgs& a, hipStream_t s) {
  const dim3 grid = grid_xy((long long)a.c.B * a.pages * a.c.Hkv);
  const bool tall = a.c.R > 64 && a.c.Ln > 64;
#define PD_APPEND(CT, DD)                                                                                  \
  do {                                                                                                     \
    if (tall) hipLaunchKernelGGL((paged_append_kernel<CT, DD, 8>), grid, dim3(512), 0, s, a);            \
    else hipLaunchKernelGGL((paged_append_kernel<CT, DD, 4>), grid, dim3(256), 0, s, a);                   \
  } while (0)
  const bool wide = a.c.D == 128;
  switch (cache_type(a.c)) {
    case kBf16: if (wide) PD_APPEND(kBf16, 128); else PD_APPEND(kBf16, 64); break;
    case kFp8: if (wide) PD_APPEND(kFp8, 128); else PD_APPEND(kFp8, 64); break;
    case kFp4: if (wide) PD_APPEND(kFp4, 128); else PD_APPEND(kFp4, 64); break;
    default: if (wide) PD_APPEND(kFp32, 128); else PD_APPEND(kFp32, 64); break;
  }
#undef PD_APPEND
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Reading rows back: a lane writes 16 bytes of the output, a wave consecutive
// rows of one (sequence, head), which lie beside each other in the pages too.
// Memory bounds it.
template <int CT, int D>
__global__ __launch_bounds__(256) void paged_read_kernel(ReadArgs a) {
  constexpr bool BF16 = CT != kFp32;
  constexpr int E = BF16 ? 8 : 4, L = D / E, RP = 256 / L, EB = BF16 ? 2 : 4, U = 4;
  const PagedArgs& p = a.c;
  const int id = uniform((int)block_id());
  const int bh = a.by_blocks.quot(id), block = a.by_blocks.rem(id, bh);
  const int b = a.by_heads.quot(bh), h = a.by_heads.rem(bh, b);
  if (b >= p.B) return;
  const int len = paged_len(p, b), c = threadIdx.x % L;
  const int row0 = block * RP * U + threadIdx.x / L;
  const int end = min(len - a.first, a.n);
  if (block * RP * U >= end) return;
  const int32_t* table = p.page_table + (long long)b * p.max_pages;
  long long at[U];
  bool bad[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int pos = a.first + min(row0 + u * RP, end - 1);
    int page = table[pos >> p.log2R];
    bad[u] = (unsigned)page >= (unsigned)p.n_pages;
    if (bad[u]) page = 0;
    at[u] = ((long long)page * p.Hkv + h) * p.R + (pos & (p.R - 1));
  }
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    const char* src = (const char*)(kv ? p.v_pages : p.k_pages);
    char* out = (char*)(kv ? a.v_out : a.k_out) + ((long long)bh * a.n * D + c * E) * EB;
    if constexpr (CT == kFp4) {
      const uint8_t* ex = kv ? p.v_exp : p.k_exp;
      uint32_t w[U];
      float s[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        w[u] = __builtin_nontemporal_load((const uint32_t*)(src + at[u] * (D / 2) + c * 4));
        const int slot = (a.first + min(row0 + u * RP, end - 1)) & (p.R - 1);
        s[u] = exp_to_scale(ex[(at[u] - slot) * (D / 32) + (long long)(c / 4) * p.R + slot]);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        Row16<true> x;
        x.v = from_fp4(w[u], s[u]);
        if (bad[u]) x.nan();
        if (row0 + u * RP < end) x.store_once(out + (long long)(row0 + u * RP) * D * EB);
      }
    } else if constexpr (CT == kFp8) {
      const uint8_t* ex = kv ? p.v_exp : p.k_exp;
      u32x2 w[U];
      float s[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        w[u] = __builtin_nontemporal_load((const u32x2*)(src + at[u] * D + c * E));
        s[u] = exp_to_scale(ex[at[u]]);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float y[8];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[u][k], false);
          const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[u][k], true);
          y[4 * k] = lo[0] * s[u];
          y[4 * k + 1] = lo[1] * s[u];
          y[4 * k + 2] = hi[0] * s[u];
          y[4 * k + 3] = hi[1] * s[u];
        }
        Row16<true> x;
        x.pack(y);
        if (bad[u]) x.nan();
        if (row0 + u * RP < end) x.store_once(out + (long long)(row0 + u * RP) * D * EB);
      }
    } else {
      Row16<BF16> x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) x[u].load_once(src + (at[u] * D + c * E) * EB);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (bad[u]) x[u].nan();
        if (row0 + u * RP < end) x[u].store_once(out + (long long)(row0 + u * RP) * D * EB);
      }
    }
  }
}

template <int CT, int D>
hipError_t read_of(ReadArgs a, hipStream_t s) {
  constexpr int rows = 256 / (D / (CT == kFp32 ? 4 : 8)) * 4;
  const int blocks = (a.n + rows - 1) / rows;
  a.by_blocks = fast_div(blocks);
  hipLaunchKernelGGL((paged_read_kernel<CT, D>), grid_xy((long long)a.c.B * a.c.Hkv * blocks), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_paged_read(const ReadArgs& a, hipStream_t s) {
  const bool wide = a.c.D == 128;
  switch (cache_type(a.c)) {
    case kBf16: return wide ? read_of<kBf16, 128>(a, s) : read_of<kBf16, 64>(a, s);
    case kFp8: return wide ? read_of<kFp8, 128>(a, s) : read_of<kFp8, 64>(a, s);
    case kFp4: return wide ? read_of<kFp4, 128>(a, s) : read_of<kFp4, 64>(a, s);
    default: return wide ? read_of<kFp32, 128>(a, s) : read_of<kFp32, 64>(a, s);
  }
}

// ---------------------------------------------------------------------------
// Page scores: max over the group's query rows of sum_i q_i * (q_i >= 0 ? hi_i : lo_i).
//
// Pages whose scores differ in the last bits of an fp32 sum have to come out in the
// same order whatever the order of summation, so products and sums are double: the
// product of two bf16 is exact there, and a sum of d of them too unless their
// exponents lie more than 30 apart.  The bounds are read once per block of query rows
// and converted once; memory bounds it for few query rows (16 lanes or more read a
// page's bounds in whole lines, a lane four pages at once: 512 pages of 8 x 32 heads 12.9 us,
// one page at a time 18.7), the double FMAs (one per element and row) for many.

constexpr int kScoreTurns = 4;   // pages of a lane
constexpr int kScoreRows = 16;   // query rows in LDS at a time
// Scores of pages j0 .. of (b, g) over the query rows of every step-th block from block r0 on, four
// pages a lane of NT threads; put(j, score).
template <bool BF16, int D, int NT, class F>
__device__ __forceinline__ void score_pages(const PageSelectArgs& a, int b, int g, int j0, int pages, int rows,
                                            int block0, int step, float (&q)[kScoreRows][D], F put) {
  constexpr int E = BF16 ? 8 : 4, L = D / E, PP = NT / L, EB = BF16 ? 2 : 4, QR = kScoreRows, U = kScoreTurns;
  const PagedArgs& p = a.c;
  const int c = threadIdx.x % L;
  Row16<BF16> lo[U], hi[U];
  bool nan[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int j = min(j0 + u * PP + (int)threadIdx.x / L, pages - 1);
    int page = p.page_table[(long long)b * p.max_pages + j];
    nan[u] = (unsigned)page >= (unsigned)p.n_pages;
    if (nan[u]) page = 0;
    const char* src = (const char*)p.k_bounds + (((long long)page * p.Hkv + g) * 2 * D + c * E) * EB;
    lo[u].load(src);
    hi[u].load(src + D * EB);
  }
  double best[U];
#pragma unroll
  for (int u = 0; u < U; ++u) best[u] = -INFINITY;
  for (int r0 = block0 * QR; r0 < rows; r0 += step * QR) {
    const int n = min(QR, rows - r0);
    __syncthreads();
    for (int i = threadIdx.x; i < n * L; i += NT) {
      const int r = r0 + i / L, ch = i % L, nr = a.by_group.quot(r);
      Row16<BF16> x;
      x.load((const char*)a.q +
             ((((long long)b * p.Ln + nr) * p.Hq + (long long)g * p.G + a.by_group.rem(r, nr)) * D + ch * E) * EB);
      x.unpack(&q[i / L][ch * E]);
    }
    __syncthreads();
    for (int r = 0; r < n; ++r) {
      float x[E];
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = q[r][c * E + e];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (u > 0 && j0 + u * PP >= pages) break;   // no pages in this turn
        float l32[E], h32[E];
        lo[u].unpack(l32);
        hi[u].unpack(h32);
        double s = 0.0;
#pragma unroll
        for (int e = 0; e < E; ++e) s = fma((double)x[e], (double)(x[e] >= 0.f ? h32[e] : l32[e]), s);
        s = lanes_sum<L>(s);
        nan[u] = nan[u] || s != s;
        best[u] = fmax(best[u], s);
      }
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int j = j0 + u * PP + threadIdx.x / L;
    if (c == 0 && j < pages) put(j, nan[u] ? (double)NAN : best[u]);
  }
}

template <bool BF16, int D>
__global__ __launch_bounds__(256) void page_score_kernel(PageSelectArgs a) {
  constexpr int PP = 256 / (D / (BF16 ? 8 : 4));
  __shared__ __align__(16) float q[kScoreRows][D];
  const PagedArgs& p = a.c;
  const int id = uniform((int)block_id());
  const int all = a.by_blocks.quot(id), bh = a.by_shares.quot(all), share = a.by_shares.rem(all, bh);
  const int b = a.by_heads.quot(bh), g = a.by_heads.rem(bh, b);
  if (b >= p.B) return;
  const int pages = (paged_len(p, b) + p.R - 1) >> p.log2R;
  const int j0 = a.by_blocks.rem(id, all) * PP * kScoreTurns;
  if (j0 >= pages) return;
  double* score = a.score + (long long)all * p.max_pages;
  score_pages<BF16, D, 256>(a, b, g, j0, pages, paged_new(p, b) * p.G, share, a.shares, q,
                            [&](int j, double s) { score[j] = s; });
}

// The top_k pages of one (sequence, KV head), ascending.  Scores map to 64-bit keys whose
// order is theirs; a radix descent of eight bits a pass, from the highest bit in which
// the keys differ down to the first digit that parts exactly the pages wanted, finds the
// least key kept.  Then the pages above it, and the lowest of those equal to it, are
// written in order.  The latency of the passes bounds it (2048 pages 7.0 us; eight
// passes over all 64 bits 13.5): a thread keeps its pages, neighbours, in registers for up to
// KPT of them (KPT = 0: reads them again from the workspace).
constexpr int kSelectThreads = 512, kSelectWaves = kSelectThreads / 64;

__device__ __forceinline__ uint64_t page_key(double s) {
  if (s != s) return ~0ull;
  const uint64_t u = __builtin_bit_cast(uint64_t, s == 0.0 ? 0.0 : s);
  return (u >> 63) ? ~u : (u | (1ull << 63));
}

// Bitwise reduction over the wave.
template <class F>
__device__ __forceinline__ uint64_t wave_bits(uint64_t x, int none, F op) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane(wave_scan((int)(uint32_t)x, none, op), 63);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane(wave_scan((int)(uint32_t)(x >> 32), none, op), 63);
  return (uint64_t)hi << 32 | lo;
}

// Exclusive sum over the workgroup of one value per thread.
__device__ __forceinline__ int block_prefix(int x, int* lds) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int incl = wave_scan(x, 0, [](int p, int q) { return p + q; });
  if (lane == 63) lds[wave] = incl;
  __syncthreads();
  int before = 0;
#pragma unroll
  for (int w = 0; w < kSelectWaves - 1; ++w) before += w < wave ? lds[w] : 0;
  return before + incl - x;
}

// score: of page j of row share i at i * stride + j.
template <int KPT>
__device__ __forceinline__ void select_pages(const PageSelectArgs& a, const double* score, int shares, int stride,
                                             int pages, int32_t* out) {
  __shared__ uint32_t hist[256];
  __shared__ uint64_t all_or[kSelectWaves], all_and[kSelectWaves];
  __shared__ int sums[2][kSelectWaves], pick[3];
  const int tid = threadIdx.x;
  const int k = min(a.top_k, pages);
  for (int i = k + tid; i < a.top_k; i += kSelectThreads) out[i] = -1;
  // Forced pages: 0..head-1 and tail..pages-1.
  const int head = min(a.n_first, pages), tail = max(head, pages - a.n_last), forced = head + pages - tail;
  if (k == pages || forced >= k) {
    for (int i = tid; i < k; i += kSelectThreads) out[i] = i < head ? i : k == pages ? i : tail + i - head;
    return;
  }
  int need = k - forced;                // pages still to be taken among those that match the prefix
  const int per = (pages + kSelectThreads - 1) / kSelectThreads, j0 = tid * per;
  auto key_of = [&](int j) {            // NaN ranks first, so the largest key is the largest score's
    uint64_t x = page_key(score[j]);
    for (int i = 1; i < shares; ++i) x = max(x, page_key(score[(long long)i * stride + j]));
    return x;
  };
  uint64_t key[KPT > 0 ? KPT : 1];
#pragma unroll
  for (int t = 0; t < KPT; ++t) key[t] = t < per && j0 + t < pages ? key_of(j0 + t) : 0;
  auto free_page = [&](int j) { return j >= head && j < tail; };
  auto each = [&](auto f) {             // f(page, key) for the thread's pages that are not forced
    if constexpr (KPT > 0) {
#pragma unroll
      for (int t = 0; t < KPT; ++t)
        if (t < per && free_page(j0 + t)) f(j0 + t, key[t]);
    } else {
      for (int t = 0; t < per; ++t)
        if (free_page(j0 + t)) f(j0 + t, key_of(j0 + t));
    }
  };
  uint64_t any = 0, every = ~0ull;
  each([&](int, uint64_t x) {
    any |= x;
    every &= x;
  });
  any = wave_bits(any, 0, [](int x, int y) { return x | y; });
  every = wave_bits(every, -1, [](int x, int y) { return x & y; });
  if ((tid & 63) == 0) {
    all_or[tid >> 6] = any;
    all_and[tid >> 6] = every;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kSelectWaves; ++w) {
    any |= all_or[w];
    every &= all_and[w];
  }
  // Bits below `low` are still open.
  int low = any == every ? 0 : 64 - __clzll((long long)(any ^ every));
  uint64_t prefix = low >= 64 ? 0 : any >> low << low;
  bool exact = false;                   // all pages from the prefix up are kept
  while (low > 0 && !exact) {
    const int shift = max(low - 8, 0);
    const uint32_t digits = (1u << (low - shift)) - 1;
    for (int i = tid; i < 256; i += kSelectThreads) hist[i] = 0;
    __syncthreads();
    each([&](int, uint64_t x) {
      if (low >= 64 || (x >> low) == (prefix >> low)) atomicAdd(&hist[(uint32_t)(x >> shift) & digits], 1u);
    });
    __syncthreads();
    if (tid < 64) {
      // Lane l owns digits 255-4l .. 252-4l, the highest first.
      int own[4], s = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) s += own[i] = (int)hist[255 - 4 * tid - i];
      int before = wave_scan(s, 0, [](int x, int y) { return x + y; }) - s;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (before < need && before + own[i] >= need) {
          pick[0] = 255 - 4 * tid - i;
          pick[1] = before;
          pick[2] = own[i];
        }
        before += own[i];
      }
    }
    __syncthreads();
    prefix |= (uint64_t)pick[0] << shift;
    need -= pick[1];
    exact = pick[2] == need;
    low = shift;
  }
  // Of the pages with the prefix's own key, all, or the lowest `need`.
  int rank = 0;
  if (!exact) {
    int same = 0;
    each([&](int, uint64_t x) { same += x == prefix; });
    rank = block_prefix(same, sums[0]);
  }
  int kept = 0, r = rank;
  auto keep = [&](uint64_t x) { return x > prefix || (x == prefix && (exact || r++ < need)); };
  each([&](int, uint64_t x) { kept += keep(x); });
  int at = block_prefix(kept, sums[1]) + head;
  r = rank;
  each([&](int j, uint64_t x) {
    if (keep(x)) out[at++] = j;
  });
  for (int i = tid; i < forced; i += kSelectThreads) {
    if (i < head) out[i] = i;
    else out[k - forced + i] = tail + i - head;
  }
}

template <int KPT>
__global__ __launch_bounds__(kSelectThreads) void page_select_kernel(PageSelectArgs a) {
  const PagedArgs& p = a.c;
  const int bh = uniform((int)block_id()), b = a.by_heads.quot(bh);
  if (b >= p.B) return;
  select_pages<KPT>(a, a.score + (long long)bh * a.shares * p.max_pages, a.shares, p.max_pages,
                    (paged_len(p, b) + p.R - 1) >> p.log2R, a.page_idx + (long long)bh * a.top_k);
}

// Scores and choice in one launch, a workgroup for each (sequence, KV head), the scores in LDS.
constexpr int kFusedPages = 128;
template <bool BF16, int D>
__global__ __launch_bounds__(kSelectThreads) void page_score_select_kernel(PageSelectArgs a) {
  constexpr int PP = kSelectThreads / (D / (BF16 ? 8 : 4));
  __shared__ __align__(16) float q[kScoreRows][D];
  __shared__ double score[kFusedPages];
  const PagedArgs& p = a.c;
  const int bh = uniform((int)block_id());
  const int b = a.by_heads.quot(bh), g = a.by_heads.rem(bh, b);
  if (b >= p.B) return;
  const int pages = (paged_len(p, b) + p.R - 1) >> p.log2R, rows = paged_new(p, b) * p.G;
  if (pages > a.top_k)   // otherwise all are kept
    for (int j0 = 0; j0 < pages; j0 += PP * kScoreTurns)
      score_pages<BF16, D, kSelectThreads>(a, b, g, j0, pages, rows, 0, 1, q, [&](int j, double s) { score[j] = s; });
  __syncthreads();
  select_pages<1>(a, score, 1, 0, pages, a.page_idx + (long long)bh * a.top_k);
}

// Whether one launch does: few pages (128 pages of 8 heads 17.2 us with the attention over 16 of
// them, 17.7 with two launches).  More are scored by more workgroups (512 pages of 8 x 32 heads
// 46.4 us in one launch, 45.4 in two).
bool page_select_fused(const PagedArgs& p) { return p.max_pages <= kFusedPages && p.G * p.Ln <= kScoreRows; }

// Shares that the query rows of a (sequence, head) are scored in, each by workgroups of its own: the
// blocks of 16 rows, at most eight shares (264 rows over 17 pages of 13 heads, and the attention over 6 of
// them: 223 us with one share, 35 with eight).
int page_score_shares(const PagedArgs& p) {
  const long long blocks = ((long long)p.G * p.Ln + kScoreRows - 1) / kScoreRows;
  return (int)(blocks < 8 ? blocks : 8);
}

int page_score_blocks(const PagedArgs& p) {
  const int per = 256 / (p.D / (p.bf16 ? 8 : 4)) * kScoreTurns;
  return (p.max_pages + per - 1) / per;
}

hipError_t launch_paged_select(const PageSelectArgs& a, hipStream_t s) {
  const PagedArgs& p = a.c;
  const dim3 sg = grid_xy((long long)p.B * p.Hkv);
  if (page_select_fused(p)) {
    if (p.bf16) {
      if (p.D == 128) hipLaunchKernelGGL((page_score_select_kernel<true, 128>), sg, dim3(kSelectThreads), 0, s, a);
      else hipLaunchKernelGGL((page_score_select_kernel<true, 64>), sg, dim3(kSelectThreads), 0, s, a);
    } else {
      if (p.D == 128) hipLaunchKernelGGL((page_score_select_kernel<false, 128>), sg, dim3(kSelectThreads), 0, s, a);
      else hipLaunchKernelGGL((page_score_select_kernel<false, 64>), sg, dim3(kSelectThreads), 0, s, a);
    }
    return hipGetLastError();
  }
  const dim3 grid = grid_xy((long long)p.B * p.Hkv * a.shares * page_score_blocks(p));
  if (p.bf16) {
    if (p.D == 128) hipLaunchKernelGGL((page_score_kernel<true, 128>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((page_score_kernel<true, 64>), grid, dim3(256), 0, s, a);
  } else {
    if (p.D == 128) hipLaunchKernelGGL((page_score_kernel<false, 128>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((page_score_kernel<false, 64>), grid, dim3(256), 0, s, a);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (p.max_pages <= kSelectThreads) hipLaunchKernelGGL(page_select_kernel<1>, sg, dim3(kSelectThreads), 0, s, a);
  else if (p.max_pages <= 4 * kSelectThreads) hipLaunchKernelGGL(page_select_kernel<4>, sg, dim3(kSelectThreads), 0, s, a);
  else if (p.max_pages <= 16 * kSelectThreads) hipLaunchKernelGGL(page_select_kernel<16>, sg, dim3(kSelectThreads), 0, s, a);
  else hipLaunchKernelGGL(page_select_kernel<0>, sg, dim3(kSelectThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace pd
