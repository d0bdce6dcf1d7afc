// Rows of a projection into the pages, with the head norms and the rotary positions on the way.
//
// y = x * w / sqrt(mean x^2 + eps), then (y_i, y_{i+d/2}) turned by pos * base^(-2i/d): query rows go to a buffer of their
// own, key rows into the pages, and value rows beside them as they are.  Every element is read and written once;
// nothing else is moved, so memory bounds it.
//
// Norm and rotation are in double precision: what is held in a few bits is next to a border now and then, and so the
// pages hold the bits of the formula whatever the order of its sums.
//
// Measured: prompts of 4 sequences of up to 4161 rows, 32 + 32 + 32 heads, bf16: 121 us, 4.2 TB/s; without norm and
// rotation 91, so that the arithmetic (counters: 60 us of the vector units) hides behind memory only in part.  One token
// of 8 sequences of 36 heads 8.4 us: a chain of lengths, page number, sine and cosine, rows.
#include <type_traits>

#include "paged_common.h"

namespace pd {

// 1 / sqrt(x): the hardware's approximation, off by some 2^-23 of itself, and one step of third order.
__device__ __forceinline__ double inv_sqrt(double x) {
  const double y = __builtin_amdgcn_rsq(x), off = fma(-x * y, y, 1.0);
  const double z = fma(y * off, fma(0.375, off, 0.5), y);
  return x < INFINITY ? z : y;   // 0 of infinity
}

// x with its sign changed where `sign` has the sign bit.
__device__ __forceinline__ double flip(double x, uint32_t sign) {
  u32x2 w = __builtin_bit_cast(u32x2, x);
  w[1] ^= sign;
  return __builtin_bit_cast(double, w);
}

// One workgroup per (sequence, page that new rows fall into, `heads` of the row's heads: queries, then keys, then
// values), so that the bounds of a page need no atomics in memory.  It walks the page's rows T at a time: sines and
// cosines of the next T rows go to LDS in double while these are worked on, and a wave takes a head of the T rows, U loads
// of HP rows, with the next head's in flight (without norm and rotation the prompts above take 90.7 us so and 93.5 otherwise,
// with them 120.6 and 120.1).  Three waves a SIMD: four spill registers, and spilled ones are written and read through memory (147 us).
template <int CT, int D>
__global__ __launch_bounds__(256, 3) void paged_append_rope_kernel(AppendRopeArgs a) {
  constexpr bool BF16 = CT != kFp32;
  constexpr int E = BF16 ? 8 : 4, L = D / E, HP = 64 / L, EB = BF16 ? 2 : 4, U = 4, T = U * HP;
  __shared__ double2 table[2][T][D / 2];
  __shared__ float bound[kRopeHeads][2][D];
  const PagedArgs& p = a.c;
  const int id = uniform((int)block_id());
  const int bj = a.by_chunks.quot(id), h0 = a.by_chunks.rem(id, bj) * a.heads;
  const int b = a.by_pages.quot(bj), jj = a.by_pages.rem(bj, b);
  if (b >= p.B) return;
  const int len = paged_len(p, b), n_new = paged_new(p, b);
  const int start = len - n_new;                       // position of new row 0; below 0: rows that only queries have
  const int j = (max(start, 0) >> p.log2R) + jj;
  const int lo = jj == 0 ? start : j << p.log2R, hi = min(len, (j + 1) << p.log2R);
  if (lo >= hi) return;
  const int heads = p.Hq + 2 * p.Hkv, h1 = min(h0 + a.heads, heads), rotated = p.Hq + p.Hkv;
  const uint32_t minus = threadIdx.x % L < L / 2 ? 0x80000000u : 0u;   // the sign of the sine
  const int wave = uniform((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, c = lane % L;
  int page = 0;
  bool there = false;
  if (h1 > p.Hq && hi > 0) {
    const int number = p.page_table[(long long)b * p.max_pages + j];
    there = (unsigned)number < (unsigned)p.n_pages;
    page = there ? number : 0;
  }
  const bool widen = (max(lo, 0) & (p.R - 1)) != 0;    // the page's row 0 is an older one
  const bool turn = a.rotate && h0 < rotated;
  // This thread's pair of the table.
  constexpr int P = D / 2;
  const int pair = threadIdx.x % P;
  double freq = 0.0, step_cos = 1.0, step_sin = 0.0;   // of the positions between a thread's rows
  if (turn) {
    const double rest = (double)pair * a.step_rest * -0.6931471805599453;
    freq = exp2(-(double)pair * a.step) * (1.0 + (rest + 0.5 * rest * rest)) * 0.15915494309189535;
    if (!a.pos && hi - lo > 256 / P) {
      const double turns = (double)(256 / P) * freq;
      sincospi(2.0 * (turns - rint(turns)), &step_sin, &step_cos);
    }
  }
  // Sines and cosines of the T rows from r0 on.  Where positions follow each other, a thread's first row has them
  // from the angle, and its others (three at most) are turned on from there.
  auto angles = [&](double2 (*to)[D / 2], int r0) {
    double sn = 0.0, cs = 1.0;
    for (int t = threadIdx.x / P; t < min(T, hi - r0); t += 256 / P) {
      const int r = r0 + t;
      if (a.pos || t < 256 / P) {
        const int at = a.pos ? a.pos[(long long)b * p.Ln + (r - start)] : r;
        const double turns = (double)at * freq;
        sincospi(2.0 * (turns - rint(turns)), &sn, &cs);
      } else {
        const double z = cs;
        cs = fma(z, step_cos, -sn * step_sin);
        sn = fma(sn, step_cos, z * step_sin);
      }
      to[t][(pair % E) * (L / 2) + pair / E] = make_double2(cs, sn);
    }
  };
  for (int i = threadIdx.x; p.k_bounds && i < kRopeHeads * 2 * D; i += 256)
    (&bound[0][0][0])[i] = (i / D) & 1 ? -INFINITY : INFINITY;
  // The rows of one head, HP in each of U loads: those of the next head (or of the next rows) are in flight while one
  // is worked on.
  auto fetch = [&](Row16<BF16>* x, int r0, int h) {
    const int kind = h < p.Hq ? 0 : h < rotated ? 1 : 2, hh = kind == 0 ? h : kind == 1 ? h - p.Hq : h - rotated;
    const long long stride = kind == 0 ? a.qs : kind == 1 ? a.ks : a.vs;
    const char* src = (const char*)(kind == 0 ? a.q : kind == 1 ? a.k : a.v) + ((long long)hh * D + c * E) * EB;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = min(r0 + u * HP + lane / L, hi - 1);
      x[u].load_once(src + ((long long)b * p.Ln + (r - start)) * stride * EB);
    }
  };
  Row16<BF16> next[U];
  if (h0 + wave < h1) fetch(next, lo, h0 + wave);
  if (turn) angles(table[0], lo);
  int buf = 0;
  for (int r0 = lo; r0 < hi; r0 += T, buf ^= 1) {
    if (turn || (r0 == lo && p.k_bounds)) __syncthreads();
    if (turn && r0 + T < hi) angles(table[buf ^ 1], r0 + T);   // which no wave reads any more
    for (int h = h0 + wave; h < h1; h += 4) {
      const int kind = h < p.Hq ? 0 : h < rotated ? 1 : 2, hh = kind == 0 ? h : kind == 1 ? h - p.Hq : h - rotated;
      Row16<BF16> x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) x[u] = next[u];
      if (h + 4 < h1) fetch(next, r0, h + 4);
      else if (r0 + T < hi) fetch(next, r0 + T, h0 + wave);
      const void* weights = kind == 0 ? a.w_q : a.w_k;
      const CacheRow<CT, D> to(p, kind == 2, ((long long)page * p.Hkv + hh) * p.R, c);
      // K: the kind of head, or 3 where it is looked at here; FULL: with norm and rotation, no branch for either, so that
      // the U loads' chains run beside each other.
      auto work = [&](auto kind_of, auto all) {
        constexpr int K = decltype(kind_of)::value;
        constexpr bool FULL = decltype(all)::value;
        const bool norm = FULL || (kind < 2 && weights), rotates = FULL || (kind < 2 && turn);
        Row16<BF16> weight;
        if (norm) weight.load((const char*)weights + c * 16);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int r = r0 + u * HP + lane / L, t = min(r, hi - 1) - r0;   // rows behind the last are that one again
          float y[E];
          x[u].unpack(y);
          if (norm || rotates) {
            double z[E], scale = 1.0;
#pragma unroll
            for (int e = 0; e < E; ++e) z[e] = (double)y[e];
            if (norm) {
              // Unpacked for each load: kept in double, the weights are eight registers more, and spilled ones cost writes.
              float w[E];
#pragma unroll
              for (int i = 0; i < 4; ++i) asm("" : "+v"(weight.v[i]));
              weight.unpack(w);
              double s = 0.0;
#pragma unroll
              for (int e = 0; e < E; ++e) {
                s = fma(z[e], z[e], s);
                z[e] *= (double)w[e];
              }
              scale = inv_sqrt(lanes_sum<L>(s) * (1.0 / D) + (double)a.eps);
            }
            if (rotates) {
#pragma unroll
              for (int e = 0; e < E; ++e) {
                const double2 cs = table[buf][t][e * (L / 2) + c % (L / 2)];
                // out_i = y_i cos - y' sin, out_{i+d/2} = y_{i+d/2} cos + y' sin
                z[e] = fma(partner<L>(z[e]), flip(cs.y, minus), z[e] * cs.x);
              }
            }
            // To fp32 and to the element type, and what the pages hold from that: keys have bounds that are theirs
            // to the bit, and the bytes that the append kernel gives for the same rows.
#pragma unroll
            for (int e = 0; e < E; ++e) {
              y[e] = (float)(z[e] * scale);
              asm("" : "+v"(y[e]));   // otherwise both roundings become one, a dozen instructions long
            }
            x[u].pack(y);
            x[u].unpack(y);
          }
          if (K == 0 || (K == 3 && kind == 0)) {
            char* at = (char*)a.q_out + ((((long long)b * p.Ln + (r - start)) * p.Hq + h) * D + c * E) * EB;
            if (r < hi) {
              if (a.stream) x[u].store_once(at);
              else x[u].store(at);
            }
          } else {
            if ((K == 1 || (K == 3 && kind == 1)) && p.k_bounds) {
              // The rows that a wave holds side by side meet in LDS; NaN is neither less nor more than what is there.
              const bool counts = FULL || r >= 0;
#pragma unroll
              for (int e = 0; e < E; ++e) {
                __hip_atomic_fetch_min(&bound[h - h0][0][e * L + c], counts ? y[e] : INFINITY, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
                __hip_atomic_fetch_max(&bound[h - h0][1][e * L + c], counts ? y[e] : -INFINITY, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
              }
            }
            to.put(x[u], y, r & (p.R - 1), r < hi && (FULL || r >= 0) && there);
          }
        }
      };
      const bool full = weights && turn && r0 >= 0;
      if (full && kind == 0) work(std::integral_constant<int, 0>{}, std::true_type{});
      else if (full && kind == 1) work(std::integral_constant<int, 1>{}, std::true_type{});
      else work(std::integral_constant<int, 3>{}, std::false_type{});
    }
  }
  if (!p.k_bounds || !there) return;
  __syncthreads();
  const int k0 = max(h0, p.Hq), k1 = min(h1, rotated);
  for (int i = threadIdx.x; i < (k1 - k0) * 2 * D; i += 256) {
    const int h = k0 + i / (2 * D);
    const bool up = (i / D) & 1;
    const long long at = ((long long)page * p.Hkv + (h - p.Hq)) * 2 * D + i % (2 * D);
    float x = bound[h - h0][up][i % E * L + i % D / E];
    if constexpr (BF16) {
      uint16_t* to = (uint16_t*)p.k_bounds + at;
      if (widen) x = up ? fmaxf(x, bf16_to_f32(*to)) : fminf(x, bf16_to_f32(*to));
      *to = f32_to_bf16(x);
    } else {
      float* to = (float*)p.k_bounds + at;
      if (widen) x = up ? fmaxf(x, *to) : fminf(x, *to);
      *to = x;
    }
  }
}

template <int CT, int D>
hipError_t append_rope_of(const AppendRopeArgs& a, hipStream_t s) {
  const int chunks = (int)a.by_chunks.d;
  hipLaunchKernelGGL((paged_append_rope_kernel<CT, D>), grid_xy((long long)a.c.B * a.pages * chunks), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_paged_append_rope(AppendRopeArgs a, hipStream_t s) {
  // As many heads a workgroup as leave four workgroups for every CU: sines and cosines are shared by its heads.  Eight
  // at most (the prompts above 121 us, 139 with sixteen, whose last round is half empty, 123 with four).
  const int heads = a.c.Hq + 2 * a.c.Hkv;
  a.heads = kRopeHeads;
  while (a.heads > 4 && (long long)a.c.B * a.pages * ((heads + a.heads - 1) / a.heads) < 4 * kNumCu) a.heads /= 2;
  a.by_chunks = fast_div((heads + a.heads - 1) / a.heads);
  a.by_pages = fast_div(a.pages);
  a.stream = (double)a.c.B * a.c.Ln * heads * a.c.D * (a.c.bf16 ? 4 : 8) >= 256e6;   // what the last cache holds
  const bool wide = a.c.D == 128;
  switch (cache_type(a.c)) {
    case kBf16: return wide ? append_rope_of<kBf16, 128>(a, s) : append_rope_of<kBf16, 64>(a, s);
    case kFp8: return wide ? append_rope_of<kFp8, 128>(a, s) : append_rope_of<kFp8, 64>(a, s);
    case kFp4: return wide ? append_rope_of<kFp4, 128>(a, s) : append_rope_of<kFp4, 64>(a, s);
    default: return wide ? append_rope_of<kFp32, 128>(a, s) : append_rope_of<kFp32, 64>(a, s);
  }
}

}  // namespace pd
