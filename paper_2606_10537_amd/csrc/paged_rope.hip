// Rows of a projection into the pages, with the head norms and the rotary positions on the way.
//
// y = x * w / sqrt(mean x^2 + eps), then (y_i, y_{i+d/2}) turned by pos * base^(-2i/d): query rows go to a buffer of their
// own, key rows into the pages, and value rows beside them as they are.  Every element is read and written once;
// nothing else is moved, so memory bounds it.
//
// Norm and rotation are in double precision: what is held in a few bits is next to a border now and then, and so the
// pages hold the bits of the formula whatever the order of its sums.  A double product costs what an fp32 one does
// here (64 a cycle and CU), and the rows' memory leaves room for them.
#include "paged_common.h"

namespace pd {

// One workgroup per (sequence, page that new rows fall into, `heads` of the row's heads: queries, then keys, then
// values), so that the bounds of a page need no atomics.  It walks the page's rows T at a time: sines and
// cosines of T rows go to LDS in double, then a wave takes a head, four loads of HP rows at once, as in the append kernel.
template <int CT, int D>
__global__ __launch_bounds__(256) void paged_append_rope_kernel(AppendRopeArgs a) {
  constexpr bool BF16 = CT != kFp32;
  constexpr int E = BF16 ? 8 : 4, L = D / E, HP = 64 / L, EB = BF16 ? 2 : 4, U = 4, T = U * HP;
  __shared__ double2 table[T][D / 2];
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
  double freq = 0.0;
  if (turn) {
    const double rest = (double)pair * a.step_rest * -0.6931471805599453;
    freq = exp2(-(double)pair * a.step) * (1.0 + (rest + 0.5 * rest * rest)) * 0.15915494309189535;
  }
  for (int i = threadIdx.x; p.k_bounds && i < kRopeHeads * 2 * D; i += 256)
    (&bound[0][0][0])[i] = (i / D) & 1 ? -INFINITY : INFINITY;
  for (int r0 = lo; r0 < hi; r0 += T) {
    if (r0 > lo || p.k_bounds) __syncthreads();
    if (turn) {
      for (int t = threadIdx.x / P; t < min(T, hi - r0); t += 256 / P) {
        const int r = r0 + t, at = a.pos ? a.pos[(long long)b * p.Ln + (r - start)] : r;
        const double turns = (double)at * freq;
        double sn, cs;
        sincospi(2.0 * (turns - rint(turns)), &sn, &cs);
        table[t][(pair % E) * (L / 2) + pair / E] = make_double2(cs, sn);
      }
      __syncthreads();
    }
    for (int h = h0 + wave; h < h1; h += 4) {
      const int kind = h < p.Hq ? 0 : h < rotated ? 1 : 2, hh = kind == 0 ? h : kind == 1 ? h - p.Hq : h - rotated;
      const long long stride = kind == 0 ? a.qs : kind == 1 ? a.ks : a.vs;
      const char* src = (const char*)(kind == 0 ? a.q : kind == 1 ? a.k : a.v) + ((long long)hh * D + c * E) * EB;
      Row16<BF16> x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int r = min(r0 + u * HP + lane / L, hi - 1);
        x[u].load(src + ((long long)b * p.Ln + (r - start)) * stride * EB);
      }
      const void* weights = kind == 0 ? a.w_q : a.w_k;
      const bool norm = kind < 2 && weights;
      float w[E], wp[E];
      if (norm) {
        Row16<BF16> t;
        t.load((const char*)weights + c * 16);
        t.unpack(w);
        t.load((const char*)weights + (c ^ (L / 2)) * 16);
        t.unpack(wp);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) w[e] = wp[e] = 1.f;
      }
      float least[E], most[E];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        least[e] = INFINITY;
        most[e] = -INFINITY;
      }
      const CacheRow<CT, D> to(p, kind == 2, ((long long)page * p.Hkv + hh) * p.R, c);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int t = u * HP + lane / L, r = r0 + t;
        float y[E];
        x[u].unpack(y);
        if (norm || (kind < 2 && turn)) {
          double z[E], scale = 1.0;
          if (norm) {
            double s = 0.0;
#pragma unroll
            for (int e = 0; e < E; ++e) s = fma((double)y[e], (double)y[e], s);
            scale = 1.0 / sqrt(lanes_sum<L>(s) * (1.0 / D) + (double)a.eps);
          }
#pragma unroll
          for (int e = 0; e < E; ++e) z[e] = (double)y[e] * (double)w[e] * scale;
          if (turn) {
            Row16<BF16> xp;
            float yp[E];
#pragma unroll
            for (int i = 0; i < 4; ++i) xp.v[i] = __float_as_uint(partner<L>(__uint_as_float(x[u].v[i])));
            xp.unpack(yp);
#pragma unroll
            for (int e = 0; e < E; ++e) {
              const double2 cs = table[t][e * (L / 2) + c % (L / 2)];
              // out_i = y_i cos - y' sin, out_{i+d/2} = y_{i+d/2} cos + y' sin
              const double zp = (double)yp[e] * (double)wp[e] * scale;
              z[e] = fma(zp, c < L / 2 ? -cs.y : cs.y, z[e] * cs.x);
            }
          }
          // To fp32 and to the element type, and what the pages hold from that: keys have bounds that are theirs
          // to the bit, and the bytes that the append kernel gives for the same rows.
#pragma unroll
          for (int e = 0; e < E; ++e) {
            y[e] = (float)z[e];
            asm("" : "+v"(y[e]));   // otherwise both roundings become one, a dozen instructions long
          }
          x[u].pack(y);
          x[u].unpack(y);
        }
        if (kind == 0) {
          if (r < hi) x[u].store((char*)a.q_out + ((((long long)b * p.Ln + (r - start)) * p.Hq + h) * D + c * E) * EB);
        } else {
          const bool live = r < hi && r >= 0 && there;
          if (kind == 1 && live) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
              least[e] = fminf(least[e], y[e]);
              most[e] = fmaxf(most[e], y[e]);
            }
          }
          to.put(x[u], y, r & (p.R - 1), live);
        }
      }
      if (kind == 1 && p.k_bounds) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
#pragma unroll
          for (int k = L; k < 64; k *= 2) {
            least[e] = fminf(least[e], __shfl_xor(least[e], k));
            most[e] = fmaxf(most[e], __shfl_xor(most[e], k));
          }
          if (lane < L) {   // of this head by this wave alone
            float* at = &bound[h - h0][0][c * E + e];
            at[0] = fminf(at[0], least[e]);
            at[D] = fmaxf(at[D], most[e]);
          }
        }
      }
    }
  }
  if (!p.k_bounds || !there) return;
  __syncthreads();
  const int k0 = max(h0, p.Hq), k1 = min(h1, rotated);
  for (int i = threadIdx.x; i < (k1 - k0) * 2 * D; i += 256) {
    const int h = k0 + i / (2 * D);
    const bool up = (i / D) & 1;
    const long long at = ((long long)page * p.Hkv + (h - p.Hq)) * 2 * D + i % (2 * D);
    float x = bound[h - h0][up][i % D];
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
  // As many heads a workgroup as leave four workgroups for every CU: sines and cosines are shared by its heads.
  const int heads = a.c.Hq + 2 * a.c.Hkv;
  a.heads = kRopeHeads;
  while (a.heads > 4 && (long long)a.c.B * a.pages * ((heads + a.heads - 1) / a.heads) < 4 * kNumCu) a.heads /= 2;
  a.by_chunks = fast_div((heads + a.heads - 1) / a.heads);
  a.by_pages = fast_div(a.pages);
  const bool wide = a.c.D == 128;
  switch (cache_type(a.c)) {
    case kBf16: return wide ? append_rope_of<kBf16, 128>(a, s) : append_rope_of<kBf16, 64>(a, s);
    case kFp8: return wide ? append_rope_of<kFp8, 128>(a, s) : append_rope_of<kFp8, 64>(a, s);
    case kFp4: return wide ? append_rope_of<kFp4, 128>(a, s) : append_rope_of<kFp4, 64>(a, s);
    default: return wide ? append_rope_of<kFp32, 128>(a, s) : append_rope_of<kFp32, 64>(a, s);
  }
}

}  // namespace pd
