// Device helpers of the paged-cache kernels.
#pragma once
#include "paged_kernels.h"
#include "pd_common.h"
#include "pd_kernels.h"

namespace pd {

typedef float f32x2 __attribute__((ext_vector_type(2)));

// 16 bytes of a row: eight bf16 or four fp32.
template <bool BF16>
struct Row16 {
  u32x4 v;
  __device__ __forceinline__ void load(const void* p) { v = *(const u32x4*)p; }
  __device__ __forceinline__ void store(void* p) const { *(u32x4*)p = v; }
  // Data that is read or written once, past the caches where it can.
  __device__ __forceinline__ void load_once(const void* p) { v = __builtin_nontemporal_load((const u32x4*)p); }
  __device__ __forceinline__ void store_once(void* p) const { __builtin_nontemporal_store(v, (u32x4*)p); }
  __device__ __forceinline__ void zero() { v = u32x4{0, 0, 0, 0}; }
  __device__ __forceinline__ void nan() { v = u32x4{kNanWord, kNanWord, kNanWord, kNanWord}; }
  __device__ __forceinline__ void unpack(float* y) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (BF16) {
        y[2 * i] = __uint_as_float(v[i] << 16);
        y[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
      } else {
        y[i] = __uint_as_float(v[i]);
      }
    }
  }
  __device__ __forceinline__ void pack(const float* y) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (BF16) v[i] = pack_bf16x2(y[2 * i], y[2 * i + 1]);
      else v[i] = __float_as_uint(y[i]);
    }
  }
};

// 2^e of an exponent byte e + 127 (27..247, in 4 bits ..253; 255, a group that is NaN, is what the conversions from 4 bits
// take for NaN).
__device__ __forceinline__ float exp_to_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// Eight E2M1 values times a power of two, to and from bf16 or fp32: element i is in bits 4 i.  Rounded to
// nearest even, at most +-6; from 4 bits the results are exact.
__device__ __forceinline__ u32x4 from_fp4(uint32_t w, float scale) {
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3))};
}
__device__ __forceinline__ uint32_t to_fp4(const float* y, float scale) {
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[0], y[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], scale, 3);
}

// Rows and new rows of a sequence, within what the cache and the call have room for.
__device__ __forceinline__ int paged_len(const PagedArgs& p, int b) {
  return min(max(p.kv_len[b], 0), p.max_pages << p.log2R);
}
__device__ __forceinline__ int paged_new(const PagedArgs& p, int b) {
  return p.new_rows ? min(max(p.new_rows[b], 0), p.Ln) : p.Ln;
}

// Inclusive scan over the wave (sums, maxima), on the vector units: 16 lanes at a time, then
// the last lane of each row handed on.
template <class F>
__device__ __forceinline__ int wave_scan(int x, int none, F op) {
#define PD_SCAN(ctrl, rows) x = op(x, __builtin_amdgcn_update_dpp(none, x, ctrl, rows, 0xf, false))
  PD_SCAN(0x111, 0xf);   // row_shr:1
  PD_SCAN(0x112, 0xf);
  PD_SCAN(0x114, 0xf);
  PD_SCAN(0x118, 0xf);
  PD_SCAN(0x142, 0xa);   // row_bcast:15
  PD_SCAN(0x143, 0xc);   // row_bcast:31
#undef PD_SCAN
  return x;
}

// The value of the lane that a DPP control names (all lanes active, none out of range).
template <int CTRL, int BANKS = 0xf>
__device__ __forceinline__ float dpp(float old, float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(old), __float_as_int(x), CTRL, 0xf, BANKS, false));
}
// The value of lane ^ L / 2, for groups of L = 8, 16 or 32 neighbouring lanes.
template <int L>
__device__ __forceinline__ float partner(float x) {
  if constexpr (L == 8) {
    // lanes 4..7 of every eight from four below, lanes 0..3 from four above
    return dpp<0x104, 0x5>(dpp<0x114, 0xa>(x, x), x);
  } else if constexpr (L == 16) {
    return dpp<0x128>(x, x);   // row_ror:8
  } else {
    return __shfl_xor(x, L / 2);
  }
}
// Sum over groups of L neighbouring lanes, the same bits in each.
template <int L>
__device__ __forceinline__ float lanes_sum(float x) {
  x += dpp<0xb1>(x, x);                            // quad_perm [1,0,3,2]
  x += dpp<0x4e>(x, x);                            // quad_perm [2,3,0,1]
  x += dpp<0x141>(x, x);                           // row_half_mirror
  if constexpr (L >= 16) x += dpp<0x140>(x, x);    // row_mirror
  if constexpr (L >= 32) x += __shfl_xor(x, 16);
  return x;
}

// The value of lane ^ L / 2 (partner).
template <int L>
__device__ __forceinline__ double partner(double x) {
  const u32x2 w = __builtin_bit_cast(u32x2, x);
  u32x2 y;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if constexpr (L == 16) y[i] = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w[i], 0x128, 0xf, 0xf, true);   // row_ror:8
    else y[i] = __float_as_uint(partner<L>(__uint_as_float(w[i])));
  }
  return __builtin_bit_cast(double, y);
}

// x + the same of the lane that `ctrl` names.
template <int CTRL>
__device__ __forceinline__ double add_dpp(double x) {
  const u32x2 w = __builtin_bit_cast(u32x2, x);
  const u32x2 y = {(uint32_t)__builtin_amdgcn_update_dpp(0, (int)w[0], CTRL, 0xf, 0xf, true),
                   (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w[1], CTRL, 0xf, 0xf, true)};
  return x + __builtin_bit_cast(double, y);
}
// Sum over groups of L neighbouring lanes, the same bits in each.
template <int L>
__device__ __forceinline__ double lanes_sum(double x) {
  x = add_dpp<0xb1>(x);                            // quad_perm [1,0,3,2]
  x = add_dpp<0x4e>(x);                            // quad_perm [2,3,0,1]
  x = add_dpp<0x141>(x);                           // row_half_mirror
  if constexpr (L >= 16) x = add_dpp<0x140>(x);    // row_mirror
  if constexpr (L >= 32) x += __shfl_xor(x, 16);
  return x;
}

// Maximum over groups of L neighbouring lanes.
template <int L>
__device__ __forceinline__ float lanes_max(float x) {
  x = fmaxf(x, dpp<0xb1>(x, x));
  x = fmaxf(x, dpp<0x4e>(x, x));
  x = fmaxf(x, dpp<0x141>(x, x));
  if constexpr (L >= 16) x = fmaxf(x, dpp<0x140>(x, x));
  if constexpr (L >= 32) x = fmaxf(x, __shfl_xor(x, 16));
  return x;
}

// What a lane needs to write its 16 bytes of rows into a page: row `base` of the pool is the page's
// row 0 (of one KV head), c the lane of a row.
template <int CT, int D>
struct CacheRow {
  static constexpr int E = CT == kFp32 ? 4 : 8, L = D / E, EB = CT == kFp32 ? 4 : 2;
  char* dst;
  uint8_t* ex;
  int c;
  __device__ __forceinline__ CacheRow(const PagedArgs& p, int kv, long long base, int lane) : ex(nullptr), c(lane) {
    char* pages = (char*)(kv ? p.v_pages : p.k_pages);
    uint8_t* exps = kv ? p.v_exp : p.k_exp;
    if constexpr (CT == kFp4) {
      dst = pages + base * (D / 2) + c * 4;
      ex = exps + base * (D / 32) + (c / 4) * p.R;   // exponent bytes of 32 channels lie by rows
    } else if constexpr (CT == kFp8) {
      dst = pages + base * D + c * 8;
      ex = exps + base;
    } else {
      dst = pages + base * (D * EB) + c * 16;
    }
  }
  // Writes row `slot` of the page, where `live`; x: the lane's 16 bytes, y: their elements.  All
  // lanes of a row are active.
  __device__ __forceinline__ void put(const Row16<CT != kFp32>& x, const float* y, int slot, bool live) const {
    if constexpr (CT == kFp8 || CT == kFp4) {
      float m = 0.f;
      bool finite = true;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float t = fabsf(y[e]);
        finite = finite && t < INFINITY;
        m = fmaxf(m, t < INFINITY ? t : 0.f);
      }
      if constexpr (CT == kFp8) {
        m = lanes_max<L>(m);
        const uint32_t bits = __float_as_uint(m);
        const int e2 = min(max((int)(bits >> 23) - 135 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0), -100), 120);
        const float inv = __uint_as_float((uint32_t)(127 - e2) << 23);
        uint32_t w[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          float z[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            z[e] = y[4 * k + e] * inv;
            z[e] = fabsf(y[4 * k + e]) < INFINITY ? z[e] : NAN;
          }
          int v = __builtin_amdgcn_cvt_pk_fp8_f32(z[0], z[1], 0, false);
          w[k] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(z[2], z[3], v, true);
        }
        if (live) {
          *(u32x2*)(dst + (long long)slot * D) = u32x2{w[0], w[1]};
          if (c == 0) ex[slot] = (uint8_t)(e2 + 127);
        }
      } else {
        // The group's four lanes: its maximum, or infinity where an element is not finite.
        m = finite ? m : INFINITY;
        m = fmaxf(m, dpp<0xb1>(m, m));
        m = fmaxf(m, dpp<0x4e>(m, m));
        const uint32_t bits = __float_as_uint(m);
        const int e2 = min(max((int)(bits >> 23) - 129 + ((bits & 0x7fffffu) > 0x400000u ? 1 : 0), -100), 126);
        const uint32_t w = to_fp4(y, exp_to_scale((uint32_t)(e2 + 127)));
        if (live) {
          *(uint32_t*)(dst + (long long)slot * (D / 2)) = w;
          if ((c & 3) == 0) ex[slot] = m < INFINITY ? (uint8_t)(e2 + 127) : (uint8_t)255;
        }
      }
    } else {
      if (live) x.store_once(dst + (long long)slot * (D * EB));
    }
  }
};

}  // namespace pd
