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

// 2^e of an exponent byte e + 127 (27..247).
__device__ __forceinline__ float exp_to_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

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

}  // namespace pd
