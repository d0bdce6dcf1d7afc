// Host-side argument validation of the paged-cache entry points under AddressSanitizer and
// UndefinedBehaviorSanitizer: every call has arguments that are refused before anything
// is launched (so no GPU is needed), plus the size queries.  Exit status 0 iff every
// call returned the expected status.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstring>

#include "pd.h"

static int failures = 0;

#define EXPECT(call, want)                                                                                   \
  do {                                                                                                       \
    const int got_ = (int)(call);                                                                            \
    if (got_ != (int)(want)) {                                                                               \
      std::printf("FAIL line %d: %s -> %d (want %d): %s\n", __LINE__, #call, got_, (int)(want), pd_last_error_message()); \
      ++failures;                                                                                            \
    }                                                                                                        \
  } while (0)

int main() {
  void* A = reinterpret_cast<void*>(uintptr_t(1) << 20);
  void* MIS = reinterpret_cast<void*>((uintptr_t(1) << 20) + 8);
  const size_t big = size_t(1) << 40;
  pd_paged_dims d;
  std::memset(&d, 0, sizeof(d));
  d.batch = 2; d.new_len = 1; d.n_heads_q = 8; d.n_heads_kv = 2; d.head_dim = 128; d.dtype = PD_BF16;
  d.cache_dtype = PD_FP8_E4M3; d.page_rows = 64; d.n_pages = 100; d.max_pages = 40; d.causal = 1;
  pd_paged_cache c{A, A, static_cast<uint8_t*>(A), static_cast<uint8_t*>(A), A, static_cast<int32_t*>(A),
                   static_cast<int32_t*>(A), nullptr};
  int32_t* I = static_cast<int32_t*>(A);
  const struct { int32_t pd_paged_dims::*f; int32_t v; pd_status want; } bad[] = {
      {&pd_paged_dims::batch, INT32_MIN, PD_ERR_BAD_DIMS},     {&pd_paged_dims::batch, INT32_MAX, PD_ERR_BAD_DIMS},
      {&pd_paged_dims::new_len, 0, PD_ERR_BAD_DIMS},           {&pd_paged_dims::new_len, INT32_MAX, PD_ERR_BAD_DIMS},
      {&pd_paged_dims::n_heads_q, INT32_MAX, PD_ERR_BAD_DIMS}, {&pd_paged_dims::n_heads_kv, INT32_MIN, PD_ERR_BAD_DIMS},
      {&pd_paged_dims::n_heads_kv, 3, PD_ERR_UNSUPPORTED},     {&pd_paged_dims::head_dim, INT32_MIN, PD_ERR_UNSUPPORTED},
      {&pd_paged_dims::dtype, 99, PD_ERR_UNSUPPORTED},         {&pd_paged_dims::cache_dtype, PD_FP32, PD_ERR_UNSUPPORTED},
      {&pd_paged_dims::page_rows, INT32_MIN, PD_ERR_BAD_DIMS}, {&pd_paged_dims::page_rows, 0, PD_ERR_BAD_DIMS},
      {&pd_paged_dims::n_pages, -1, PD_ERR_BAD_DIMS},          {&pd_paged_dims::max_pages, INT32_MAX, PD_ERR_BAD_DIMS},
      {&pd_paged_dims::max_pages, INT32_MIN, PD_ERR_BAD_DIMS}, {&pd_paged_dims::causal, -1, PD_ERR_BAD_DIMS},
  };
  for (const auto& b : bad) {
    pd_paged_dims x = d;
    x.*(b.f) = b.v;
    EXPECT(pd_paged_append(&x, &c, A, 256, A, 256, nullptr), b.want);
    EXPECT(pd_paged_read(&x, &c, 0, 1, A, A, nullptr), b.want);
    EXPECT(pd_paged_select(&x, &c, A, 4, 0, 0, I, A, big, nullptr), b.want);
    EXPECT(pd_paged_attn(&x, &c, A, nullptr, 0, A, nullptr, A, big, nullptr), b.want);
    for (int which = 0; which < 2; ++which)
      if (pd_paged_workspace_bytes(&x, 4, which) != 0) { std::printf("FAIL: size query accepted bad dims\n"); ++failures; }
  }
  pd_paged_dims huge = d;   // sizes whose products pass 32 and 64 bits
  huge.batch = 65536; huge.n_heads_q = 65536; huge.n_heads_kv = 65536; huge.new_len = 1; huge.max_pages = 1 << 24;
  EXPECT(pd_paged_attn(&huge, &c, A, nullptr, 0, A, nullptr, A, big, nullptr), PD_ERR_BAD_DIMS);
  huge.n_heads_q = huge.n_heads_kv = 16384;
  huge.new_len = 2;
  EXPECT(pd_paged_append(&huge, &c, A, 16384 * 128, A, 16384 * 128, nullptr), PD_ERR_BAD_DIMS);
  EXPECT(pd_paged_read(&huge, &c, 0, 1 << 30, A, A, nullptr), PD_ERR_BAD_DIMS);
  EXPECT(pd_paged_select(&huge, &c, A, 4, 0, 0, I, A, big, nullptr), PD_ERR_BAD_DIMS);
  EXPECT(pd_paged_workspace_bytes(&huge, 0, 1), 0);
  EXPECT(pd_paged_append(nullptr, &c, A, 256, A, 256, nullptr), PD_ERR_NULL_PTR);
  EXPECT(pd_paged_attn(&d, nullptr, A, nullptr, 0, A, nullptr, A, big, nullptr), PD_ERR_NULL_PTR);
  EXPECT(pd_paged_append(&d, &c, MIS, 256, A, 256, nullptr), PD_ERR_MISALIGNED);
  EXPECT(pd_paged_append(&d, &c, A, INT64_MIN, A, 256, nullptr), PD_ERR_BAD_DIMS);
  EXPECT(pd_paged_append(&d, &c, A, 256, A, INT64_MAX, nullptr), PD_ERR_BAD_DIMS);
  EXPECT(pd_paged_read(&d, &c, INT32_MAX, INT32_MAX, A, A, nullptr), PD_ERR_BAD_DIMS);
  EXPECT(pd_paged_select(&d, &c, A, INT32_MAX, 0, 0, I, A, big, nullptr), PD_ERR_BAD_DIMS);
  EXPECT(pd_paged_select(&d, &c, A, 4, 0, INT32_MIN, I, A, big, nullptr), PD_ERR_BAD_DIMS);
  EXPECT(pd_paged_attn(&d, &c, A, nullptr, 0, A, nullptr, A, pd_paged_workspace_bytes(&d, 0, 1) - 1, nullptr), PD_ERR_WORKSPACE);
  EXPECT(pd_paged_attn(&d, &c, A, I, 41, A, nullptr, A, big, nullptr), PD_ERR_BAD_DIMS);
  EXPECT(pd_qk_norm_rope(INT32_MAX, 65536, 65536, 128, PD_BF16, A, 1 << 23, A, 1 << 23, A, A, 1e-6f, I, 1e4, A, 1 << 23, A, 1 << 23, nullptr), PD_ERR_BAD_DIMS);
  EXPECT(pd_qk_norm_rope(1, INT32_MAX, INT32_MAX, 128, PD_BF16, A, 256, A, 256, A, A, 1e-6f, I, 1e4, A, 256, A, 256, nullptr), PD_ERR_BAD_DIMS);
  EXPECT(pd_qk_norm_rope(1, 2, 2, 128, PD_BF16, A, INT64_MIN, A, 256, A, A, 1e-6f, I, 1e4, A, 256, A, 256, nullptr), PD_ERR_BAD_DIMS);
  EXPECT(pd_qk_norm_rope(1, 2, 2, 128, PD_BF16, A, 256, A, 256, A, A, NAN, I, 1e4, A, 256, A, 256, nullptr), PD_ERR_BAD_DIMS);
  EXPECT(pd_qk_norm_rope(0, 2, 2, 128, PD_BF16, nullptr, 0, nullptr, 0, nullptr, nullptr, 0.f, I, 1e4, nullptr, 0, nullptr, 0, nullptr), PD_OK);
  std::printf("%s (%d failures)\n", failures ? "FAILED" : "ok", failures);
  return failures ? 1 : 0;
}
