// Host-side argument validation of pd_paged_window_attn, pd_paged_append_rope and of caches in 4 bits under AddressSanitizer and
// UndefinedBehaviorSanitizer: every call has arguments that are refused before anything is launched (so no GPU is
// needed), plus the size queries.  Exit status 0 iff every call returned the expected status.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <initializer_list>

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
  int32_t* I = static_cast<int32_t*>(A);
  const size_t big = size_t(1) << 40;
  pd_paged_dims d;
  std::memset(&d, 0, sizeof(d));
  d.batch = 2; d.new_len = 1; d.n_heads_q = 8; d.n_heads_kv = 2; d.head_dim = 128; d.dtype = PD_BF16;
  d.cache_dtype = PD_FP4_E2M1; d.page_rows = 64; d.n_pages = 100; d.max_pages = 40; d.causal = 1;
  pd_paged_cache c{A, A, static_cast<uint8_t*>(A), static_cast<uint8_t*>(A), A, I, I, nullptr};
  auto window = [&](const pd_paged_dims& x, int32_t w, int32_t s, size_t n) {
    return pd_paged_window_attn(&x, &c, A, w, s, A, nullptr, A, n, nullptr);
  };
  auto rope = [&](const pd_paged_dims& x, int64_t qs, int64_t ks, int64_t vs, float eps, double base, void* qo) {
    return pd_paged_append_rope(&x, &c, A, qs, A, ks, A, vs, A, A, eps, I, base, qo, nullptr);
  };
  const struct { int32_t pd_paged_dims::*f; int32_t v; pd_status want; } bad[] = {
      {&pd_paged_dims::batch, INT32_MIN, PD_ERR_BAD_DIMS},     {&pd_paged_dims::batch, INT32_MAX, PD_ERR_BAD_DIMS},
      {&pd_paged_dims::new_len, INT32_MAX, PD_ERR_BAD_DIMS},   {&pd_paged_dims::n_heads_q, INT32_MAX, PD_ERR_BAD_DIMS},
      {&pd_paged_dims::n_heads_kv, 3, PD_ERR_UNSUPPORTED},     {&pd_paged_dims::head_dim, INT32_MIN, PD_ERR_UNSUPPORTED},
      {&pd_paged_dims::dtype, PD_FP4_E2M1, PD_ERR_UNSUPPORTED}, {&pd_paged_dims::dtype, PD_FP32, PD_ERR_UNSUPPORTED},
      {&pd_paged_dims::cache_dtype, 4, PD_ERR_UNSUPPORTED},    {&pd_paged_dims::page_rows, INT32_MIN, PD_ERR_BAD_DIMS},
      {&pd_paged_dims::max_pages, INT32_MAX, PD_ERR_BAD_DIMS}, {&pd_paged_dims::causal, -1, PD_ERR_BAD_DIMS},
  };
  for (const auto& b : bad) {
    pd_paged_dims x = d;
    x.*(b.f) = b.v;
    EXPECT(window(x, 100, 4, big), b.want);
    EXPECT(rope(x, 1024, 256, 256, 1e-6f, 1e4, A), b.want);
    EXPECT(pd_paged_window_workspace_bytes(&x, 100, 4), 0);
  }
  for (int32_t w : {0, -1, INT32_MIN}) {
    EXPECT(window(d, w, 0, big), PD_ERR_BAD_DIMS);
    EXPECT(pd_paged_window_workspace_bytes(&d, w, 0), 0);
  }
  EXPECT(window(d, 1, INT32_MIN, big), PD_ERR_BAD_DIMS);
  for (int32_t w : {2000, INT32_MAX})
    for (int32_t s : {0, 1, INT32_MAX}) {
      const size_t need = pd_paged_window_workspace_bytes(&d, w, s);
      if (need == 0) { std::printf("FAIL: no size for window=%d, n_sinks=%d\n", w, s); ++failures; }
      EXPECT(window(d, w, s, need - 1), PD_ERR_WORKSPACE);
    }
  pd_paged_dims huge = d;   // sizes whose products pass 32 and 64 bits
  huge.batch = 65536; huge.n_heads_q = 16384; huge.n_heads_kv = 16384; huge.new_len = 2; huge.max_pages = 1 << 24;
  EXPECT(window(huge, INT32_MAX, INT32_MAX, big), PD_ERR_BAD_DIMS);
  EXPECT(rope(huge, 1 << 21, 1 << 21, 1 << 21, 1e-6f, 1e4, A), PD_ERR_BAD_DIMS);
  huge.batch = 1; huge.n_heads_q = huge.n_heads_kv = 1; huge.new_len = 1 << 13; huge.causal = 0;
  if (pd_paged_window_workspace_bytes(&huge, INT32_MAX, INT32_MAX) == 0) { std::printf("FAIL: no size for many new rows\n"); ++failures; }
  huge.new_len = 1 << 24;   // row blocks that fill the card: nothing is cut
  EXPECT(pd_paged_window_workspace_bytes(&huge, INT32_MAX, INT32_MAX), 0);
  for (int64_t s : {INT64_MIN, int64_t(0), INT64_MAX}) {
    EXPECT(rope(d, s, 256, 256, 1e-6f, 1e4, A), PD_ERR_BAD_DIMS);
    EXPECT(rope(d, 1024, s, 256, 1e-6f, 1e4, A), PD_ERR_BAD_DIMS);
    EXPECT(rope(d, 1024, 256, s, 1e-6f, 1e4, A), PD_ERR_BAD_DIMS);
  }
  EXPECT(rope(d, 1024, 256, 256, NAN, 1e4, A), PD_ERR_BAD_DIMS);
  EXPECT(rope(d, 1024, 256, 256, 1e-6f, INFINITY, A), PD_ERR_BAD_DIMS);
  EXPECT(rope(d, 1032, 256, 256, 1e-6f, 1e4, A), PD_ERR_BAD_DIMS);
  EXPECT(rope(d, 1024, 256, 256, 1e-6f, 1e4, nullptr), PD_ERR_NULL_PTR);
  EXPECT(rope(d, 1024, 256, 256, 1e-6f, 1e4, MIS), PD_ERR_MISALIGNED);
  EXPECT(pd_paged_append_rope(&d, &c, nullptr, INT64_MIN, nullptr, 256, A, 256, A, A, 0.f, nullptr, 0.0, nullptr, nullptr), PD_ERR_NULL_PTR);
  EXPECT(pd_paged_window_attn(nullptr, &c, A, 1, 0, A, nullptr, A, big, nullptr), PD_ERR_NULL_PTR);
  EXPECT(pd_paged_append(&d, &c, MIS, 256, A, 256, nullptr), PD_ERR_MISALIGNED);
  c.v_exp = nullptr;
  EXPECT(window(d, 100, 4, big), PD_ERR_NULL_PTR);
  EXPECT(rope(d, 1024, 256, 256, 1e-6f, 1e4, A), PD_ERR_NULL_PTR);
  EXPECT(pd_paged_read(&d, &c, 0, 1, A, A, nullptr), PD_ERR_NULL_PTR);
  std::printf("%s (%d failures)\n", failures ? "FAILED" : "ok", failures);
  return failures ? 1 : 0;
}
