// C-ABI entry points of the paged cache: argument validation, workspace layout,
// launches.  Everything here runs on the host.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "paged_kernels.h"
#include "pd.h"
#include "pd_host.h"
#include "pd_kernels.h"

namespace {

using namespace pd_host;

constexpr int kMaxBatch = 1 << 16;
constexpr int kMaxSelectPages = 1 << 16;
constexpr long long kMaxPositions = 1LL << 30;   // the kernels mark absent keys with this position
constexpr long long kMaxGrid = 1LL << 31;

pd_status check_paged_dims(const pd_paged_dims* d) {
  if (!d) return fail(PD_ERR_NULL_PTR, "dims is NULL");
  if (d->batch < 1 || d->batch > kMaxBatch)
    return fail(PD_ERR_BAD_DIMS, "batch=%d must be in 1..%d", d->batch, kMaxBatch);
  if (d->new_len < 1 || d->new_len > (1 << 24))
    return fail(PD_ERR_BAD_DIMS, "new_len=%d must be in 1..2^24", d->new_len);
  if (d->n_heads_q < 1 || d->n_heads_kv < 1 || d->n_heads_q > (1 << 16))
    return fail(PD_ERR_BAD_DIMS, "head counts %d/%d must be in 1..65536", d->n_heads_q, d->n_heads_kv);
  if (d->n_heads_q % d->n_heads_kv != 0)
    return fail(PD_ERR_UNSUPPORTED, "n_heads_q=%d is not a multiple of n_heads_kv=%d", d->n_heads_q, d->n_heads_kv);
  if (d->head_dim != 64 && d->head_dim != 128)
    return fail(PD_ERR_UNSUPPORTED, "head_dim=%d must be 64 or 128", d->head_dim);
  if (d->dtype != PD_BF16 && d->dtype != PD_FP32)
    return fail(PD_ERR_UNSUPPORTED, "dtype=%d is neither PD_BF16 nor PD_FP32", d->dtype);
  if (d->cache_dtype != d->dtype &&
      !((d->cache_dtype == PD_FP8_E4M3 || d->cache_dtype == PD_FP4_E2M1) && d->dtype == PD_BF16))
    return fail(PD_ERR_UNSUPPORTED, "cache_dtype=%d must be dtype=%d, or PD_FP8_E4M3 or PD_FP4_E2M1 with PD_BF16",
                d->cache_dtype, d->dtype);
  if (d->page_rows < 16 || d->page_rows > 256 || (d->page_rows & (d->page_rows - 1)) != 0)
    return fail(PD_ERR_BAD_DIMS, "page_rows=%d must be 16, 32, 64, 128 or 256", d->page_rows);
  if (d->n_pages < 1) return fail(PD_ERR_BAD_DIMS, "n_pages=%d must be >= 1", d->n_pages);
  if (d->max_pages < 1 || (long long)d->max_pages * d->page_rows > kMaxPositions)
    return fail(PD_ERR_BAD_DIMS, "max_pages=%d must be >= 1 and max_pages*page_rows at most 2^30", d->max_pages);
  if (!std::isfinite(d->sm_scale)) return fail(PD_ERR_BAD_DIMS, "sm_scale is not finite");
  if (d->causal != 0 && d->causal != 1) return fail(PD_ERR_BAD_DIMS, "causal=%d must be 0 or 1", d->causal);
  if ((long long)d->batch * d->n_heads_q * d->new_len >= kMaxGrid)
    return fail(PD_ERR_BAD_DIMS, "batch*n_heads_q*new_len must stay below 2^31");
  return PD_OK;
}

pd_status check_cache(const pd_paged_dims* d, const pd_paged_cache* c, bool pages, bool bounds) {
  if (!c) return fail(PD_ERR_NULL_PTR, "cache is NULL");
  const bool scaled = d->cache_dtype == PD_FP8_E4M3 || d->cache_dtype == PD_FP4_E2M1;
  if (pages) {
    PD_REQUIRE_PTR(c->k_pages);
    PD_REQUIRE_PTR(c->v_pages);
    if (scaled) {
      PD_REQUIRE_PTR(c->k_exp);
      PD_REQUIRE_PTR(c->v_exp);
    }
  }
  if (bounds) PD_REQUIRE_PTR(c->k_bounds);
  if (c->k_bounds && !aligned16(c->k_bounds))
    return fail(PD_ERR_MISALIGNED, "pointer 'k_bounds' is not 16-byte aligned");
  PD_REQUIRE_PTR(c->page_table);
  PD_REQUIRE_PTR(c->kv_len);
  if (c->new_rows && !aligned16(c->new_rows))
    return fail(PD_ERR_MISALIGNED, "pointer 'new_rows' is not 16-byte aligned");
  return PD_OK;
}

pd_status check_norm(float eps, double rope_base) {
  if (!std::isfinite(eps) || eps < 0.f) return fail(PD_ERR_BAD_DIMS, "eps must be finite and >= 0");
  if (!std::isfinite(rope_base) || rope_base < 0.0)
    return fail(PD_ERR_BAD_DIMS, "rope_base must be finite and >= 0 (0: no rotation)");
  return PD_OK;
}

pd_status check_stride(const char* name, int64_t stride, long long least, int elem) {
  if (stride < least || stride % (16 / elem) != 0 || stride > (1LL << 40))
    return fail(PD_ERR_BAD_DIMS, "%s=%lld must be at least %lld, a multiple of 16 bytes and at most 2^40", name,
                (long long)stride, least);
  return PD_OK;
}

pd::PagedArgs paged_args(const pd_paged_dims* d, const pd_paged_cache* c) {
  pd::PagedArgs a{};
  a.k_pages = c->k_pages;
  a.v_pages = c->v_pages;
  a.k_exp = c->k_exp;
  a.v_exp = c->v_exp;
  a.k_bounds = c->k_bounds;
  a.page_table = c->page_table;
  a.kv_len = c->kv_len;
  a.new_rows = c->new_rows;
  a.B = d->batch;
  a.Ln = d->new_len;
  a.Hq = d->n_heads_q;
  a.Hkv = d->n_heads_kv;
  a.G = a.Hq / a.Hkv;
  a.D = d->head_dim;
  a.R = d->page_rows;
  a.log2R = __builtin_ctz((unsigned)d->page_rows);
  a.n_pages = d->n_pages;
  a.max_pages = d->max_pages;
  a.causal = d->causal;
  a.bf16 = d->dtype == PD_BF16;
  a.fp8 = d->cache_dtype == PD_FP8_E4M3;
  a.fp4 = d->cache_dtype == PD_FP4_E2M1;
  const float scale = d->sm_scale > 0.f ? d->sm_scale : 1.0f / std::sqrt((float)d->head_dim);
  a.scale_log2 = scale * 1.4426950408889634f;
  return a;
}

// Pages that up to new_len consecutive rows can touch.
long long touched_pages(const pd_paged_dims* d) {
  return std::min<long long>(d->max_pages, (d->new_len + d->page_rows - 2) / d->page_rows + 1);
}

// --- attention: how the keys are cut, and the workspace of the parts -----------
struct AttnPlan {
  int row_blocks, part_rows, parts, max_chunks;
  long long grid;
  size_t o_bytes, ml_bytes, unit_bytes, total;
  bool planned;
};
// whole: the keys of a unit are not cut.
pd_status attn_plan(const pd_paged_dims* d, int top_k, long long most_keys, bool whole, AttnPlan* p) {
  const long long rows = (long long)(d->n_heads_q / d->n_heads_kv) * d->new_len;
  p->row_blocks = cdiv(rows, pd::kPagedRows);
  p->part_rows = (int)std::min<long long>(rows, pd::kPagedRows);
  const long long units = (long long)d->batch * d->n_heads_kv * p->row_blocks;
  const long long keys = std::min((long long)(top_k > 0 ? top_k : d->max_pages) * d->page_rows, most_keys);
  const long long blocks = cdiv(keys, pd::paged_block_keys(d->dtype == PD_FP32));
  if (units >= kMaxGrid / 2 || (double)units * (double)blocks >= 9e18)
    return fail(PD_ERR_BAD_DIMS, "attention of batch=%d with new_len=%d is too large for one launch", d->batch,
                d->new_len);
  p->parts = pd::paged_parts(rows);
  p->max_chunks = whole || blocks <= pd::paged_whole_blocks(units) ? 1 : (int)std::min<long long>(blocks, p->parts);
  // The kernels cut with a quota of at least all blocks / parts: at most so many whole
  // quotas, and one part that is not whole for each unit.
  p->grid = p->max_chunks == 1 ? units : std::min(units + p->parts, units * p->max_chunks);
  const size_t slots = p->max_chunks == 1 ? 0 : (size_t)p->grid * p->part_rows;
  p->o_bytes = round_up(slots * d->head_dim * sizeof(float));
  p->ml_bytes = round_up(slots * 2 * sizeof(float));
  p->unit_bytes = slots ? round_up((size_t)units * 4 * sizeof(int32_t)) : 0;
  p->planned = slots && d->batch > pd::kPlanBatch;
  p->total = p->o_bytes + p->ml_bytes + p->unit_bytes +
             (p->planned ? round_up((2 + 2 * (size_t)cdiv(d->batch, 64)) * sizeof(int32_t)) : 0);
  return PD_OK;
}

// What the kernels go by of the sizes alone.
pd::PagedArgs sizes_of(const pd_paged_dims* d) {
  const pd_paged_cache none{};
  return paged_args(d, &none);
}

size_t select_bytes(const pd_paged_dims* d) {
  const int shares = pd::page_score_shares(sizes_of(d));
  return round_up((size_t)d->batch * d->n_heads_kv * shares * d->max_pages * sizeof(double));
}

pd_status check_select_dims(const pd_paged_dims* d, int top_k) {
  if (d->max_pages > kMaxSelectPages)
    return fail(PD_ERR_BAD_DIMS, "max_pages=%d must be at most %d to select pages", d->max_pages, kMaxSelectPages);
  if (top_k < 1 || top_k > d->max_pages)
    return fail(PD_ERR_BAD_DIMS, "top_k=%d must be in 1..max_pages=%d", top_k, d->max_pages);
  if ((double)d->batch * d->n_heads_kv * d->max_pages * pd::page_score_shares(sizes_of(d)) >= (double)kMaxGrid)
    return fail(PD_ERR_BAD_DIMS, "selection of batch=%d over %d pages is too large for one launch", d->batch,
                d->max_pages);
  return PD_OK;
}

pd_status check_attn_pages(const pd_paged_dims* d, const int32_t* page_idx, int top_k) {
  if (page_idx ? (top_k < 1 || top_k > d->max_pages) : top_k != 0)
    return fail(PD_ERR_BAD_DIMS, "top_k=%d must be in 1..max_pages=%d with page_idx and 0 without", top_k,
                d->max_pages);
  if (page_idx && !aligned16(page_idx)) return fail(PD_ERR_MISALIGNED, "pointer 'page_idx' is not 16-byte aligned");
  return PD_OK;
}

struct Window {
  int window, n_sinks, keys;   // keys: of a row block, see PagedAttnArgs
  long long most_keys;         // of any
  int tile_rows;               // paged_tile_rows
};
pd_status check_window(int window, int n_sinks) {
  if (window < 1) return fail(PD_ERR_BAD_DIMS, "window=%d must be >= 1", window);
  if (n_sinks < 0) return fail(PD_ERR_BAD_DIMS, "n_sinks=%d must be >= 0", n_sinks);
  return PD_OK;
}
Window window_of(const pd_paged_dims* d, int window, int n_sinks) {
  // Beyond all positions and new rows a window or a count has no further effect.
  constexpr long long most = kMaxPositions + (1 << 24);
  Window w{};
  w.window = (int)std::min<long long>(window, most);
  w.n_sinks = (int)std::min<long long>(n_sinks, kMaxPositions);
  const int G = d->n_heads_q / d->n_heads_kv;
  const long long rows = std::min<long long>(d->new_len, (pd::kPagedRows + G - 1) / G + 1);   // new rows of a row block
  const long long keys = pd::paged_window_keys(w.window, w.n_sinks, d->causal ? rows : 0);
  w.keys = (int)std::min<long long>(keys, kMaxPositions);
  w.most_keys = w.keys + (d->causal ? 0 : (long long)d->new_len);
  // The tile kernel scales scores that it has masked with -inf: not where the scale may vanish in fp32.
  if (!(d->sm_scale > 0.f) || d->sm_scale >= 1e-30f)
    w.tile_rows = pd::paged_tile_rows(d->dtype == PD_BF16, (long long)d->batch * d->n_heads_kv, (long long)G * d->new_len, w.most_keys);
  return w;
}

pd_status launch_attn(const pd_paged_dims* d, const pd_paged_cache* cache, const void* q, const int32_t* page_idx,
                      int top_k, const Window* w, void* o, float* lse, void* workspace, size_t ws_bytes,
                      void* stream) {
  AttnPlan plan;
  PD_RETURN_IF(attn_plan(d, top_k, w ? w->most_keys : kMaxPositions, w && w->tile_rows, &plan));
  PD_RETURN_IF(check_ws(workspace, ws_bytes, plan.total));
  pd::PagedAttnArgs a{};
  a.c = paged_args(d, cache);
  a.q = q;
  a.page_idx = page_idx;
  a.top_k = top_k;
  if (w) {
    a.window = w->window;
    a.n_sinks = w->n_sinks;
    a.window_keys = w->keys;
  }
  a.o = o;
  a.lse = lse;
  a.o_part = (float*)workspace;
  a.ml_part = (float*)((char*)workspace + plan.o_bytes);
  a.unit = (int32_t*)((char*)workspace + plan.o_bytes + plan.ml_bytes);
  a.plan = plan.planned ? (int32_t*)((char*)workspace + plan.o_bytes + plan.ml_bytes + plan.unit_bytes) : nullptr;
  a.row_blocks = plan.row_blocks;
  a.part_rows = plan.part_rows;
  a.max_chunks = plan.max_chunks;
  a.per_part = 1.0f / plan.parts;
  a.places = (float)pd::paged_places(a.c.fp4, (long long)a.c.G * a.c.Ln);
  a.grid = plan.grid;
  a.by_group = pd::fast_div(a.c.G);
  a.by_heads = pd::fast_div(a.c.Hkv);
  a.by_rows = pd::fast_div(a.c.G * a.c.Ln);
  a.by_blocks = pd::fast_div(a.row_blocks);
  a.by_units = pd::fast_div(a.c.Hkv * a.row_blocks);
  if (w && w->tile_rows) return hip_status(pd::launch_paged_tile(a, w->tile_rows, (hipStream_t)stream), "paged attention kernel");
  return hip_status(pd::launch_paged_attn(a, (hipStream_t)stream), "paged attention kernels");
}

}  // namespace

extern "C" {

pd_status pd_qk_norm_rope(int32_t n_rows, int32_t n_heads_q, int32_t n_heads_kv, int32_t head_dim, int32_t dtype,
                          const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* w_q,
                          const void* w_k, float eps, const int32_t* pos, double rope_base, void* q_out,
                          int64_t q_out_stride, void* k_out, int64_t k_out_stride, void* stream) {
  if (n_rows < 0) return fail(PD_ERR_BAD_DIMS, "n_rows=%d must be >= 0", n_rows);
  if (n_heads_q < 0 || n_heads_kv < 0 || n_heads_q + (long long)n_heads_kv < 1 || n_heads_q > (1 << 16) ||
      n_heads_kv > (1 << 16))
    return fail(PD_ERR_BAD_DIMS, "head counts %d/%d must be in 0..65536 and not both 0", n_heads_q, n_heads_kv);
  if (head_dim != 64 && head_dim != 128) return fail(PD_ERR_UNSUPPORTED, "head_dim=%d must be 64 or 128", head_dim);
  if (dtype != PD_BF16 && dtype != PD_FP32)
    return fail(PD_ERR_UNSUPPORTED, "dtype=%d is neither PD_BF16 nor PD_FP32", dtype);
  PD_RETURN_IF(check_norm(eps, rope_base));
  // A wave takes at least two heads (fp32, d = 128).
  if ((double)n_rows * ((n_heads_q + (long long)n_heads_kv + 1) / 2) >= 2147483640.0)
    return fail(PD_ERR_BAD_DIMS, "n_rows=%d rows of %lld heads are too large for one launch", n_rows,
                n_heads_q + (long long)n_heads_kv);
  if (n_rows == 0) return ok();
  const int eb = dtype == PD_BF16 ? 2 : 4;
  if (n_heads_q > 0) {
    PD_REQUIRE_PTR(q);
    PD_REQUIRE_PTR(q_out);
    PD_RETURN_IF(check_stride("q_stride", q_stride, (long long)n_heads_q * head_dim, eb));
    PD_RETURN_IF(check_stride("q_out_stride", q_out_stride, (long long)n_heads_q * head_dim, eb));
  }
  if (n_heads_kv > 0) {
    PD_REQUIRE_PTR(k);
    PD_REQUIRE_PTR(k_out);
    PD_RETURN_IF(check_stride("k_stride", k_stride, (long long)n_heads_kv * head_dim, eb));
    PD_RETURN_IF(check_stride("k_out_stride", k_out_stride, (long long)n_heads_kv * head_dim, eb));
  }
  if (w_q && !aligned16(w_q)) return fail(PD_ERR_MISALIGNED, "pointer 'w_q' is not 16-byte aligned");
  if (w_k && !aligned16(w_k)) return fail(PD_ERR_MISALIGNED, "pointer 'w_k' is not 16-byte aligned");
  if (rope_base > 0.0) PD_REQUIRE_PTR(pos);
  pd::NormRopeArgs a{};
  a.x[0] = q;
  a.x[1] = k;
  a.y[0] = q_out;
  a.y[1] = k_out;
  a.w[0] = w_q;
  a.w[1] = w_k;
  a.xs[0] = q_stride;
  a.xs[1] = k_stride;
  a.ys[0] = q_out_stride;
  a.ys[1] = k_out_stride;
  a.pos = rope_base > 0.0 ? pos : nullptr;
  a.rows = n_rows;
  a.Hq = n_heads_q;
  a.Hkv = n_heads_kv;
  a.D = head_dim;
  a.eps = eps;
  a.log2_step = rope_base > 0.0 ? std::log2(rope_base) * 2.0 / head_dim : 0.0;
  a.bf16 = dtype == PD_BF16;
  return hip_status(pd::launch_qk_norm_rope(a, (hipStream_t)stream), "norm and rotation kernel");
}

pd_status pd_paged_append(const pd_paged_dims* d, const pd_paged_cache* cache, const void* k_new, int64_t k_stride,
                          const void* v_new, int64_t v_stride, void* stream) {
  PD_RETURN_IF(check_paged_dims(d));
  PD_RETURN_IF(check_cache(d, cache, true, false));
  PD_REQUIRE_PTR(k_new);
  PD_REQUIRE_PTR(v_new);
  const int eb = d->dtype == PD_BF16 ? 2 : 4;
  const long long row = (long long)d->n_heads_kv * d->head_dim;
  PD_RETURN_IF(check_stride("k_stride", k_stride, row, eb));
  PD_RETURN_IF(check_stride("v_stride", v_stride, row, eb));
  if ((double)d->batch * d->n_heads_kv * touched_pages(d) >= (double)kMaxGrid)
    return fail(PD_ERR_BAD_DIMS, "append of batch=%d with new_len=%d is too large for one launch", d->batch,
                d->new_len);
  pd::AppendArgs a{};
  a.c = paged_args(d, cache);
  a.k_new = k_new;
  a.v_new = v_new;
  a.ks = k_stride;
  a.vs = v_stride;
  a.pages = (int)touched_pages(d);
  a.by_heads = pd::fast_div(a.c.Hkv);
  a.by_pages = pd::fast_div(a.pages);
  return hip_status(pd::launch_paged_append(a, (hipStream_t)stream), "append kernel");
}

pd_status pd_paged_append_rope(const pd_paged_dims* d, const pd_paged_cache* cache, const void* q, int64_t q_stride,
                               const void* k_new, int64_t k_stride, const void* v_new, int64_t v_stride,
                               const void* w_q, const void* w_k, float eps, const int32_t* pos, double rope_base,
                               void* q_out, void* stream) {
  PD_RETURN_IF(check_paged_dims(d));
  PD_RETURN_IF(check_norm(eps, rope_base));
  PD_RETURN_IF(check_cache(d, cache, true, false));
  PD_REQUIRE_PTR(k_new);
  PD_REQUIRE_PTR(v_new);
  const int eb = d->dtype == PD_BF16 ? 2 : 4;
  const long long row = (long long)d->n_heads_kv * d->head_dim, q_row = (long long)d->n_heads_q * d->head_dim;
  if (q || q_out) {
    PD_REQUIRE_PTR(q);
    PD_REQUIRE_PTR(q_out);
    PD_RETURN_IF(check_stride("q_stride", q_stride, q_row, eb));
    if (q == q_out && q_stride != q_row)
      return fail(PD_ERR_BAD_DIMS, "q_out may be q only where its rows lie without gaps, q_stride=%lld", (long long)q_stride);
  }
  PD_RETURN_IF(check_stride("k_stride", k_stride, row, eb));
  PD_RETURN_IF(check_stride("v_stride", v_stride, row, eb));
  if (w_q && !aligned16(w_q)) return fail(PD_ERR_MISALIGNED, "pointer 'w_q' is not 16-byte aligned");
  if (w_k && !aligned16(w_k)) return fail(PD_ERR_MISALIGNED, "pointer 'w_k' is not 16-byte aligned");
  if (pos && !aligned16(pos)) return fail(PD_ERR_MISALIGNED, "pointer 'pos' is not 16-byte aligned");
  // A workgroup takes at least four of the heads of a page's rows.
  const long long chunks = ((q ? d->n_heads_q : 0) + 2LL * d->n_heads_kv + 3) / 4;
  if ((double)d->batch * (double)chunks * touched_pages(d) >= (double)kMaxGrid)
    return fail(PD_ERR_BAD_DIMS, "append of batch=%d with new_len=%d is too large for one launch", d->batch,
                d->new_len);
  pd::AppendRopeArgs a{};
  a.c = paged_args(d, cache);
  if (!q) a.c.Hq = 0;
  a.q = q;
  a.k = k_new;
  a.v = v_new;
  a.qs = q_stride;
  a.ks = k_stride;
  a.vs = v_stride;
  a.w_q = w_q;
  a.w_k = w_k;
  a.q_out = q_out;
  a.pos = pos;
  a.eps = eps;
  a.rotate = rope_base > 0.0;
  if (a.rotate) {
    const long double step = std::log2((long double)rope_base) * 2 / d->head_dim;
    a.step = (double)(float)step;
    a.step_rest = (double)(step - (long double)a.step);
  }
  a.pages = (int)touched_pages(d);
  return hip_status(pd::launch_paged_append_rope(a, (hipStream_t)stream), "append kernel with norms and rotation");
}

pd_status pd_paged_read(const pd_paged_dims* d, const pd_paged_cache* cache, int32_t first, int32_t n_rows,
                        void* k_out, void* v_out, void* stream) {
  PD_RETURN_IF(check_paged_dims(d));
  PD_RETURN_IF(check_cache(d, cache, true, false));
  if (first < 0 || n_rows < 1 || (long long)first + n_rows > (long long)d->max_pages * d->page_rows)
    return fail(PD_ERR_BAD_DIMS, "first=%d, n_rows=%d must lie within max_pages*page_rows=%lld", first, n_rows,
                (long long)d->max_pages * d->page_rows);
  PD_REQUIRE_PTR(k_out);
  PD_REQUIRE_PTR(v_out);
  if ((double)d->batch * d->n_heads_kv * cdiv(n_rows, 32) >= (double)kMaxGrid)
    return fail(PD_ERR_BAD_DIMS, "read-back of batch=%d with n_rows=%d is too large for one launch", d->batch, n_rows);
  pd::ReadArgs a{};
  a.c = paged_args(d, cache);
  a.k_out = k_out;
  a.v_out = v_out;
  a.first = first;
  a.n = n_rows;
  a.by_heads = pd::fast_div(a.c.Hkv);
  return hip_status(pd::launch_paged_read(a, (hipStream_t)stream), "read-back kernel");
}

pd_status pd_paged_select(const pd_paged_dims* d, const pd_paged_cache* cache, const void* q, int32_t top_k,
                          int32_t n_first, int32_t n_last, int32_t* page_idx, void* workspace, size_t ws_bytes,
                          void* stream) {
  PD_RETURN_IF(check_paged_dims(d));
  PD_RETURN_IF(check_select_dims(d, top_k));
  if (n_first < 0 || n_last < 0)
    return fail(PD_ERR_BAD_DIMS, "n_first=%d and n_last=%d must be >= 0", n_first, n_last);
  PD_RETURN_IF(check_cache(d, cache, false, true));
  PD_REQUIRE_PTR(q);
  PD_REQUIRE_PTR(page_idx);
  PD_RETURN_IF(check_ws(workspace, ws_bytes, select_bytes(d)));
  pd::PageSelectArgs a{};
  a.c = paged_args(d, cache);
  a.q = q;
  a.top_k = top_k;
  a.n_first = n_first;
  a.n_last = n_last;
  a.page_idx = page_idx;
  a.score = (double*)workspace;
  a.by_group = pd::fast_div(a.c.G);
  a.by_heads = pd::fast_div(a.c.Hkv);
  a.shares = pd::page_score_shares(a.c);
  a.by_blocks = pd::fast_div(pd::page_score_blocks(a.c));
  a.by_shares = pd::fast_div(a.shares);
  return hip_status(pd::launch_paged_select(a, (hipStream_t)stream), "page selection kernels");
}

pd_status pd_paged_attn(const pd_paged_dims* d, const pd_paged_cache* cache, const void* q, const int32_t* page_idx,
                        int32_t top_k, void* o, float* lse, void* workspace, size_t ws_bytes, void* stream) {
  PD_RETURN_IF(check_paged_dims(d));
  PD_RETURN_IF(check_cache(d, cache, true, false));
  PD_RETURN_IF(check_attn_pages(d, page_idx, top_k));
  PD_REQUIRE_PTR(q);
  PD_REQUIRE_PTR(o);
  if (lse && !aligned16(lse)) return fail(PD_ERR_MISALIGNED, "pointer 'lse' is not 16-byte aligned");
  return launch_attn(d, cache, q, page_idx, top_k, nullptr, o, lse, workspace, ws_bytes, stream);
}

pd_status pd_paged_window_attn(const pd_paged_dims* d, const pd_paged_cache* cache, const void* q, int32_t window,
                               int32_t n_sinks, void* o, float* lse, void* workspace, size_t ws_bytes, void* stream) {
  PD_RETURN_IF(check_paged_dims(d));
  PD_RETURN_IF(check_window(window, n_sinks));
  PD_RETURN_IF(check_cache(d, cache, true, false));
  PD_REQUIRE_PTR(q);
  PD_REQUIRE_PTR(o);
  if (lse && !aligned16(lse)) return fail(PD_ERR_MISALIGNED, "pointer 'lse' is not 16-byte aligned");
  const Window w = window_of(d, window, n_sinks);
  return launch_attn(d, cache, q, nullptr, 0, &w, o, lse, workspace, ws_bytes, stream);
}
size_t pd_paged_workspace_bytes(const pd_paged_dims* d, int32_t top_k, int32_t which) {
  if (check_paged_dims(d) != PD_OK || top_k < 0 || top_k > d->max_pages) return 0;
  if (which == 0) return check_select_dims(d, top_k) == PD_OK ? select_bytes(d) : 0;
  if (which != 1) return 0;
  AttnPlan plan;
  return attn_plan(d, top_k, kMaxPositions, false, &plan) == PD_OK ? plan.total : 0;
}

size_t pd_paged_window_workspace_bytes(const pd_paged_dims* d, int32_t window, int32_t n_sinks) {
  if (check_paged_dims(d) != PD_OK || check_window(window, n_sinks) != PD_OK) return 0;
  AttnPlan plan;
  const Window w = window_of(d, window, n_sinks);
  return attn_plan(d, 0, w.most_keys, w.tile_rows > 0, &plan) == PD_OK ? plan.total : 0;
}

}  // extern "C"
