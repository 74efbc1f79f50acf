// C ABI of rotated appends, the 8-bit KV cache and attention over a window:
// argument validation, planning and launches.  As in api.cpp the plans travel
// in the kernel arguments; nothing is uploaded or synchronised.
#include "plan_common.h"
#include "window_internal.h"

namespace {

using namespace rg;

rg_status validate_rotation(const rg_attn_layout* L, const rg_rotation* R) {
  if (R == nullptr) return RG_OK;
  if (R->dims < 0 || R->dims > L->head_dim || R->dims % 16) return RG_ERR_SHAPE;
  if (R->dims > 0 && !R->inv_freq) return RG_ERR_NULL;
  if ((R->inv_freq && !aligned(R->inv_freq, 4)) || (R->positions && !aligned(R->positions, 4))) return RG_ERR_UNSUPPORTED;
  return RG_OK;
}

// Rows of `width` elements, `stride` apart.
rg_status validate_rows(const void* rows, int64_t stride, int64_t width) {
  if (stride < width) return RG_ERR_SHAPE;
  return stride % 8 || !aligned(rows, 16) ? RG_ERR_UNSUPPORTED : RG_OK;
}

// Pages that the rows of request r touch.
int64_t touched_pages(const rg_attn_layout* L, int r) {
  const int64_t n = L->q_indptr[r + 1] - L->q_indptr[r];
  return n == 0 ? 0 : (L->ctx_len[r] + n - 1) / kPageSize - L->ctx_len[r] / kPageSize + 1;
}
int64_t touched_pages(const rg_attn_layout* L) {
  int64_t pages = 0;
  for (int r = 0; r < L->num_requests; ++r) pages += touched_pages(L, r);
  return pages;
}

// Launches over the touched pages, `each` items a page.
template <typename Launch>
rg_status launch_pages(const rg_attn_layout* L, int64_t each, Launch launch) {
  auto items = [&](int r) { return touched_pages(L, r) * each; };
  if (L->num_requests > kMaxReqPerLaunch) {
    const rg_status fits = check_plans(L, kAppendThreads, items);
    if (fits != RG_OK) return fits;
  }
  return each_plan(L, kAppendThreads, items, launch);
}

rg_status run_append(const rg_attn_layout* L, const rg_rotation* R, const uint16_t* q, int64_t q_stride, uint16_t* q_out,
                     const uint16_t* k, int64_t k_stride, const uint16_t* v, int64_t v_stride, uint16_t* k_cache,
                     uint16_t* v_cache, uint8_t* cache, float* scales, bool kv8, void* stream) {
  rg_status st = validate_layout(L);
  if (st != RG_OK) return st;
  if (!k || !v || (kv8 ? !cache || !scales : !k_cache || !v_cache) || !q != !q_out) return RG_ERR_NULL;
  st = validate_rotation(L, R);
  if (st != RG_OK) return st;
  const int64_t width = (int64_t)L->num_kv_heads * L->head_dim, q_width = (int64_t)L->num_q_heads * L->head_dim;
  st = validate_rows(k, k_stride, width);
  if (st == RG_OK) st = validate_rows(v, v_stride, width);
  if (st == RG_OK && q) st = validate_rows(q, q_stride, q_width);
  if (st != RG_OK) return st;
  if (q && q == q_out && q_stride != q_width) return RG_ERR_SHAPE;
  if (!aligned(q_out, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(cache, 16) ||
      !aligned(scales, 4) || !aligned(L->page_indices, 4))
    return RG_ERR_UNSUPPORTED;
  AppendArgs a;
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_out = q_out;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.k_cache = k_cache;
  a.v_cache = v_cache;
  a.cache = cache;
  a.scales = scales;
  a.page_indices = L->page_indices;
  a.positions = R ? R->positions : nullptr;
  a.inv_freq = R ? R->inv_freq : nullptr;
  a.hq = L->num_q_heads;
  a.hkv = L->num_kv_heads;
  a.dims = R ? R->dims : 0;
  a.interleaved = R && R->interleaved ? 1 : 0;
  // Where there are pages enough a work group takes all heads of one, and makes
  // its angles once.
  const bool many = touched_pages(L) > 1024;
  const int kv_heads = many ? L->num_kv_heads : 1, q_heads = many ? L->num_q_heads : std::min(L->num_q_heads, 8);
  const int64_t each = (L->num_kv_heads + kv_heads - 1) / kv_heads + (q ? (L->num_q_heads + q_heads - 1) / q_heads : 0);
  return launch_pages(L, each, [&](AttnPlan& p) {
    p.chunk = kv_heads;
    p.cols_per_group = q ? q_heads : 0;
    return launch_append(a, p, L->head_dim, kv8, static_cast<hipStream_t>(stream));
  });
}

}  // namespace

extern "C" {

rg_status rg_kv_append(const rg_attn_layout* layout, const rg_rotation* rotation, const uint16_t* q, int64_t q_stride,
                       uint16_t* q_out, const uint16_t* k, int64_t k_stride, const uint16_t* v, int64_t v_stride,
                       uint16_t* k_cache, uint16_t* v_cache, void* stream) {
  return run_append(layout, rotation, q, q_stride, q_out, k, k_stride, v, v_stride, k_cache, v_cache, nullptr, nullptr,
                    false, stream);
}

rg_status rg_kv8_append(const rg_attn_layout* layout, const rg_rotation* rotation, const uint16_t* q, int64_t q_stride,
                        uint16_t* q_out, const uint16_t* k, int64_t k_stride, const uint16_t* v, int64_t v_stride,
                        uint8_t* cache, float* scales, void* stream) {
  return run_append(layout, rotation, q, q_stride, q_out, k, k_stride, v, v_stride, nullptr, nullptr, cache, scales, true,
                    stream);
}

rg_status rg_kv8_read(const rg_attn_layout* layout, const uint8_t* cache, const float* scales, uint16_t* k,
                      int64_t k_stride, uint16_t* v, int64_t v_stride, void* stream) {
  rg_status st = validate_layout(layout);
  if (st != RG_OK) return st;
  if (!k || !v || !cache || !scales) return RG_ERR_NULL;
  const int64_t width = (int64_t)layout->num_kv_heads * layout->head_dim;
  st = validate_rows(k, k_stride, width);
  if (st == RG_OK) st = validate_rows(v, v_stride, width);
  if (st != RG_OK) return st;
  if (!aligned(cache, 16) || !aligned(scales, 4) || !aligned(layout->page_indices, 4)) return RG_ERR_UNSUPPORTED;
  Kv8ReadArgs a;
  a.cache = cache;
  a.scales = scales;
  a.k = k;
  a.v = v;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.page_indices = layout->page_indices;
  a.hkv = layout->num_kv_heads;
  const int heads = touched_pages(layout) > 1024 ? layout->num_kv_heads : 1;
  return launch_pages(layout, (layout->num_kv_heads + heads - 1) / heads, [&](AttnPlan& p) {
    p.chunk = heads;
    return launch_kv8_read(a, p, layout->head_dim, static_cast<hipStream_t>(stream));
  });
}

}  // extern "C"
