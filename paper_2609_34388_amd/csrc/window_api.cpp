// C ABI of rotated appends, the 8-bit KV cache and attention over a window:
// argument validation, planning and launches.  As in api.cpp the plans travel
// in the kernel arguments; nothing is uploaded or synchronised.
#include <new>
#include <numeric>
#include <vector>

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
  // Heads of q in an item, whose rows at 4 of D = 128 or 8 of D = 64 weigh what those of
  // its KV heads do.  At D = 128 eight in few pages, where angles and starts count, and in
  // 8 bits (us with 4, 8 and 16 heads of 32: 128 requests' steps 12.6, 11.7, 13.2, 256
  // pages of a prompt 20.5, 18.7, 18.6, 512 pages 40.7, 42.8, 46.4, 2307 168, 172, 180; in
  // 8 bits 64 steps 17.0, 16.9, 17.2, 2048 pages 173, 176, 184; D = 64 28.7, 29.2, 40.3, in
  // 8 bits 48.4, 47.3, 59.7).
  const bool many = touched_pages(L) >= 512;
  const int q_heads = std::min(L->num_q_heads, L->head_dim == 128 && !kv8 && many ? 4 : 8), kv_heads = append_heads(L->head_dim);
  const int64_t each = (L->num_kv_heads + kv_heads - 1) / kv_heads + (q ? (L->num_q_heads + q_heads - 1) / q_heads : 0);
  return launch_pages(L, each, [&](AttnPlan& p) {
    p.cols_per_group = q ? q_heads : 0;
    return launch_append(a, p, L->head_dim, kv8, static_cast<hipStream_t>(stream));
  });
}

// ---------------------------------------------------------------------------
template <typename Plan>
struct FullPlan {
  std::vector<Plan> launches;
  size_t ml_offset = 0, ws_bytes = 0;
};

// Limits of the window; without one, all keys.
struct Limits {
  int size, sink;
};
constexpr int kAllKeys = 1 << 30;
Limits limits_of(const rg_window* W) {
  if (W == nullptr) return {kAllKeys, 0};
  return {std::min(W->size, kAllKeys), std::min(W->sink, kAllKeys)};
}
rg_status validate_window(const rg_window* W) {
  return W != nullptr && (W->size < 1 || W->sink < 0) ? RG_ERR_SHAPE : RG_OK;
}

// Hundredths of a microsecond, as below.  In one, two and three rounds 40 long requests
// take 718, 566 and 568 us; rounds of less than 80 us are best left one (102, 110, 122;
// 34, 42, 48), and among longer ones those that fill it evenly (184, 195, 198).
constexpr int64_t kLongRound = 8000;
// A merge's launch, and what it takes for each run: not for what a split saves below that.
// 100 tokens over 500 keys of D = 64 whole 15.9 us, split to fill the chip 21.1; in 8 bits
// 11.5 and 16.7.  5 requests of 17 to 29 rows over 600 to 4900 keys (D = 64, 8 bits) in 608
// items of one step 24.7, in half as many 21.6.
constexpr int64_t kMerge = 450, kMergeRun = 16;
// How a kernel takes a batch: column groups of up to `group` tiles, dealt evenly or
// full but for the last; steps of `keys` keys; work groups that run at once; the time of
// a step of so many tiles, of an item's start and end, and of its partials where it is one
// of several runs, a part for each and one for each 32 columns of D = 128, in hundredths
// of a microsecond; and the least that a step takes where few items run, which share bytes
// and SIMDs with fewer, in percent.
//
// A step of a work group with every place taken, for 1 to 4 tiles: in bf16 2.75, 2.77, 2.89
// and 3.22 us, and of D = 64 (96 keys) 3.14, 3.28, 3.61 and 4.02; in 8 bits 2.78, 2.90,
// 4.60 and 4.82, and of D = 64 2.11, 2.63, 4.38 and 4.49.  The constants do not know D: in
// bf16 they are those of D = 128; in 8 bits they are fitted, a third to a half of what was
// measured, the best of a sweep over batches of all sizes, where work groups seldom start
// together.  Partials: 90 requests of 5 to 45 rows over 2945 keys 247
// us; with 2 us for them in all, and so split, 286.  Few items: 48 requests of 8 to 63 rows
// over 701 keys (D = 64, 8 bits) whole in a third of the places 22.1 us, split to fill them,
// as with 90 or 100 percent, 27.5; with 60 a longer batch takes 102 us against 83.
struct Shape {
  int group, keys, per_cu;
  bool even;
  int64_t (*step)(int64_t tiles);
  int64_t start, parts, part_tile, least, alone;
};
Shape kv8_shape(int head_dim) {
  return {kKv8Waves, kKv8Step, head_dim == 64 ? 3 : 2, false, [](int64_t tiles) -> int64_t {
            constexpr int64_t t[] = {0, 6, 9, 16, 16};
            return 16 * t[tiles];
          }, 600, 300, 100, 128, 80};
}
Shape bf16_shape(int head_dim) {
  return {kWindowWaves, window_keys(head_dim), head_dim == 64 ? 3 : 2, true, [](int64_t tiles) { return std::max<int64_t>(270, 130 + 47 * tiles); },
          600, 200, 200, 270, 60};
}

// A request's column groups.
struct Groups {
  int64_t count = 0, tiles = 0, per = 0;  // groups, tiles in all, tiles of a group at most
  int64_t steps = 0, cols = 0;            // of the longest, and columns of a group at most
};
template <bool BR>
Groups groups_of(const rg_attn_layout* L, int r, Limits w, const Shape& shape, int g) {
  Groups q;
  const int n = L->q_indptr[r + 1] - L->q_indptr[r];
  if (n == 0) return q;
  q.tiles = ((int64_t)n * g + 31) / 32;
  q.count = 1;
  q.per = q.tiles;
  int keys = 0;
  if (q.tiles <= shape.group) {
    keys = window_span<BR>(L->ctx_len[r], L->n_verify[r], n, 0, n, w.size, w.sink).keys;
  } else {
    q.count = (q.tiles + shape.group - 1) / shape.group;
    q.per = shape.even ? (q.tiles + q.count - 1) / q.count : shape.group;
    q.count = (q.tiles + q.per - 1) / q.per;
    for (int64_t k = 0; k < q.count; ++k) {
      const int64_t c0 = k * q.per * 32, c1 = std::min((int64_t)n * g, (k + 1) * q.per * 32);
      const WindowSpan s = window_span<BR>(L->ctx_len[r], L->n_verify[r], n, (int)(c0 / g), (int)((c1 - 1) / g) + 1, w.size, w.sink);
      keys = std::max(keys, s.keys);
    }
  }
  q.steps = (keys + shape.keys - 1) / shape.keys;
  q.cols = std::min<int64_t>((int64_t)n * g, q.per * 32);
  return q;
}

template <typename Plan, int MaxReq>
rg_status plan_window(const rg_attn_layout* L, const rg_branch_layout* B, Limits w, bool kv8, FullPlan<Plan>& fp) {
  constexpr bool BR = __is_same(Plan, WindowPlanBr);
  const int R = L->num_requests, hkv = L->num_kv_heads, cus = device_cus();
  const Shape shape = kv8 ? kv8_shape(L->head_dim) : bf16_shape(L->head_dim);
  for (int r = 0; r < R; ++r)  // columns of a request: 32 bits
    if ((int64_t)(L->q_indptr[r + 1] - L->q_indptr[r]) * (L->num_q_heads / hkv) >= int64_t(1) << 30) return RG_ERR_UNSUPPORTED;
  std::vector<Groups> groups(R);
  for (int r = 0; r < R; ++r) groups[r] = groups_of<BR>(L, r, w, shape, L->num_q_heads / hkv);
  auto runs_of = [&](const Groups& q, int64_t target) {
    // in 32 bits, whose divisions are the faster
    const uint32_t steps = (uint32_t)q.steps, step = (uint32_t)shape.step(q.per);
    const uint32_t most = std::min<uint32_t>(kMaxRunSteps, std::max(1u, (uint32_t)std::min<int64_t>(target, UINT32_MAX) / step));
    if (most >= steps) return (int64_t)1;
    const uint32_t n = (steps + most - 1) / most, each = (steps + n - 1) / n;  // steps of a run
    return (int64_t)((steps + each - 1) / each);
  };
  // Cost of an item at most: of no split, of one round of items or 0.7 of one, and
  // where a round is long (kLongRound) of more, what promises the earliest end: a long
  // round ends unevenly, an item's start, its partials and their merge cost.
  struct Load {
    Groups q;
    int64_t items;  // whole
  };
  std::vector<Load> loads;  // those alike together: a batch has few kinds
  int64_t work = 0, whole = 0, whole_cost = 0;
  for (const Groups& q : groups) {
    if (q.count == 0) continue;
    work += q.count * hkv * q.steps * shape.step(q.per);
    whole += q.count * hkv;
    whole_cost = std::max(whole_cost, q.steps * shape.step(q.per));
    auto same = std::find_if(loads.begin(), loads.end(), [&](const Load& x) { return x.q.steps == q.steps && x.q.cols == q.cols; });
    if (same == loads.end()) loads.push_back({q, q.count * hkv});
    else same->items += q.count * hkv;
  }
  // Places of all launches, which run one after the other.
  const int64_t slots = (int64_t)cus * shape.per_cu * std::max(R, MaxReq) / MaxReq;
  auto items_of = [&](int64_t target) {
    int64_t items = 0;
    for (const Load& x : loads) items += x.items * runs_of(x.q, target);
    return items;
  };
  auto fit = [&](int64_t room) {  // the least for so many items, to 3 %
    if (whole >= room) return whole_cost;
    int64_t lo = std::max<int64_t>(shape.least, work / room), hi = std::max(lo, whole_cost);
    if (items_of(lo) <= room) return lo;
    while (hi - lo > 1 + lo / 32) {
      const int64_t mid = (lo + hi) / 2;
      if (items_of(mid) <= room) hi = mid;
      else lo = mid;
    }
    return hi;
  };
  auto time_of = [&](int64_t target) {
    const int64_t items = items_of(target), share = std::min<int64_t>(100, std::max(shape.alone, 100 * items / slots));
    int64_t longest = 0, total = 0, most_runs = 0;
    for (const Load& x : loads) {
      const int64_t n = runs_of(x.q, target), steps = (x.q.steps + n - 1) / n;
      int64_t each = steps * shape.step(x.q.per) * share / 100 + shape.start;
      if (n > 1) each += shape.parts + shape.part_tile * x.q.cols * L->head_dim / (32 * 128);
      total += x.items * n * each;
      longest = std::max(longest, each);
      most_runs = std::max(most_runs, n);
    }
    const int64_t end = items <= slots ? longest : std::max(longest, total / slots + total / items / 2);
    return end + (items > whole ? kMerge + kMergeRun * most_runs : 0);
  };
  int64_t target = whole_cost, best = time_of(target);
  auto consider = [&](int64_t t) {
    const int64_t time = time_of(t);
    if (time < best) {
      target = t;
      best = time;
    }
  };
  const int64_t one_round = fit(slots);
  consider(one_round);
  if (whole < slots) consider(fit(slots * 7 / 10));
  if (one_round > kLongRound)
    for (int64_t rounds = 2; rounds <= 4; ++rounds) consider(fit(rounds * slots));
  // Costliest work items first.
  std::vector<int> order(R);
  std::iota(order.begin(), order.end(), 0);
  std::vector<int64_t> cost(R, 0);
  std::vector<int32_t> runs(R, 0), each(R, 0);  // of a request, and steps of one
  for (int r = 0; r < R; ++r) {
    const Groups& q = groups[r];
    if (q.count == 0) continue;
    runs[r] = (int32_t)runs_of(q, target);
    each[r] = (int32_t)((q.steps + runs[r] - 1) / runs[r]);
    cost[r] = each[r] * shape.step(q.per);
  }
  std::stable_sort(order.begin(), order.end(), [&](int x, int y) { return cost[x] > cost[y]; });
  int64_t most_part = 0;
  for (int r0 = 0; r0 < R; r0 += MaxReq) {
    Plan p;
    std::memset(&p, 0, sizeof(p));
    p.num_req = std::min(MaxReq, R - r0);
    int64_t items = 0, part = 0, comb = 0;
    for (int k = 0; k < p.num_req; ++k) {
      const int r = order[r0 + k];
      const Groups& q = groups[r];
      auto& x = p.req[k];
      if constexpr (BR) pack_branches(B, r, x.br, x.rep);
      x.q_start = L->q_indptr[r];
      x.ctx = L->ctx_len[r];
      x.nv = (int32_t)((uint32_t)(L->q_indptr[r + 1] - L->q_indptr[r]) | ((uint32_t)L->n_verify[r] << 16));
      x.page_start = L->page_indptr[r];
      x.item_start = (int32_t)items;
      x.part_start = (int32_t)part;
      if (q.count == 0) continue;
      const int64_t nch = runs[r];
      if (nch > 0xffff) return RG_ERR_UNSUPPORTED;  // packed in 16 bits
      x.runs = (uint32_t)nch | (uint32_t)each[r] << 16;
      items += hkv * q.count * nch;
      if (nch > 1) {
        p.max_chunks = std::max(p.max_chunks, (int32_t)nch);
        part += hkv * nch * q.tiles;
        comb += hkv * q.tiles * (L->head_dim / 8);
      }
      if (items > INT32_MAX / 2 || part > INT32_MAX / 64 || comb > INT32_MAX / 2) return RG_ERR_UNSUPPORTED;
    }
    p.req[p.num_req].item_start = p.total_items = (int32_t)items;
    p.req[p.num_req].part_start = (int32_t)part;
    p.total_comb = (int32_t)comb;
    if (!fits_launch(items, 64 * shape.group) || !fits_launch(comb, 64 * kWindowMergeWaves)) return RG_ERR_UNSUPPORTED;
    most_part = std::max(most_part, part);
    if (items > 0) fp.launches.push_back(p);
  }
  fp.ml_offset = align256((size_t)most_part * 32 * L->head_dim * sizeof(float));
  fp.ws_bytes = most_part ? fp.ml_offset + align256((size_t)most_part * 32 * 2 * sizeof(float)) : 0;
  return RG_OK;
}

// Calls f(plan) with the plan of a layout and its branches (or NULL).
template <typename F>
rg_status with_window_plan(const rg_attn_layout* L, const rg_branch_layout* B, const rg_window* W, bool kv8, F f) try {
  rg_status st = validate_layout(L);
  if (st == RG_OK) st = validate_window(W);
  if (st != RG_OK) return st;
  if (B == nullptr) {
    FullPlan<WindowPlan> fp;
    st = plan_window<WindowPlan, kMaxReqPerLaunch>(L, nullptr, limits_of(W), kv8, fp);
    return st != RG_OK ? st : f(fp);
  }
  st = validate_branches(L, B);
  if (st != RG_OK) return st;
  FullPlan<WindowPlanBr> fp;
  st = plan_window<WindowPlanBr, kMaxReqPerLaunchBr>(L, B, limits_of(W), kv8, fp);
  return st != RG_OK ? st : f(fp);
} catch (const std::bad_alloc&) {  // nothing is launched before a plan is whole
  return RG_ERR_WORKSPACE;
}

rg_status query_workspace(const rg_attn_layout* L, const rg_branch_layout* B, const rg_window* W, bool kv8, size_t* bytes) {
  if (bytes == nullptr) return RG_ERR_NULL;
  return with_window_plan(L, B, W, kv8, [&](const auto& fp) {
    *bytes = fp.ws_bytes;
    return RG_OK;
  });
}

rg_status run_attention(const rg_attn_layout* L, const rg_branch_layout* B, const rg_window* W, const uint16_t* q,
                        const void* k_cache, const void* v_cache, const float* scales, bool kv8, uint16_t* out, float* lse,
                        void* ws, size_t ws_bytes, void* stream) {
  return with_window_plan(L, B, W, kv8, [&](const auto& fp) -> rg_status {
    if (!q || !k_cache || !out || (kv8 ? !scales : !v_cache)) return RG_ERR_NULL;
    if (!aligned(q, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(scales, 4) || !aligned(out, 16) ||
        !aligned(lse, 4) || !aligned(L->page_indices, 4))
      return RG_ERR_UNSUPPORTED;
    if (fp.ws_bytes > 0 && (ws == nullptr || ws_bytes < fp.ws_bytes || !aligned(ws, 16))) return RG_ERR_WORKSPACE;
    WindowArgs a;
    a.q = q;
    a.k_cache = static_cast<const uint8_t*>(k_cache);
    a.v_cache = static_cast<const uint8_t*>(v_cache);
    a.scales = scales;
    a.out = out;
    a.lse = lse;
    a.page_indices = L->page_indices;
    a.part_o = fp.ws_bytes ? static_cast<float*>(ws) : nullptr;
    a.part_ml = fp.ws_bytes ? reinterpret_cast<float*>(static_cast<char*>(ws) + fp.ml_offset) : nullptr;
    a.hq = L->num_q_heads;
    a.hkv = L->num_kv_heads;
    a.g = a.hq / a.hkv;
    set_divisor(a.g, a.g_mul, a.g_shift);
    set_divisor(a.hkv, a.hkv_mul, a.hkv_shift);
    const Limits w = limits_of(W);
    a.size = w.size;
    a.sink = w.sink;
    a.sm_scale = softmax_scale(L);
    a.scale_log2 = a.sm_scale * 1.4426950408889634f;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    for (const auto& p : fp.launches)
      if ((kv8 ? launch_kv8_attention(a, p, L->head_dim, s) : launch_window_attention(a, p, L->head_dim, s)) !=
          hipSuccess)
        return RG_ERR_HIP;
    return RG_OK;
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
  const int heads = kv8_read_heads(layout->head_dim);
  return launch_pages(layout, (layout->num_kv_heads + heads - 1) / heads, [&](const AttnPlan& p) {
    return launch_kv8_read(a, p, layout->head_dim, static_cast<hipStream_t>(stream));
  });
}

rg_status rg_kv8_attention_workspace(const rg_attn_layout* layout, const rg_branch_layout* branches,
                                     const rg_window* window, size_t* bytes) {
  return query_workspace(layout, branches, window, true, bytes);
}

rg_status rg_kv8_attention(const rg_attn_layout* layout, const rg_branch_layout* branches, const rg_window* window,
                           const uint16_t* q, const uint8_t* cache, const float* scales, uint16_t* out, float* lse, void* ws,
                           size_t ws_bytes, void* stream) {
  return run_attention(layout, branches, window, q, cache, nullptr, scales, true, out, lse, ws, ws_bytes, stream);
}

rg_status rg_window_attention_workspace(const rg_attn_layout* layout, const rg_branch_layout* branches,
                                        const rg_window* window, size_t* bytes) {
  if (bytes == nullptr || window == nullptr) return RG_ERR_NULL;
  return query_workspace(layout, branches, window, false, bytes);
}

rg_status rg_window_attention(const rg_attn_layout* layout, const rg_branch_layout* branches, const rg_window* window,
                              const uint16_t* q, const uint16_t* k_cache, const uint16_t* v_cache, uint16_t* out, float* lse,
                              void* ws, size_t ws_bytes, void* stream) {
  if (window == nullptr) return RG_ERR_NULL;
  return run_attention(layout, branches, window, q, k_cache, v_cache, nullptr, false, out, lse, ws, ws_bytes, stream);
}

}  // extern "C"
