// C ABI of the 4-bit KV cache, the attention mass and the eviction of tokens:
// argument validation, planning and launches.  As in api.cpp the plans travel
// in the kernel arguments; nothing is uploaded or synchronised.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <numeric>
#include <vector>

#include "cache_internal.h"
#include "plan_common.h"

namespace {

using namespace rg;

// Calls launch(plan) for a layout's requests, in order, a plan's worth at a
// time; items(r) is request r's number of work items (0: left out).
template <typename Items, typename Launch>
rg_status each_plan(const rg_attn_layout* L, int threads, Items items, Launch launch) {
  AttnPlan p;
  for (int r0 = 0; r0 < L->num_requests; r0 += kMaxReqPerLaunch) {
    const int cnt = std::min(kMaxReqPerLaunch, L->num_requests - r0);
    std::memset(&p, 0, sizeof(p));
    p.num_req = cnt;
    int64_t total = 0;
    for (int k = 0; k < cnt; ++k) {
      const int r = r0 + k;
      AttnReq& q = p.req[k];
      q.q_start = L->q_indptr[r];
      q.ctx = L->ctx_len[r];
      q.nv = (int32_t)((uint32_t)(L->q_indptr[r + 1] - L->q_indptr[r]) | ((uint32_t)L->n_verify[r] << 16));
      q.page_start = L->page_indptr[r];
      q.item_start = (int32_t)total;
      q.part_start = r;
      total += items(r);
      if (total > INT32_MAX / 2 || !fits_launch(total, threads)) return RG_ERR_UNSUPPORTED;
    }
    p.req[cnt].item_start = p.total_items = (int32_t)total;
    if (total > 0 && launch(p) != hipSuccess) return RG_ERR_HIP;
  }
  return RG_OK;
}
// Whether every plan can be launched: asked before the first launch wherever a
// later plan could refuse.
template <typename Items>
rg_status check_plans(const rg_attn_layout* L, int threads, Items items) {
  return each_plan(L, threads, items, [](const AttnPlan&) { return hipSuccess; });
}

// ---------------------------------------------------------------------------
// Blocks from which on a work item takes kRowHeads of them: 1400 blocks take
// 6.6 us in and 5.1 out one by one, 7.4 and 4.7 in fours; 217 thousand take 483 us
// out one by one, 409 in fours, 413 in eights.
constexpr int64_t kRowBlocks = 4096;
rg_status run_rows(const rg_attn_layout* L, const uint16_t* k, int64_t k_stride, const uint16_t* v, int64_t v_stride,
                   const uint8_t* cache, bool append, void* stream) {
  const rg_status st = validate_layout(L);
  if (st != RG_OK) return st;
  if (!k || !v || !cache) return RG_ERR_NULL;
  const int64_t width = (int64_t)L->num_kv_heads * L->head_dim;
  if (k_stride < width || v_stride < width) return RG_ERR_SHAPE;
  if (k_stride % 8 || v_stride % 8 || !aligned(k, 16) || !aligned(v, 16) || !aligned(cache, 16) ||
      !aligned(L->page_indices, 4))
    return RG_ERR_UNSUPPORTED;
  Kv4RowArgs a;
  a.k = const_cast<uint16_t*>(k);
  a.v = const_cast<uint16_t*>(v);
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.cache = const_cast<uint8_t*>(cache);
  a.page_indices = L->page_indices;
  a.hkv = L->num_kv_heads;
  auto pages = [&](int r) -> int64_t {
    const int64_t n = L->q_indptr[r + 1] - L->q_indptr[r];
    return n == 0 ? 0 : (L->ctx_len[r] + n - 1) / kPageSize - L->ctx_len[r] / kPageSize + 1;
  };
  int64_t blocks = 0;
  for (int r = 0; r < L->num_requests; ++r) blocks += pages(r) * L->num_kv_heads;
  const int heads = blocks > kRowBlocks ? kRowHeads : 1;
  auto items = [&](int r) { return pages(r) * ((L->num_kv_heads + heads - 1) / heads); };
  if (L->num_requests > kMaxReqPerLaunch) {
    const rg_status fits = check_plans(L, 256, items);
    if (fits != RG_OK) return fits;
  }
  return each_plan(L, 256, items, [&](AttnPlan& p) {
    p.chunk = heads;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    return append ? launch_kv4_append(a, p, L->head_dim, s) : launch_kv4_read(a, p, L->head_dim, s);
  });
}

// ---------------------------------------------------------------------------
template <typename Plan>
struct Kv4Plan {
  std::vector<Plan> launches;
  int64_t max_partial_cols = 0;
  size_t ml_offset = 0, ws_bytes = 0;
};

// Column groups of a request: `full` of four tiles, then one of `rest` tiles
// unless that is 0.
struct Kv4Cols {
  int64_t full;
  int rest;
};
Kv4Cols kv4_cols(const rg_attn_layout* L, int r) {
  const int64_t M = (int64_t)(L->q_indptr[r + 1] - L->q_indptr[r]) * (L->num_q_heads / L->num_kv_heads);
  const int64_t tiles = (M + 31) / 32;
  return {tiles / kKv4Waves, (int)(tiles % kKv4Waves)};
}

// Units (kv4_rate) of a work item at most: the least that gives one round of
// items on the compute units (two work groups each, at head size 64 three), or
// as many rounds as keep items below kKv4Long units: a long round ends unevenly.
// Measured (a call, merge included): 40 requests of 8k to 32k keys 568 us in one
// round, 493 in three, 571 in eleven, 695 in 22; 16 requests of 1k to 8k keys with
// branches 71 us in one round, 84 in two.  Equal shares of a request's segments, a
// work group ending one and beginning the next, took 73 us where these runs then
// took 67: a second start costs more than even lengths give.
// kKv4Least is two steps of a wave on one tile, or one on four: one token over
// 4097 keys takes 12.5 us with it, 13.3 with three quarters of it, 12.6 with one
// and a half.
constexpr int kKv4Least = 32, kKv4Long = 4096;
int kv4_target(const rg_attn_layout* L, int cus) {
  const int64_t slots = (int64_t)(L->head_dim == 64 ? 3 : 2) * cus;
  struct Group {
    int T, tiles;
    int64_t count;
  };
  std::vector<Group> groups;
  int64_t work = 0, least = 0;
  for (int r = 0; r < L->num_requests; ++r) {
    const Kv4Cols c = kv4_cols(L, r);
    const int T = L->ctx_len[r] + (L->q_indptr[r + 1] - L->q_indptr[r]);
    auto add = [&](int tiles, int64_t count) {
      if (count == 0) return;
      groups.push_back({T, tiles, count});
      least += count;
      work += count * ((T + 31) / 32) * kv4_rate(tiles);
    };
    add(kKv4Waves, c.full * L->num_kv_heads);
    add(c.rest, c.rest ? L->num_kv_heads : 0);
  }
  auto fit = [&](int64_t rounds) {  // the least target whose items fit the rounds
    for (int64_t t = std::max<int64_t>(kKv4Least, work / (rounds * slots));; t += 1 + t / 16) {
      int64_t items = 0;
      for (const Group& q : groups) items += q.count * kv4_run_count(q.T, q.tiles, (int)std::min<int64_t>(t, INT32_MAX));
      if (items <= std::max(least, rounds * slots)) return t;
    }
  };
  const int64_t one = fit(1), lim = kKv4Long;
  return (int)std::min<int64_t>(INT32_MAX, one <= lim ? one : fit((one + lim - 1) / lim));
}

template <typename Plan, int MaxReq>
rg_status plan_kv4(const rg_attn_layout* L, const rg_branch_layout* B, Kv4Plan<Plan>& fp) {
  const int R = L->num_requests, hkv = L->num_kv_heads;
  const int target = kv4_target(L, device_cus());
  auto keys_of = [&](int r) { return L->ctx_len[r] + (L->q_indptr[r + 1] - L->q_indptr[r]); };
  auto runs_of = [&](int r, int tiles) { return kv4_run_count(keys_of(r), tiles, target); };
  // Costliest work items first.
  std::vector<int> order(R);
  std::iota(order.begin(), order.end(), 0);
  std::vector<int64_t> cost(R);
  for (int r = 0; r < R; ++r) {
    const Kv4Cols c = kv4_cols(L, r);
    if (c.full) cost[r] = (int64_t)kv4_run_keys(keys_of(r), runs_of(r, kKv4Waves)) * kv4_rate(kKv4Waves);
    if (c.rest) cost[r] = std::max(cost[r], (int64_t)kv4_run_keys(keys_of(r), runs_of(r, c.rest)) * kv4_rate(c.rest));
  }
  std::stable_sort(order.begin(), order.end(), [&](int x, int y) { return cost[x] > cost[y]; });
  for (int r0 = 0; r0 < R; r0 += MaxReq) {
    const int cnt = std::min(MaxReq, R - r0);
    Plan p;
    std::memset(&p, 0, sizeof(p));
    p.num_req = cnt;
    p.chunk = target;
    int64_t items = 0, part = 0, comb = 0;
    for (int k = 0; k < cnt; ++k) {
      const int r = order[r0 + k];
      const int64_t n = L->q_indptr[r + 1] - L->q_indptr[r];
      auto& q = p.req[k];
      if constexpr (__is_same(Plan, AttnPlanBr)) pack_branches(B, r, q.br, q.rep);
      q.q_start = L->q_indptr[r];
      q.ctx = L->ctx_len[r];
      q.nv = (int32_t)((uint32_t)n | ((uint32_t)L->n_verify[r] << 16));
      q.page_start = L->page_indptr[r];
      q.item_start = (int32_t)items;
      q.part_start = (int32_t)part;
      q.comb_start = (int32_t)comb;
      if (n == 0) continue;
      const Kv4Cols c = kv4_cols(L, r);
      auto add = [&](int tiles, int64_t groups) {
        const int64_t nch = runs_of(r, tiles);
        items += hkv * groups * nch;
        if (nch == 1) return;
        p.max_chunks = std::max<int32_t>(p.max_chunks, (int32_t)nch);
        part += hkv * groups * nch * 32 * tiles;
        comb += hkv * groups * tiles * (L->head_dim / 8);
      };
      if (c.full) add(kKv4Waves, c.full);
      if (c.rest) add(c.rest, 1);
      if (items > INT32_MAX / 2 || part > INT32_MAX / 2 || comb > INT32_MAX / 2) return RG_ERR_UNSUPPORTED;
    }
    p.req[cnt].item_start = (int32_t)items;
    p.req[cnt].part_start = (int32_t)part;
    p.req[cnt].comb_start = (int32_t)comb;
    p.total_items = (int32_t)items;
    p.total_comb = (int32_t)comb;
    p.grid_items = (int32_t)round_up(items, 8);
    p.grid_comb = (int32_t)round_up(comb, 8);
    if (!fits_launch(items, 64 * kKv4Waves) || !fits_launch(comb, 64 * kKv4MergeParts))
      return RG_ERR_UNSUPPORTED;
    fp.max_partial_cols = std::max(fp.max_partial_cols, part);
    if (items > 0) fp.launches.push_back(p);
  }
  fp.ml_offset = align256((size_t)fp.max_partial_cols * L->head_dim * sizeof(float));
  fp.ws_bytes = fp.max_partial_cols ? fp.ml_offset + align256((size_t)fp.max_partial_cols * 2 * sizeof(float)) : 0;
  return RG_OK;
}

// Calls f(plan) with the plan of a layout and its branches (or NULL).
template <typename F>
rg_status with_kv4_plan(const rg_attn_layout* L, const rg_branch_layout* B, F f) try {
  rg_status st = validate_layout(L);
  if (st != RG_OK) return st;
  if (B == nullptr) {
    Kv4Plan<AttnPlan> fp;
    st = plan_kv4<AttnPlan, kMaxReqPerLaunch>(L, nullptr, fp);
    return st != RG_OK ? st : f(fp);
  }
  st = validate_branches(L, B);
  if (st != RG_OK) return st;
  Kv4Plan<AttnPlanBr> fp;
  st = plan_kv4<AttnPlanBr, kMaxReqPerLaunchBr>(L, B, fp);
  return st != RG_OK ? st : f(fp);
} catch (const std::bad_alloc&) {  // nothing is launched before a plan is whole
  return RG_ERR_WORKSPACE;
}

// The factor and shift that divide by d (quotient in kv4_device.h): with 2^l >= d,
// mul = ceil(2^(31 + l) / d) fits 32 bits and mul d exceeds 2^(31 + l) by e < d, so
// x mul / 2^(31 + l) exceeds x / d by x e / (d 2^(31 + l)) < 1 / d for every x below
// 2^31: the floors agree.
void set_divisor(int32_t d, uint32_t& mul, int32_t& shift) {
  shift = 0;
  while ((1ll << shift) < d) ++shift;
  mul = (uint32_t)(((uint64_t(1) << (31 + shift)) + d - 1) / d);
}

float softmax_scale(const rg_attn_layout* L) {
  return L->sm_scale > 0.f ? L->sm_scale : 1.0f / std::sqrt((float)L->head_dim);
}

// ---------------------------------------------------------------------------
rg_status run_mass(const rg_attn_layout* L, const uint16_t* q, const void* keys, bool kv4, const float* lse,
                   const int32_t* row_count, float decay, float* mass, void* stream) {
  rg_status st = validate_layout(L);
  if (st != RG_OK) return st;
  // launch_mass_rows addresses a request's rows by 32-bit offsets
  for (int r = 0; r < L->num_requests; ++r)
    if ((int64_t)L->n_verify[r] * L->num_q_heads * L->head_dim * 2 > INT32_MAX) return RG_ERR_UNSUPPORTED;
  if (!q || !keys || !lse || !mass) return RG_ERR_NULL;
  if (!(decay >= 0.f) || std::isinf(decay)) return RG_ERR_SHAPE;
  if (!aligned(q, 16) || !aligned(keys, 16) || !aligned(lse, 4) || !aligned(mass, 4) || !aligned(L->page_indices, 4) ||
      (row_count && !aligned(row_count, 4)))
    return RG_ERR_UNSUPPORTED;
  MassArgs a;
  a.q = q;
  a.keys = keys;
  a.lse = lse;
  a.row_count = row_count;
  a.mass = mass;
  a.page_indices = L->page_indices;
  a.hq = L->num_q_heads;
  a.hkv = L->num_kv_heads;
  a.g = a.hq / a.hkv;
  set_divisor(a.g, a.g_mul, a.g_shift);
  a.scale_log2 = softmax_scale(L) * 1.4426950408889634f;
  a.decay = decay;
  // A request without query rows need not own pages for its context.
  auto len = [&](int r) { return L->q_indptr[r + 1] == L->q_indptr[r] ? 0 : (int64_t)L->ctx_len[r] + L->n_verify[r]; };
  auto runs = [&](int r, int64_t step) { return (len(r) + step - 1) / step * L->num_kv_heads; };
  // launch_mass goes over a key's columns kMassCols at a time, in one work group;
  // launch_mass_rows shares them among a work group's waves, with fewer keys each.  The
  // latter is the faster of the two where there are few keys (it has more work groups,
  // each done sooner) or many columns; the former, which decodes and reads a key and
  // starts a work group for more of them at once, else.  So up to `most` times kMassCols
  // columns go to the former, by the work groups of kMassKeys keys that the batch gives
  // a compute unit.  us, former / latter, heads 32/8/128, by columns (* not taken):
  //                             132          256          512          1024
  //   40 of 8k-32k keys, bf16   482 / 1081   613 / 1164   1059 / 1496  1957 / 2320
  //                      4-bit  341 / 637    474 / 711    883 / 1107   *1763 / 1851
  //   16 of 1k-8k keys, bf16    51 / 100     66 / 107     114 / 140    218 / 224
  //                     4-bit   41 / 61      56 / 67      *109 / 106   *224 / 178
  //   one of 4096 keys, bf16    *10 / 11     *13 / 12     *22 / 14     *37 / 20
  //                     4-bit   *13 / 9      *18 / 9      *30 / 11     *57 / 16
  auto chunks = [&](int r) { return ((int64_t)L->n_verify[r] * a.g + kMassCols - 1) / kMassCols; };
  const int64_t limit = kv4 ? 4 : 8;
  int64_t groups = 0;
  bool asked = kv4;  // whether the compute units matter: asking for them takes the host a while
  for (int r = 0; r < L->num_requests; ++r) {
    if (chunks(r) <= limit) groups += runs(r, kMassKeys);
    asked = asked || chunks(r) > 1;
  }
  const int cus = asked ? device_cus() : 1;
  const int64_t most = std::min(limit, std::max<int64_t>(1, groups / (kv4 ? 4 * cus : cus)));
  auto many = [&](int r) { return chunks(r) > most; };
  bool wide = false;
  for (int r = 0; r < L->num_requests; ++r) wide = wide || (!many(r) && chunks(r) > 1);
  // 4-bit: the longest run that still gives every compute unit four work
  // groups, so that a run's start is a small part of it (40 long requests take 146
  // us so, as with eight or two, 188 with as many as bf16 keys give).
  int64_t all = 0;
  for (int r = 0; r < L->num_requests; ++r)
    if (!many(r)) all += len(r) * L->num_kv_heads;
  const int64_t run = kv4 ? std::min<int64_t>(kMassRun, std::max<int64_t>(128, all / (4 * cus) / 128 * 128)) : kMassKeys;
  const auto few_items = [&](int r) { return many(r) ? 0 : runs(r, run); };
  const auto many_items = [&](int r) { return many(r) ? runs(r, kMassRowKeys) : 0; };
  const int threads = 64 * kMassWaves;
  st = check_plans(L, threads, few_items);
  if (st == RG_OK) st = check_plans(L, threads, many_items);
  if (st != RG_OK) return st;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  st = each_plan(L, threads, many_items, [&](const AttnPlan& p) { return launch_mass_rows(a, p, L->head_dim, kv4, s); });
  if (st != RG_OK) return st;
  return each_plan(L, threads, few_items, [&](AttnPlan& p) {
    p.chunk = (int32_t)run;
    return launch_mass(a, p, L->head_dim, kv4, wide, s);
  });
}

// ---------------------------------------------------------------------------
rg_status validate_evict(const rg_evict_layout* L) {
  if (L == nullptr) return RG_ERR_NULL;
  if (!L->ctx_len || !L->keep || !L->tracked || !L->evicted || !L->page_indptr || !L->page_indices) return RG_ERR_NULL;
  if (L->num_requests < 1 || L->num_kv_heads < 1 || L->num_pages < 1) return RG_ERR_SHAPE;
  if (L->head_dim != 64 && L->head_dim != 128) return RG_ERR_UNSUPPORTED;
  if (L->page_size != kPageSize) return RG_ERR_UNSUPPORTED;
  if (L->sink < 0 || L->recent < 0 || L->page_indptr[0] != 0) return RG_ERR_SHAPE;
  for (int r = 0; r < L->num_requests; ++r) {
    const int64_t n = L->ctx_len[r], pages = (int64_t)L->page_indptr[r + 1] - L->page_indptr[r];
    if (n < 0 || pages < 0 || L->keep[r] < 0 || L->evicted[r] < 0) return RG_ERR_SHAPE;
    if (L->tracked[r] < 0 || L->tracked[r] > n) return RG_ERR_SHAPE;
    if (n > (int64_t(1) << 30) || n + L->evicted[r] > INT32_MAX) return RG_ERR_UNSUPPORTED;
    if (pages * kPageSize < n) return RG_ERR_SHAPE;
    // every protected token has to fit
    if (L->keep[r] < n && (int64_t)L->sink + L->recent > L->keep[r]) return RG_ERR_SHAPE;
  }
  return RG_OK;
}

// Calls f(plan) for the requests of a layout, a plan's worth at a time.  The
// launches share the workspace one after another; `words` returns its size.
template <typename F>
rg_status each_evict_plan(const rg_evict_layout* L, int64_t& words, F f) {
  words = 0;
  for (int r0 = 0; r0 < L->num_requests; r0 += kMaxEvictReq) {
    EvictPlan p;
    std::memset(&p, 0, sizeof(p));
    p.num_req = std::min(kMaxEvictReq, L->num_requests - r0);
    int64_t ws = 0, moves = 0;
    // The longest requests first: a choice takes as long as its request, and two
    // work groups at a time share a compute unit.
    int order[kMaxEvictReq];
    std::iota(order, order + p.num_req, r0);
    std::stable_sort(order, order + p.num_req, [&](int x, int y) { return L->ctx_len[x] > L->ctx_len[y]; });
    for (int k = 0; k < p.num_req; ++k) {
      const int r = order[k];
      EvictReq& q = p.req[k];
      q.ctx = L->ctx_len[r];
      q.keep = std::min(L->keep[r], L->ctx_len[r]);
      q.tracked = L->tracked[r];
      q.evicted = L->evicted[r];
      q.page_start = L->page_indptr[r];
      q.most = std::min(q.keep, q.ctx - q.keep);
      q.ws_start = (int32_t)ws;
      q.move_start = (int32_t)moves;
      if (q.most == 0) continue;
      p.longest = std::max(p.longest, q.ctx);
      ws += (int64_t)L->num_kv_heads * evict_words(q.keep, q.most);
      moves += (int64_t)L->num_kv_heads * (((q.keep + 15) / 16 + kMoveWaves - 1) / kMoveWaves);
      if (ws > INT32_MAX / 2 || !fits_launch(moves, kMoveThreads)) return RG_ERR_UNSUPPORTED;
    }
    if (!fits_launch((int64_t)p.num_req * L->num_kv_heads, kEvictThreads)) return RG_ERR_UNSUPPORTED;
    p.move_items = (int32_t)moves;
    p.req[p.num_req].move_start = (int32_t)moves;
    words = std::max(words, ws);
    const rg_status st = f(p);
    if (st != RG_OK) return st;
  }
  return RG_OK;
}

rg_status run_evict(const rg_evict_layout* L, uint8_t* k_cache, uint8_t* v_cache, bool kv4, const float* score,
                    float* mass, int32_t* positions, void* ws, size_t ws_bytes, void* stream) {
  rg_status st = validate_evict(L);
  if (st != RG_OK) return st;
  if (!k_cache || !v_cache || !score || !positions) return RG_ERR_NULL;
  if (!aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(score, 4) || !aligned(positions, 4) ||
      (mass && !aligned(mass, 4)) || !aligned(L->page_indices, 4))
    return RG_ERR_UNSUPPORTED;
  int64_t words = 0;
  st = each_evict_plan(L, words, [](const EvictPlan&) { return RG_OK; });
  if (st != RG_OK) return st;
  if (words > 0 && (ws == nullptr || ws_bytes < (size_t)words * 4 || !aligned(ws, 16))) return RG_ERR_WORKSPACE;
  EvictArgs a;
  a.score = score;
  a.mass = mass;
  a.positions = positions;
  a.k_cache = k_cache;
  a.v_cache = v_cache;
  a.page_indices = L->page_indices;
  a.ws = static_cast<int32_t*>(ws);
  a.hkv = L->num_kv_heads;
  a.sink = L->sink;
  a.recent = L->recent;
  return each_evict_plan(L, words, [&](const EvictPlan& p) {
    return launch_evict(a, p, L->head_dim, kv4, static_cast<hipStream_t>(stream)) == hipSuccess ? RG_OK : RG_ERR_HIP;
  });
}

}  // namespace

extern "C" {

rg_status rg_kv4_append(const rg_attn_layout* layout, const uint16_t* k, int64_t k_stride, const uint16_t* v,
                        int64_t v_stride, uint8_t* cache, void* stream) {
  return run_rows(layout, k, k_stride, v, v_stride, cache, true, stream);
}

rg_status rg_kv4_read(const rg_attn_layout* layout, const uint8_t* cache, uint16_t* k, int64_t k_stride, uint16_t* v,
                      int64_t v_stride, void* stream) {
  return run_rows(layout, k, k_stride, v, v_stride, cache, false, stream);
}

rg_status rg_kv4_attention_workspace(const rg_attn_layout* layout, const rg_branch_layout* branches, size_t* bytes) {
  if (bytes == nullptr) return RG_ERR_NULL;
  return with_kv4_plan(layout, branches, [&](const auto& fp) {
    *bytes = fp.ws_bytes;
    return RG_OK;
  });
}

rg_status rg_kv4_attention(const rg_attn_layout* layout, const rg_branch_layout* branches, const uint16_t* q,
                           const uint8_t* cache, uint16_t* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  return with_kv4_plan(layout, branches, [&](const auto& fp) -> rg_status {
    if (!q || !cache || !out) return RG_ERR_NULL;
    if (!aligned(q, 16) || !aligned(cache, 16) || !aligned(out, 16) || (lse && !aligned(lse, 4)) ||
        !aligned(layout->page_indices, 4))
      return RG_ERR_UNSUPPORTED;
    if (fp.ws_bytes > 0 && (ws == nullptr || ws_bytes < fp.ws_bytes || !aligned(ws, 16))) return RG_ERR_WORKSPACE;
    Kv4AttnArgs a;
    a.q = q;
    a.cache = cache;
    a.out = out;
    a.lse = lse;
    a.page_indices = layout->page_indices;
    a.part_o = fp.ws_bytes ? static_cast<float*>(ws) : nullptr;
    a.part_ml = fp.ws_bytes ? reinterpret_cast<float*>(static_cast<char*>(ws) + fp.ml_offset) : nullptr;
    a.hq = layout->num_q_heads;
    a.hkv = layout->num_kv_heads;
    a.g = a.hq / a.hkv;
    set_divisor(a.g, a.g_mul, a.g_shift);
    set_divisor(a.hkv, a.hkv_mul, a.hkv_shift);
    a.sm_scale = softmax_scale(layout);
    a.scale_log2 = a.sm_scale * 1.4426950408889634f;
    for (const auto& p : fp.launches)
      if (launch_kv4_attention(a, p, layout->head_dim, static_cast<hipStream_t>(stream)) != hipSuccess) return RG_ERR_HIP;
    return RG_OK;
  });
}

rg_status rg_attention_mass(const rg_attn_layout* layout, const uint16_t* q, const uint16_t* k_cache, const float* lse,
                            const int32_t* row_count, float decay, float* mass, void* stream) {
  return run_mass(layout, q, k_cache, false, lse, row_count, decay, mass, stream);
}

rg_status rg_kv4_attention_mass(const rg_attn_layout* layout, const uint16_t* q, const uint8_t* cache, const float* lse,
                                const int32_t* row_count, float decay, float* mass, void* stream) {
  return run_mass(layout, q, cache, true, lse, row_count, decay, mass, stream);
}

rg_status rg_evict_workspace(const rg_evict_layout* layout, size_t* bytes) {
  if (bytes == nullptr) return RG_ERR_NULL;
  rg_status st = validate_evict(layout);
  if (st != RG_OK) return st;
  int64_t words = 0;
  st = each_evict_plan(layout, words, [](const EvictPlan&) { return RG_OK; });
  if (st == RG_OK) *bytes = (size_t)words * 4;
  return st;
}

rg_status rg_evict_tokens(const rg_evict_layout* layout, uint16_t* k_cache, uint16_t* v_cache, const float* score,
                          float* mass, int32_t* positions, void* ws, size_t ws_bytes, void* stream) {
  return run_evict(layout, reinterpret_cast<uint8_t*>(k_cache), reinterpret_cast<uint8_t*>(v_cache), false, score, mass,
                   positions, ws, ws_bytes, stream);
}

rg_status rg_kv4_evict_tokens(const rg_evict_layout* layout, uint8_t* cache, const float* score, float* mass,
                              int32_t* positions, void* ws, size_t ws_bytes, void* stream) {
  return run_evict(layout, cache, cache, true, score, mass, positions, ws, ws_bytes, stream);
}

}  // extern "C"
