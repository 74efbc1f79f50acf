// Host helpers shared by the API files: argument checks and planning rules
// (validation, branches and device_cus defined in api.cpp).
#pragma once

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>

#include "recguide.h"
#include "rg_internal.h"

namespace rg {

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

inline int64_t round_up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

// Whether a grid of this many work groups, rounded up to 8, is one launch.
inline bool fits_launch(int64_t groups, int threads) { return round_up(groups, 8) * threads <= kMaxLaunchThreads; }

rg_status validate_layout(const rg_attn_layout* L);
rg_status validate_branches(const rg_attn_layout* L, const rg_branch_layout* B);
bool pack_branches(const rg_branch_layout* B, int r, int32_t (&w)[3], int32_t& rep);

int device_cus();

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

// The factor and shift that divide by d (quotient in attention_device.h): with 2^l >= d,
// mul = ceil(2^(31 + l) / d) fits 32 bits and mul d exceeds 2^(31 + l) by e < d, so
// x mul / 2^(31 + l) exceeds x / d by x e / (d 2^(31 + l)) < 1 / d for every x below
// 2^31: the floors agree.
inline void set_divisor(int32_t d, uint32_t& mul, int32_t& shift) {
  shift = 0;
  while ((1ll << shift) < d) ++shift;
  mul = (uint32_t)(((uint64_t(1) << (31 + shift)) + d - 1) / d);
}

inline float softmax_scale(const rg_attn_layout* L) {
  return L->sm_scale > 0.f ? L->sm_scale : 1.0f / std::sqrt((float)L->head_dim);
}

}  // namespace rg
