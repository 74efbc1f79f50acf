// Launch-side structures of rotated appends, the 8-bit KV cache and attention
// over a window, shared by window_api.cpp and their kernels.
#pragma once

#include "rg_internal.h"

namespace rg {

// Rows into, or out of, a cache.  Plans: AttnPlan; a page that a request's rows
// touch has items of plan.chunk KV heads, then of plan.cols_per_group heads of
// q (0: no q).
constexpr int kAppendThreads = 256;
struct AppendArgs {
  const uint16_t* q;  // or NULL
  const uint16_t* k;
  const uint16_t* v;
  uint16_t* q_out;
  int64_t q_stride, k_stride, v_stride;  // elements
  uint16_t* k_cache;                     // bf16 pools, or
  uint16_t* v_cache;
  uint8_t* cache;                        // the 8-bit pool
  float* scales;
  const int32_t* page_indices;
  const int32_t* positions;  // or NULL
  const float* inv_freq;
  int32_t hq, hkv, dims, interleaved;
};
hipError_t launch_append(const AppendArgs& a, const AttnPlan& p, int head_dim, bool kv8, hipStream_t stream);

struct Kv8ReadArgs {
  const uint8_t* cache;
  const float* scales;
  uint16_t* k;
  uint16_t* v;
  int64_t k_stride, v_stride;
  const int32_t* page_indices;
  int32_t hkv;
};
hipError_t launch_kv8_read(const Kv8ReadArgs& a, const AttnPlan& p, int head_dim, hipStream_t stream);

}  // namespace rg
