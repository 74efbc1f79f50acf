// Launch-side structures of the 4-bit KV cache, the attention mass and the
// eviction of tokens, shared by cache_api.cpp and their kernels.
#pragma once

#include "rg_internal.h"

namespace rg {

// Rows into, or out of, the 4-bit cache.  Plans: AttnPlan with a work item per
// page that a request's rows touch and plan.chunk KV heads (1 .. kRowHeads).
constexpr int kRowHeads = 4;
struct Kv4RowArgs {
  uint16_t* k;  // rows (appended: read, read back: written)
  uint16_t* v;
  int64_t k_stride, v_stride;  // elements
  uint8_t* cache;
  const int32_t* page_indices;
  int32_t hkv;
};
hipError_t launch_kv4_append(const Kv4RowArgs& a, const AttnPlan& p, int head_dim, hipStream_t stream);
hipError_t launch_kv4_read(const Kv4RowArgs& a, const AttnPlan& p, int head_dim, hipStream_t stream);

// Attention over the 4-bit cache.
constexpr int kKv4Waves = 4;                       // waves of a work group
constexpr int kKv4Cols = 32 * kKv4Waves;           // query columns of a work group at most
constexpr int kKv4MergeRows = 2;                   // rows of a wave of the merge
constexpr int kKv4MergeParts = 4;                  // waves of a work group of the merge
// A request's 32-column tiles form column groups of four, and a last one of
// what remains.  Time of 32 keys in a group of 1 .. 4 tiles, in units of a
// sixteenth of that of four, as work groups' own clocks gave it (three tiles: of
// the two wave pairs one has a single tile and waits for the other).
__host__ __device__ inline int kv4_rate(int tiles) { return tiles == 1 ? 6 : tiles == 2 ? 9 : tiles == 3 ? 15 : 16; }
// Runs that the T keys of such a group are cut into, for items of at most
// `target` units, and the keys of a run: all but the last alike.
__host__ __device__ inline int kv4_run_count(int T, int tiles, int target) {
  const uint32_t steps = ((uint32_t)T + 31) / 32, rate = kv4_rate(tiles);
  const uint32_t most = (uint32_t)target > rate ? (uint32_t)target / rate : 1;  // steps of a run at most
  const uint32_t n = (steps + most - 1) / most, each = (steps + n - 1) / n;
  return (int)((steps + each - 1) / each);
}
__host__ __device__ inline int kv4_run_keys(int T, int count) {
  const uint32_t steps = ((uint32_t)T + 31) / 32;
  return (int)(32 * ((steps + count - 1) / count));
}
struct Kv4AttnArgs {
  const uint16_t* q;
  const uint8_t* cache;
  uint16_t* out;
  float* lse;
  const int32_t* page_indices;
  float* part_o;   // per 32-column tile: 32 x D fp32 sums, 16-byte rows lane-interleaved
  float* part_ml;  // [partial columns][2] (running maximum of raw scores, sum)
  int32_t hq, hkv, g;
  uint32_t g_mul, hkv_mul;  // quotient by g, by hkv
  int32_t g_shift, hkv_shift;
  float sm_scale, scale_log2;
};
hipError_t launch_kv4_attention(const Kv4AttnArgs& a, const AttnPlan& p, int head_dim, hipStream_t stream);
hipError_t launch_kv4_attention(const Kv4AttnArgs& a, const AttnPlanBr& p, int head_dim, hipStream_t stream);

// Attention mass.  Plans: AttnPlan, part_start the request's number.  Requests
// of few query columns a KV head take launch_mass (`wide` where one has more than
// kMassCols), with work items of kMassKeys keys (bf16) or plan.chunk (4-bit) of a KV
// head; the others launch_mass_rows, with items of kMassRowKeys keys.  Where the line
// lies: run_mass in cache_api.cpp.
constexpr int kMassWaves = 4;
constexpr int kMassCols = 128;
constexpr int kMassSub = 2;                            // 32-key tiles of a bf16 wave
constexpr int kMassKeys = 32 * kMassWaves * kMassSub;
constexpr int kMassRun = 2048;                         // plan.chunk at most
constexpr int kMassRowKeys = 64;
struct MassArgs {
  const uint16_t* q;
  const void* keys;  // bf16 K pool, or the 4-bit pool
  const float* lse;
  const int32_t* row_count;  // or NULL
  float* mass;
  const int32_t* page_indices;
  int32_t hq, hkv, g;
  float scale_log2, decay;
  uint32_t g_mul;  // quotient by g
  int32_t g_shift;
};
hipError_t launch_mass(const MassArgs& a, const AttnPlan& p, int head_dim, bool kv4, bool wide, hipStream_t stream);
hipError_t launch_mass_rows(const MassArgs& a, const AttnPlan& p, int head_dim, bool kv4, hipStream_t stream);

// Eviction.
constexpr int kEvictThreads = 1024;  // select: a work group per (request, KV head)
constexpr int kMoveWaves = 4;        // move: a page per wave
constexpr int kMoveThreads = 64 * kMoveWaves;
// Workspace words of a (request, head): two for every kept slot and for every
// move at most.
__host__ __device__ inline size_t evict_words(int keep, int most) { return (2 * (size_t)keep + 2 * (size_t)most + 3) / 4 * 4; }
struct EvictReq {
  int32_t ctx, keep, tracked, evicted;  // keep <= ctx
  int32_t page_start;
  int32_t ws_start;    // first word of the request's move lists in the workspace
  int32_t most;        // moves of a head at most
  int32_t move_start;  // first move item
};
constexpr int kMaxEvictReq = 96;
struct EvictPlan {
  int32_t num_req, move_items;
  int32_t longest;  // most tokens of a request that is cut
  EvictReq req[kMaxEvictReq + 1];
};
static_assert(sizeof(EvictPlan) <= 3700, "plan must fit the kernel argument block");
struct EvictArgs {
  const float* score;
  float* mass;  // or NULL
  int32_t* positions;
  uint8_t* k_cache;  // bf16 K pool, or the 4-bit pool
  uint8_t* v_cache;  // bf16 V pool
  const int32_t* page_indices;
  int32_t* ws;       // per (request, head): evict_words
  int32_t hkv, sink, recent;
};
hipError_t launch_evict(const EvictArgs& a, const EvictPlan& p, int head_dim, bool kv4, hipStream_t stream);

}  // namespace rg
