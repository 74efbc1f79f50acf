// Launch-side structures of rotated appends, the 8-bit KV cache and attention
// over a window, shared by window_api.cpp and their kernels.
#pragma once

#include "rg_internal.h"

namespace rg {

// Rows into, or out of, a cache.  Plans: AttnPlan; a page that a request's rows
// touch has items of append_heads KV heads, and of plan.cols_per_group heads of q
// (0: no q).
constexpr int kAppendThreads = 256;
__host__ __device__ constexpr int append_heads(int head_dim) { return 256 / head_dim; }
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
// KV heads of an item of the read.
__host__ __device__ constexpr int kv8_read_heads(int head_dim) { return kAppendThreads / (2 * head_dim); }
hipError_t launch_kv8_read(const Kv8ReadArgs& a, const AttnPlan& p, int head_dim, hipStream_t stream);

// Attention over a window, or all, of the keys of a bf16 or an 8-bit cache.
//
// A request's 32-column tiles are dealt evenly to column groups of up to
// kWindowWaves tiles.  A group's keys are those that its rows may see: the sinks'
// pages and those from the first row's window on, counted without the gap between
// them.  They are cut into runs, alike for all groups of a request; runs past a
// group's keys are empty.
constexpr int kWindowWaves = 4;  // waves of a work group; two (D = 128) or three share a compute unit
// Keys a buffer of a work group holds: two of K and two of V leave room for two work
// groups of D = 128 in a compute unit, three of D = 64 (15 prompts of 555 rows over 3806
// keys 216 us; with buffers of 128 and two work groups 250, of 64 the same 216, but 100
// tokens over 500 keys 21 us against 17).
__host__ __device__ constexpr int window_keys(int head_dim) { return head_dim == 64 ? 96 : 64; }
constexpr int kWindowMergeWaves = 4;  // waves of a work group of the merge
constexpr int kWindowMergeRows = 2;   // rows of one
struct WindowReq {
  int32_t q_start, ctx, nv, page_start, item_start;  // as in AttnReq
  int32_t part_start;                                // first partial tile in the workspace
  uint32_t runs;                                     // their number (low 16 bits) | keys of one / keys of a step << 16
};
struct WindowReqBr : WindowReq {
  int32_t br[3], rep;  // as in AttnReqBr
};
constexpr int kMaxRunSteps = 0xffff;
template <typename Req, int MaxReq>
struct WindowPlanT {
  int32_t num_req, total_items, total_comb, max_chunks;
  Req req[MaxReq + 1];  // entry num_req holds the end sentinel of item_start
};
using WindowPlan = WindowPlanT<WindowReq, kMaxReqPerLaunch>;
using WindowPlanBr = WindowPlanT<WindowReqBr, kMaxReqPerLaunchBr>;
static_assert(sizeof(WindowPlan) <= 3700 && sizeof(WindowPlanBr) <= 3700, "plan must fit the kernel argument block");

struct WindowArgs {
  const uint16_t* q;
  const uint8_t* k_cache;  // bf16 K pool, or the 8-bit pool
  const uint8_t* v_cache;  // bf16 V pool
  const float* scales;     // of the 8-bit pool
  uint16_t* out;
  float* lse;
  const int32_t* page_indices;
  float* part_o;   // per 32-column tile: 32 x D fp32 sums, 16-byte rows lane-interleaved
  float* part_ml;  // [partial columns][2] (reference of raw scores, sum)
  int32_t hq, hkv, g;
  uint32_t g_mul, hkv_mul;  // quotient by g, by hkv
  int32_t g_shift, hkv_shift;
  int32_t size, sink;  // of the window; size 2^30 for all keys
  float sm_scale, scale_log2;
};
// The keys that rows i0 .. i1 - 1 of a request may see.
struct WindowSpan {
  int32_t keys;  // their number, with the sinks' pages' other slots
  int32_t gap;   // key k >= head stands for token k + gap; a multiple of 16
  int32_t head;  // keys of the sinks' pages where there is a gap
  int32_t lo;    // the first key of the window
};
template <bool BR>
__host__ __device__ inline WindowSpan window_span(int L, int V, int n, int i0, int i1, int size, int sink) {
  WindowSpan s;
  // a branch may keep none of the verify rows
  const int first = BR && i1 > V ? L : L + i0;
  int lo = first + 1 - size;
  if (lo > L + V) lo = L + V;  // draft rows see all of their block
  if (BR && i1 > V && lo > L) lo = L;
  if (lo < 0) lo = 0;
  const int end = i1 <= V ? L + i1 : L + n;
  s.head = (sink + 15) / 16 * 16;
  s.gap = lo / 16 * 16 - s.head;
  if (s.gap < 0) s.gap = 0;
  s.lo = lo - s.gap;
  s.keys = end - s.gap;
  return s;
}
#ifdef __HIPCC__
// Scores of a 32 x 32 tile: value i of a lane is key 8 lh + place_of(i) of the tile.  A mask
// is made as bits of the lane's places, and a score hidden in two instructions, without
// branches or condition registers.
__device__ __forceinline__ constexpr int place_of(int i) { return 16 * (i >> 3) + 4 * ((i >> 2) & 1) + (i & 3); }
__device__ __forceinline__ uint32_t places_below(int x) { return (1u << min(max(x, 0), 24)) - 1; }
template <typename Scores>
__device__ __forceinline__ void hide_places(Scores& sc, uint32_t hidden) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const uint32_t all = (uint32_t)__builtin_amdgcn_sbfe((int)hidden, place_of(i), 1);
    sc[i] = __uint_as_float((all & 0xff800000u) | (~all & __float_as_uint(sc[i])));  // minus infinity
  }
}
#endif
hipError_t launch_window_attention(const WindowArgs& a, const WindowPlan& p, int head_dim, hipStream_t stream);
hipError_t launch_window_attention(const WindowArgs& a, const WindowPlanBr& p, int head_dim, hipStream_t stream);

// Over the 8-bit cache: column groups of kKv8Waves tiles and a last one of what
// remains, steps of kKv8Step keys.
constexpr int kKv8Waves = 4, kKv8Step = 128;
// The first of the four dims of row v of a lane in half-wave lh there.
__host__ __device__ constexpr int kv8_dim(int dt, int v, int lh) { return 8 * dt * (v / dt) + 4 * dt * lh + 4 * (v % dt); }
hipError_t launch_kv8_attention(const WindowArgs& a, const WindowPlan& p, int head_dim, hipStream_t stream);
hipError_t launch_kv8_attention(const WindowArgs& a, const WindowPlanBr& p, int head_dim, hipStream_t stream);
// The merge of both, of split requests' runs (nothing where there are none).
hipError_t launch_window_merge(const WindowArgs& a, const WindowPlan& p, int head_dim, hipStream_t stream);
hipError_t launch_window_merge(const WindowArgs& a, const WindowPlanBr& p, int head_dim, hipStream_t stream);

}  // namespace rg
