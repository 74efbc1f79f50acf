// Eviction of tokens from a paged cache by score.
//
// Per (request, KV head) the L tokens are cut to the `keep` that are
// protected (first positions, latest positions) or have the largest scores.
// Tokens do not keep their order (attention does not look at it, and the
// positions pool says which token a slot holds), so only the kept tokens
// behind slot `keep` move: into the evicted slots before it, both in ascending
// order.  No slot is both read and written, so moves run in any order.
//
// select: one work group per (request, KV head).  A radix selection over the
// scores as ordered 32-bit words (protected tokens the largest word) finds the
// word of the keep-th largest, then each wave walks a contiguous part of the
// slots: ties are taken from the lowest slot on, holes and movers get their
// ranks from wave ballots.  It writes the move list, the positions and the
// mass.  move: copies K and V of 16 moves per work group.
#include "cache_internal.h"
#include "kv4_device.h"

namespace rg {
namespace {

constexpr int kWaves = kEvictThreads / 64;

__device__ __forceinline__ int evict_request(const EvictPlan& p, int item) {
  const int lane = threadIdx.x & 63;
  int r = 0;
  for (int base = 1; base < p.num_req; base += 64) {
    const int k = base + lane;
    r += __popcll(__ballot(k < p.num_req && p.req[k].move_start <= item));
  }
  return __builtin_amdgcn_readfirstlane(r);
}

__device__ __forceinline__ int32_t* move_list(const EvictArgs& a, const EvictReq& q, int hk) {
  return a.ws + q.ws_start + (size_t)hk * (4 + 2 * (size_t)q.most);
}

__global__ __launch_bounds__(kEvictThreads) void evict_select_kernel(EvictArgs a, EvictPlan p) {
  __shared__ uint32_t hist[256];
  __shared__ uint32_t s_digit, s_left;
  __shared__ uint32_t s_count[kWaves][3];
  const int r = (int)blockIdx.x / a.hkv, hk = (int)blockIdx.x % a.hkv;
  const EvictReq q = p.req[r];
  const int L = q.ctx, keep = q.keep, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int32_t* pages = a.page_indices + q.page_start;
  const int recent_from = L + q.evicted - a.recent;  // positions from here on are protected

  auto place = [&](int j) { return ((size_t)pages[j >> 4] * a.hkv + hk) * kPageSize + (j & 15); };
  auto position = [&](int j, size_t at) { return j < q.tracked ? a.positions[at] : j + q.evicted; };
  // A slot's score as a word of the same order: protected tokens the largest.
  auto word = [&](int j) {
    const size_t at = place(j);
    const int pos = position(j, at);
    if (pos < a.sink || pos >= recent_from) return 0xffffffffu;
    const uint32_t u = __float_as_uint(a.score[at] + 0.f);  // -0 becomes 0
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
  };

  if (keep == 0) {  // (also an empty request)
    if (tid == 0) move_list(a, q, hk)[0] = 0;
    return;
  }
  uint32_t prefix = 0, left = (uint32_t)keep;  // of the tokens whose words begin with the prefix, `left` are kept
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
    const uint32_t mask = shift == 24 ? 0u : ~0u << (shift + 8);
    for (int j = tid; j < L; j += kEvictThreads) {
      const uint32_t u = word(j);
      if ((u & mask) == prefix) atomicAdd(&hist[(u >> shift) & 255], 1u);
    }
    __syncthreads();
    if (wave == 0) {  // lane l holds bins 255 - 4 l .. 252 - 4 l
      uint32_t b[4], sum = 0;
      for (int e = 0; e < 4; ++e) sum += b[e] = hist[255 - 4 * lane - e];
      uint32_t upto = sum;
      for (int off = 1; off < 64; off <<= 1) {
        const uint32_t x = __shfl_up(upto, off);
        if (lane >= off) upto += x;
      }
      uint32_t before = upto - sum;
      if (before < left && left <= upto) {
        int e = 0;
        while (before + b[e] < left) before += b[e++];
        s_digit = 255 - 4 * lane - e;
        s_left = left - before;
      }
    }
    __syncthreads();
    prefix |= s_digit << shift;
    left = s_left;
  }

  // Slots of this wave, a multiple of 64 from a multiple of 64 on.
  const int seg = ((L + 64 * kWaves - 1) / (64 * kWaves)) * 64;
  const int j0 = min(L, wave * seg), j1 = min(L, j0 + seg);
  const uint64_t below = (1ull << lane) - 1;
  uint32_t ties = 0;
  for (int b = j0; b < j1; b += 64) ties += __popcll(__ballot(b + lane < j1 && word(b + lane) == prefix));
  if (lane == 0) s_count[wave][0] = ties;
  __syncthreads();
  uint32_t tie0 = 0;
  for (int w = 0; w < wave; ++w) tie0 += s_count[w][0];

  auto walk = [&](auto visit) {  // visit(j, kept, rank of a hole or mover among the wave's)
    uint32_t tie = tie0, holes = 0, movers = 0;
    for (int b = j0; b < j1; b += 64) {
      const int j = b + lane;
      const uint32_t u = j < j1 ? word(j) : 0;
      const uint64_t eq = __ballot(j < j1 && u == prefix);
      const bool kept = j < j1 && (u > prefix || (u == prefix && tie + __popcll(eq & below) < left));
      const uint64_t hole = __ballot(j < j1 && j < keep && !kept), mover = __ballot(kept && j >= keep);
      if (j < j1) visit(j, kept, j < keep ? holes + __popcll(hole & below) : movers + __popcll(mover & below));
      tie += __popcll(eq);
      holes += __popcll(hole);
      movers += __popcll(mover);
    }
    return make_uint2(holes, movers);
  };
  const uint2 mine = walk([](int, bool, uint32_t) {});
  if (lane == 0) {
    s_count[wave][1] = mine.x;
    s_count[wave][2] = mine.y;
  }
  __syncthreads();
  uint32_t hole0 = 0, mover0 = 0, count = 0;
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) hole0 += s_count[w][1], mover0 += s_count[w][2];
    count += s_count[w][2];
  }
  int32_t* list = move_list(a, q, hk);
  if (tid == 0) list[0] = (int32_t)count;
  walk([&](int j, bool kept, uint32_t rank) {
    if (j < keep && !kept) list[4 + 2 * (size_t)(hole0 + rank)] = j;
    if (j >= keep && kept) list[5 + 2 * (size_t)(mover0 + rank)] = j;
  });
  __syncthreads();
  for (int j = max(q.tracked, 0) + tid; j < keep; j += kEvictThreads) a.positions[place(j)] = j + q.evicted;
  __syncthreads();
  for (uint32_t k = tid; k < count; k += kEvictThreads) {
    const int to = list[4 + 2 * (size_t)k], from = list[5 + 2 * (size_t)k];
    const size_t dst = place(to), src = place(from);
    a.positions[dst] = position(from, src);
    if (a.mass) a.mass[dst] = a.mass[src];
  }
}

template <int D, bool KV4>
__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(EvictArgs a, EvictPlan p) {
  const int item = blockIdx.x;
  const int r = evict_request(p, item);
  const EvictReq q = p.req[r];
  const int groups = (q.most + kMoveTokens - 1) / kMoveTokens;
  const int local = item - q.move_start;
  const int hk = local / groups;
  const int32_t* list = move_list(a, q, hk);
  const int k = local % groups * kMoveTokens + (int)threadIdx.x / 16, t = threadIdx.x % 16;
  if (k >= list[0]) return;
  const int to = list[4 + 2 * (size_t)k], from = list[5 + 2 * (size_t)k];
  const int32_t* pages = a.page_indices + q.page_start;
  const size_t dst = (size_t)pages[to >> 4] * a.hkv + hk, src = (size_t)pages[from >> 4] * a.hkv + hk;
  const int ds = to & 15, ss = from & 15;
  if constexpr (KV4) {
    using B = Kv4<D>;
    uint8_t* x = a.k_cache + dst * B::BLOCK;
    const uint8_t* y = a.k_cache + src * B::BLOCK;
    if constexpr (D == 128) {
      *(uint32_t*)(x + B::k_code(ds, 8 * t)) = *(const uint32_t*)(y + B::k_code(ss, 8 * t));
#pragma unroll
      for (int e = 0; e < 2; ++e) *(uint16_t*)(x + B::v_unit(ds, t + 16 * e)) = *(const uint16_t*)(y + B::v_unit(ss, t + 16 * e));
    } else {
      *(uint16_t*)(x + B::k_code(ds, 4 * t)) = *(const uint16_t*)(y + B::k_code(ss, 4 * t));
#pragma unroll
      for (int e = 0; e < 2; ++e) x[B::v_unit(ds, t + 16 * e)] = y[B::v_unit(ss, t + 16 * e)];
    }
    if (t < B::DT) x[B::k_scale(ds, t)] = y[B::k_scale(ss, t)];
    else if (t < 2 * B::DT) x[B::v_scale(ds, t - B::DT)] = y[B::v_scale(ss, t - B::DT)];
  } else {
    constexpr int E = D / 16;  // elements of a thread
    uint16_t* k_cache = reinterpret_cast<uint16_t*>(a.k_cache);
    uint16_t* v_cache = reinterpret_cast<uint16_t*>(a.v_cache);
    uint16_t* kd = k_cache + (dst * kPageSize + ds) * D + E * t;
    const uint16_t* ks = k_cache + (src * kPageSize + ss) * D + E * t;
    if constexpr (D == 128) *(u32x4*)kd = *(const u32x4*)ks;
    else *(u32x2*)kd = *(const u32x2*)ks;
    uint16_t x[E];
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = v_cache[(src * D + t + 16 * e) * kPageSize + ss];
#pragma unroll
    for (int e = 0; e < E; ++e) v_cache[(dst * D + t + 16 * e) * kPageSize + ds] = x[e];
  }
}

}  // namespace

hipError_t launch_evict(const EvictArgs& a, const EvictPlan& p, int head_dim, bool kv4, hipStream_t stream) {
  hipLaunchKernelGGL(evict_select_kernel, dim3(p.num_req * a.hkv), dim3(kEvictThreads), 0, stream, a, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.move_items == 0) return e;
  const dim3 grid(p.move_items), block(kMoveThreads);
  if (head_dim == 128 && kv4) hipLaunchKernelGGL((evict_move_kernel<128, true>), grid, block, 0, stream, a, p);
  else if (head_dim == 128) hipLaunchKernelGGL((evict_move_kernel<128, false>), grid, block, 0, stream, a, p);
  else if (kv4) hipLaunchKernelGGL((evict_move_kernel<64, true>), grid, block, 0, stream, a, p);
  else hipLaunchKernelGGL((evict_move_kernel<64, false>), grid, block, 0, stream, a, p);
  return hipGetLastError();
}

}  // namespace rg
