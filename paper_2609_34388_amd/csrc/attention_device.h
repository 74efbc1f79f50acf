// Device helpers shared by the attention kernels (bf16 and 4-bit caches).
#pragma once

#include "rg_internal.h"

namespace rg {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr float kNegInf = -__builtin_huge_valf();

__device__ __forceinline__ int swap23(int r) {
  return (r & ~12) | ((r & 4) << 1) | ((r & 8) >> 1);
}

__device__ __forceinline__ uint32_t pack_bf16x2(float a, float b) {
  const f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

// Request owning work item `item` of `count` requests: the last r with start(r) <=
// item (starts are nondecreasing, empty requests share their successor's start).
// Every lane tests one request, so the search is one round of loads, not a chain.
template <typename Start>
__device__ __forceinline__ int find_start(int count, int item, Start start) {
  const int lane = threadIdx.x & 63;
  int r = 0;
  for (int base = 1; base < count; base += 64) {
    const int k = base + lane;
    r += __popcll(__ballot(k < count && start(k) <= item));
  }
  return __builtin_amdgcn_readfirstlane(r);
}
template <typename Plan>
__device__ __forceinline__ int find_request(const Plan& p, int item, bool combine) {
  return find_start(p.num_req, item, [&](int k) {
    if constexpr (__is_same(Plan, AttnPlanBrPacked)) return p.req[k].item_start;
    else return combine ? p.req[k].comb_start : p.req[k].item_start;
  });
}

// Consecutive work items of one (request, KV head) land on one XCD: the
// dispatcher deals work groups to the 8 XCDs round-robin, so block b runs on
// XCD b % 8; give XCD x the item range [x*per, (x+1)*per).
__device__ __forceinline__ int xcd_item(int grid_items) {
  const int per = grid_items >> 3;
  return (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
}

// Work-group barrier that orders LDS only.  __syncthreads() also fences
// global memory, which makes every wave wait for all of its outstanding
// vector-memory operations -- the copy waves' loads of the next buffers --
// at each barrier.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// 16 bytes of every lane from base + off to LDS, byte `lds` + 16 * lane (below
// 64 KiB).  No register waits for the data: they are there once s_waitcnt vmcnt
// says so.
__device__ __forceinline__ void load_to_lds(uint32_t lds, const void* base, uint32_t off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void load_to_lds(uint32_t lds, const void* lane_address) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(lane_address) : "memory", "m0");
}
// A pointer's byte of LDS.
__device__ __forceinline__ uint32_t lds_place(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char*)p;
}

// x over the divisor that the factor and shift stand for: exact below 2^31
// (set_divisor in plan_common.h).
__device__ __forceinline__ int quotient(int x, uint32_t mul, int shift) {
  return (int)(__umulhi(2u * (uint32_t)x, mul) >> shift);
}
// Query row of a column.
template <typename Args>
__device__ __forceinline__ int row_of(const Args& a, int col) {
  return quotient(col, a.g_mul, a.g_shift);
}

// Request r of a plan.
__device__ __forceinline__ AttnReq request_of(const AttnPlan& p, int r) { return p.req[r]; }
__device__ __forceinline__ AttnReqBr request_of(const AttnPlanBr& p, int r) { return p.req[r]; }
__device__ __forceinline__ AttnReqBr request_of(const AttnPlanBrPacked& p, int r) { return p.req[r].unpack(); }

// Keys a column of query row `tok` sees: those below lim, and with overlap
// branches also its branch's own rows slo .. shi - 1 (Eq. 1 on the branch's
// sequence: the kept canonical prefix, then the branch's committed lead rows
// causally, then its draft rows seeing the whole branch).  Both clipped to the
// chunk's end.
template <typename Req, bool BR = !__is_same(Req, AttnReq)>
__device__ __forceinline__ void key_limits(const Req& rq, bool valid, int tok, int kend, int& lim, int& slo, int& shi) {
  const int n = rq.nv & 0xffff, nver = (int)((uint32_t)rq.nv >> 16), L = rq.ctx, T = L + n;
  slo = shi = 0;
  if (!valid) {
    lim = 0;
  } else if (!BR || tok < nver) {
    lim = min(kend, tok < nver ? L + tok + 1 : T);
  } else {
    int t = tok - nver, start = L + nver, prefix = nver, lead = 0, rows = n - nver;
    if constexpr (BR) {
      // Word `last` stands for `cnt` branches of its shape whose prefixes
      // grow by `stp`; the words before it for one branch each.
      const int cnt = rq.rep & 0xffff, stp = (rq.rep >> 16) & 0xfff, last = (int)((uint32_t)rq.rep >> 28);
      bool found = false;
#pragma unroll
      for (int bb = 0; bb < 3; ++bb) {
        const int w = rq.br[bb];
        const int rb = w & 0xffff;
        if (w != 0 && !found) {
          const int span = bb == last ? rb * cnt : rb;
          if (t < span) {
            const int k = bb == last ? t / rb : 0;
            t -= k * rb;
            start += k * rb;
            prefix = ((w >> 16) & 0xfff) + k * stp;
            lead = (int)((uint32_t)w >> 28);
            rows = rb;
            found = true;
          } else {
            t -= span;
            start += span;
          }
        }
      }
    }
    lim = min(kend, L + prefix);
    slo = start;
    // empty (shi = slo) when the chunk ends before the branch's rows begin
    shi = max(slo, min(kend, start + (t < lead ? t + 1 : rows)));
  }
}

}  // namespace
}  // namespace rg
