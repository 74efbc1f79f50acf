// Rows into the 4-bit paged cache, and out of it.
//
// Per group of 32 elements with largest magnitude a the scale is the power of
// two with 3.5 <= a / scale < 7, so the largest element is off by at most half
// a step of the grid (a tie to 8 cannot occur, 6 saturates only what rounds to
// it); the codes are the nearest elements of 0, .5, 1, 1.5, 2, 3, 4, 6.  As
// the scale is a power of two the quotient is exact and the result does not
// depend on how it is computed.  A group with an infinity or a NaN, which the
// grid has no element for, gets the scale byte that makes every element a NaN.
//
// A work item is one page that a request's rows touch, of plan.chunk neighbouring
// KV heads (blocks that lie together): no two work groups write the same block,
// and blocks go through LDS, where their codes change between the order of rows
// and that of the block.  A block whose tokens are all new is written with
// 16-byte stores; of any other only the new tokens' bytes are.  Bound by the
// bytes, at short calls by the launch.  128 requests' steps 6.6 us in and 4.9 out;
// 28 thousand rows of 8 heads of 128 36 us in (4.1 TB/s: more reads than writes), 27
// out (5.4 TB/s); 400 thousand rows out 410 us (5.4 TB/s; 483 with a head a work
// group, which starts four times as many).  Rows are written past the caches: with
// ordinary stores the appends and evictions between them took 9 us longer.
#include "cache_internal.h"
#include "kv4_device.h"

namespace rg {
namespace {

constexpr int kRowThreads = 256;

// The tokens of a work item: slots s0 .. s1 - 1 of heads h .. h + heads - 1, rows row0 ...
struct RowItem {
  size_t block;  // of the pool, head h's
  int s0, s1, h, heads;
  int64_t row0;  // row of slot 0 (may lie before the request's first)
};
__device__ __forceinline__ RowItem row_item(const Kv4RowArgs& a, const AttnPlan& p) {
  const int item = blockIdx.x;
  const int r = find_request(p, item, false);
  const AttnReq rq = p.req[r];
  const int n = rq.nv & 0xffff;
  const uint32_t local = item - rq.item_start, each = ((uint32_t)a.hkv + p.chunk - 1) / p.chunk;
  const int page = (rq.ctx >> 4) + local / each;
  RowItem it;
  it.h = local % each * p.chunk;
  it.heads = min(p.chunk, a.hkv - it.h);
  it.block = (size_t)a.page_indices[rq.page_start + page] * a.hkv + it.h;
  it.s0 = max(rq.ctx - page * 16, 0);
  it.s1 = min(rq.ctx + n - page * 16, 16);
  it.row0 = (int64_t)rq.q_start + (page * 16 - rq.ctx);
  return it;
}

// Units of 8 elements of K, or V, of a block; a thread has PER of both, those of
// thread + e kRowThreads.
template <int D>
struct Units {
  static constexpr int N = 16 * D / 8, PER = 2 * N / kRowThreads;
  int kv, slot, d0;
  __device__ __forceinline__ explicit Units(int e) {
    const int u = threadIdx.x + e * kRowThreads;
    kv = u / N;
    slot = u % N / (D / 8);
    d0 = u % (D / 8) * 8;
  }
};

template <int D>
__global__ __launch_bounds__(kRowThreads) void kv4_append_kernel(Kv4RowArgs a, AttnPlan p) {
  using B = Kv4<D>;
  constexpr int PER = Units<D>::PER;
  __shared__ __attribute__((aligned(16))) uint8_t lds[kRowHeads * B::BLOCK];
  const RowItem it = row_item(a, p);
  u32x4 x[kRowHeads][PER];  // all loads first
#pragma unroll
  for (int h = 0; h < kRowHeads; ++h)
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const Units<D> u(e);
      x[h][e] = u32x4{0u, 0u, 0u, 0u};
      if (h < it.heads && u.slot >= it.s0 && u.slot < it.s1) {
        const uint16_t* rows = u.kv ? a.v + (it.row0 + u.slot) * a.v_stride : a.k + (it.row0 + u.slot) * a.k_stride;
        x[h][e] = *(const u32x4*)(rows + (size_t)(it.h + h) * D + u.d0);
      }
    }
#pragma unroll
  for (int h = 0; h < kRowHeads; ++h) {
    if (h >= it.heads) break;
    uint8_t* blk = lds + h * B::BLOCK;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const Units<D> u(i);
      const u32x4 w = x[h][i];
      uint32_t m = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) m = max(m, max(w[e] & 0x7fffu, (w[e] >> 16) & 0x7fffu));
      m = max(m, (uint32_t)__shfl_xor((int)m, 1));  // four lanes hold a group
      m = max(m, (uint32_t)__shfl_xor((int)m, 2));
      const uint32_t scale = (uint32_t)min(max((int)((m + 0x20) >> 7) - 2, 1), 252);
      const uint32_t c = encode8(w, scale_of(scale)), b = m >= 0x7f80u ? kNanScale : scale;
      if (u.kv == 0) {
        *(uint32_t*)(blk + B::k_code(u.slot, u.d0)) = c;
        if ((u.d0 & 31) == 0) blk[B::k_scale(u.slot, u.d0 >> 5)] = (uint8_t)b;
      } else {
#pragma unroll
        for (int e = 0; e < 8 / B::DT; ++e) {
          uint8_t* at = blk + B::v_unit(u.slot, u.d0 / B::DT + e);
          if constexpr (D == 128) *(uint16_t*)at = (uint16_t)(c >> (16 * e));
          else *at = (uint8_t)(c >> (8 * e));
        }
        if ((u.d0 & 31) == 0) blk[B::v_scale(u.slot, u.d0 >> 5)] = (uint8_t)b;
      }
    }
  }
  __syncthreads();
  uint8_t* dst = a.cache + it.block * B::BLOCK;
  if (it.s0 == 0 && it.s1 == 16) {
    for (int u = threadIdx.x; u < it.heads * B::BLOCK / 16; u += kRowThreads)
      *(u32x4*)(dst + 16 * u) = *(const u32x4*)(lds + 16 * u);
    return;
  }
  constexpr int N = Units<D>::N;
  for (int u = threadIdx.x; u < it.heads * N; u += kRowThreads) {
    const int slot = u % N / (D / 8), c = u % (D / 8), d0 = 8 * c, block = u / N * B::BLOCK;
    if (slot < it.s0 || slot >= it.s1) continue;
    const uint8_t* from = lds + block;
    uint8_t* to = dst + block;
    *(uint32_t*)(to + B::k_code(slot, d0)) = *(const uint32_t*)(from + B::k_code(slot, d0));
#pragma unroll
    for (int e = 0; e < 8 / B::DT; ++e) {
      const int at = B::v_unit(slot, d0 / B::DT + e);
      if constexpr (D == 128) *(uint16_t*)(to + at) = *(const uint16_t*)(from + at);
      else to[at] = from[at];
    }
    if (c < B::DT) to[B::k_scale(slot, c)] = from[B::k_scale(slot, c)];
    else if (c < 2 * B::DT) to[B::v_scale(slot, c - B::DT)] = from[B::v_scale(slot, c - B::DT)];
  }
}

template <int D>
__global__ __launch_bounds__(kRowThreads) void kv4_read_kernel(Kv4RowArgs a, AttnPlan p) {
  using B = Kv4<D>;
  __shared__ __attribute__((aligned(16))) uint8_t lds[kRowHeads * B::BLOCK];
  const RowItem it = row_item(a, p);
  const uint8_t* src = a.cache + it.block * B::BLOCK;
  constexpr int LOADS = (kRowHeads * B::BLOCK / 16 + kRowThreads - 1) / kRowThreads;
  const int units = it.heads * B::BLOCK / 16;
  u32x4 x[LOADS];
#pragma unroll
  for (int e = 0; e < LOADS; ++e)
    if (threadIdx.x + e * kRowThreads < units) x[e] = *(const u32x4*)(src + 16 * (threadIdx.x + e * kRowThreads));
#pragma unroll
  for (int e = 0; e < LOADS; ++e)
    if (threadIdx.x + e * kRowThreads < units) *(u32x4*)(lds + 16 * (threadIdx.x + e * kRowThreads)) = x[e];
  __syncthreads();
  for (int h = 0; h < it.heads; ++h) {
    const uint8_t* blk = lds + h * B::BLOCK;
#pragma unroll
    for (int i = 0; i < Units<D>::PER; ++i) {
      const Units<D> u(i);
      if (u.slot < it.s0 || u.slot >= it.s1) continue;
      uint32_t c, b;
      uint16_t* rows;
      if (u.kv == 0) {
        c = *(const uint32_t*)(blk + B::k_code(u.slot, u.d0));
        b = blk[B::k_scale(u.slot, u.d0 >> 5)];
        rows = a.k + (it.row0 + u.slot) * a.k_stride;
      } else {
        c = 0;
#pragma unroll
        for (int e = 0; e < 8 / B::DT; ++e) {
          const uint8_t* at = blk + B::v_unit(u.slot, u.d0 / B::DT + e);
          if constexpr (D == 128) c |= (uint32_t)*(const uint16_t*)at << (16 * e);
          else c |= (uint32_t)*at << (8 * e);
        }
        b = blk[B::v_scale(u.slot, u.d0 >> 5)];
        rows = a.v + (it.row0 + u.slot) * a.v_stride;
      }
      __builtin_nontemporal_store(decode8(c, scale_of(b)), (u32x4*)(rows + (size_t)(it.h + h) * D + u.d0));
    }
  }
}

}  // namespace

hipError_t launch_kv4_append(const Kv4RowArgs& a, const AttnPlan& p, int head_dim, hipStream_t stream) {
  if (head_dim == 128)
    hipLaunchKernelGGL((kv4_append_kernel<128>), dim3(p.total_items), dim3(kRowThreads), 0, stream, a, p);
  else
    hipLaunchKernelGGL((kv4_append_kernel<64>), dim3(p.total_items), dim3(kRowThreads), 0, stream, a, p);
  return hipGetLastError();
}

hipError_t launch_kv4_read(const Kv4RowArgs& a, const AttnPlan& p, int head_dim, hipStream_t stream) {
  if (head_dim == 128)
    hipLaunchKernelGGL((kv4_read_kernel<128>), dim3(p.total_items), dim3(kRowThreads), 0, stream, a, p);
  else
    hipLaunchKernelGGL((kv4_read_kernel<64>), dim3(p.total_items), dim3(kRowThreads), 0, stream, a, p);
  return hipGetLastError();
}

}  // namespace rg
