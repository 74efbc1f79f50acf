// Rows into the 4-bit paged cache, and out of it.
//
// Per group of 32 elements with largest magnitude a the scale is the power of
// two with 3.5 <= a / scale < 7, so the largest element is off by at most half
// a step of the grid (a tie to 8 cannot occur, 6 saturates only what rounds to
// it); the codes are the nearest elements of 0, .5, 1, 1.5, 2, 3, 4, 6.  As
// the scale is a power of two the quotient is exact and the result does not
// depend on how it is computed.
//
// A work item is one page that a request's rows touch, for all KV heads: no
// two work groups write the same block.  Four lanes hold a group, 8 elements
// (16 bytes) each.
#include "cache_internal.h"
#include "kv4_device.h"

namespace rg {
namespace {

constexpr int kRowThreads = 256;

// Row units of a work item: calls f(slot, h, d0, kv, row) for every 8 elements.
template <int D, typename F>
__device__ __forceinline__ void each_unit(const Kv4RowArgs& a, const AttnPlan& p, F f) {
  const int item = blockIdx.x;
  const int r = find_request(p, item, false);
  const AttnReq rq = p.req[r];
  const int n = rq.nv & 0xffff;
  const int page = (rq.ctx >> 4) + (item - rq.item_start);
  const int t0 = max(rq.ctx, page * 16), cnt = min(rq.ctx + n, page * 16 + 16) - t0;
  const size_t block = (size_t)a.page_indices[rq.page_start + page] * a.hkv;
  const int units = cnt * a.hkv * (D / 8) * 2;
  for (int u = threadIdx.x; u < units; u += kRowThreads) {
    const int c = u % (D / 8);
    const int h = u / (D / 8) % a.hkv;
    const int tok = u / (D / 8) / a.hkv;  // K rows of the page, then V rows
    const int kv = tok >= cnt;
    const int t = t0 + tok - kv * cnt;
    f(a.cache + (block + h) * Kv4<D>::BLOCK, t & 15, h, 8 * c, kv, (int64_t)rq.q_start + (t - rq.ctx));
  }
}

template <int D>
__global__ __launch_bounds__(kRowThreads) void kv4_append_kernel(Kv4RowArgs a, AttnPlan p) {
  using B = Kv4<D>;
  each_unit<D>(a, p, [&](uint8_t* block, int slot, int h, int d0, int kv, int64_t row) {
    const uint16_t* src = kv ? a.v + row * a.v_stride : a.k + row * a.k_stride;
    const u32x4 x = *(const u32x4*)(src + (size_t)h * D + d0);
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) m = max(m, max(x[e] & 0x7fffu, (x[e] >> 16) & 0x7fffu));
    m = max(m, (uint32_t)__shfl_xor((int)m, 1));
    m = max(m, (uint32_t)__shfl_xor((int)m, 2));
    const uint32_t b = (uint32_t)min(max((int)((m + 0x20) >> 7) - 2, 1), 252);
    const uint32_t c = encode8(x, scale_of(b));
    if (kv == 0) {
      *(uint32_t*)(block + B::k_code(slot, d0)) = c;
      if ((d0 & 31) == 0) block[B::k_scale(slot, d0 >> 5)] = (uint8_t)b;
    } else {
#pragma unroll
      for (int e = 0; e < 8 / B::DT; ++e) {
        uint8_t* at = block + B::v_unit(slot, d0 / B::DT + e);
        if constexpr (D == 128) *(uint16_t*)at = (uint16_t)(c >> (16 * e));
        else *at = (uint8_t)(c >> (8 * e));
      }
      if ((d0 & 31) == 0) block[B::v_scale(slot, d0 >> 5)] = (uint8_t)b;
    }
  });
}

template <int D>
__global__ __launch_bounds__(kRowThreads) void kv4_read_kernel(Kv4RowArgs a, AttnPlan p) {
  using B = Kv4<D>;
  each_unit<D>(a, p, [&](const uint8_t* block, int slot, int h, int d0, int kv, int64_t row) {
    uint32_t c, b;
    uint16_t* dst;
    if (kv == 0) {
      c = *(const uint32_t*)(block + B::k_code(slot, d0));
      b = block[B::k_scale(slot, d0 >> 5)];
      dst = a.k + row * a.k_stride;
    } else {
      c = 0;
#pragma unroll
      for (int e = 0; e < 8 / B::DT; ++e) {
        const uint8_t* at = block + B::v_unit(slot, d0 / B::DT + e);
        if constexpr (D == 128) c |= (uint32_t)*(const uint16_t*)at << (16 * e);
        else c |= (uint32_t)*at << (8 * e);
      }
      b = block[B::v_scale(slot, d0 >> 5)];
      dst = a.v + row * a.v_stride;
    }
    *(u32x4*)(dst + (size_t)h * D + d0) = decode8(c, scale_of(b));
  });
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
