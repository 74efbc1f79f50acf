// Attention mass: what the verify rows of a step give to each key,
//   w_j = sum over counted rows i (j <= L + i) and the KV head's query heads
//         of exp(scale q_i . k_j - lse_i),
// added to the key's history, mass_j = (j < L ? decay * mass_j : 0) + w_j.
//
// One pass over K after the attention (whose lse it needs): the products of
// the scores once more, no V.  A work item is (request, KV head, 256 keys); a
// wave holds two 32-key tiles of K in registers as the columns of S = Q K^T,
// so a lane's 16 scores are 16 query columns of one key and the sum over
// columns stays in the lane.  Query columns pass through LDS, 128 at a time.
// No atomics: a key belongs to one lane pair, its sum to one order.
#include "cache_internal.h"
#include "kv4_device.h"

namespace rg {
namespace {

constexpr int kThreads = 64 * kMassWaves;
constexpr int kCols = 128;  // query columns staged at a time

template <int D, bool KV4>
__global__ __launch_bounds__(kThreads, 2) void mass_kernel(MassArgs a, AttnPlan p) {
  constexpr int NCH = D / 8, KSTEPS = D / 16;
  __shared__ __attribute__((aligned(16))) uint16_t qs[kCols * D];
  __shared__ float lse2[kCols];
  const int item = blockIdx.x;
  const int r = find_request(p, item, false);
  const AttnReq rq = p.req[r];
  const int V = (int)((uint32_t)rq.nv >> 16), L = rq.ctx, T = L + V;
  const int g = a.g;
  const int nch = (T + kMassKeys - 1) / kMassKeys;
  const int local = item - rq.item_start;
  const int hk = local / nch, kbeg = local % nch * kMassKeys;
  const int count = a.row_count ? min(max(a.row_count[rq.part_start], 0), V) : V;
  const int M = count * g;

  const int tid = threadIdx.x, lane = tid & 63, lc = lane & 31, lh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  // K of the wave's tiles: keys kbeg + 32 (wave + 4 s) + lc
  bf16x8 kf[kMassSub][KSTEPS];
  const int last_page = (T - 1) / kPageSize;
  const int32_t* pages = a.page_indices + rq.page_start;
#pragma unroll
  for (int s = 0; s < kMassSub; ++s) {
    const int key = kbeg + 32 * (wave + kMassWaves * s) + lc;
    const size_t block = (size_t)pages[min(key >> 4, last_page)] * a.hkv + hk;
    if constexpr (KV4) {
      using B = Kv4<D>;
      const uint8_t* b = static_cast<const uint8_t*>(a.keys) + block * B::BLOCK;
#pragma unroll
      for (int i = 0; i < D / 64; ++i) {
        const u32x4 w = *(const u32x4*)(b + B::k_code(key & 15, 64 * i + 32 * lh));
        const float sc = scale_of(b[B::k_scale(key & 15, 2 * i + lh)]);
#pragma unroll
        for (int e = 0; e < 4; ++e) kf[s][4 * i + e] = __builtin_bit_cast(bf16x8, decode8(w[e], sc));
      }
    } else {
      const uint16_t* b = static_cast<const uint16_t*>(a.keys) + (block * kPageSize + (key & 15)) * D;
#pragma unroll
      for (int ks = 0; ks < KSTEPS; ++ks) kf[s][ks] = *(const bf16x8*)(b + 16 * ks + 8 * lh);
    }
  }

  float w[kMassSub];
  for (int s = 0; s < kMassSub; ++s) w[s] = 0.f;
  // The first columns whose rows see a key of this item.
  const int first = max(0, kbeg - L);
  for (int c0 = (int)((int64_t)first * g / kCols) * kCols; c0 < M; c0 += kCols) {
    __syncthreads();
    for (int u = tid; u < kCols * NCH; u += kThreads) {
      const int row = u / NCH, ch = u % NCH, col = c0 + row;
      u32x4 x = {0u, 0u, 0u, 0u};
      if (col < M) {
        const int tok = col / g;
        x = *(const u32x4*)(a.q + ((size_t)(rq.q_start + tok) * a.hq + hk * g + (col - tok * g)) * D + 8 * ch);
      }
      *(u32x4*)(qs + row * D + ((ch ^ (row & (NCH - 1))) * 8)) = x;
    }
    if (tid < kCols) {
      const int col = c0 + tid, tok = col / g;
      // a column that does not count weighs exp2(-inf) = 0
      lse2[tid] = col < M ? a.lse[(size_t)(rq.q_start + tok) * a.hq + hk * g + (col - tok * g)] * 1.4426950408889634f
                          : -kNegInf;
    }
    __syncthreads();
    for (int t = 0; t < kCols / 32 && c0 + 32 * t < M; ++t) {
      const int low = L + (c0 + 32 * t) / g;                      // last key the tile's first row sees
      const int high = L + (min(c0 + 32 * t + 31, M - 1)) / g;    // ... its last row
      bf16x8 qf[KSTEPS];
#pragma unroll
      for (int ks = 0; ks < KSTEPS; ++ks) {
        const int ch = KV4 ? 8 * (ks / 4) + 4 * lh + ks % 4 : 2 * ks + lh;
        qf[ks] = *(const bf16x8*)(qs + (32 * t + lc) * D + ((ch ^ (lc & (NCH - 1))) * 8));
      }
      float ls[16];
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) {
        const float4 x = *(const float4*)(lse2 + 32 * t + 8 * i4 + 4 * lh);
        ls[4 * i4] = x.x, ls[4 * i4 + 1] = x.y, ls[4 * i4 + 2] = x.z, ls[4 * i4 + 3] = x.w;
      }
#pragma unroll
      for (int s = 0; s < kMassSub; ++s) {
        const int kb = kbeg + 32 * (wave + kMassWaves * s);
        if (kb > high) continue;
        f32x16 sc;
        for (int i = 0; i < 16; ++i) sc[i] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf[ks], kf[s][ks], sc, 0, 0, 0);
        if (kb + 31 > low) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int col = c0 + 32 * t + 8 * (i >> 2) + 4 * lh + (i & 3);
            if (kb + lc > L + col / g) sc[i] = kNegInf;
          }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) w[s] += __builtin_amdgcn_exp2f(__builtin_fmaf(sc[i], a.scale_log2, -ls[i]));
      }
    }
  }
#pragma unroll
  for (int s = 0; s < kMassSub; ++s) {
    const float sum = w[s] + __shfl_xor(w[s], 32);
    const int key = kbeg + 32 * (wave + kMassWaves * s) + lc;
    if (lh == 0 && key < T) {
      float* at = a.mass + ((size_t)pages[key >> 4] * a.hkv + hk) * kPageSize + (key & 15);
      *at = key < L && a.decay != 0.f ? a.decay * *at + sum : sum;
    }
  }
}

}  // namespace

hipError_t launch_mass(const MassArgs& a, const AttnPlan& p, int head_dim, bool kv4, hipStream_t stream) {
  const dim3 grid(p.total_items), block(kThreads);
  if (head_dim == 128 && kv4) hipLaunchKernelGGL((mass_kernel<128, true>), grid, block, 0, stream, a, p);
  else if (head_dim == 128) hipLaunchKernelGGL((mass_kernel<128, false>), grid, block, 0, stream, a, p);
  else if (kv4) hipLaunchKernelGGL((mass_kernel<64, true>), grid, block, 0, stream, a, p);
  else hipLaunchKernelGGL((mass_kernel<64, false>), grid, block, 0, stream, a, p);
  return hipGetLastError();
}

}  // namespace rg
