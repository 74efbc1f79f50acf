// Rows into a paged cache, bf16 or 8 bits, with the rotation of their positions
// on the way, and rows out of the 8-bit cache.
//
// A row of position p turns the pairs (x, y) of its first dims to (x c - y s,
// y c + x s), c and s the cosine and sine of p inv_freq.  The angle is the exact
// product, up to 55 bits as the sum of two doubles, reduced by multiples of pi / 2
// there, so that a far position turns as exactly as a near one; c and s are rounded to
// fp32 once.  A work group makes the angles of a page's 16 rows once for all of its heads.
//
// 8-bit blocks: the largest magnitude of the new rows of a (page, head) gives
// the block's scale, the one it has is kept where that is larger and older tokens
// stay; those are decoded and rounded again with the new rows (at an unchanged
// scale to the codes they had).  A thread holds 16 elements of a row in
// registers between the two.
//
// A work item is one page that a request's rows touch and 256 dims of KV heads, or some
// heads of q: no two work groups write the same block.  V, which lies by dims,
// and 8-bit blocks go through LDS.
//
// Prompts are bound by their bytes: 36862 rows of 32 + 2 x 8 heads of 128, 906 MB
// read and written, in 168 us (5.4 TB/s; a copy reaches 5.2).  Steps are bound by their
// one chain of page number, angles, rows, LDS and stores, not by the launch: 128 requests
// of 4 to 32 rows, 34 MB, 11.7 us in a captured graph, where an empty kernel of the same
// grid takes 1.8; vector instructions, the angles of every work group among them, fill
// 63 % of the cycles of a compute unit with work.  In 8 bits they come to that for prompts
// too (68 %): 33194 rows of 16 + 2 x 4 heads of 64 38 us.
#include "kv8_device.h"
#include "window_internal.h"

namespace rg {
namespace {

// Sine and cosine of the angle position x freq (to about 2^40 in magnitude), each to
// about 1e-14 of one.  The product is x + rest: a position has 31 bits and a frequency
// 24, a double 53.  With k = round(x 2 / pi) the remainder is x + rest - k pi / 2, pi / 2
// as the sum of two doubles (the first product and difference in one rounding), and
// Taylor's series on [-pi / 4, pi / 4] end below 3e-14 (r^15 / 15!) and 2e-15 (r^16 / 16!).
__device__ __forceinline__ float2 turn_of(double position, double freq) {
  const double x = position * freq, rest = __builtin_fma(position, freq, -x);
  const double k = __builtin_rint(x * 0.63661977236758134308);
  double r = __builtin_fma(-k, 1.57079632679489655800, x) + rest;
  r = __builtin_fma(-k, 6.12323399573676603587e-17, r);
  const double z = r * r;
  double s = 1. / 6227020800.;
  s = __builtin_fma(s, z, -1. / 39916800.);
  s = __builtin_fma(s, z, 1. / 362880.);
  s = __builtin_fma(s, z, -1. / 5040.);
  s = __builtin_fma(s, z, 1. / 120.);
  s = __builtin_fma(s, z, -1. / 6.);
  s = __builtin_fma(s * z, r, r);
  double c = -1. / 87178291200.;
  c = __builtin_fma(c, z, 1. / 479001600.);
  c = __builtin_fma(c, z, -1. / 3628800.);
  c = __builtin_fma(c, z, 1. / 40320.);
  c = __builtin_fma(c, z, -1. / 720.);
  c = __builtin_fma(c, z, 1. / 24.);
  c = __builtin_fma(c, z, -0.5);
  c = __builtin_fma(c, z, 1.);
  const int q = (int)(k - 4. * __builtin_floor(0.25 * k));
  const float fs = (float)(q & 1 ? c : s), fc = (float)(q & 1 ? s : c);
  // quarters: (c, s), (-s, c), (-c, -s), (s, -c)
  return make_float2(q == 1 || q == 2 ? -fc : fc, q >= 2 ? -fs : fs);
}

// Slots s0 .. s1 - 1 of page entry `page` of a request, row0 the row of slot 0
// (it may lie before the request's first).
struct PageItem {
  int pool_page, s0, s1, first_position;
  int local;  // item of the page
  int64_t row0;
};
__device__ __forceinline__ PageItem page_item(const int32_t* page_indices, const AttnPlan& p, int per_page) {
  const int item = blockIdx.x;
  const int r = find_request(p, item, false);
  const AttnReq rq = p.req[r];
  const int n = rq.nv & 0xffff;
  const uint32_t local = item - rq.item_start;
  const uint32_t nth = local / (uint32_t)per_page;
  const int page = (rq.ctx >> 4) + (int)nth;
  PageItem it;
  // from page to page another item first: an XCD has all kinds (eight items a page,
  // the prompts above: 178 us without, 170 with)
  it.local = (int)((local + nth + (uint32_t)r) % (uint32_t)per_page);
  it.pool_page = page_indices[rq.page_start + page];
  it.s0 = max(rq.ctx - page * 16, 0);
  it.s1 = min(rq.ctx + n - page * 16, 16);
  it.first_position = page * 16;
  it.row0 = (int64_t)rq.q_start + (page * 16 - rq.ctx);
  return it;
}

// Sixteen elements of a row: the units of 8 dims c0 and c1 of pair unit m.  Dims
// (j, j + dims / 2) of a pair lie in the two units of one; the units behind the
// turned dims, and all units of neighbours' pairs, go two by two.
struct Units {
  int c0, c1;
  bool halves;  // the two units turn with each other
};
template <bool NEXT>
__device__ __forceinline__ Units units_of(int m, int dims) {
  if (!NEXT && m < dims / 16) return {m, m + dims / 16, true};
  return {2 * m, 2 * m + 1, false};
}

__device__ __forceinline__ void unpack8(u32x4 w, float* x) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = __uint_as_float(w[e] << 16);
    x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
  }
}
__device__ __forceinline__ u32x4 pack8(const float* x) {
  return u32x4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
}

// Turns x (units c0, c1 of a row) by the row's angles; products and sums each
// rounded.  NEXT: neighbours are pairs.
template <bool NEXT>
__device__ __forceinline__ void turn(float (&x)[16], const Units& u, const float2* angle, int dims) {
#pragma clang fp contract(off)
  auto pair = [](float& a, float& b, float2 t) {
    const float ac = a * t.x, bs = b * t.y, bc = b * t.x, as = a * t.y;
    a = ac - bs;
    b = bc + as;
  };
  if constexpr (NEXT) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (8 * (e < 4 ? u.c0 : u.c1) < dims) pair(x[2 * e], x[2 * e + 1], angle[4 * (e < 4 ? u.c0 : u.c1) + (e & 3)]);
  } else if (u.halves) {
#pragma unroll
    for (int e = 0; e < 8; ++e) pair(x[e], x[8 + e], angle[8 * u.c0 + e]);
  }
}

template <int D, bool KV8, bool NEXT>
__global__ __launch_bounds__(kAppendThreads) void append_kernel(AppendArgs a, AttnPlan p) {
  using B = Kv8<D>;
  constexpr int HALF = D / 2;                          // angles of a row at most
  constexpr int PAIRS = D / 16;                        // pair units of a row
  constexpr int HEADS = append_heads(D);               // KV heads of an item
  constexpr int PER = HEADS * 2 * D / kAppendThreads;  // units of a thread; 4 take registers and are slower
  constexpr int BLOCK = 32 * D;                        // bytes of V of a page and head in bf16, or of an 8-bit block
  __shared__ float2 angle[16 * HALF];
  __shared__ __attribute__((aligned(16))) uint8_t lds[HEADS * BLOCK];
  __shared__ float top[PER][kAppendThreads / 64];
  const int kv_items = (a.hkv + HEADS - 1) / HEADS;
  const int q_items = p.cols_per_group > 0 ? (a.hq + p.cols_per_group - 1) / p.cols_per_group : 0;
  const PageItem it = page_item(a.page_indices, p, kv_items + q_items);
  const int tid = threadIdx.x;

  // Angles: a thread has one frequency and every `apart`-th of the page's new rows.
  const int half = a.dims / 2;
  if (half > 0) {
    const int apart = kAppendThreads / half, first = tid / half, j = tid - first * half;
    if (first < apart) {
      const double freq = a.inv_freq[j];
      for (int slot = it.s0 + first; slot < it.s1; slot += apart) {
        const int at = a.positions ? a.positions[it.row0 + slot] : it.first_position + slot;
        angle[slot * HALF + j] = turn_of((double)at, freq);
      }
    }
  }
  __syncthreads();

  if (it.local >= kv_items) {  // heads of q
    const int h0 = (it.local - kv_items) * p.cols_per_group, heads = min(p.cols_per_group, a.hq - h0);
    const int each = heads * PAIRS;  // of a row
    for (int i = it.s0 * each + tid; i < it.s1 * each; i += kAppendThreads) {
      const int slot = i / each, h = h0 + (i - slot * each) / PAIRS, m = i % PAIRS;
      const Units u = units_of<NEXT>(m, a.dims);
      const int64_t row = it.row0 + slot;
      const uint16_t* from = a.q + row * a.q_stride + (size_t)h * D;
      const u32x4 w0 = *(const u32x4*)(from + 8 * u.c0), w1 = *(const u32x4*)(from + 8 * u.c1);
      float x[16];
      unpack8(w0, x);
      unpack8(w1, x + 8);
      turn<NEXT>(x, u, angle + slot * HALF, a.dims);
      uint16_t* to = a.q_out + ((size_t)row * a.hq + h) * D;
      *(u32x4*)(to + 8 * u.c0) = pack8(x);
      *(u32x4*)(to + 8 * u.c1) = pack8(x + 8);
    }
    return;
  }

  const int h0 = it.local * HEADS, heads = min(HEADS, a.hkv - h0);
  const size_t block0 = (size_t)it.pool_page * a.hkv + h0;
  // Pair unit e of this thread: head h0 + head, K (kv 0) or V of slot's row.
  auto head_of = [&](int e) { return (tid + e * kAppendThreads) / (2 * D); };
  const int kv = tid / D & 1, slot = tid % D / PAIRS, m = tid % PAIRS;  // alike for every e
  const Units u = kv ? Units{2 * m, 2 * m + 1, false} : units_of<NEXT>(m, a.dims);
  const bool fresh = slot >= it.s0 && slot < it.s1;
  float x[PER][16];
  {
    u32x4 w[PER][2];
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      w[e][0] = w[e][1] = u32x4{0u, 0u, 0u, 0u};
      if (fresh && head_of(e) < heads) {
        const int64_t row = it.row0 + slot;
        const uint16_t* from = (kv ? a.v + row * a.v_stride : a.k + row * a.k_stride) + (size_t)(h0 + head_of(e)) * D;
        w[e][0] = *(const u32x4*)(from + 8 * u.c0);
        w[e][1] = *(const u32x4*)(from + 8 * u.c1);
      }
    }
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      unpack8(w[e][0], x[e]);
      unpack8(w[e][1], x[e] + 8);
      if (kv == 0 && fresh) turn<NEXT>(x[e], u, angle + slot * HALF, a.dims);
    }
  }
  if constexpr (!KV8) {
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      if (!fresh || head_of(e) >= heads) continue;
      if (kv == 0) {
        uint16_t* to = a.k_cache + ((block0 + head_of(e)) * 16 + slot) * D;
        *(u32x4*)(to + 8 * u.c0) = pack8(x[e]);
        *(u32x4*)(to + 8 * u.c1) = pack8(x[e] + 8);
      } else {
        uint16_t* by_dim = reinterpret_cast<uint16_t*>(lds + head_of(e) * BLOCK) + slot;
#pragma unroll
        for (int i = 0; i < 16; ++i) by_dim[(16 * m + i) * 16] = (uint16_t)(__float_as_uint(x[e][i]) >> 16);  // as it came
      }
    }
    __syncthreads();
    uint16_t* to = a.v_cache + block0 * 16 * D;
    if (it.s0 == 0 && it.s1 == 16) {
      for (int i = tid; i < heads * BLOCK / 16; i += kAppendThreads) *(u32x4*)(to + 8 * i) = *(const u32x4*)(lds + 16 * i);
    } else {
      const int count = it.s1 - it.s0;
      for (int i = tid; i < heads * D * count; i += kAppendThreads) {
        const int row = i / count, s = it.s0 + i - row * count;
        to[(size_t)row * 16 + s] = reinterpret_cast<const uint16_t*>(lds)[row * 16 + s];
      }
    }
  } else {
    // Blocks that are not written whole come in as they are.
    const bool part = it.s0 > 0 || it.s1 < 16;
    uint8_t* to = a.cache + block0 * B::BLOCK;
    if (part)
      for (int i = tid; i < heads * B::BLOCK / 16; i += kAppendThreads) *(u32x4*)(lds + 16 * i) = *(const u32x4*)(to + 16 * i);
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      float t = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float y = fabsf(x[e][i]);
        t = y < __builtin_huge_valf() ? fmaxf(t, y) : t;
      }
      for (int off = 32; off >= 1; off >>= 1) t = fmaxf(t, __shfl_xor(t, off));
      if ((tid & 63) == 0) top[e][tid >> 6] = t;
    }
    __syncthreads();
    float scales[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      if (head_of(e) >= heads) continue;
      const int wave = tid >> 6;
      const float t = D == 128 ? fmaxf(top[e][wave], top[e][wave ^ 1]) : top[e][wave];
      const float old = it.s0 > 0 ? a.scales[2 * (block0 + head_of(e)) + kv] : 0.f;
      const float scale = fmaxf(__uint_as_float((uint32_t)kv8_exponent(__float_as_uint(t)) << 23), old);
      scales[e] = scale;
      if (slot < it.s0) {  // an older token: its codes' values
        const uint8_t* blk = lds + head_of(e) * B::BLOCK;
        uint32_t w[4] = {0u, 0u, 0u, 0u};
        if (kv == 0) {
#pragma unroll
          for (int k = 0; k < 4; ++k) w[k] = *(const uint32_t*)(blk + B::k_code(slot, 8 * (k < 2 ? u.c0 : u.c1) + 4 * (k & 1)));
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) w[i >> 2] |= (uint32_t)blk[B::v_code(slot, 16 * m + i)] << (8 * (i & 3));
        }
        unpack8(decode8_8(w[0], w[1], old), x[e]);
        unpack8(decode8_8(w[2], w[3], old), x[e] + 8);
      }
      if (slot < it.s1) {
        // its exponent is 254 less the scale's: a power of two again
        const float inv = __uint_as_float(0x7f000000u - __float_as_uint(scale));
        uint8_t* blk = lds + head_of(e) * B::BLOCK;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t w = encode4_8(x[e][4 * k], x[e][4 * k + 1], x[e][4 * k + 2], x[e][4 * k + 3], inv);
          if (kv == 0) {
            *(uint32_t*)(blk + B::k_code(slot, 8 * (k < 2 ? u.c0 : u.c1) + 4 * (k & 1))) = w;
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) blk[B::v_code(slot, 16 * m + 4 * k + i)] = (uint8_t)(w >> (8 * i));
          }
        }
      }
    }
    __syncthreads();  // the old scales are read, the codes are in
#pragma unroll
    for (int e = 0; e < PER; ++e)
      if (head_of(e) < heads && slot == it.s0 && m == 0) a.scales[2 * (block0 + head_of(e)) + kv] = scales[e];
    for (int i = tid; i < heads * B::BLOCK / 16; i += kAppendThreads) *(u32x4*)(to + 16 * i) = *(const u32x4*)(lds + 16 * i);
  }
}

// Rows out of the 8-bit cache: an item is a page's kv8_read_heads heads, a thread 16
// elements of a row.  Bound by the bytes, and by the launch where they are few.  Few
// heads an item, not a page's all: append and read of 32768 rows (8 heads of 128, with
// 32 of q) 183 us against 194 with 2 heads, 200 with 4 or 8; 33194 rows of 4 heads of
// 64 55, 53.5 and 58 us with 1, 2 and 4.
template <int D>
__global__ __launch_bounds__(kAppendThreads) void kv8_read_kernel(Kv8ReadArgs a, AttnPlan p) {
  using B = Kv8<D>;
  constexpr int PAIRS = D / 16, HEADS = kv8_read_heads(D);
  __shared__ __attribute__((aligned(16))) uint8_t lds[HEADS * B::BLOCK];
  const PageItem it = page_item(a.page_indices, p, (a.hkv + HEADS - 1) / HEADS);
  const int tid = threadIdx.x, h = tid / (2 * D), kv = tid / D & 1, slot = tid % D / PAIRS, m = tid % PAIRS;
  const int h0 = it.local * HEADS, heads = min(HEADS, a.hkv - h0);
  const size_t block0 = (size_t)it.pool_page * a.hkv + h0;
  const uint8_t* from = a.cache + block0 * B::BLOCK;
  for (int i = tid; i < heads * B::BLOCK / 16; i += kAppendThreads) *(u32x4*)(lds + 16 * i) = *(const u32x4*)(from + 16 * i);
  __syncthreads();
  if (slot < it.s0 || slot >= it.s1 || h >= heads) return;
  // after the barrier: before it the D = 64 rows take 4 us longer
  const float scale = a.scales[2 * (block0 + h) + kv];
  const uint8_t* blk = lds + h * B::BLOCK;
  u32x4 w = {0u, 0u, 0u, 0u};
  if (kv == 0) {
    w = *(const u32x4*)(blk + B::k_code(slot, 16 * m));
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) w[i >> 2] |= (uint32_t)blk[B::v_code(slot, 16 * m + i)] << (8 * (i & 3));
  }
  const int64_t row = it.row0 + slot;
  uint16_t* to = (kv ? a.v + row * a.v_stride : a.k + row * a.k_stride) + (size_t)(h0 + h) * D + 16 * m;
  __builtin_nontemporal_store(decode8_8(w[0], w[1], scale), (u32x4*)to);
  __builtin_nontemporal_store(decode8_8(w[2], w[3], scale), (u32x4*)(to + 8));
}

}  // namespace

template <int D, bool KV8>
static hipError_t launch_impl(const AppendArgs& a, const AttnPlan& p, hipStream_t stream) {
  const dim3 grid(p.total_items), threads(kAppendThreads);
  if (a.interleaved) hipLaunchKernelGGL((append_kernel<D, KV8, true>), grid, threads, 0, stream, a, p);
  else hipLaunchKernelGGL((append_kernel<D, KV8, false>), grid, threads, 0, stream, a, p);
  return hipGetLastError();
}

hipError_t launch_append(const AppendArgs& a, const AttnPlan& p, int head_dim, bool kv8, hipStream_t stream) {
  if (head_dim == 128) return kv8 ? launch_impl<128, true>(a, p, stream) : launch_impl<128, false>(a, p, stream);
  return kv8 ? launch_impl<64, true>(a, p, stream) : launch_impl<64, false>(a, p, stream);
}

hipError_t launch_kv8_read(const Kv8ReadArgs& a, const AttnPlan& p, int head_dim, hipStream_t stream) {
  if (head_dim == 128)
    hipLaunchKernelGGL((kv8_read_kernel<128>), dim3(p.total_items), dim3(kAppendThreads), 0, stream, a, p);
  else
    hipLaunchKernelGGL((kv8_read_kernel<64>), dim3(p.total_items), dim3(kAppendThreads), 0, stream, a, p);
  return hipGetLastError();
}

}  // namespace rg
