// Hybrid-mask attention over the 4-bit paged cache (gfx950): the mask, the
// columns and the split over keys of attention.hip, on a quarter of the bytes.
//
// A work item is (request, KV head, column group of up to 128 columns, run of
// keys).  Its four waves are (32-column tiles) x (key groups): one tile gives
// four key groups, two tiles two each, three or four tiles one.  A wave reads
// its keys' codes straight from the pool into registers, as the block is laid
// out for that: a lane's 16 bytes of K codes are the 32 dims of one scale
// group of its key, and its 16 bytes of V codes are 8 tokens of its D / 32
// dims, the operand rows of S^T = K Q^T and O^T += V^T P^T.  So the main loop
// has no LDS and no barrier, and a decoded element costs half a conversion
// (v_cvt_scalef32_pk_bf16_fp4, which multiplies by the group's scale), for V
// plus half a byte permutation that pairs two tokens.
//
// The dims go through the products in another order than in memory: K step ks
// of S^T holds dims 64 (ks / 4) + 32 lh + 8 (ks % 4) .. + 7 of half-wave lh (Q
// is read alike), and row l of output tile dt is dim DT l + dt, DT = D / 32.
//
// Softmax online in base 2; the running sum adds P in fp32, the product takes
// it rounded to bf16 (off by at most 2^-8 of each term, as the output's own
// rounding).  Runs of a request's keys meet in fp32 in the workspace.
#include "cache_internal.h"
#include "kv4_device.h"

namespace rg {
namespace {

constexpr int kThreads = 64 * kKv4Waves;

// A lane's codes of a 32-key tile: K of its key (scale groups lh, 2 + lh of
// its token), V of tokens 8 lh .. 8 lh + 7 of both pages.
template <int D>
struct Tile4 {
  u32x4 kc[D / 64];
  uint32_t ks;
  uint32_t vc[2][D / 32];
  u32x2 vs[2];
};

template <int D, typename Plan>
__global__ __launch_bounds__(kThreads, 2) void kv4_attn_kernel(Kv4AttnArgs a, Plan p) {
  using B = Kv4<D>;
  constexpr bool BR = !__is_same(Plan, AttnPlan);
  constexpr int DT = D / 32, KSTEPS = D / 16;
  constexpr int SLOT = 64 * 16 * DT + 128;  // floats of a wave's state in LDS
  __shared__ __attribute__((aligned(16))) float area[(kKv4Waves - 1) * SLOT];

  const int item = p.num_req == 1 ? xcd_item(p.grid_items) : (int)blockIdx.x;
  if (item >= p.total_items) return;
  const int r = find_request(p, item, false);
  const auto rq = request_of(p, r);
  const int n = rq.nv & 0xffff, L = rq.ctx, T = L + n;
  const int g = a.g;
  const int M = n * g;
  const int tiles = (M + 31) / 32, ncg = (M + kKv4Cols - 1) / kKv4Cols;
  const int tpg = (tiles + ncg - 1) / ncg;  // tiles are dealt evenly to the column groups
  const int nch = (T + p.chunk - 1) / p.chunk;
  int local = item - rq.item_start;
  const int c = local % nch;
  local /= nch;
  const int hk = local % a.hkv;
  const int cg = local / a.hkv;
  const int kbeg = c * p.chunk, kend = min(T, kbeg + p.chunk);

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lc = lane & 31, lh = lane >> 5;
  const int nct = min(tpg, tiles - cg * tpg);
  const int per = nct == 1 ? 1 : nct == 2 ? 2 : 4;  // waves of one key group
  const int ct = wave % per, kg = kKv4Waves / per, kgi = wave / per;
  if (ct >= nct) return;  // the fourth wave of three tiles; no merge waits for it

  const int col = (cg * tpg + ct) * 32 + lc;
  const bool valid = col < M;
  const int tok = valid ? col / g : 0;
  const int hh = col - tok * g;
  int lim, slo, shi;
  key_limits(rq, valid, tok, kend, lim, slo, shi);
  int wave_min_lim = valid ? lim : kend;
  for (int off = 32; off >= 1; off >>= 1) wave_min_lim = min(wave_min_lim, __shfl_xor(wave_min_lim, off));

  bf16x8 qf[KSTEPS];
  {
    const uint16_t* qrow = a.q + ((size_t)(rq.q_start + tok) * a.hq + hk * g + hh) * D;
#pragma unroll
    for (int s = 0; s < KSTEPS; ++s) {
      u32x4 w = {0u, 0u, 0u, 0u};
      if (valid) w = *(const u32x4*)(qrow + 64 * (s / 4) + 32 * lh + 8 * (s % 4));
      qf[s] = __builtin_bit_cast(bf16x8, w);
    }
  }

  f32x16 acc[DT];
  for (int dt = 0; dt < DT; ++dt)
    for (int i = 0; i < 16; ++i) acc[dt][i] = 0.f;
  float m_run = kNegInf, l_run = 0.f;

  typedef const int32_t __attribute__((address_space(4))) * cpage_ptr;
  const int pg0 = kbeg / kPageSize;
  const int npg = (kend + kPageSize - 1) / kPageSize - pg0;
  const cpage_ptr pages = (cpage_ptr)(a.page_indices + rq.page_start + pg0);
  const uint8_t* pool = a.cache + (size_t)hk * B::BLOCK;
  const size_t page_bytes = (size_t)a.hkv * B::BLOCK;
  const int ktok = swap23(lc) & 15;
  const uint32_t koff = (uint32_t)(ktok * 32 + 16 * lh), ksoff = (uint32_t)B::k_scale(ktok, 0);
  const uint32_t voff = (uint32_t)B::v_unit(8 * lh, lc), vsoff = (uint32_t)B::v_scale(8 * lh, lc * DT / 32);

  // Pages of tile j of the run; one past the run's last page is that page again.
  auto load = [&](int j) {
    Tile4<D> t;
    const uint8_t* b0 = pool + (size_t)pages[2 * j] * page_bytes;
    const uint8_t* b1 = pool + (size_t)pages[min(2 * j + 1, npg - 1)] * page_bytes;
    const uint8_t* bk = lc < 16 ? b0 : b1;
#pragma unroll
    for (int i = 0; i < D / 64; ++i) t.kc[i] = *(const u32x4*)(bk + koff + 512 * i);
    t.ks = D == 128 ? *(const uint32_t*)(bk + ksoff) : *(const uint16_t*)(bk + ksoff);
#pragma unroll
    for (int pp = 0; pp < 2; ++pp) {
      const uint8_t* b = pp ? b1 : b0;
      if constexpr (D == 128) {
        const u32x4 w = *(const u32x4*)(b + voff);
        for (int e = 0; e < 4; ++e) t.vc[pp][e] = w[e];
      } else {
        const u32x2 w = *(const u32x2*)(b + voff);
        for (int e = 0; e < 2; ++e) t.vc[pp][e] = w[e];
      }
      t.vs[pp] = *(const u32x2*)(b + vsoff);
    }
    return t;
  };

  auto compute = [&](Tile4<D>& t, int kbase) {
    f32x16 sc;
    for (int i = 0; i < 16; ++i) sc[i] = 0.f;
    const uint32_t kscale = t.ks >> (8 * lh);
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      const float s = scale_of((kscale >> (16 * i)) & 0xff);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, decode8(t.kc[i][e], s)), qf[4 * i + e], sc,
                                                     0, 0, 0);
    }
    if (kbase + 32 > wave_min_lim) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = kbase + 16 * (i >> 3) + 8 * lh + 4 * ((i >> 2) & 1) + (i & 3);
        if (key >= lim && (!BR || (uint32_t)(key - slo) >= (uint32_t)(shi - slo))) sc[i] = kNegInf;
      }
    }
    if (kbase + 32 > kend) {
      // Slots past the last key may hold anything: scale bytes of infinity
      // become those of small numbers, which weigh zero.
#pragma unroll
      for (int pp = 0; pp < 2; ++pp)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (kbase + 16 * pp + 8 * lh + e >= kend) t.vs[pp][e >> 2] = (t.vs[pp][e >> 2] & ~(0xffu << (8 * (e & 3)))) | (1u << (8 * (e & 3)));
    }
    float mx = sc[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, sc[i]);
    {
      const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
      mx = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
    }
    // The reference maximum moves when a score exceeds it by 2^8 in
    // probability: P stays below 256, and the sums are rescaled rarely.
    const bool grew = mx > m_run + a.rescale_gap;
    if (__any(grew)) {
      const float m_new = grew ? mx : m_run;
      const float alpha = grew ? __builtin_amdgcn_exp2f((m_run - m_new) * a.scale_log2) : 1.f;
      l_run *= alpha;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[dt][i] *= alpha;
      m_run = m_new;
    }
    const float mc = (m_run == kNegInf) ? 0.f : m_run * a.scale_log2;
    u32x4 pk[2];
#pragma unroll
    for (int pp = 0; pp < 2; ++pp)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[8 * pp + 2 * e], a.scale_log2, -mc));
        const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[8 * pp + 2 * e + 1], a.scale_log2, -mc));
        l_run += x + y;
        pk[pp][e] = pack_bf16x2(x, y);
      }
#pragma unroll
    for (int pp = 0; pp < 2; ++pp) {
      u32x4 vf[DT];
#pragma unroll
      for (int w = 0; w < 4; ++w) {  // tokens 2 w, 2 w + 1 of the lane's eight
        const float s0 = scale_of((t.vs[pp][w >> 1] >> (16 * (w & 1))) & 0xff);
        const float s1 = scale_of((t.vs[pp][w >> 1] >> (16 * (w & 1) + 8)) & 0xff);
        auto pair = [&](int dt, uint32_t x, uint32_t y) {  // dims dt, dt + 1 of both tokens
          vf[dt][w] = __builtin_amdgcn_perm(y, x, 0x05040100u);
          vf[dt + 1][w] = __builtin_amdgcn_perm(y, x, 0x07060302u);
        };
        if constexpr (D == 128) {
          const uint32_t u = t.vc[pp][w];
          pair(0, decode2<0>(u, s0), decode2<2>(u, s1));
          pair(2, decode2<1>(u, s0), decode2<3>(u, s1));
        } else {
          const uint32_t u = t.vc[pp][w >> 1];
          if (w & 1) pair(0, decode2<2>(u, s0), decode2<3>(u, s1));
          else pair(0, decode2<0>(u, s0), decode2<1>(u, s1));
        }
      }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
        acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf[dt]),
                                                          __builtin_bit_cast(bf16x8, pk[pp]), acc[dt], 0, 0, 0);
    }
  };

  const int ntile = (kend - kbeg + 31) / 32;
  if (kgi < ntile) {
    Tile4<D> cur = load(kgi);
    for (int j = kgi; j < ntile; j += kg) {
      Tile4<D> next = cur;
      if (j + kg < ntile) next = load(j + kg);
      compute(cur, kbeg + 32 * j);
      cur = next;
    }
  }

  // Element f of run i4 of a lane: dim 8 DT i4 + 4 DT lh + f, f < 4 DT.
  auto at = [&](int i4, int f) { return acc[f % DT][4 * i4 + f / DT]; };
  float l_tot = l_run + __shfl_xor(l_run, 32);
  if (kg > 1) {  // key groups meet in LDS (lane-wise: same columns, same dims)
    if (kgi > 0) {
      float* slot = area + (wave - 1) * SLOT;
#pragma unroll
      for (int v = 0; v < 4 * DT; ++v)
        *(float4*)(slot + (v * 64 + lane) * 4) = make_float4(at(v / DT, 4 * (v % DT)), at(v / DT, 4 * (v % DT) + 1),
                                                             at(v / DT, 4 * (v % DT) + 2), at(v / DT, 4 * (v % DT) + 3));
      slot[64 * 16 * DT + lane] = m_run;
      slot[64 * 16 * DT + 64 + lane] = l_tot;
    }
    __syncthreads();
    if (kgi > 0) return;
    for (int k = 1; k < kg; ++k) {
      const float* slot = area + (wave + k * per - 1) * SLOT;
      const float mk = slot[64 * 16 * DT + lane];
      if (mk == kNegInf) continue;
      const float lk = slot[64 * 16 * DT + 64 + lane];
      const float m_new = fmaxf(m_run, mk);
      const float a0 = __builtin_amdgcn_exp2f((m_run - m_new) * a.scale_log2);
      const float a1 = __builtin_amdgcn_exp2f((mk - m_new) * a.scale_log2);
#pragma unroll
      for (int v = 0; v < 4 * DT; ++v) {
        const float4 o = *(const float4*)(slot + (v * 64 + lane) * 4);
        const float x[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int f = 4 * (v % DT) + e;
          acc[f % DT][4 * (v / DT) + f / DT] = at(v / DT, f) * a0 + x[e] * a1;
        }
      }
      l_tot = l_tot * a0 + lk * a1;
      m_run = m_new;
    }
  }
  if (!valid) return;

  if (nch == 1) {
    const size_t orow = (size_t)(rq.q_start + tok) * a.hq + hk * g + hh;
    const float inv = 1.f / l_tot;
    uint16_t* dst = a.out + orow * D + 4 * DT * lh;
#pragma unroll
    for (int i4 = 0; i4 < 4; ++i4)
#pragma unroll
      for (int f = 0; f < 4 * DT; f += 8) {
        u32x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = pack_bf16x2(at(i4, f + 2 * e) * inv, at(i4, f + 2 * e + 1) * inv);
        *(u32x4*)(dst + 8 * DT * i4 + f) = w;
      }
    if (a.lse != nullptr && lh == 0) a.lse[orow] = m_run * a.sm_scale + __logf(l_tot);
  } else {
    const int M32 = (M + 31) & ~31;
    const size_t tile0 = (size_t)rq.part_start + ((size_t)hk * nch + c) * M32 + (size_t)((cg * tpg + ct) * 32);
    float* dst = a.part_o + tile0 * D;
#pragma unroll
    for (int v = 0; v < 4 * DT; ++v)
      *(float4*)(dst + (v * 64 + lane) * 4) = make_float4(at(v / DT, 4 * (v % DT)), at(v / DT, 4 * (v % DT) + 1),
                                                          at(v / DT, 4 * (v % DT) + 2), at(v / DT, 4 * (v % DT) + 3));
    if (lh == 0) *(float2*)(a.part_ml + 2 * (tile0 + lc)) = make_float2(m_run, l_tot);
  }
}

// Merge of the runs of split requests.  A work item is (request, KV head,
// 32-column tile, row v): 64 rows of 16 bytes, 4 dims of a column each.  PARTS
// threads share a row, part j taking runs j, j + PARTS, ..., and meet in LDS.
template <int D, int PARTS, typename Plan>
__global__ __launch_bounds__(kKv4MergeRows * PARTS) void kv4_merge_kernel(Kv4AttnArgs a, Plan p) {
  constexpr int DT = D / 32;
  __shared__ float st[PARTS > 1 ? (PARTS - 1) * 6 * 64 : 1];
  const int item = xcd_item(p.grid_comb);
  if (item >= p.total_comb) return;
  const int r = find_request(p, item, true);
  const auto rq = p.req[r];
  const int n = rq.nv & 0xffff, T = rq.ctx + n;
  const int g = a.g, M = n * g, M32 = (M + 31) & ~31;
  const int nch = (T + p.chunk - 1) / p.chunk;
  int local = item - rq.comb_start;
  const int v = local % (4 * DT);
  local /= 4 * DT;
  const int tile = local % (M32 / 32), hk = local / (M32 / 32);
  const int lane = threadIdx.x & 63, lc = lane & 31, lh = lane >> 5;
  const int part = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int col = tile * 32 + lc;
  const size_t base = (size_t)rq.part_start + (size_t)hk * nch * M32 + (size_t)tile * 32;

  float m = kNegInf, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  auto absorb = [&](float mc, float lc_, const float (&oc)[4]) {
    if (mc == kNegInf) return;  // no key of that run is visible to the column
    const float m_new = fmaxf(m, mc);
    const float a0 = __builtin_amdgcn_exp2f((m - m_new) * a.scale_log2);
    const float a1 = __builtin_amdgcn_exp2f((mc - m_new) * a.scale_log2);
    l = l * a0 + lc_ * a1;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = o[e] * a0 + oc[e] * a1;
    m = m_new;
  };
  if (col < M) {
    for (int c0 = part; c0 < nch; c0 += 8 * PARTS) {
      float2 ml[8];
      float4 x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int c = c0 + u * PARTS;
        ml[u] = make_float2(kNegInf, 0.f);
        if (c < nch) {
          const size_t t0 = base + (size_t)c * M32;
          ml[u] = *(const float2*)(a.part_ml + 2 * (t0 + lc));
          x[u] = *(const float4*)(a.part_o + t0 * D + (v * 64 + lane) * 4);
        }
      }
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (c0 + u * PARTS < nch) absorb(ml[u].x, ml[u].y, {x[u].x, x[u].y, x[u].z, x[u].w});
    }
  }
  if (PARTS > 1) {
    if (part > 0) {
      float* s = st + (part - 1) * 6 * 64 + lane;
      s[0] = m;
      s[64] = l;
#pragma unroll
      for (int e = 0; e < 4; ++e) s[(2 + e) * 64] = o[e];
    }
    __syncthreads();
    if (part > 0) return;
#pragma unroll
    for (int j = 0; j < PARTS - 1; ++j) {
      const float* s = st + j * 6 * 64 + lane;
      absorb(s[0], s[64], {s[2 * 64], s[3 * 64], s[4 * 64], s[5 * 64]});
    }
  }
  if (col >= M) return;
  const int tok = col / g, hh = col - tok * g;
  const size_t orow = (size_t)(rq.q_start + tok) * a.hq + hk * g + hh;
  const float inv = 1.f / l;
  u32x2 w;
  w[0] = pack_bf16x2(o[0] * inv, o[1] * inv);
  w[1] = pack_bf16x2(o[2] * inv, o[3] * inv);
  *(u32x2*)(a.out + orow * D + 8 * DT * (v / DT) + 4 * DT * lh + 4 * (v % DT)) = w;
  if (a.lse != nullptr && v == 0 && lh == 0) a.lse[orow] = m * a.sm_scale + __logf(l);
}

template <int D, typename Plan>
hipError_t launch_impl(const Kv4AttnArgs& a, const Plan& p, hipStream_t stream) {
  hipLaunchKernelGGL((kv4_attn_kernel<D, Plan>), dim3(p.grid_items), dim3(kThreads), 0, stream, a, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.total_comb == 0) return e;
  if (p.max_chunks > 8)
    hipLaunchKernelGGL((kv4_merge_kernel<D, kKv4MergeParts, Plan>), dim3(p.grid_comb),
                       dim3(kKv4MergeRows * kKv4MergeParts), 0, stream, a, p);
  else
    hipLaunchKernelGGL((kv4_merge_kernel<D, 1, Plan>), dim3(p.grid_comb), dim3(kKv4MergeRows), 0, stream, a, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv4_attention(const Kv4AttnArgs& a, const AttnPlan& p, int head_dim, hipStream_t stream) {
  return head_dim == 128 ? launch_impl<128>(a, p, stream) : launch_impl<64>(a, p, stream);
}
hipError_t launch_kv4_attention(const Kv4AttnArgs& a, const AttnPlanBr& p, int head_dim, hipStream_t stream) {
  return head_dim == 128 ? launch_impl<128>(a, p, stream) : launch_impl<64>(a, p, stream);
}

}  // namespace rg
