// Hybrid-mask attention over a sliding window with sinks of the bf16 paged cache
// (gfx950), and the merge of it and of attention over the 8-bit cache.
//
// The mathematics is that of attention.hip: S^T = K Q^T, P = exp2 of the scaled
// scores less a running reference, O^T += V^T P^T, in matrix instructions with
// columns (query row, query head) of a KV head.  A row of position p sees, of the
// keys before its own draft block or branch, those of positions > p - size and <
// sink.  A column group visits only the keys that one of its rows may see
// (window_span): the sinks' pages, then those from its first row's window on; keys
// are counted without the gap between, and limits moved alike.  So a group of a
// prompt reads its window, not the context, and no key behind its last row.
//
// Keys pass through LDS, a buffer at a time and two buffers of LDS, in the layout of
// attention.hip: all waves load their share of the next buffer straight into LDS while
// one is computed, and wait for it before the one barrier of a buffer.  V of slots that
// no row may see, which can hold anything, is made zero there.
//
// Softmax online in base 2; the product takes P rounded to bf16 (off by at most
// 2^-8 of each term, as the output's own rounding).  Two sums run in fp32: of P,
// for the lse, and of the rounded P, by which the product is divided, so that the
// weights add up to one.  Runs of a request's keys meet in fp32 in the workspace.
//
// Tokens are bound by the bytes: 64 requests of one, 4096 keys each of 8 heads of 128,
// 1.07 GB in 185 us (5.8 TB/s).  Prompts: 10002 rows over windows of 1024 225 us (740
// TFLOP/s), 8192 rows over all keys 587 (936): products and the softmax of two waves
// overlap in part, and the rest waits for LDS, barriers, starts and ends of groups.  Keys
// through registers into LDS took 236 and 612, V's fragments read after the softmax,
// with a wave's priority raised for the products, 242 and 629 then, scalar loads of the
// page numbers and waits for Q in the loop 228 and 588; K's fragments read a
// sub-tile ahead were 4 % slower, eight waves a group 2 % faster here and up to 50 %
// slower in steps, two sub-tiles at once do not fit the registers.
#include "attention_device.h"
#include "window_internal.h"

namespace rg {
namespace {

// Swizzle of the two 16-byte halves of a dimension row of a V page in LDS.
__device__ __forceinline__ int vswz(int d) { return ((d >> 2) ^ (d >> 3)) & 1; }

template <int D>
struct WindowShape {
  static constexpr int DT = D / 32;
  static constexpr int NW = kWindowWaves, KEYS = window_keys(D);
  static constexpr int PAGES = KEYS / kPageSize;
  static constexpr int BUF = KEYS * D * 2;          // bytes of K, or V, of a buffer
  static constexpr int STATE = 64 * 16 * DT + 192;  // floats of a wave's state
  static constexpr int LDS = 4 * BUF > NW * STATE * 4 ? 4 * BUF : NW * STATE * 4;
};

template <int D, typename Plan>
__global__ __launch_bounds__(64 * kWindowWaves, D == 64 ? 3 : 2) void window_attn_kernel(WindowArgs a, Plan p) {
  using S = WindowShape<D>;
  constexpr int NW = S::NW;
  constexpr bool BR = __is_same(Plan, WindowPlanBr);
  constexpr int DT = S::DT, KSTEPS = D / 16, NCH = D / 8, THREADS = 64 * NW;
  constexpr int UNITS = 2 * D;                     // 16-byte units of K, and of V, of a page and head
  constexpr int PER = S::PAGES * UNITS / THREADS;  // of a thread and buffer
  constexpr int STEP = THREADS / UNITS;            // pages between two of them
  constexpr int PAGE_LDS = 32 * D;                 // bytes of K, or V, of a page in LDS
  static_assert(STEP >= 1 && PER * STEP == S::PAGES && UNITS % 64 == 0, "a wave's unit is of one page");
  __shared__ __attribute__((aligned(16))) char lds[S::LDS];

  const int item = (int)blockIdx.x;
  const int r = find_start(p.num_req, item, [&](int k) { return p.req[k].item_start; });
  const auto rq = p.req[r];
  const int n = rq.nv & 0xffff, nver = (int)((uint32_t)rq.nv >> 16), L = rq.ctx;
  const int g = a.g, M = n * g, tiles = (M + 31) / 32;
  const int nch = rq.runs & 0xffff, run = (int)(rq.runs >> 16) * S::KEYS;
  const int ncg = (tiles + NW - 1) / NW, tpg = (tiles + ncg - 1) / ncg;
  // Items of a request: KV heads, then column groups from the last, which sees most
  // keys, then runs: a group's neighbours, which share most keys, follow on one XCD (8
  // KV heads), and the short groups fill the end.  A prompt of 8192 rows over all keys
  // 1160 us with an XCD's items in a row, 819 dealt to the XCDs in turn, 727 so (8-bit
  // cache 879, 644, 596); over a window of 1024, where groups are alike, 201, 211, 208.
  // A division by the groups only where there are several.
  const int local = item - rq.item_start;
  int cg = 0, c = quotient(local, a.hkv_mul, a.hkv_shift);
  const int hk = local - c * a.hkv;
  if (ncg > 1) {
    const int of = c;
    c /= ncg;
    cg = ncg - 1 - (of - c * ncg);
  }
  const int tile0 = cg * tpg, nct = min(tpg, tiles - tile0);
  const int row0 = row_of(a, tile0 * 32), row1 = row_of(a, min(M, (tile0 + nct) * 32) - 1) + 1;
  const WindowSpan span = window_span<BR>(L, nver, n, row0, row1, a.size, a.sink);
  const int kbeg = c * run, kend = min(span.keys, kbeg + run);

  const int tid = threadIdx.x, lane = tid & 63, lc = lane & 31, lh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  // A wave's column tile ct and key group kgi of kg, the tile's waves `apart` apart.
  const int apart = nct <= 1 ? 1 : nct <= 2 ? 2 : 4, ct = wave % apart, kg = NW / apart, kgi = wave / apart;
  // Columns behind the last are that one again, and not written.
  const bool on = ct < nct, valid = on && (tile0 + ct) * 32 + lc < M;
  const int col = min((tile0 + ct) * 32 + lc, M - 1);
  const int tok = row_of(a, col), hh = col - tok * g;

  // ---- copies
  // By vector loads: waits for LDS would wait for scalar ones too.
  const int32_t* pages = a.page_indices + rq.page_start;
  const int page0 = kbeg / kPageSize, last_page = max((kend - 1) / kPageSize, 0);
  const int head_pages = span.head / kPageSize, gap_pages = span.gap / kPageSize;
  const int my_page = wave * 64 / UNITS, w = tid % UNITS;
  const size_t head_bytes = UNITS * 16, page_bytes = a.hkv * head_bytes;
  // Unit w of a page in LDS is unit w of its memory but for the order in a row of K and
  // of V's pairs; the first key of V's unit.
  const int kslot = w / NCH, vd = w / 2, vhalf = (w & 1) ^ vswz(vd), vkey = 8 * vhalf;
  const uint8_t* kbase = a.k_cache + (size_t)hk * head_bytes + 16 * (w ^ (swap23(kslot) & (NCH - 1)));
  const uint8_t* vbase = a.v_cache + (size_t)hk * head_bytes + 16 * (2 * vd + vhalf);
  int pg[PER];  // pages of the next buffer to be loaded
  // Pages of this wave's units of buffer s; past the run's last page that page again.
  auto pages_of = [&](int s) {
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const int at = min(page0 + s * S::PAGES + my_page + e * STEP, last_page);
      pg[e] = pages[at < head_pages ? at : at + gap_pages];
    }
  };
  // Straight into LDS: a wave's 64 units of 16 bytes lie behind one another there.
  static_assert(4 * S::BUF <= 65536, "load_to_lds reaches 64 KiB");
  const uint32_t at0 = lds_place(lds) + my_page * PAGE_LDS + (wave * 64 % UNITS) * 16;
  auto load = [&](int s) {
    const uint32_t at = at0 + (s & 1) * S::BUF;
#pragma unroll
    for (int e = 0; e < PER; ++e) load_to_lds(at + e * STEP * PAGE_LDS, kbase + (size_t)pg[e] * page_bytes);
#pragma unroll
    for (int e = 0; e < PER; ++e) load_to_lds(at + 2 * S::BUF + e * STEP * PAGE_LDS, vbase + (size_t)pg[e] * page_bytes);
  };
  // Waits for buffer s; V of slots behind the last key, and of those between the sinks
  // and every window, becomes zero.
  auto arrive = [&](int s) {
    // vmcnt(0), as the compiler understands it: else it waits for Q's loads, and with
    // them for the buffer in flight, at every product
    __builtin_amdgcn_s_waitcnt(0x0f70);
    asm volatile("" ::: "memory");
    const int k0 = kbeg + s * S::KEYS;
    if (k0 + S::KEYS > kend || (k0 < span.lo && k0 + S::KEYS > a.sink)) {
      char* vto = lds + (2 + (s & 1)) * S::BUF + my_page * PAGE_LDS + 16 * w;
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        u32x4 v = *(const u32x4*)(vto + e * STEP * PAGE_LDS);
        const int key = k0 + (my_page + e * STEP) * kPageSize + vkey;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          auto seen = [&](int k) { return k < kend && (k < a.sink || k >= span.lo); };
          v[i] &= (seen(key + 2 * i) ? 0xffffu : 0u) | (seen(key + 2 * i + 1) ? 0xffff0000u : 0u);
        }
        *(u32x4*)(vto + e * STEP * PAGE_LDS) = v;
      }
    }
  };
  const int nbuf = kend > kbeg ? (kend - kbeg + S::KEYS - 1) / S::KEYS : 0;
  if (nbuf > 0) {
    pages_of(0);
    load(0);
    if (nbuf > 1) pages_of(1);
  }

  // ---- columns
  bf16x8 qf[KSTEPS];
  {
    const uint16_t* qrow = a.q + ((size_t)(rq.q_start + tok) * a.hq + hk * g + hh) * D;
#pragma unroll
    for (int s = 0; s < KSTEPS; ++s) qf[s] = *(const bf16x8*)(qrow + s * 16 + 8 * lh);
  }
  // Limits of the column: keys lo .. lim - 1 and below the sink, and slo .. shi - 1.
  int lim, slo, shi, lo;
  if constexpr (BR) {
    key_limits<WindowReqBr, true>(rq, true, tok, INT_MAX, lim, slo, shi);
    // a branch row's position: the kept prefix and its place in the branch
    lo = tok < nver ? lim - a.size : min(lim, lim + (L + tok - slo) + 1 - a.size);
    slo -= span.gap;
    shi -= span.gap;
  } else {
    key_limits<WindowReq, false>(rq, true, tok, INT_MAX, lim, slo, shi);
    lo = tok < nver ? lim - a.size : min(L + nver, L + tok + 1 - a.size);
  }
  lim -= span.gap;
  lo = max(lo - span.gap, 0);
  if (lo <= a.sink) lo = 0;
  // Of the wave's columns, from its first and last row: below min_lim no column has
  // an upper limit, from max_lo on none a lower one; nobody sees keys from `end` on,
  // or of sink .. min_lo - 1.  Where branches are among them, bounds of these.
  const int ra = row_of(a, (tile0 + ct) * 32), rb = row_of(a, min(M, (tile0 + ct) * 32 + 32) - 1);
  const bool branched = BR && rb >= nver;
  auto lo_of = [&](int row) { return min(L + nver, L + row + 1 - a.size) - span.gap; };
  const int min_lim = (branched ? L : ra < nver ? L + ra + 1 : L + n) - span.gap;
  const int end = min(kend, (rb < nver ? L + rb + 1 : L + n) - span.gap);
  const int max_lo = lo_of(branched ? n : rb), min_lo = branched ? min(L, L + 1 - a.size) - span.gap : lo_of(ra);

  f32x16 acc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
    for (int i = 0; i < 16; ++i) acc[dt][i] = 0.f;
  float m_run = kNegInf, l_run = 0.f, r_run = 0.f;  // reference, sum of P, of the rounded P
  bool open = true;                                 // some column has no reference yet
  const bf16x2 ones = {(__bf16)1.f, (__bf16)1.f};

  // Byte of this lane's K fragment ks inside a 32-key sub-tile: row swap23(lc),
  // 16-byte chunk (2 ks + lh) ^ (lc % NCH) = 2 (ks ^ kw) + kb.
  const int kx = lc & (NCH - 1), kw = kx >> 1;
  const uint32_t krow = (uint32_t)(swap23(lc) * D * 2 + ((lh ^ (kx & 1)) * 16));

  auto sub_tile = [&](const char* kt, const char* vt, int kbase) {
    f32x16 sc;
    {
      bf16x8 kf[KSTEPS];
#pragma unroll
      for (int ks = 0; ks < KSTEPS; ++ks) kf[ks] = *(const bf16x8*)(kt + krow + ((ks ^ kw) << 5));
      for (int i = 0; i < 16; ++i) sc[i] = 0.f;
      __builtin_amdgcn_sched_barrier(0);  // all reads before the products
#pragma unroll
      for (int ks = 0; ks < KSTEPS; ++ks) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[ks], qf[ks], sc, 0, 0, 0);
    }
    // V's fragments are on their way during the softmax
    bf16x8 vf[2][DT];
#pragma unroll
    for (int pp = 0; pp < 2; ++pp)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const int d = 32 * dt + lc;
        vf[pp][dt] = *(const bf16x8*)(vt + pp * PAGE_LDS + d * 32 + ((lh ^ vswz(d)) * 16));
      }
    __builtin_amdgcn_sched_barrier(0);
    // Keys behind a column's limits, and those before its window.
    const bool behind = kbase + 32 > min_lim, before = kbase < max_lo && kbase + 32 > a.sink;
    if (behind || before) {
      const int base = kbase + 8 * lh;
      uint32_t hidden = 0;
      if (behind) {
        uint32_t seen = places_below(lim - base);
        if constexpr (BR) seen |= places_below(shi - base) & ~places_below(slo - base);
        hidden = ~seen;
      }
      if (before) hidden |= places_below(lo - base) & ~places_below(a.sink - base);
      hide_places(sc, hidden);
    }
    // P against the running reference, a maximum of earlier scores.  A sum of a
    // lane's 16 past 2^12 (overflow included), or a column without a reference,
    // moves the references to the maxima of this tile: P stays below 2^12, and no
    // maximum is taken where nothing moves.
    float sum, rsum;
    u32x4 pk[2];
    auto weigh = [&]() {
      const float mc = (m_run == kNegInf) ? 0.f : m_run * a.scale_log2;
      sum = rsum = 0.f;
#pragma unroll
      for (int pp = 0; pp < 2; ++pp)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[8 * pp + 2 * e], a.scale_log2, -mc));
          const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[8 * pp + 2 * e + 1], a.scale_log2, -mc));
          sum += x + y;
          const uint32_t xy = pack_bf16x2(x, y);
          rsum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, xy), ones, rsum, false);
          pk[pp][e] = xy;
        }
    };
    weigh();
    if (open || __any(!(sum <= 4096.f))) {
      float mx = sc[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) mx = fmaxf(mx, sc[i]);
      const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
      const float m_new = fmaxf(m_run, fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])));
      const float alpha = m_new == kNegInf ? 1.f : __builtin_amdgcn_exp2f((m_run - m_new) * a.scale_log2);
      l_run *= alpha;
      r_run *= alpha;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[dt][i] *= alpha;
      m_run = m_new;
      open = __any(m_new == kNegInf);
      weigh();
    }
    l_run += sum;
    r_run += rsum;
#pragma unroll
    for (int pp = 0; pp < 2; ++pp)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
        acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[pp][dt], __builtin_bit_cast(bf16x8, pk[pp]), acc[dt], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);  // the next sub-tile's loads stay after this one's products
  };
  auto compute = [&](int s) {
    if (!on) return;
    const char* kt = lds + (s & 1) * S::BUF;
    const char* vt = lds + (2 + (s & 1)) * S::BUF;
#pragma unroll 1
    for (int q = 0; q < S::KEYS / 32; ++q) {
      const int kbase = kbeg + s * S::KEYS + 32 * q;
      if (((S::KEYS / 32 * s + q) & (kg - 1)) != kgi || kbase >= end) continue;
      if (kbase + 32 <= min_lo && kbase >= a.sink) continue;
      sub_tile(kt + 64 * q * D, vt + 64 * q * D, kbase);
    }
  };

  // ---- keys
#pragma unroll 1
  for (int s = 0; s < nbuf; ++s) {
    arrive(s);
    lds_barrier();
    if (s + 1 < nbuf) {  // into LDS of buffer s - 1, with which every wave was done before the barrier
      load(s + 1);
      if (s + 2 < nbuf) pages_of(s + 2);
    }
    compute(s);
  }

  l_run += __shfl_xor(l_run, 32);
  r_run += __shfl_xor(r_run, 32);
  // what makes the products sums of weights l; one where nothing was added
  const float whole = r_run > 0.f ? l_run / r_run : 1.f;
  const size_t orow = (size_t)(rq.q_start + tok) * a.hq + hk * g + hh;
  const size_t tile = (size_t)rq.part_start + (size_t)(hk * nch + c) * tiles + (tile0 + ct);
  // Element e of row v of a lane: dim 32 (v / 4) + 8 (v % 4) + 4 lh + e.
  auto put = [&](int v, float4 o, float f) {
    if (nch == 1) {
      const u32x2 y = {pack_bf16x2(o.x * f, o.y * f), pack_bf16x2(o.z * f, o.w * f)};
      *(u32x2*)(a.out + orow * D + 8 * v + 4 * lh) = y;
    } else {
      *(float4*)(a.part_o + tile * 32 * D + (v * 64 + lane) * 4) = make_float4(o.x * f, o.y * f, o.z * f, o.w * f);
    }
  };
  auto put_sums = [&](float m, float l) {
    if (lh != 0) return;
    if (nch > 1) *(float2*)(a.part_ml + 2 * (tile * 32 + lc)) = make_float2(m, l);
    else if (a.lse != nullptr) a.lse[orow] = m * a.sm_scale + __logf(l);
  };
  if (kg == 1) {
    if (!valid) return;
    const float f = nch == 1 ? 1.f / r_run : whole;
#pragma unroll
    for (int v = 0; v < 4 * DT; ++v) {
      float4 o = make_float4(acc[v / 4][4 * (v % 4)], acc[v / 4][4 * (v % 4) + 1], acc[v / 4][4 * (v % 4) + 2],
                             acc[v / 4][4 * (v % 4) + 3]);
      put(v, o, f);
    }
    put_sums(m_run, l_run);
    return;
  }
  // The key groups' states meet in LDS (lane-wise: same columns, same dims), and
  // each group's wave joins a share of the rows.
  lds_barrier();
  float* area = reinterpret_cast<float*>(lds);
  {
    float* state = area + wave * S::STATE;
#pragma unroll
    for (int v = 0; v < 4 * DT; ++v)
      *(float4*)(state + (v * 64 + lane) * 4) = make_float4(acc[v / 4][4 * (v % 4)], acc[v / 4][4 * (v % 4) + 1],
                                                            acc[v / 4][4 * (v % 4) + 2], acc[v / 4][4 * (v % 4) + 3]);
    state[64 * 16 * DT + lane] = m_run;
    state[64 * 16 * DT + 64 + lane] = l_run;
    state[64 * 16 * DT + 128 + lane] = whole;
  }
  lds_barrier();
  if (!valid) return;
  const float* states = area + ct * S::STATE;
  const int stride = apart * S::STATE, share = 4 * DT / kg;
  float m = kNegInf, l = 0.f, weight[NW];
#pragma unroll
  for (int k = 0; k < NW; ++k) {
    weight[k] = k < kg ? states[k * stride + 64 * 16 * DT + lane] : kNegInf;
    m = fmaxf(m, weight[k]);
  }
#pragma unroll
  for (int k = 0; k < NW; ++k) {
    // a group none of whose keys the column sees weighs nothing
    weight[k] = weight[k] == kNegInf ? 0.f : __builtin_amdgcn_exp2f((weight[k] - m) * a.scale_log2);
    if (k < kg) {
      l += weight[k] * states[k * stride + 64 * 16 * DT + 64 + lane];
      weight[k] *= states[k * stride + 64 * 16 * DT + 128 + lane];
    }
  }
  const float f = nch == 1 ? 1.f / l : 1.f;
#pragma unroll 1
  for (int v = kgi * share; v < kgi * share + share; ++v) {
    float4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < NW; ++k) {
      const float4 y = *(const float4*)(states + (k < kg ? k : 0) * stride + (v * 64 + lane) * 4);
      o.x += weight[k] * y.x, o.y += weight[k] * y.y, o.z += weight[k] * y.z, o.w += weight[k] * y.w;
    }
    put(v, o, f);
  }
  if (kgi == 0) put_sums(m, l);
}

// Merge of the runs of split requests, bound by the latency of a load or two and the
// launch (5 to 10 us; 40 requests of 8 to 64 rows 21 us).  Rows of 16 bytes, 4 dims of a column
// each, are counted by (request, KV head, 32-column tile, v); a wave has the 32
// columns of a v, one half of the dims in each half-wave.  PARTS 1: a wave takes
// kWindowMergeRows of a tile's v.  Else the waves of a work group share a v, wave j
// taking runs j, j + PARTS, ..., and meet in LDS.
template <int D, int PARTS, typename Plan>
__global__ __launch_bounds__(64 * kWindowMergeWaves) void window_merge_kernel(WindowArgs a, Plan p) {
  constexpr int DT = D / 32, ROWS = PARTS > 1 ? 1 : kWindowMergeRows, N = 8;  // N: runs in flight
  __shared__ float st[PARTS > 1 ? (PARTS - 1) * 6 * 64 : 1];
  const int part = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int item = PARTS > 1 ? (int)blockIdx.x : ((int)blockIdx.x * kWindowMergeWaves + part) * ROWS;
  if (item >= p.total_comb) return;
  // The request: a lane counts the items of one, and of all before it.
  int r = 0, before = 0;
  for (int base = 0; base < p.num_req; base += 64) {
    const int k = base + ((int)threadIdx.x & 63);
    int count = 0;
    if (k < p.num_req) {
      const uint32_t tiles = ((uint32_t)(p.req[k].nv & 0xffff) * a.g + 31) / 32;
      if ((p.req[k].runs & 0xffff) > 1) count = (int)(tiles * a.hkv * 4 * DT);
    }
    int sum = count;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int x = __shfl_up(sum, off);
      if (((int)threadIdx.x & 63) >= off) sum += x;
    }
    const int all = __shfl(sum, 63);
    if (item < before + all) {
      const int at = __popcll(__ballot(before + sum <= item));
      r = base + at;
      before += __shfl(sum - count, at);
      break;
    }
    before += all;
  }
  r = __builtin_amdgcn_readfirstlane(r);
  const auto rq = p.req[r];
  const int n = rq.nv & 0xffff, g = a.g, M = n * g, tiles = (M + 31) / 32, nch = rq.runs & 0xffff;
  int local = item - __builtin_amdgcn_readfirstlane(before);
  const int v = local % (4 * DT);
  local /= 4 * DT;
  const int hk = local / tiles, tile = local - hk * tiles;
  const size_t base = (size_t)rq.part_start + (size_t)hk * nch * tiles + tile;
  const int lane = threadIdx.x & 63, lc = lane & 31, lh = lane >> 5;
  const int col = tile * 32 + lc;

  float m = kNegInf, l = 0.f, o[ROWS][4] = {};
  auto absorb = [&](const auto& mc, const auto& ls, const auto& oc) {
    constexpr int C = sizeof(ls) / sizeof(ls[0]);
    float m_new = m, weight[C];
#pragma unroll
    for (int u = 0; u < C; ++u) m_new = fmaxf(m_new, mc[u]);
    const float a0 = m == kNegInf ? 0.f : __builtin_amdgcn_exp2f((m - m_new) * a.scale_log2);
    l *= a0;
#pragma unroll
    for (int u = 0; u < C; ++u) {
      weight[u] = mc[u] == kNegInf ? 0.f : __builtin_amdgcn_exp2f((mc[u] - m_new) * a.scale_log2);
      l += weight[u] * ls[u];
    }
#pragma unroll
    for (int q = 0; q < ROWS; ++q)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        o[q][e] *= a0;
#pragma unroll
        for (int u = 0; u < C; ++u) o[q][e] += weight[u] * oc[u][q][e];
      }
    m = m_new;
  };
  if (col < M) {
    for (int c0 = PARTS > 1 ? part : 0; c0 < nch; c0 += N * PARTS) {
      float mc[N], ls[N], x[N][ROWS][4];
#pragma unroll
      for (int u = 0; u < N; ++u) {
        const int c = min(c0 + u * PARTS, nch - 1);  // past the last: that one again, for nothing
        const size_t t0 = base + (size_t)c * tiles;
        const float2 ml = *(const float2*)(a.part_ml + 2 * (t0 * 32 + lc));
        mc[u] = c0 + u * PARTS < nch ? ml.x : kNegInf;
        ls[u] = ml.y;
#pragma unroll
        for (int q = 0; q < ROWS; ++q) {
          const float4 y = *(const float4*)(a.part_o + t0 * 32 * D + ((v + q) * 64 + lane) * 4);
          x[u][q][0] = y.x, x[u][q][1] = y.y, x[u][q][2] = y.z, x[u][q][3] = y.w;
        }
      }
      absorb(mc, ls, x);
    }
  }
  if (PARTS > 1) {
    if (part > 0) {
      float* s = st + (part - 1) * 6 * 64 + lane;
      s[0] = m;
      s[64] = l;
#pragma unroll
      for (int e = 0; e < 4; ++e) s[(2 + e) * 64] = o[0][e];
    }
    __syncthreads();
    if (part > 0) return;
#pragma unroll
    for (int j = 0; j < PARTS - 1; ++j) {
      const float* s = st + j * 6 * 64 + lane;
      const float mc[1] = {s[0]}, ls[1] = {s[64]}, x[1][1][4] = {{{s[2 * 64], s[3 * 64], s[4 * 64], s[5 * 64]}}};
      if constexpr (PARTS > 1) absorb(mc, ls, x);
    }
  }
  if (col >= M) return;
  const int tok = row_of(a, col), hh = col - tok * g;
  const size_t orow = (size_t)(rq.q_start + tok) * a.hq + hk * g + hh;
  const float inv = 1.f / l;
#pragma unroll
  for (int q = 0; q < ROWS; ++q) {
    const u32x2 w = {pack_bf16x2(o[q][0] * inv, o[q][1] * inv), pack_bf16x2(o[q][2] * inv, o[q][3] * inv)};
    const int d = a.scales != nullptr ? kv8_dim(DT, v + q, lh) : 8 * (v + q) + 4 * lh;
    *(u32x2*)(a.out + orow * D + d) = w;
  }
  if (a.lse != nullptr && v == 0 && lh == 0) a.lse[orow] = m * a.sm_scale + __logf(l);
}

template <int D, typename Plan>
hipError_t merge_impl(const WindowArgs& a, const Plan& p, hipStream_t stream) {
  if (p.total_comb == 0) return hipSuccess;
  const dim3 threads(64 * kWindowMergeWaves);
  // Many runs, and few enough rows to be bound by latency: a token over 1024, 4096 and
  // 32768 keys, attention and merge, 12.0, 12.3 and 20.8 us against 13.1, 19.4 and 30.8;
  // more rows or fewer runs 107 and 43 against 94 and 34.
  if (p.max_chunks > 8 && p.total_comb <= 1024)
    hipLaunchKernelGGL((window_merge_kernel<D, kWindowMergeWaves, Plan>), dim3(p.total_comb), threads, 0, stream, a, p);
  else
    hipLaunchKernelGGL((window_merge_kernel<D, 1, Plan>),
                       dim3((p.total_comb + kWindowMergeRows * kWindowMergeWaves - 1) / (kWindowMergeRows * kWindowMergeWaves)),
                       threads, 0, stream, a, p);
  return hipGetLastError();
}
template <int D, typename Plan>
hipError_t launch_impl(const WindowArgs& a, const Plan& p, hipStream_t stream) {
  hipLaunchKernelGGL((window_attn_kernel<D, Plan>), dim3(p.total_items), dim3(64 * kWindowWaves), 0, stream, a, p);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess ? e : merge_impl<D>(a, p, stream);
}

}  // namespace

hipError_t launch_window_attention(const WindowArgs& a, const WindowPlan& p, int head_dim, hipStream_t stream) {
  return head_dim == 128 ? launch_impl<128>(a, p, stream) : launch_impl<64>(a, p, stream);
}
hipError_t launch_window_attention(const WindowArgs& a, const WindowPlanBr& p, int head_dim, hipStream_t stream) {
  return head_dim == 128 ? launch_impl<128>(a, p, stream) : launch_impl<64>(a, p, stream);
}
hipError_t launch_window_merge(const WindowArgs& a, const WindowPlan& p, int head_dim, hipStream_t stream) {
  return head_dim == 128 ? merge_impl<128>(a, p, stream) : merge_impl<64>(a, p, stream);
}
hipError_t launch_window_merge(const WindowArgs& a, const WindowPlanBr& p, int head_dim, hipStream_t stream) {
  return head_dim == 128 ? merge_impl<128>(a, p, stream) : merge_impl<64>(a, p, stream);
}

}  // namespace rg
