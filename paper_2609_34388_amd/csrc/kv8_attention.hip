// Hybrid-mask attention over the 8-bit paged cache (gfx950), over all keys or a
// window: the mask of window_attention.hip, on half of the bytes.
//
// A work item is (request, KV head, column group of up to four 32-column tiles,
// run of keys), a column group's keys those that its rows may see (window_span).
// A wave holds one or two of the tiles (two share every decoded element) and takes
// every kg-th 32-key tile of the run: one pair of tiles gives the four waves four
// key groups, two pairs two each.  The main loop has no barrier.
//
// Codes come straight into registers, a key tile ahead: K's when the tile's scores
// are made, V's when its product is.  The block is laid out for that: 16 bytes of K
// are 16 dims of the lane's key, 8 bytes of V 8 tokens of a dim, so a load of the
// wave is whole lines, and the decoded bytes are the operand rows of S^T = K Q^T and
// O^T += V^T P^T as they lie.  A conversion makes two bf16 of two codes and applies
// the block's scale (exact).  Q is read from LDS for each key tile; in registers it
// would leave one wave per SIMD.  (Through LDS as bf16, as window_attention.hip has
// its keys: 238 us where this takes 199, 127 for 97 and 638 for 565.)
//
// Tokens are bound by the bytes: 128 requests of one over 512 to 8192 keys, 8 KV
// heads of 128, 1.15 GB in 199 us (5.8 TB/s).  Many rows are bound by what a SIMD's two
// waves issue, and by the clock under the power limit: 40 requests of 8 to 64 rows over
// 8192 to 32768 keys 546 us (720 TFLOP/s) at 2.0 GHz, a wave at work 46 % of its time,
// waiting to issue 34 % and for data 20 %; 8 vector instructions a product.
//
// The dims go through the products in another order than in memory: K step s of S^T
// holds dims 32 (s / 2) + 16 lh + 8 (s % 2) .. + 7 of half-wave lh (Q is read alike),
// and row l of output tile dt is dim DT l + dt, DT = D / 32.
//
// Softmax, its sums and the runs' merge: window_attention.hip.
#include "kv8_device.h"
#include "window_internal.h"

namespace rg {
namespace {

constexpr int kThreads = 64 * kKv8Waves;

template <int D>
struct Kv8Shape {
  static constexpr int DT = D / 32;
  static constexpr int QROW = 2 * D + 16;           // bytes of a column of Q in LDS: 16 more, so that a
                                                    // fragment read meets every bank once
  static constexpr int STATE = 64 * 16 * DT + 192;  // floats of a wave's state of one tile
  static constexpr int Q = 32 * kKv8Waves * QROW, STATES = kKv8Waves * STATE * 4;
  static constexpr int LDS = Q > STATES ? Q : STATES;
};

struct Kv8Item {
  int hk, c, nch, kbeg, kend;  // KV head, run of how many, its keys
  int n, nver, L, M, tiles;    // of the request
  int tile0, nct;              // first tile, tiles of the column group
  WindowSpan span;
};

// The TILES column tiles of this wave: pair `pair` of `np`, key group `kgi`.
template <int D, int TILES, typename Req>
__device__ __forceinline__ void kv8_wave(const WindowArgs& a, const Req& rq, const Kv8Item& it, int pair, int np, int kgi,
                                         char* lds) {
  using S = Kv8Shape<D>;
  constexpr bool BR = __is_same(Req, WindowReqBr);
  constexpr int DT = S::DT, KU = D / 32, VU = D / 64;  // 16-byte units of K, and of V of a block, of a lane
  const int lane = threadIdx.x & 63, lc = lane & 31, lh = lane >> 5;
  const int kg = kKv8Waves / np, g = a.g, L = it.L, n = it.n, nver = it.nver;
  const int kbeg = it.kbeg, kend = it.kend;
  const WindowSpan& span = it.span;

  typedef const int32_t __attribute__((address_space(4))) * cpage_ptr;
  typedef const float __attribute__((address_space(4))) * cscale_ptr;
  const cpage_ptr pages = (cpage_ptr)(a.page_indices + rq.page_start);
  const int page0 = kbeg / kPageSize, last_page = max((kend - 1) / kPageSize, 0);
  const int head_pages = span.head / kPageSize, gap_pages = span.gap / kPageSize;
  const uint8_t* pool = a.k_cache + (size_t)it.hk * Kv8<D>::BLOCK;
  const size_t page_bytes = (size_t)a.hkv * Kv8<D>::BLOCK;
  const int ktok = swap23(lc) & 15;
  const uint32_t koff = ktok * 32 + 16 * lh, voff = 16 * D + (lh * D + DT * lc) * 8;
  const char* qlane = lds + (2 * pair * 32 + lc) * S::QROW + 32 * lh;
  const int ntile = kend > kbeg ? (kend - kbeg + 31) / 32 : 0;

  // Pages of key tile j; past the run's last page that page again.
  struct Pair {
    int p0, p1;
  };
  auto pages_of = [&](int j) {
    const int x = min(page0 + 2 * j, last_page), y = min(page0 + 2 * j + 1, last_page);
    return Pair{pages[x < head_pages ? x : x + gap_pages], pages[y < head_pages ? y : y + gap_pages]};
  };
  u32x4 kc[KU], vc[2][VU];
  float kscale, vscale[2];
  auto load_k = [&](Pair x) {
    const uint8_t* at = pool + (size_t)(lc < 16 ? x.p0 : x.p1) * page_bytes + koff;
#pragma unroll
    for (int i = 0; i < KU; ++i) kc[i] = *(const u32x4*)(at + 512 * i);
    const float s0 = ((cscale_ptr)a.scales)[2 * ((size_t)x.p0 * a.hkv + it.hk)];
    const float s1 = ((cscale_ptr)a.scales)[2 * ((size_t)x.p1 * a.hkv + it.hk)];
    kscale = lc < 16 ? s0 : s1;
  };
  auto load_v = [&](Pair x) {
#pragma unroll
    for (int pp = 0; pp < 2; ++pp) {
      const int page = pp ? x.p1 : x.p0;
#pragma unroll
      for (int i = 0; i < VU; ++i) vc[pp][i] = *(const u32x4*)(pool + (size_t)page * page_bytes + voff + 16 * i);
      vscale[pp] = ((cscale_ptr)a.scales)[2 * ((size_t)page * a.hkv + it.hk) + 1];
    }
  };
  Pair now{0, 0}, ahead{0, 0};
  if (kgi < ntile) {
    now = pages_of(kgi);
    load_k(now);
    load_v(now);
    ahead = pages_of(kgi + kg);
  }
  // Q of the column group, by the whole work group, behind the first codes.
  {
    constexpr int N = 32 * kKv8Waves * (D / 8) / kThreads;  // loads of a thread, all before the stores
    const int rows = it.nct > 2 ? 128 : 32 * it.nct;  // three tiles: of the fourth too
    u32x4 x[N];
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const int u = threadIdx.x + e * kThreads, row = u / (D / 8), ch = u % (D / 8);
      const int col = min(it.tile0 * 32 + row, it.M - 1);  // behind the last that one again
      if (row < rows) {
        const int tok = row_of(a, col);
        x[e] = *(const u32x4*)(a.q + ((size_t)(rq.q_start + tok) * a.hq + it.hk * g + (col - tok * g)) * D + 8 * ch);
      }
    }
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const int u = threadIdx.x + e * kThreads, row = u / (D / 8), ch = u % (D / 8);
      if (row < rows) *(u32x4*)(lds + row * S::QROW + 16 * ch) = x[e];
    }
  }
  // Limits of a lane's columns: keys lo .. lim - 1 and below the sink, and slo .. shi
  // - 1.  Over the wave: below min_lim no column has an upper limit, from max_lo on
  // none a lower one.
  int lim[TILES], slo[TILES], shi[TILES], lo[TILES];
  int min_lim = INT_MAX, max_lo = 0;
#pragma unroll
  for (int u = 0; u < TILES; ++u) {
    const int first = (it.tile0 + 2 * pair + u) * 32, col = min(first + lc, it.M - 1);
    const int tok = row_of(a, col);
    key_limits<Req, BR>(rq, true, tok, INT_MAX, lim[u], slo[u], shi[u]);
    if constexpr (BR)  // a branch row's position: the kept prefix and its place in the branch
      lo[u] = tok < nver ? lim[u] - a.size : min(lim[u], lim[u] + (L + tok - slo[u]) + 1 - a.size);
    else
      lo[u] = tok < nver ? lim[u] - a.size : min(L + nver, L + tok + 1 - a.size);
    lim[u] -= span.gap;
    slo[u] -= span.gap;
    shi[u] -= span.gap;
    lo[u] = max(lo[u] - span.gap, 0);
    if (lo[u] <= a.sink) lo[u] = 0;
    // of the tile's first and last row; bounds where branches are among them
    const int ra = row_of(a, min(first, it.M - 1)), rb = row_of(a, min(first + 31, it.M - 1));
    const bool branched = BR && rb >= nver;
    min_lim = min(min_lim, (branched ? L : ra < nver ? L + ra + 1 : L + n) - span.gap);
    max_lo = max(max_lo, min(L + nver, L + (branched ? n : rb) + 1 - a.size) - span.gap);
  }

  f32x16 acc[TILES][DT];
  float m_run[TILES], l_run[TILES], r_run[TILES];  // reference, sum of P, of the rounded P
  bool open[TILES];                                // some column has no reference yet
#pragma unroll
  for (int u = 0; u < TILES; ++u) {
    for (int dt = 0; dt < DT; ++dt)
      for (int i = 0; i < 16; ++i) acc[u][dt][i] = 0.f;
    m_run[u] = kNegInf;
    l_run[u] = r_run[u] = 0.f;
    open[u] = true;
  }

  lds_barrier();

#pragma unroll 1
  for (int j = kgi; j < ntile; j += kg) {
    const int kbase = kbeg + 32 * j;
    f32x16 sc[TILES];
#pragma unroll
    for (int u = 0; u < TILES; ++u)
      for (int i = 0; i < 16; ++i) sc[u][i] = 0.f;
    // Products before the other wave's softmax: a product occupies the matrix core
    // for longer than its issue takes, the softmax fills what is between.
    __builtin_amdgcn_s_setprio(1);
    {
      // Q fragments are read two K steps ahead
      constexpr int N = D / 16, AHEAD = 2;
      bf16x8 qf[AHEAD + 1][TILES];
      auto read_q = [&](int s) {
#pragma unroll
        for (int u = 0; u < TILES; ++u)
          qf[s % (AHEAD + 1)][u] = *(const bf16x8*)(qlane + u * 32 * S::QROW + 64 * (s / 2) + 16 * (s % 2));
      };
#pragma unroll
      for (int s = 0; s < AHEAD; ++s) read_q(s);
#pragma unroll
      for (int s = 0; s < N; ++s) {
        if (s + AHEAD < N) read_q(s + AHEAD);
        const bf16x8 kf = __builtin_bit_cast(bf16x8, decode8_8(kc[s / 2][2 * (s % 2)], kc[s / 2][2 * (s % 2) + 1], kscale));
#pragma unroll
        for (int u = 0; u < TILES; ++u)
          sc[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[s % (AHEAD + 1)][u], sc[u], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    __builtin_amdgcn_s_setprio(0);
    load_k(ahead);
    u32x4 pk[TILES][2];
    const bf16x2 ones = {(__bf16)1.f, (__bf16)1.f};
#pragma unroll
    for (int u = 0; u < TILES; ++u) {
      // Keys behind a column's limits, and those before its window.
      const bool behind = kbase + 32 > min_lim, before = kbase < max_lo && kbase + 32 > a.sink;
      if (behind || before) {
        const int base = kbase + 8 * lh;
        uint32_t hidden = 0;
        if (behind) {
          uint32_t seen = places_below(lim[u] - base);
          if constexpr (BR) seen |= places_below(shi[u] - base) & ~places_below(slo[u] - base);
          hidden = ~seen;
        }
        if (before) hidden |= places_below(lo[u] - base) & ~places_below(a.sink - base);
        hide_places(sc[u], hidden);
      }
      // P against the running reference, a maximum of earlier scores.  A sum of a
      // lane's 16 past 2^12 (overflow included), or a column without a reference,
      // moves the references to the maxima of this tile: P stays below 2^12, and no
      // maximum is taken where nothing moves.
      float sum, rsum;
      auto weigh = [&]() {
        const float mc = (m_run[u] == kNegInf) ? 0.f : m_run[u] * a.scale_log2;
        sum = rsum = 0.f;
#pragma unroll
        for (int pp = 0; pp < 2; ++pp)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[u][8 * pp + 2 * e], a.scale_log2, -mc));
            const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[u][8 * pp + 2 * e + 1], a.scale_log2, -mc));
            sum += x + y;
            const uint32_t xy = pack_bf16x2(x, y);
            rsum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, xy), ones, rsum, false);
            pk[u][pp][e] = xy;
          }
      };
      weigh();
      if (open[u] || __any(!(sum <= 4096.f))) {
        float mx = sc[u][0];
#pragma unroll
        for (int i = 1; i < 16; ++i) mx = fmaxf(mx, sc[u][i]);
        const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
        const float m_new = fmaxf(m_run[u], fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])));
        const float alpha = m_new == kNegInf ? 1.f : __builtin_amdgcn_exp2f((m_run[u] - m_new) * a.scale_log2);
        l_run[u] *= alpha;
        r_run[u] *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[u][dt][i] *= alpha;
        m_run[u] = m_new;
        open[u] = __any(m_new == kNegInf);
        weigh();
      }
      l_run[u] += sum;
      r_run[u] += rsum;
    }
    // V of slots behind the last key, and of those between the sinks and every
    // window, is zero.
    if (kbase + 32 > kend || (kbase < span.lo && kbase + 32 > a.sink)) {
#pragma unroll
      for (int pp = 0; pp < 2; ++pp) {
        const int key = kbase + 16 * pp + 8 * lh;
        uint32_t keep[2] = {0u, 0u};
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (key + i < kend && (key + i < a.sink || key + i >= span.lo)) keep[i >> 2] |= 0xffu << (8 * (i & 3));
#pragma unroll
        for (int i = 0; i < VU; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) vc[pp][i][e] &= keep[e & 1];
      }
    }
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int pp = 0; pp < 2; ++pp)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const bf16x8 vf = __builtin_bit_cast(
            bf16x8, decode8_8(vc[pp][dt / 2][2 * (dt % 2)], vc[pp][dt / 2][2 * (dt % 2) + 1], vscale[pp]));
#pragma unroll
        for (int u = 0; u < TILES; ++u)
          acc[u][dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, __builtin_bit_cast(bf16x8, pk[u][pp]), acc[u][dt], 0, 0, 0);
      }
    __builtin_amdgcn_s_setprio(0);
    load_v(ahead);
    ahead = pages_of(j + 2 * kg);
  }

  // The key groups' states meet in LDS, one tile of a wave at a time (lane-wise:
  // same columns, same dims), and each group's wave joins a share of the rows.
  // In loops: this code runs once an item, so its fetch is what it costs.
  const int wave = kgi * np + pair;
  float* area = reinterpret_cast<float*>(lds);
  const float* states = area + pair * S::STATE;  // of the pair, np apart
  const int step = np * S::STATE, share = 4 * DT / kg;
  auto put = [&](const f32x16(&o)[DT], float m, float l, float rounded) {
    float* state = area + wave * S::STATE;
#pragma unroll
    for (int v = 0; v < 4 * DT; ++v) {
      const int i4 = v / DT, f = 4 * (v % DT);
      *(float4*)(state + (v * 64 + lane) * 4) =
          make_float4(o[f % DT][4 * i4 + f / DT], o[(f + 1) % DT][4 * i4 + (f + 1) / DT],
                      o[(f + 2) % DT][4 * i4 + (f + 2) / DT], o[(f + 3) % DT][4 * i4 + (f + 3) / DT]);
    }
    state[64 * 16 * DT + lane] = m;
    l += __shfl_xor(l, 32);
    rounded += __shfl_xor(rounded, 32);
    state[64 * 16 * DT + 64 + lane] = l;
    // what makes the products sums of weights l; one where nothing was added
    state[64 * 16 * DT + 128 + lane] = rounded > 0.f ? l / rounded : 1.f;
  };
#pragma unroll 1
  for (int u = 0; u < 2; ++u) {
    if (u == 1 && it.nct == 1) break;
    lds_barrier();  // Q, or the states before, are no longer read
    if (u == 0) put(acc[0], m_run[0], l_run[0], r_run[0]);
    else if (TILES == 2) put(acc[TILES - 1], m_run[TILES - 1], l_run[TILES - 1], r_run[TILES - 1]);
    lds_barrier();
    const int col = (it.tile0 + 2 * pair + u) * 32 + lc;
    if (u >= TILES || col >= it.M) continue;
    float m = kNegInf, l = 0.f, w[kKv8Waves];
#pragma unroll
    for (int k = 0; k < kKv8Waves; ++k) {
      w[k] = k < kg ? states[k * step + 64 * 16 * DT + lane] : kNegInf;
      m = fmaxf(m, w[k]);
    }
#pragma unroll
    for (int k = 0; k < kKv8Waves; ++k) {
      // a group none of whose keys the column sees weighs nothing
      w[k] = w[k] == kNegInf ? 0.f : __builtin_amdgcn_exp2f((w[k] - m) * a.scale_log2);
      if (k < kg) {
        l += w[k] * states[k * step + 64 * 16 * DT + 64 + lane];
        w[k] *= states[k * step + 64 * 16 * DT + 128 + lane];
      }
    }
    const int tok = row_of(a, col);
    const size_t orow = (size_t)(rq.q_start + tok) * a.hq + it.hk * g + (col - tok * g);
    const size_t tile = (size_t)rq.part_start + (size_t)(it.hk * it.nch + it.c) * it.tiles + (it.tile0 + 2 * pair + u);
    const float inv = 1.f / l;
#pragma unroll 1
    for (int v = kgi * share; v < kgi * share + share; ++v) {
      float4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < kKv8Waves; ++k) {
        const float4 x = *(const float4*)(states + (k < kg ? k : 0) * step + (v * 64 + lane) * 4);
        o.x += w[k] * x.x, o.y += w[k] * x.y, o.z += w[k] * x.z, o.w += w[k] * x.w;
      }
      if (it.nch == 1) {
        const u32x2 x = {pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv)};
        *(u32x2*)(a.out + orow * D + kv8_dim(DT, v, lh)) = x;
      } else {
        *(float4*)(a.part_o + tile * 32 * D + (v * 64 + lane) * 4) = o;
      }
    }
    if (kgi == 0 && lh == 0) {
      if (it.nch > 1) *(float2*)(a.part_ml + 2 * (tile * 32 + lc)) = make_float2(m, l);
      else if (a.lse != nullptr) a.lse[orow] = m * a.sm_scale + __logf(l);
    }
  }
}

template <int D, typename Plan>
__global__ __launch_bounds__(kThreads, D == 64 ? 3 : 2) void kv8_attn_kernel(WindowArgs a, Plan p) {
  __shared__ __attribute__((aligned(16))) char lds[Kv8Shape<D>::LDS];
  constexpr bool BR = __is_same(Plan, WindowPlanBr);

  const int item = (int)blockIdx.x;
  const int r = find_start(p.num_req, item, [&](int k) { return p.req[k].item_start; });
  const auto rq = p.req[r];
  Kv8Item it;
  it.n = rq.nv & 0xffff;
  it.nver = (int)((uint32_t)rq.nv >> 16);
  it.L = rq.ctx;
  it.M = it.n * a.g;
  it.tiles = (it.M + 31) / 32;
  it.nch = rq.runs & 0xffff;
  const int ncg = (it.tiles + kKv8Waves - 1) / kKv8Waves;
  // Items of a request: KV heads, then column groups from the last, which sees most
  // keys, then runs; a division by the groups only where there are several.
  const int local = item - rq.item_start;
  int cg = 0;
  it.c = quotient(local, a.hkv_mul, a.hkv_shift);
  it.hk = local - it.c * a.hkv;
  if (ncg > 1) {
    const int of = it.c;
    it.c /= ncg;
    cg = ncg - 1 - (of - it.c * ncg);
  }
  it.tile0 = cg * kKv8Waves;
  it.nct = min(kKv8Waves, it.tiles - it.tile0);
  const int row0 = row_of(a, it.tile0 * 32), row1 = row_of(a, min(it.M, (it.tile0 + it.nct) * 32) - 1) + 1;
  it.span = window_span<BR>(it.L, it.nver, it.n, row0, row1, a.size, a.sink);
  const int run = (int)(rq.runs >> 16) * kKv8Step;
  it.kbeg = it.c * run;
  it.kend = min(it.span.keys, it.kbeg + run);

  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  // Two tiles a wave where there are two, though each alone would give more key
  // groups: 16 requests with branches 95 us against 107, 40 long ones 547 against 622;
  // a few requests, bound by latency, 16 to 26 us against 15 to 25.
  const int np = it.nct > 2 ? 2 : 1, pair = wave % np;
  // Of three tiles the second pair's waves make one twice: alone it would run ahead
  // of the other's, and each would read the keys from memory (2.66 us against 2.34 for
  // 128 keys, a compute unit full).
  if (it.nct >= 2) kv8_wave<D, 2>(a, rq, it, pair, np, wave / np, lds);
  else kv8_wave<D, 1>(a, rq, it, pair, np, wave / np, lds);
}

template <typename Plan>
hipError_t launch_any(const WindowArgs& a, const Plan& p, int head_dim, hipStream_t stream) {
  if (head_dim == 128)
    hipLaunchKernelGGL((kv8_attn_kernel<128, Plan>), dim3(p.total_items), dim3(kThreads), 0, stream, a, p);
  else
    hipLaunchKernelGGL((kv8_attn_kernel<64, Plan>), dim3(p.total_items), dim3(kThreads), 0, stream, a, p);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess ? e : launch_window_merge(a, p, head_dim, stream);
}

}  // namespace

hipError_t launch_kv8_attention(const WindowArgs& a, const WindowPlan& p, int head_dim, hipStream_t stream) {
  return launch_any(a, p, head_dim, stream);
}
hipError_t launch_kv8_attention(const WindowArgs& a, const WindowPlanBr& p, int head_dim, hipStream_t stream) {
  return launch_any(a, p, head_dim, stream);
}

}  // namespace rg
