// Hybrid-mask attention over the 4-bit paged cache (gfx950): the mask, the
// columns and the split over keys of attention.hip, on a quarter of the bytes.
//
// A work item is (request, KV head, column group of up to four 32-column tiles,
// run of keys).  A wave holds one or two of the tiles (two share every decoded
// element: decoding is more than half of a tile's vector instructions) and
// takes every kg-th 32-key tile of the run: one pair of tiles gives the four
// waves four key groups, two pairs two each.  The main loop has no barrier.
//
// A wave copies both blocks of a key tile as they lie in the pool into its own
// ring of two in LDS, by loads that need no register, two tiles ahead; the block
// is laid out for what the lanes take from there: 16 bytes of K codes are the 32
// dims of one scale group of the lane's key, 16 bytes of V codes 8 tokens of its
// D / 32 dims, the operand rows of S^T = K Q^T and O^T += V^T P^T.  A decoded
// element costs half a conversion (v_cvt_scalef32_pk_bf16_fp4, which multiplies
// by the group's scale), for V plus half a byte permutation that pairs two
// tokens.  Q is read from LDS for each key tile; in registers it would leave one
// wave per SIMD.
//
// The dims go through the products in another order than in memory: K step ks
// of S^T holds dims 64 (ks / 4) + 32 lh + 8 (ks % 4) .. + 7 of half-wave lh (Q
// is read alike), and row l of output tile dt is dim DT l + dt, DT = D / 32.
//
// Softmax online in base 2; the product takes P rounded to bf16 (off by at most
// 2^-8 of each term, as the output's own rounding).  Two sums run in fp32: of P,
// for the lse, and of the rounded P, by which the product is divided, so that the
// weights add up to one (a dominant key's V comes out as it is; over the exact
// sum it would be off by up to 2^-8).  The second sum costs 1.5 % of a call at head
// size 128, 5 % at 64, by v_dot2 (by unpacking and adding 4 and 9 %).  No maximum is
// taken where the running reference holds (below).
// Runs of a request's keys meet in fp32 in the workspace.
//
// Measured (query heads / KV heads / head size 32/8/128 unless said):
// one token over 4097 keys 8.0 us + 4.2 of the merge, bound by the chain of its
// start, one key tile a wave, and its end; 16 requests of 1k to 8k keys with
// branches 61 + 9 us; 48 of up to 6k keys, heads 16/4/64, 29 + 6 us; 40 of 8k to
// 32k keys 471 + 21 us, 775 TFLOP/s of bf16 products at 2.0 GHz, to which the
// chip's power limit takes the clock: vector instructions fill 59 % of the
// cycles, products 40 %.  (After half a second of the same; after idle time calls
// take up to 20 % longer.)  Codes read straight into registers measured the same
// within 2 % at head size 128 and leave no registers for a second wave at 64.
#include "cache_internal.h"
#include "kv4_device.h"

namespace rg {
namespace {

constexpr int kThreads = 64 * kKv4Waves;

// Scale byte E of a word as a float whose exponent is the byte, all that the
// conversion takes of its scale (the other bits are the word's other bytes).
template <int E>
__device__ __forceinline__ float scale_at(uint32_t word) {
  return __uint_as_float(E < 3 ? word << (23 - 8 * E) : word >> 1);
}

// What a work group of a wave's tiles works on.
struct Kv4Item {
  int hk, kbeg, kend;  // KV head, keys of the run
  int nch;             // runs that the column group's keys are cut into
  int n, L, M;         // rows, context, columns of the request
  int tile0, nct;      // first tile, tiles of the column group
  int part;            // first partial column of the item
};

template <int D>
struct Kv4Shape {
  static constexpr int DT = D / 32;
  static constexpr int QROW = 2 * D + 16;             // bytes of a column of Q in LDS: 16 more, so that
                                                      // a fragment read meets every bank once
  static constexpr int STATE = 64 * 16 * DT + 192;    // floats of a wave's state of one tile
  static constexpr int RING = 2;                      // key tiles of a wave in LDS
  static constexpr int SLOT = 2 * Kv4<D>::BLOCK;      // bytes of one: two blocks
  // Loads of 16 bytes a lane that fill a slot: FULL of each block, and one of the
  // REST bytes of both; the slot holds them in this order.
  static constexpr int FULL = Kv4<D>::BLOCK / 1024, REST = Kv4<D>::BLOCK % 1024, LOADS = 2 * FULL + 1;
  static_assert(2 * REST <= 1024, "one load");
  // Place of byte x of block pp in a slot.
  static __device__ __forceinline__ int place(int pp, int x) {
    return x < 1024 * FULL ? 1024 * FULL * pp + x : 2 * 1024 * FULL + REST * pp + (x - 1024 * FULL);
  }
  // The rings come first: a load to LDS takes a 16-bit place.  Q behind them.
  static constexpr int Q = kKv4Waves * RING * SLOT;
  static constexpr int LDS = Q + kKv4Cols * QROW;
  static_assert(Q <= 1 << 16, "places of loads to LDS");
  static_assert(kKv4Waves * STATE * 4 <= LDS, "the states fit where Q and the codes were");
};

// The TILES column tiles of this wave: pair `pair` of `np`, key group `kgi`.
template <int D, int TILES, typename Plan, typename Req>
__device__ __forceinline__ void kv4_wave(const Kv4AttnArgs& a, const Req& rq, const Kv4Item& it, int pair, int np, int kgi,
                                         char* lds) {
  using B = Kv4<D>;
  using S = Kv4Shape<D>;
  constexpr bool BR = !__is_same(Plan, AttnPlan);
  constexpr int DT = D / 32;
  const int lane = threadIdx.x & 63, lc = lane & 31, lh = lane >> 5;
  const int kg = kKv4Waves / np, g = a.g;
  const int kbeg = it.kbeg, kend = it.kend;

  typedef const int32_t __attribute__((address_space(4))) * cpage_ptr;
  const int pg0 = kbeg / kPageSize;
  const int npg = (kend + kPageSize - 1) / kPageSize - pg0;
  const cpage_ptr pages = (cpage_ptr)(a.page_indices + rq.page_start + pg0);
  const uint8_t* pool = a.cache + (size_t)it.hk * B::BLOCK;
  const size_t page_bytes = (size_t)a.hkv * B::BLOCK;
  const int ktok = swap23(lc) & 15;
  const char* qlane = lds + S::Q + (2 * pair * 32 + lc) * S::QROW + 64 * lh;

  // The wave's ring of key tiles in LDS: both blocks as they lie in the pool.
  // The loads of a tile go out two tiles ahead; a lane's share of a block is
  // read from LDS when it is needed.
  const int wave = kgi * np + pair;
  char* ring = lds + wave * S::RING * S::SLOT;
  const uint32_t ring_at = lds_place(ring);
  const int koff = S::place(lc >> 4, ktok * 32 + 16 * lh);  // K codes and scales lie in the full part
  const int ksoff = S::place(lc >> 4, B::k_scale(ktok, 0));
  const int voff[2] = {S::place(0, B::v_unit(8 * lh, lc)), S::place(1, B::v_unit(8 * lh, lc))};
  const int vsoff[2] = {S::place(0, B::v_scale(8 * lh, lc * DT / 32)), S::place(1, B::v_scale(8 * lh, lc * DT / 32))};
  const int ntile = (kend - kbeg + 31) / 32;
  // Pages of key tile j; past the run's last page that page again.
  struct Pair {
    int p0, p1;
  };
  auto pages_of = [&](int j) { return Pair{pages[min(2 * j, npg - 1)], pages[min(2 * j + 1, npg - 1)]}; };
  auto load = [&](int slot, Pair x) {
    const uint8_t* b0 = pool + (size_t)x.p0 * page_bytes;
    const uint8_t* b1 = pool + (size_t)x.p1 * page_bytes;
    const uint32_t to = ring_at + slot * S::SLOT;
#pragma unroll
    for (int i = 0; i < S::FULL; ++i) {
      load_to_lds(to + 1024 * i, b0 + 1024 * i, 16 * lane);
      load_to_lds(to + 1024 * (S::FULL + i), b1 + 1024 * i, 16 * lane);
    }
    if (lane < 2 * S::REST / 16)  // from two places: the lanes' own addresses
      load_to_lds(to + 1024 * 2 * S::FULL,
                  (lane < S::REST / 16 ? b0 : b1 - S::REST) + 1024 * S::FULL + 16 * lane);
  };

  Pair ahead{0, 0};
  if (kgi < ntile) {
    load(0, pages_of(kgi));
    if (kgi + kg < ntile) load(1, pages_of(kgi + kg));
    ahead = pages_of(kgi + 2 * kg);
  }
  // Q of the column group, by the whole work group, behind the first codes.
  {
    constexpr int N = kKv4Cols * (D / 8) / kThreads;  // loads of a thread, all before the stores
    u32x4 x[N];
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const int u = threadIdx.x + e * kThreads, row = u / (D / 8), ch = u % (D / 8), col = it.tile0 * 32 + row;
      x[e] = u32x4{0u, 0u, 0u, 0u};
      if (row < 32 * it.nct && col < it.M) {
        const int tok = row_of(a, col);
        x[e] = *(const u32x4*)(a.q + ((size_t)(rq.q_start + tok) * a.hq + it.hk * g + (col - tok * g)) * D + 8 * ch);
      }
    }
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const int u = threadIdx.x + e * kThreads, row = u / (D / 8), ch = u % (D / 8);
      if (row < 32 * it.nct) *(u32x4*)(lds + S::Q + row * S::QROW + 16 * ch) = x[e];
    }
  }
  int lim[TILES], slo[TILES], shi[TILES], min_lim[TILES];
  bool open[TILES];  // some column that sees keys of the run has no reference yet
#pragma unroll
  for (int u = 0; u < TILES; ++u) {
    const int col = (it.tile0 + 2 * pair + u) * 32 + lc;
    key_limits(rq, col < it.M, row_of(a, col), kend, lim[u], slo[u], shi[u]);
    int m = col < it.M ? lim[u] : kend;
    for (int off = 32; off >= 1; off >>= 1) m = min(m, __shfl_xor(m, off));
    min_lim[u] = __builtin_amdgcn_readfirstlane(m);
    open[u] = true;
  }

  f32x16 acc[TILES][DT];
  float m_run[TILES], l_run[TILES], r_run[TILES];  // reference, sum of P, of the rounded P
#pragma unroll
  for (int u = 0; u < TILES; ++u) {
    for (int dt = 0; dt < DT; ++dt)
      for (int i = 0; i < 16; ++i) acc[u][dt][i] = 0.f;
    m_run[u] = kNegInf;
    l_run[u] = r_run[u] = 0.f;
  }

  lds_barrier();

  int slot = 0;
  for (int j = kgi; j < ntile; j += kg, slot ^= 1) {
    const int kbase = kbeg + 32 * j;
    if (j + kg < ntile) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(S::LOADS) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    const char* code = ring + slot * S::SLOT;
    u32x4 kc[D / 64];
#pragma unroll
    for (int i = 0; i < D / 64; ++i) kc[i] = *(const u32x4*)(code + koff + 512 * i);
    const uint32_t kscale = (D == 128 ? *(const uint32_t*)(code + ksoff) : *(const uint16_t*)(code + ksoff)) >> (8 * lh);
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
          qf[s % (AHEAD + 1)][u] = *(const bf16x8*)(qlane + u * 32 * S::QROW + 128 * (s / 4) + 16 * (s % 4));
      };
#pragma unroll
      for (int s = 0; s < AHEAD; ++s) read_q(s);
#pragma unroll
      for (int s = 0; s < N; ++s) {
        if (s + AHEAD < N) read_q(s + AHEAD);
        const bf16x8 kf = __builtin_bit_cast(bf16x8, decode8(kc[s / 4][s % 4], s < 4 ? scale_at<0>(kscale) : scale_at<2>(kscale)));
#pragma unroll
        for (int u = 0; u < TILES; ++u)
          sc[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[s % (AHEAD + 1)][u], sc[u], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    __builtin_amdgcn_s_setprio(0);
    u32x4 pk[TILES][2];
    const bf16x2 ones = {(__bf16)1.f, (__bf16)1.f};
#pragma unroll
    for (int u = 0; u < TILES; ++u) {
      if (kbase + 32 > min_lim[u]) {
        // key - kbase = 8 lh + place, place a constant of i
        const int seen = lim[u] - kbase - 8 * lh, from = slo[u] - kbase - 8 * lh, to = shi[u] - kbase - 8 * lh;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int place = 16 * (i >> 3) + 4 * ((i >> 2) & 1) + (i & 3);
          if (place >= seen && (!BR || place < from || place >= to)) sc[u][i] = kNegInf;
        }
      }
      // P against the running reference, a maximum of earlier scores.  A sum
      // of a lane's 16 past 2^12 (overflow included), or a column without a
      // reference, moves the references to the maxima of this tile: P stays
      // below 2^12, and no maximum is taken where nothing moves.
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
        open[u] = __any(m_new == kNegInf && (lim[u] > kbeg || (BR && shi[u] > max(slo[u], kbeg))));
        weigh();
      }
      l_run[u] += sum;
      r_run[u] += rsum;
    }
    uint32_t vc[2][DT];
    u32x2 vs[2];
#pragma unroll
    for (int pp = 0; pp < 2; ++pp) {
      if constexpr (D == 128) {
        const u32x4 w = *(const u32x4*)(code + voff[pp]);
        for (int e = 0; e < 4; ++e) vc[pp][e] = w[e];
      } else {
        const u32x2 w = *(const u32x2*)(code + voff[pp]);
        for (int e = 0; e < 2; ++e) vc[pp][e] = w[e];
      }
      vs[pp] = *(const u32x2*)(code + vsoff[pp]);
    }
    if (j + 2 * kg < ntile) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the slot is read
      load(slot, ahead);
      ahead = pages_of(j + 3 * kg);
    }
    if (kbase + 32 > kend) {
      // Slots past the last key may hold anything: scale bytes of infinity
      // become those of small numbers, which weigh zero.
#pragma unroll
      for (int pp = 0; pp < 2; ++pp) {
        const int live = min(max(kend - kbase - 16 * pp - 8 * lh, 0), 8);
        const uint64_t keep = live == 8 ? ~0ull : (1ull << (8 * live)) - 1;
        const uint64_t w = (((uint64_t)vs[pp][1] << 32 | vs[pp][0]) & keep) | (0x0101010101010101ull & ~keep);
        vs[pp] = u32x2{(uint32_t)w, (uint32_t)(w >> 32)};
      }
    }
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int pp = 0; pp < 2; ++pp) {
      u32x4 vf[DT];
      // tokens 2 w, 2 w + 1 of the lane's eight
      auto unit = [&](int w, uint32_t codes, float s0, float s1) {
        auto both = [&](int dt, uint32_t x, uint32_t y) {  // dims dt, dt + 1 of both tokens
          vf[dt][w] = __builtin_amdgcn_perm(y, x, 0x05040100u);
          vf[dt + 1][w] = __builtin_amdgcn_perm(y, x, 0x07060302u);
        };
        if constexpr (D == 128) {
          both(0, decode2<0>(codes, s0), decode2<2>(codes, s1));
          both(2, decode2<1>(codes, s0), decode2<3>(codes, s1));
        } else if (w & 1) {
          both(0, decode2<2>(codes, s0), decode2<3>(codes, s1));
        } else {
          both(0, decode2<0>(codes, s0), decode2<1>(codes, s1));
        }
      };
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const uint32_t w = vs[pp][x];
        unit(2 * x, vc[pp][D == 128 ? 2 * x : x], scale_at<0>(w), scale_at<1>(w));
        unit(2 * x + 1, vc[pp][D == 128 ? 2 * x + 1 : x], scale_at<2>(w), scale_at<3>(w));
      }
#pragma unroll
      for (int u = 0; u < TILES; ++u)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
          acc[u][dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf[dt]),
                                                               __builtin_bit_cast(bf16x8, pk[u][pp]), acc[u][dt], 0, 0, 0);
    }
    __builtin_amdgcn_s_setprio(0);
  }

  // The key groups' states meet in LDS, one tile of a wave at a time (lane-wise:
  // same columns, same dims), and each group's wave joins a share of the rows.
  // In loops: this code runs once an item, so its fetch is what it costs.
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
    lds_barrier();  // Q and the codes, or the states before, are no longer read
    if (u == 0) put(acc[0], m_run[0], l_run[0], r_run[0]);
    else if (TILES == 2) put(acc[TILES - 1], m_run[TILES - 1], l_run[TILES - 1], r_run[TILES - 1]);
    lds_barrier();
    const int col = (it.tile0 + 2 * pair + u) * 32 + lc;
    if (u >= TILES || col >= it.M) continue;
    float m = kNegInf, l = 0.f, w[kKv4Waves];
#pragma unroll
    for (int k = 0; k < kKv4Waves; ++k) {
      w[k] = k < kg ? states[k * step + 64 * 16 * DT + lane] : kNegInf;
      m = fmaxf(m, w[k]);
    }
#pragma unroll
    for (int k = 0; k < kKv4Waves; ++k) {
      // a group none of whose keys the column sees weighs nothing
      w[k] = w[k] == kNegInf ? 0.f : __builtin_amdgcn_exp2f((w[k] - m) * a.scale_log2);
      if (k < kg) {
        l += w[k] * states[k * step + 64 * 16 * DT + 64 + lane];
        w[k] *= states[k * step + 64 * 16 * DT + 128 + lane];
      }
    }
    const int tok = row_of(a, col);
    const size_t orow = (size_t)(rq.q_start + tok) * a.hq + it.hk * g + (col - tok * g);
    const size_t tile = (size_t)it.part + (2 * pair + u) * 32;
    const float inv = 1.f / l;
    // Element e of row v of a lane: dim 8 DT (v / DT) + 4 DT lh + 4 (v % DT) + e.
#pragma unroll 1
    for (int v = kgi * share; v < kgi * share + share; ++v) {
      float4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < kKv4Waves; ++k) {
        const float4 x = *(const float4*)(states + (k < kg ? k : 0) * step + (v * 64 + lane) * 4);
        o.x += w[k] * x.x, o.y += w[k] * x.y, o.z += w[k] * x.z, o.w += w[k] * x.w;
      }
      if (it.nch == 1) {
        const u32x2 x = {pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv)};
        *(u32x2*)(a.out + orow * D + 8 * DT * (v / DT) + 4 * DT * lh + 4 * (v % DT)) = x;
      } else {
        *(float4*)(a.part_o + tile * D + (v * 64 + lane) * 4) = o;
      }
    }
    if (kgi == 0 && lh == 0) {
      if (it.nch > 1) *(float2*)(a.part_ml + 2 * (tile + lc)) = make_float2(m, l);
      else if (a.lse != nullptr) a.lse[orow] = m * a.sm_scale + __logf(l);
    }
  }
}

template <int D, typename Plan>
__global__ __launch_bounds__(kThreads, D == 64 ? 3 : 2) void kv4_attn_kernel(Kv4AttnArgs a, Plan p) {
  using S = Kv4Shape<D>;
  __shared__ __attribute__((aligned(16))) char lds[S::LDS];

  const int item = p.num_req == 1 ? xcd_item(p.grid_items) : (int)blockIdx.x;
  if (item >= p.total_items) return;
  const int r = find_request(p, item, false);
  const auto rq = request_of(p, r);
  const int g = a.g;
  Kv4Item it;
  it.n = rq.nv & 0xffff;
  it.L = rq.ctx;
  it.M = it.n * g;
  // Items of the full column groups (groups, then runs, then KV heads), then those
  // of the last one; their partials lie in the same order.  The last one's runs
  // follow from the number of items: an integer division here costs 0.16 us, and an
  // item of one token's batch lasts 7.
  const int T = it.L + it.n;
  const int tiles = (it.M + 31) / 32, full = tiles / kKv4Waves;
  int local = item - rq.item_start;
  it.nct = kKv4Waves;
  it.tile0 = 0;
  it.nch = 0;
  it.part = rq.part_start;
  if (full > 0) {
    it.nch = kv4_run_count(T, kKv4Waves, p.chunk);
    const int group = a.hkv * it.nch;  // items of a column group
    const int group0 = min((int)((uint32_t)local / (uint32_t)group), full);
    local -= group0 * group;
    it.tile0 = group0 * kKv4Waves;
    if (it.nch > 1) it.part += it.tile0 * 32 * group;
  }
  if (it.tile0 == full * kKv4Waves) {
    it.nct = tiles - it.tile0;
    it.nch = quotient(p.req[r + 1].item_start - rq.item_start, a.hkv_mul, a.hkv_shift) - full * it.nch;
  }
  const int run = quotient(local, a.hkv_mul, a.hkv_shift), keys = kv4_run_keys(T, it.nch);
  it.hk = local - run * a.hkv;
  it.kbeg = run * keys;
  it.kend = min(T, it.kbeg + keys);
  if (it.nch > 1) it.part += local * it.nct * 32;

  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int np = it.nct > 2 ? 2 : 1, pair = wave % np;
  if (it.nct - 2 * pair >= 2) kv4_wave<D, 2, Plan>(a, rq, it, pair, np, wave / np, lds);
  else kv4_wave<D, 1, Plan>(a, rq, it, pair, np, wave / np, lds);
}

// Merge of the runs of split requests.  Rows of 16 bytes, 4 dims of a column
// each, are counted by (request, KV head, 32-column tile, v); a wave has the 32
// columns of a v, one half of the dims in each half-wave.  PARTS 1: a wave takes
// kKv4MergeRows of a tile's v, in work groups of four waves (for 6700 of them 9.6 us;
// with one v a wave, bound by the rate at which waves start, 11.6, in work groups
// of one wave 13.0, with four v 10.5).  Else four waves share a v, wave j taking
// runs j, j + PARTS, ..., and meet in LDS.
template <int D, int PARTS, typename Plan>
__global__ __launch_bounds__(64 * kKv4MergeParts) void kv4_merge_kernel(Kv4AttnArgs a, Plan p) {
  constexpr int DT = D / 32;
  __shared__ float st[PARTS > 1 ? (PARTS - 1) * 6 * 64 : 1];
  const int part = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  constexpr int ROWS = PARTS > 1 ? 1 : kKv4MergeRows;  // row numbers of a wave
  const int item = PARTS > 1 ? xcd_item(gridDim.x) : (xcd_item(gridDim.x) * kKv4MergeParts + part) * ROWS;
  if (item >= p.total_comb) return;
  const int r = find_request(p, item, true);
  const auto rq = p.req[r];
  const int n = rq.nv & 0xffff, T = rq.ctx + n;
  const int g = a.g, M = n * g, tiles = (M + 31) / 32, full = tiles / kKv4Waves;
  // merge items: those of the full column groups' tiles where they are split, then the last one's
  int local = item - rq.comb_start;
  const int v = local % (4 * DT);
  local /= 4 * DT;
  int nch = full > 0 ? kv4_run_count(T, kKv4Waves, p.chunk) : 0;
  const int split = nch > 1 ? full * kKv4Waves : 0;  // tiles of the former
  int nct = kKv4Waves, tile, hk;
  size_t base = rq.part_start;
  if (local < split * a.hkv) {
    tile = quotient(local, a.hkv_mul, a.hkv_shift);
    hk = local - tile * a.hkv;
  } else {
    local -= split * a.hkv;
    nct = tiles - full * kKv4Waves;
    tile = quotient(local, a.hkv_mul, a.hkv_shift);
    hk = local - tile * a.hkv;
    tile += full * kKv4Waves;
    if (split) base += (size_t)split * 32 * a.hkv * nch;
    nch = quotient(p.req[r + 1].item_start - rq.item_start, a.hkv_mul, a.hkv_shift) - full * nch;
  }
  const int tile0 = tile / kKv4Waves * kKv4Waves;  // of its group
  if (nct == kKv4Waves) base += (size_t)tile0 * 32 * a.hkv * nch;
  base += (size_t)hk * nct * 32 + (size_t)(tile - tile0) * 32;
  const size_t stride = (size_t)a.hkv * nct * 32;  // partial columns from run to run
  const int lane = threadIdx.x & 63, lc = lane & 31, lh = lane >> 5;
  const int col = tile * 32 + lc;

  float m = kNegInf, l = 0.f, o[ROWS][4] = {};
  // Joins N states; those of runs that the column sees no key of weigh nothing.
  auto absorb = [&](const auto& mc, const auto& lc_, const auto& oc) {
    constexpr int N = sizeof(lc_) / sizeof(lc_[0]);
    float m_new = m, w[N];
#pragma unroll
    for (int u = 0; u < N; ++u) m_new = fmaxf(m_new, mc[u]);
    const float a0 = m == kNegInf ? 0.f : __builtin_amdgcn_exp2f((m - m_new) * a.scale_log2);
    l *= a0;
#pragma unroll
    for (int u = 0; u < N; ++u) {
      w[u] = mc[u] == kNegInf ? 0.f : __builtin_amdgcn_exp2f((mc[u] - m_new) * a.scale_log2);
      l += w[u] * lc_[u];
    }
#pragma unroll
    for (int r4 = 0; r4 < ROWS; ++r4)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        o[r4][e] *= a0;
#pragma unroll
        for (int u = 0; u < N; ++u) o[r4][e] += w[u] * oc[u][r4][e];
      }
    m = m_new;
  };
  if (col < M) {
    constexpr int N = 8;  // runs in flight
    for (int c0 = PARTS > 1 ? part : 0; c0 < nch; c0 += N * PARTS) {
      float mc[N], lc_[N], x[N][ROWS][4];
#pragma unroll
      for (int u = 0; u < N; ++u) {
        const int c = min(c0 + u * PARTS, nch - 1);  // past the last: that one again, for nothing
        const size_t t0 = base + (size_t)c * stride;
        const float2 ml = *(const float2*)(a.part_ml + 2 * (t0 + lc));
        mc[u] = c0 + u * PARTS < nch ? ml.x : kNegInf;
        lc_[u] = ml.y;
#pragma unroll
        for (int r4 = 0; r4 < ROWS; ++r4) {
          const float4 y = *(const float4*)(a.part_o + t0 * D + ((v + r4) * 64 + lane) * 4);
          x[u][r4][0] = y.x, x[u][r4][1] = y.y, x[u][r4][2] = y.z, x[u][r4][3] = y.w;
        }
      }
      absorb(mc, lc_, x);
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
      const float mc[1] = {s[0]}, lc_[1] = {s[64]}, x[1][1][4] = {{{s[2 * 64], s[3 * 64], s[4 * 64], s[5 * 64]}}};
      if constexpr (PARTS > 1) absorb(mc, lc_, x);
    }
  }
  if (col >= M) return;
  const int tok = row_of(a, col), hh = col - tok * g;
  const size_t orow = (size_t)(rq.q_start + tok) * a.hq + hk * g + hh;
  const float inv = 1.f / l;
#pragma unroll
  for (int r4 = 0; r4 < ROWS; ++r4) {
    const u32x2 w = {pack_bf16x2(o[r4][0] * inv, o[r4][1] * inv), pack_bf16x2(o[r4][2] * inv, o[r4][3] * inv)};
    *(u32x2*)(a.out + orow * D + 8 * DT * ((v + r4) / DT) + 4 * DT * lh + 4 * ((v + r4) % DT)) = w;
  }
  if (a.lse != nullptr && v == 0 && lh == 0) a.lse[orow] = m * a.sm_scale + __logf(l);
}

template <int D, typename Plan>
hipError_t launch_impl(const Kv4AttnArgs& a, const Plan& p, hipStream_t stream) {
  hipLaunchKernelGGL((kv4_attn_kernel<D, Plan>), dim3(p.grid_items), dim3(kThreads), 0, stream, a, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.total_comb == 0) return e;
  // Many runs, and few enough rows to be bound by latency: one token over 26 runs
  // takes 4.2 us so, 10.7 with a wave for each row; 40 long requests 75 and 21.
  if (p.max_chunks > 8 && p.grid_comb <= 1024)
    hipLaunchKernelGGL((kv4_merge_kernel<D, kKv4MergeParts, Plan>), dim3(p.grid_comb),
                       dim3(64 * kKv4MergeParts), 0, stream, a, p);
  else
    hipLaunchKernelGGL((kv4_merge_kernel<D, 1, Plan>), dim3((p.total_comb / (kKv4MergeRows * kKv4MergeParts) + 8) / 8 * 8),
                       dim3(64 * kKv4MergeParts), 0, stream, a, p);
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
