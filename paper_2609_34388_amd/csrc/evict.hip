// Eviction of tokens from a paged cache by score.
//
// Per (request, KV head) the L tokens are cut to the `keep` that are
// protected (first positions, latest positions) or have the largest scores.
// Tokens do not keep their order (attention does not look at it, and the
// positions pool says which token a slot holds), so only the kept tokens
// behind slot `keep` move: into the evicted slots before it, both in ascending
// order.  No slot is both read and written, so moves run in any order.
//
// select: one work group per (request, KV head), its slots' scores as ordered
// 32-bit words (protected tokens the largest word) in registers.  A radix
// selection of 11, 11 and 10 bits finds the word of the keep-th largest, ending
// where all tokens of a prefix are kept; then each wave goes over a contiguous
// part of the slots: ties are taken from the lowest slot on, holes and movers get
// their ranks from wave ballots.  It writes for every kept slot which token it
// takes, if any.  Bound by latency: a few thousand tokens give one compute unit
// work that 255 others cannot share.  One request of 4128 tokens 11.4 us, 16 of 1k
// to 8k 13.3, 40 of 8k to 32k 50 (8 heads each; the start 1.2 us, the first bits 1.8,
// each later pass 1.1, ranks and lists 4).  Comparing the last few hundred
// candidates each with all, instead of further bits, took 2.0 us; copies of the
// bins, so that fewer lanes meet in one, changed nothing.
//
// move: a wave per page of the kept slots, which writes their positions and
// fills the page's holes: mass and K rows as they are.  In V, where a 16-byte
// unit holds eight tokens of few dims, a token is a 2-byte piece (1 byte, 4-bit
// at head size 64) of every unit: the wave reads its sources' units whole, all
// at once, and moves the pieces in registers.  Bound by the lines that the pieces
// lie in, of which a page with any hole has most: 16 requests cut to 3/4, bf16,
// 300 MB of lines in 69 us; 40 long ones cut to half, 4-bit, 1.2 GB in 342 us.
// Pieces written one by one, without reading the page's units: 67 and 353 us.
#include <type_traits>

#include "cache_internal.h"
#include "kv4_device.h"

namespace rg {
namespace {

constexpr int kWaves = kEvictThreads / 64;
constexpr int kBins = 2048;
static_assert(kBins == 2 * kEvictThreads, "two bins a thread");

// Workspace of a (request, head): for every kept slot the token that moves
// there, as its slot (-1: none) and the page of the pool it is in; then the
// slots of the holes and of the movers, in order.
struct MoveList {
  int2* take;
  int32_t *hole, *mover;
};
__device__ __forceinline__ MoveList move_list(const EvictArgs& a, const EvictReq& q, int hk) {
  int32_t* at = a.ws + q.ws_start + (size_t)hk * evict_words(q.keep, q.most);
  return {reinterpret_cast<int2*>(at), at + 2 * (size_t)q.keep, at + 2 * (size_t)q.keep + q.most};
}

// Sum over this lane and those before it (data moves within the vector unit).
__device__ __forceinline__ uint32_t scan64(uint32_t x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // row_shr:1, 2, 4, 8: rows of 16
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast:15: row 0 to 1, 2 to 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // row_bcast:31: both to 2 and 3
  return x;
}

// Sum of the counts of the waves before `wave`, and of all: one read and a scan,
// where a loop over the waves would wait for each of its reads.
__device__ __forceinline__ uint2 before_wave(const uint32_t (&counts)[kWaves], int wave) {
  const int lane = threadIdx.x & 63;
  const uint32_t upto = scan64(lane < kWaves ? counts[lane] : 0u);
  const uint32_t before = __builtin_amdgcn_readlane(upto, wave > 0 ? wave - 1 : 0);
  return make_uint2(wave > 0 ? before : 0u, __builtin_amdgcn_readlane(upto, kWaves - 1));
}

// Lanes of a mask before this one, added to `x`.
__device__ __forceinline__ uint32_t count_below(uint64_t mask, uint32_t x) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, x));
}

// KW: words of a thread in registers; slots past them are read again in each pass.
// 64 registers let two work groups share a compute unit (40 long requests: 59 us
// where they do not, 51).  As few words as the longest request needs: every step
// is in the code as often as there are words (4128 tokens: 12.3 us with 8, 16.5 with 32).
template <int KW>
__global__ __launch_bounds__(kEvictThreads, 8) void evict_select_kernel(EvictArgs a, EvictPlan p) {
  __shared__ uint32_t hist[kBins];  // later the lists of holes and movers, where they fit
  __shared__ uint32_t s_wave[kWaves], s_word, s_left, s_in;
  __shared__ uint32_t s_count[3][kWaves];
  const int r = (int)blockIdx.x / a.hkv, hk = (int)blockIdx.x % a.hkv;
  const EvictReq q = p.req[r];
  const int L = q.ctx, keep = q.keep, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int32_t* pages = a.page_indices + q.page_start;

  auto place = [&](int j) { return ((size_t)pages[j >> 4] * a.hkv + hk) * kPageSize + (j & 15); };
  auto position = [&](int j, size_t at) { return j < q.tracked ? a.positions[at] : j + q.evicted; };
  if (q.most == 0) {  // nothing moves: every token stays, or none does
    for (int j = q.tracked + tid; j < keep; j += kEvictThreads) a.positions[place(j)] = j + q.evicted;
    return;
  }
  const int recent_from = L + q.evicted - a.recent;  // positions from here on are protected
  // Slots of this wave: 64 i + lane from first on.
  const int steps = (L + kEvictThreads - 1) / kEvictThreads;
  const int first = wave * steps * 64, j0 = first + lane;
  // A slot's score as a word of the same order: protected tokens the largest.
  constexpr uint32_t kProtected = 0xffffffffu;
  auto word = [&](float score, int pos) {
    const uint32_t u = __float_as_uint(score + 0.f);  // -0 becomes 0
    return pos < a.sink || pos >= recent_from ? kProtected : (u & 0x80000000u) ? ~u : u | 0x80000000u;
  };
  auto fetch = [&](int i) {
    const int j = min(j0 + 64 * i, L - 1);
    const size_t at = place(j);
    return word(a.score[at], position(j, at));
  };
  // Page numbers of a batch, then its scores (and positions): two round trips.
  // Slots past the last repeat it and are never asked for (see each()).
  constexpr int kBatch = KW < 8 ? KW : KW < 32 ? 8 : 4;  // 32 held words leave registers for four
  uint32_t held[KW];
#pragma unroll
  for (int i0 = 0; i0 < KW; i0 += kBatch) {
    if (i0 >= steps) break;
    size_t at[kBatch];
    float score[kBatch];
    int pos[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int j = min(j0 + 64 * (i0 + i), L - 1);
      at[i] = place(j);
      pos[i] = j + q.evicted;
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) score[i] = a.score[at[i]];
    if (q.tracked > 0) {
#pragma unroll
      for (int i = 0; i < kBatch; ++i)
        if (min(j0 + 64 * (i0 + i), L - 1) < q.tracked) pos[i] = a.positions[at[i]];
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) held[i0 + i] = word(score[i], pos[i]);
  }
  // Calls f(i, word, in range) over the wave's slots, in order.
  auto each = [&](auto f) {
#pragma unroll
    for (int i = 0; i < KW; ++i)
      if (i < steps) f(i, held[i], j0 + 64 * i < L);
    for (int i = KW; i < steps; ++i) f(i, fetch(i), j0 + 64 * i < L);
  };

  // Of the tokens whose words begin with the prefix (under the mask) `left` are
  // kept; where that is all `in` of them the other bits need not be looked at.
  uint32_t prefix = 0, mask = 0, left = (uint32_t)keep, in_prefix = 0;
  auto pass = [&](auto shift_of) {  // true: the next bits have to be looked at
    constexpr int shift = decltype(shift_of)::value;
    constexpr uint32_t bins = shift == 0 ? 1024u : 2048u;
    hist[tid] = 0;
    hist[tid + kEvictThreads] = 0;
    __syncthreads();
    if constexpr (shift == 21) {  // protected tokens, one word for all, are counted by the wave
      uint32_t safe = 0;
      each([&](int, uint32_t u, bool in) {
        safe += __popcll(__ballot(in && u == kProtected));
        if (in && u != kProtected) atomicAdd(&hist[u >> shift], 1u);
      });
      if (lane == 0 && safe > 0) atomicAdd(&hist[bins - 1], safe);
    } else {
      each([&](int, uint32_t u, bool in) {
        if (in && (u & mask) == prefix) atomicAdd(&hist[(u >> shift) & (bins - 1)], 1u);
      });
    }
    __syncthreads();
    // from the top bin down, two bins a thread
    const uint32_t b0 = hist[kBins - 1 - 2 * tid], b1 = hist[kBins - 2 - 2 * tid];
    const uint32_t upto = scan64(b0 + b1);
    if (lane == 63) s_wave[wave] = upto;
    __syncthreads();
    const uint32_t before = upto - b0 - b1 + before_wave(s_wave, wave).x;
    if (before < left && left <= before + b0 + b1) {
      const bool second = left > before + b0;
      s_word = (uint32_t)(kBins - 1 - 2 * tid) - second;
      s_left = left - before - (second ? b0 : 0u);
      s_in = second ? b1 : b0;
    }
    __syncthreads();
    prefix |= s_word << shift;
    mask = ~0u << shift;
    left = s_left;
    in_prefix = s_in;
    return left != in_prefix;
  };
  if (pass(std::integral_constant<int, 21>()) && pass(std::integral_constant<int, 10>()))
    pass(std::integral_constant<int, 0>());

  // Ties: those that share the prefix and lie in waves before this one.
  uint32_t tie0 = 0;
  if (left < in_prefix) {
    uint32_t ties = 0;
    each([&](int, uint32_t u, bool in) { ties += __popcll(__ballot(in && (u & mask) == prefix)); });
    if (lane == 0) s_count[0][wave] = ties;
    __syncthreads();
    tie0 = before_wave(s_count[0], wave).x;
  }
  // Lanes whose slot is kept; `tie` counts the ties so far.
  auto kept_lanes = [&](uint32_t u, bool in, uint32_t& tie) -> uint64_t {
    uint64_t kept = __ballot(in && (u & mask) > prefix);
    const uint64_t eq = __ballot(in && (u & mask) == prefix);
    if (eq != 0) {
      const uint32_t n = (uint32_t)__popcll(eq);
      if (tie + n <= left) kept |= eq;
      else if (tie < left) kept |= eq & __ballot(count_below(eq, tie) < left);
      tie += n;
    }
    return kept;
  };
  // Lanes of step i whose slot lies before `keep`.
  auto low_lanes = [&](int i) -> uint64_t {
    const int n = keep - first - 64 * i;
    return n >= 64 ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1;
  };

  // Masks held, in scalar registers and, where these are full, in lanes of a vector
  // register (the compiler's own spills: 10 words with 8 held slots, 60 with 16, 132
  // with 32, none of them in memory); the others are made again.
  constexpr int kMasks = KW < 16 ? KW : 16;
  uint64_t kept[kMasks];
  uint32_t tie = tie0, holes = 0, movers = 0, tie_past = 0;  // tie_past: at the first of those
  each([&](int i, uint32_t u, bool in) {
    if (i == kMasks) tie_past = tie;
    const uint64_t m = kept_lanes(u, in, tie), low = low_lanes(i);
    if (i < kMasks) kept[i < kMasks ? i : 0] = m;
    holes += (uint32_t)__popcll(low & ~m);
    movers += (uint32_t)__popcll(m & ~low);
  });
  if (lane == 0) {
    s_count[1][wave] = holes;
    s_count[2][wave] = movers;
  }
  __syncthreads();
  uint32_t hole0 = before_wave(s_count[1], wave).x;
  const uint2 moves = before_wave(s_count[2], wave);
  uint32_t mover0 = moves.x;
  const uint32_t count = moves.y;
  const MoveList list = move_list(a, q, hk);
  const bool near = count <= kBins / 2;  // the lists fit LDS: no trip to memory and back
  auto visit = [&](int i, uint64_t m) {
    const int j = j0 + 64 * i;
    const uint64_t low = low_lanes(i), hole = low & ~m, mover = m & ~low;
    if (low >> lane & 1) {
      if (m >> lane & 1) {
        list.take[j] = make_int2(-1, 0);
      } else {
        const uint32_t k = count_below(hole, hole0);
        if (near) hist[k] = j;
        else list.hole[k] = j;
      }
    } else if (m >> lane & 1) {
      const uint32_t k = count_below(mover, mover0);
      if (near) hist[kBins / 2 + k] = j;
      else list.mover[k] = j;
    }
    hole0 += (uint32_t)__popcll(hole);
    mover0 += (uint32_t)__popcll(mover);
  };
#pragma unroll
  for (int i = 0; i < KW; ++i)
    if (i < steps) visit(i, i < kMasks ? kept[i < kMasks ? i : 0] : kept_lanes(held[i], j0 + 64 * i < L, tie_past));
  for (int i = KW; i < steps; ++i) visit(i, kept_lanes(fetch(i), j0 + 64 * i < L, tie_past));
  if (near) lds_barrier();  // not for what went to memory, which no one reads here
  else __syncthreads();
  for (uint32_t k0 = tid; k0 < count; k0 += 4 * kEvictThreads) {  // four at a time in flight
    int to[4], from[4], page[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const uint32_t k = min(k0 + u * kEvictThreads, count - 1);
      to[u] = near ? (int)hist[k] : list.hole[k];
      from[u] = near ? (int)hist[kBins / 2 + k] : list.mover[k];
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) page[u] = pages[from[u] >> 4];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (k0 + u * kEvictThreads < count) list.take[to[u]] = make_int2(from[u], page[u]);
  }
}

// Units of V of one lane: both formats hold eight tokens of a few dims in a
// unit of E bytes a token; half h of a page's slots has its own units.
template <int D, bool KV4>
struct VUnits {
  static constexpr int E = KV4 ? D / 64 : 2;          // bytes of a token
  static constexpr int N = KV4 ? 1 : D / 32;          // units of a lane
  static constexpr int WORDS = 2 * E;                 // 32-bit words of a unit
  // Half that the lane's units belong to, and byte of its unit i for half h in a block.
  static __device__ __forceinline__ int half(int lane) { return KV4 ? lane >> 5 : lane & 1; }
  static __device__ __forceinline__ int at(int lane, int i, int h) {
    if constexpr (KV4) return Kv4<D>::v_unit(8 * h, lane & 31);
    else return (((lane >> 1) + 32 * i) * kPageSize + 8 * h) * 2;
  }
};

template <int D, bool KV4>
__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(EvictArgs a, EvictPlan p) {
  using B = Kv4<D>;
  using V = VUnits<D, KV4>;
  const int item = blockIdx.x;
  int r = 0;
  {
    const int lane = threadIdx.x & 63;
    for (int base = 1; base < p.num_req; base += 64) {
      const int k = base + lane;
      r += __popcll(__ballot(k < p.num_req && p.req[k].move_start <= item));
    }
    r = __builtin_amdgcn_readfirstlane(r);
  }
  const EvictReq q = p.req[r];
  const int npage = (q.keep + 15) / 16;
  // heads fastest: with 8 of them a head's pages stay on one XCD, whose L2 then
  // holds the sources that neighbouring pages share
  const int local = item - q.move_start, hk = local % a.hkv;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int page = local / a.hkv * kMoveWaves + wave;
  if (page >= npage) return;
  if (q.most == 0) return;  // (its select wrote the positions)
  const MoveList list = move_list(a, q, hk);
  const int lane = threadIdx.x & 63;
  const int32_t* pages = a.page_indices + q.page_start;
  const size_t dst = (size_t)pages[page] * a.hkv + hk;
  // lane l < 16: what slot l takes, its mass and position
  const int j = page * 16 + lane;
  const int2 take = lane < 16 && j < q.keep ? list.take[j] : make_int2(-1, 0);
  const bool filled = take.x >= 0;
  const uint64_t holes = __ballot(filled);
  const int cnt = __popcll(holes);
  if (filled) {
    const size_t src = ((size_t)take.y * a.hkv + hk) * kPageSize + (take.x & 15);
    a.positions[dst * kPageSize + lane] = take.x < q.tracked ? a.positions[src] : take.x + q.evicted;
    if (a.mass) a.mass[dst * kPageSize + lane] = a.mass[src];
  } else if (lane < 16 && j >= q.tracked && j < q.keep) {
    a.positions[dst * kPageSize + lane] = j + q.evicted;
  }
  if (cnt == 0) return;
  // lane k < cnt: the k-th hole (others of the wave send to a lane past the holes)
  const int rank = filled ? __popcll(holes & ((1ull << lane) - 1)) : 32 + (lane & 31);
  const int nth = __builtin_amdgcn_ds_permute(4 * rank, lane);
  const int to = lane < cnt ? nth : 16;
  const int from = __shfl(take.x, nth & 15), from_page = __shfl(take.y, nth & 15);
  auto source = [&](int k) { return (size_t)__shfl(from_page, k) * a.hkv + hk; };

  constexpr size_t KBLOCK = KV4 ? (size_t)B::BLOCK : (size_t)kPageSize * D * 2;  // bytes of a block of the K pool
  constexpr size_t VBLOCK = KV4 ? (size_t)B::BLOCK : (size_t)kPageSize * D * 2;
  uint8_t* vdst = (KV4 ? a.k_cache : a.v_cache) + dst * VBLOCK;
  const uint8_t* vpool = KV4 ? a.k_cache : a.v_cache;
  uint8_t* kdst = a.k_cache + dst * KBLOCK;

  // K: 16 lanes a move, four moves at a time; the loads go out before the stores.
  constexpr int KW = KV4 ? 1 : D / 32;  // 32-bit words of a lane (one of two or four bytes, 4-bit)
  uint32_t kx[4][KW];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int k = 4 * i + (lane >> 4), t = lane & 15, c = min(k, cnt - 1);
    const int ss = __shfl(from, c) & 15;
    const uint8_t* src = a.k_cache + source(c) * KBLOCK;
    if (k >= cnt) continue;
    if constexpr (KV4 && D == 128) kx[i][0] = *(const uint32_t*)(src + B::k_code(ss, 8 * t));
    else if constexpr (KV4) kx[i][0] = *(const uint16_t*)(src + B::k_code(ss, 4 * t));
    else
#pragma unroll
      for (int e = 0; e < KW; ++e) kx[i][e] = *(const uint32_t*)(src + ss * 2 * D + 4 * KW * t + 4 * e);
  }
  uint8_t ks = 0, vs = 0;  // scales: a lane per (move, group)
  if constexpr (KV4) {
    const int k = lane / B::DT, c = min(k, cnt - 1), g = lane % B::DT;
    const int ss = __shfl(from, c) & 15;
    const uint8_t* src = a.k_cache + source(c) * KBLOCK;
    if (k < cnt) {
      ks = src[B::k_scale(ss, g)];
      vs = src[B::v_scale(ss, g)];
    }
  }

  // V: the lane's units of its half, patched by that half's moves, kBatch at a time.
  constexpr int kBatch = KV4 ? 4 : 2;
  const int h = V::half(lane);
  const int n0 = __popcll(__ballot(to < 8)), mine0 = h ? n0 : 0, mine = h ? cnt - n0 : n0;
  const int most = max(n0, cnt - n0);
  uint32_t unit[V::N][V::WORDS];
  auto read = [&](const uint8_t* block, int hh, uint32_t (&u)[V::N][V::WORDS]) {
#pragma unroll
    for (int i = 0; i < V::N; ++i) {
      if constexpr (V::WORDS == 4) {
        const u32x4 x = *(const u32x4*)(block + V::at(lane, i, hh));
#pragma unroll
        for (int e = 0; e < 4; ++e) u[i][e] = x[e];
      } else {
        const u32x2 x = *(const u32x2*)(block + V::at(lane, i, hh));
        u[i][0] = x[0], u[i][1] = x[1];
      }
    }
  };
  // A half that holds slots of `keep` and on, sources perhaps: its pieces are written alone.
  const bool whole = page * 16 + 8 * h + 8 <= q.keep;
  if (mine > 0 && whole) read(vdst, h, unit);
  for (int i0 = 0; i0 < most; i0 += kBatch) {
    uint32_t x[kBatch][V::N][V::WORDS];
    int ds[kBatch], ss[kBatch];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const int c = min(mine0 + i0 + b, cnt - 1);  // shuffles are done by every lane
      const int f = __shfl(from, c);
      ds[b] = __shfl(to, c) & 7;
      ss[b] = f & 7;
      const size_t src = source(c);
      if (i0 + b < mine) read(vpool + src * VBLOCK, (f >> 3) & 1, x[b]);
    }
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      if (i0 + b >= mine) continue;
      constexpr int PER = 4 / V::E;  // tokens of a word
      const uint32_t mask = V::E == 2 ? 0xffffu : 0xffu;
      const int sh = 8 * V::E * (ds[b] % PER);
#pragma unroll
      for (int n = 0; n < V::N; ++n) {
        uint32_t w = x[b][n][0];
#pragma unroll
        for (int e = 1; e < V::WORDS; ++e) w = ss[b] / PER == e ? x[b][n][e] : w;
        const uint32_t piece = (w >> (8 * V::E * (ss[b] % PER))) & mask;
        if (whole) {
#pragma unroll
          for (int e = 0; e < V::WORDS; ++e)
            if (ds[b] / PER == e) unit[n][e] = (unit[n][e] & ~(mask << sh)) | (piece << sh);
        } else {
          uint8_t* at = vdst + V::at(lane, n, h) + V::E * ds[b];
          if constexpr (V::E == 2) *(uint16_t*)at = (uint16_t)piece;
          else *at = (uint8_t)piece;
        }
      }
    }
  }
  if (mine > 0 && whole) {
#pragma unroll
    for (int i = 0; i < V::N; ++i) {
      if constexpr (V::WORDS == 4) *(u32x4*)(vdst + V::at(lane, i, h)) = u32x4{unit[i][0], unit[i][1], unit[i][2], unit[i][3]};
      else *(u32x2*)(vdst + V::at(lane, i, h)) = u32x2{unit[i][0], unit[i][1]};
    }
  }

#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int k = 4 * i + (lane >> 4), t = lane & 15, ds = __shfl(to, min(k, cnt - 1));
    if (k >= cnt) continue;
    if constexpr (KV4 && D == 128) *(uint32_t*)(kdst + B::k_code(ds, 8 * t)) = kx[i][0];
    else if constexpr (KV4) *(uint16_t*)(kdst + B::k_code(ds, 4 * t)) = (uint16_t)kx[i][0];
    else
#pragma unroll
      for (int e = 0; e < KW; ++e) *(uint32_t*)(kdst + ds * 2 * D + 4 * KW * t + 4 * e) = kx[i][e];
  }
  if constexpr (KV4) {
    const int k = lane / B::DT, g = lane % B::DT, ds = __shfl(to, min(k, cnt - 1));
    if (k < cnt) {
      kdst[B::k_scale(ds, g)] = ks;
      kdst[B::v_scale(ds, g)] = vs;
    }
  }
}

}  // namespace

hipError_t launch_evict(const EvictArgs& a, const EvictPlan& p, int head_dim, bool kv4, hipStream_t stream) {
  const dim3 heads(p.num_req * a.hkv), threads(kEvictThreads);
  const int steps = (p.longest + kEvictThreads - 1) / kEvictThreads;
  if (steps <= 4) hipLaunchKernelGGL((evict_select_kernel<4>), heads, threads, 0, stream, a, p);
  else if (steps <= 8) hipLaunchKernelGGL((evict_select_kernel<8>), heads, threads, 0, stream, a, p);
  else if (steps <= 16) hipLaunchKernelGGL((evict_select_kernel<16>), heads, threads, 0, stream, a, p);
  else hipLaunchKernelGGL((evict_select_kernel<32>), heads, threads, 0, stream, a, p);
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
