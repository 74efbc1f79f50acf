// Attention mass: what the verify rows of a step give to each key,
//   w_j = sum over counted rows i (j <= L + i) and the KV head's query heads
//         of exp(scale q_i . k_j - lse_i),
// added to the key's history, mass_j = (j < L ? decay * mass_j : 0) + w_j.
//
// One pass over K after the attention (whose lse it needs): the products of
// the scores once more, no V.  Keys are the columns of S = Q K^T, so a lane's
// 16 scores of a 32 x 32 tile are 16 query columns of one key and the sum over
// columns stays in the lane.  No atomics: a key's sum has one order.
//
// With few query columns (mass_kernel) the bytes of K bound it: up to 128 of them
// lie in LDS, waves take key tiles; mass_wide_kernel takes more, 128 after 128.
// A bf16 wave holds two key tiles, read straight from the pool; four times fewer
// bytes of a 4-bit key would leave a work group that small waiting for its start, so
// it takes a longer run of keys, two tiles a step, with the next step's codes in
// flight.  With many columns
// (mass_rows_kernel, prompts) the products and exponentials bound it: a work
// group takes 64 keys, held in registers by each of its waves, and the waves
// share the column tiles, whose Q comes through LDS of the wave's own.
//
// Measured (heads 32/8/128): 16 requests' steps over 1k to 8k bf16 keys 34 us (144 MB,
// 4.2 TB/s); 40 over 8k to 32k 4-bit keys 146 us (531 MB, 3.6 TB/s, where a kernel
// that only reads reaches 5.6: decoding and the columns' exponentials keep the vector
// units busy for 43 % of the cycles); two prompts of 2048 and 1555 rows 103 us, 68 of
// products at a large product's rate and 56 of exponentials and sums, which overlap
// little.  Prompts through mass_kernel, Q read from LDS by each key tile anew, took
// 406 us; the next tile's products placed between a wave's exponentials, at two
// waves a SIMD, took 157 where the plain order then took 135; 32, 96 or 128 keys a
// work group took 146, 106 and 110 where 64 took 106.
#include "cache_internal.h"
#include "kv4_device.h"

namespace rg {
namespace {

constexpr int kThreads = 64 * kMassWaves;
constexpr float kLog2e = 1.4426950408889634f;

// Request and range of a work item.
struct MassItem {
  int L, T, M;  // context, keys, counted columns
  int seen;     // keys that a counted row sees
  int hk, kbeg;
  int q_start, page_start;
};
__device__ __forceinline__ MassItem mass_item(const MassArgs& a, const AttnPlan& p, int keys) {
  const int item = blockIdx.x;
  const int r = find_request(p, item, false);
  const AttnReq rq = p.req[r];
  MassItem it;
  const int V = (int)((uint32_t)rq.nv >> 16);
  const int rows = a.row_count ? min(max(a.row_count[rq.part_start], 0), V) : V;
  it.L = rq.ctx;
  it.T = it.L + V;
  it.M = rows * a.g;
  it.seen = it.L + rows;
  const int local = item - rq.item_start;  // heads fastest: a prompt's costliest keys, its first, come first
  it.hk = local % a.hkv;
  it.kbeg = local / a.hkv * keys;
  it.q_start = rq.q_start;
  it.page_start = rq.page_start;
  return it;
}

// Row of q and lse of a column.
__device__ __forceinline__ size_t column_row(const MassArgs& a, const MassItem& it, int col) {
  const int tok = row_of(a, col);
  return (size_t)(it.q_start + tok) * a.hq + it.hk * a.g + (col - tok * a.g);
}

// K of key tile `kb`'s lane key as the columns' operand, straight from the pool.
template <int D, bool KV4>
__device__ __forceinline__ void load_keys(const MassArgs& a, const MassItem& it, int kb, bf16x8 (&kf)[D / 16]) {
  const int lane = threadIdx.x & 63, lc = lane & 31, lh = lane >> 5, key = kb + lc;
  const size_t block = (size_t)a.page_indices[it.page_start + min(key >> 4, (it.T - 1) / kPageSize)] * a.hkv + it.hk;
  if constexpr (KV4) {
    using B = Kv4<D>;
    const uint8_t* b = static_cast<const uint8_t*>(a.keys) + block * B::BLOCK;
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      const u32x4 w = *(const u32x4*)(b + B::k_code(key & 15, 64 * i + 32 * lh));
      const float sc = scale_of(b[B::k_scale(key & 15, 2 * i + lh)]);
#pragma unroll
      for (int e = 0; e < 4; ++e) kf[4 * i + e] = __builtin_bit_cast(bf16x8, decode8(w[e], sc));
    }
  } else {
    const uint16_t* b = static_cast<const uint16_t*>(a.keys) + (block * kPageSize + (key & 15)) * D;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) kf[ks] = *(const bf16x8*)(b + 16 * ks + 8 * lh);
  }
}

// 16-byte chunk of a row of Q that K step ks takes (the 4-bit block's order of dims).
template <bool KV4>
__device__ __forceinline__ int q_chunk(int ks, int lh) {
  return KV4 ? 8 * (ks / 4) + 4 * lh + ks % 4 : 2 * ks + lh;
}

// Adds a tile's weights: 32 columns from col0 on, keys kb + lc.
__device__ __forceinline__ void add_weights(const MassArgs& a, const MassItem& it, f32x16 sc, const float (&ls)[16], int col0,
                                            int kb, float& w) {
  const int lane = threadIdx.x & 63, lc = lane & 31, lh = lane >> 5;
  if (kb + 31 > it.L + row_of(a, col0)) {  // some row does not see every key
    int first = col0 + 4 * lh;
    asm volatile("" : "+v"(first));  // or the rows are found, 96 instructions, for every tile
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (kb + lc > it.L + row_of(a, first + 8 * (i >> 2) + (i & 3))) sc[i] = kNegInf;
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) w += __builtin_amdgcn_exp2f(__builtin_fmaf(sc[i], a.scale_log2, -ls[i]));
}

__device__ __forceinline__ void write_mass(const MassArgs& a, const MassItem& it, int key, float sum) {
  if (key >= it.seen) sum = 0.f;  // whatever it holds: a column that does not count may see it
  float* at = a.mass + ((size_t)a.page_indices[it.page_start + (key >> 4)] * a.hkv + it.hk) * kPageSize + (key & 15);
  *at = key < it.L && a.decay != 0.f ? a.decay * *at + sum : sum;
}

// A run of keys over up to kMassCols columns, or with WIDE over any number of
// them, kMassCols at a time: bf16 keys stay in registers, 4-bit ones are read
// again (from a cache, as a run's codes are 140 KB at most) and their sums stay in LDS.
template <int D, bool KV4, bool WIDE>
__device__ __forceinline__ void mass_run(const MassArgs& a, const AttnPlan& p) {
  constexpr int KSTEPS = D / 16, QROW = 2 * D + 16;  // 16 bytes more: a fragment read meets every bank once
  __shared__ __attribute__((aligned(16))) char lds[kMassCols * QROW + kMassCols * 4 + (KV4 ? kMassRun * 4 : 0)];
  char* qs = lds;
  float* lse2 = reinterpret_cast<float*>(qs + kMassCols * QROW);
  float* sums = lse2 + kMassCols;  // 4-bit: of the run's keys
  const int run = KV4 ? p.chunk : kMassKeys;
  const MassItem it = mass_item(a, p, run);
  const int tid = threadIdx.x, lane = tid & 63, lc = lane & 31, lh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int c0 = 0;                                           // first column in LDS
  int tiles = (WIDE ? min(it.M, kMassCols) + 31 : it.M + 31) / 32;  // column tiles there

  // 4-bit: codes and scales of two key tiles; their loads go out first
  typedef const int32_t __attribute__((address_space(4))) * cpage_ptr;
  const cpage_ptr pages = (cpage_ptr)(a.page_indices + it.page_start);
  const int last = (it.T - 1) / kPageSize, kend = min(it.T, it.kbeg + run);
  constexpr int STEP = 32 * kMassWaves;  // keys from a wave's tile to its next
  u32x4 kc[2][D / 64];
  uint32_t ksc[2];
  auto load = [&](int kb) {
    using B = Kv4<D>;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int pg = (kb + STEP * s) >> 4;
      const int p0 = pages[min(pg, last)], p1 = pages[min(pg + 1, last)];
      const uint8_t* b = static_cast<const uint8_t*>(a.keys) + ((size_t)(lc < 16 ? p0 : p1) * a.hkv + it.hk) * B::BLOCK;
#pragma unroll
      for (int i = 0; i < D / 64; ++i) kc[s][i] = *(const u32x4*)(b + B::k_code(lc & 15, 64 * i + 32 * lh));
      const uint8_t* sc = b + B::k_scale(lc & 15, 0);
      ksc[s] = D == 128 ? *(const uint32_t*)sc : *(const uint16_t*)sc;
    }
  };
  if constexpr (KV4) load(it.kbeg + 32 * wave);
  bf16x8 kf[KV4 ? 1 : kMassSub][KSTEPS];
  if constexpr (!KV4) {
#pragma unroll
    for (int s = 0; s < kMassSub; ++s) load_keys<D, false>(a, it, it.kbeg + 32 * (wave + kMassWaves * s), kf[s]);
    asm volatile("" ::: "memory");  // these loads go out before those of Q
  }

  auto load_columns = [&](int tid) {
    u32x4 qx[kMassCols * (D / 8) / kThreads];  // all loads, then all stores
#pragma unroll
    for (int e = 0; e < kMassCols * (D / 8) / kThreads; ++e) {
      const int u = tid + e * kThreads, col = c0 + u / (D / 8), ch = u % (D / 8);
      qx[e] = u32x4{0u, 0u, 0u, 0u};
      if (col < it.M) qx[e] = *(const u32x4*)(a.q + column_row(a, it, col) * D + 8 * ch);
    }
#pragma unroll
    for (int e = 0; e < kMassCols * (D / 8) / kThreads; ++e) {
      const int u = tid + e * kThreads, row = u / (D / 8), ch = u % (D / 8);
      if (row < 32 * tiles) *(u32x4*)(qs + row * QROW + 16 * ch) = qx[e];
    }
    // a column that does not count weighs exp2(-inf) = 0
    if (tid < 32 * tiles) lse2[tid] = c0 + tid < it.M ? a.lse[column_row(a, it, c0 + tid)] * kLog2e : -kNegInf;
    lds_barrier();
  };
  load_columns(tid);
  // The next columns, if there are any.
  auto next_columns = [&]() {
    c0 += kMassCols;
    if (!WIDE || c0 >= it.M) return false;
    tiles = (min(it.M - c0, kMassCols) + 31) / 32;
    lds_barrier();  // those before are no longer read
    int again = tid;
    asm volatile("" : "+v"(again));  // or places in LDS and q stay in registers all the while
    load_columns(again);
    return true;
  };

  // Adds the weights of N key tiles, 32 * kMassWaves keys apart, over the columns in LDS.
  auto weigh = [&](const auto& k, int kb, auto& w) {
    constexpr int N = sizeof(w) / sizeof(w[0]);
    for (int t = 0; t < tiles; ++t) {
      f32x16 sc[N];
#pragma unroll
      for (int s = 0; s < N; ++s)
        for (int i = 0; i < 16; ++i) sc[s][i] = 0.f;
      const char* row = qs + (32 * t + lc) * QROW;
      bf16x8 qf[KSTEPS];
#pragma unroll
      for (int ks = 0; ks < KSTEPS; ++ks) qf[ks] = *(const bf16x8*)(row + 16 * q_chunk<KV4>(ks, lh));
#pragma unroll
      for (int ks = 0; ks < KSTEPS; ++ks)
#pragma unroll
        for (int s = 0; s < N; ++s) sc[s] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf[ks], k[s][ks], sc[s], 0, 0, 0);
      float ls[16];
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) {
        const float4 x = *(const float4*)(lse2 + 32 * t + 8 * i4 + 4 * lh);
        ls[4 * i4] = x.x, ls[4 * i4 + 1] = x.y, ls[4 * i4 + 2] = x.z, ls[4 * i4 + 3] = x.w;
      }
#pragma unroll
      for (int s = 0; s < N; ++s) add_weights(a, it, sc[s], ls, c0 + 32 * t, kb + 32 * kMassWaves * s, w[s]);
    }
  };
  if constexpr (KV4) {
    do {
      // two key tiles a step: half the reads of Q, two chains of products
      for (int kb = it.kbeg + 32 * wave; kb < kend; kb += 2 * STEP) {
        bf16x8 k[2][KSTEPS];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int i = 0; i < D / 64; ++i) {
            const float f = scale_of((ksc[s] >> (8 * lh + 16 * i)) & 0xff);
#pragma unroll
            for (int e = 0; e < 4; ++e) k[s][4 * i + e] = __builtin_bit_cast(bf16x8, decode8(kc[s][i][e], f));
          }
        // the next step's codes, or the first's for the next columns
        if (kb + 2 * STEP < kend) load(kb + 2 * STEP);
        else if (WIDE && c0 + kMassCols < it.M) load(it.kbeg + 32 * wave);
        float w[2] = {0.f, 0.f};
        weigh(k, kb, w);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const float sum = w[s] + __shfl_xor(w[s], 32);
          if (lh == 0 && kb + STEP * s < kend) {
            float& at = sums[kb + STEP * s - it.kbeg + lc];  // always this lane's
            at = WIDE && c0 > 0 ? at + sum : sum;
          }
        }
      }
    } while (next_columns());
    // behind the loop: a load or store of the mass in it would wait for the codes
    lds_barrier();
    for (int key = it.kbeg + tid; key < kend; key += kThreads) write_mass(a, it, key, sums[key - it.kbeg]);
  } else {
    const int kb = it.kbeg + 32 * wave;
    float w[kMassSub] = {};
    do
      if (kb < it.T) weigh(kf, kb, w);
    while (next_columns());
#pragma unroll
    for (int s = 0; s < kMassSub; ++s) {
      const float sum = w[s] + __shfl_xor(w[s], 32);
      const int key = kb + 32 * kMassWaves * s + lc;
      if (lh == 0 && key < it.T) write_mass(a, it, key, sum);
    }
  }
}

template <int D, bool KV4>
__global__ __launch_bounds__(kThreads, KV4 ? 3 : 2) void mass_kernel(MassArgs a, AttnPlan p) {
  mass_run<D, KV4, false>(a, p);
}
template <int D, bool KV4>
__global__ __launch_bounds__(kThreads, KV4 ? 3 : 2) void mass_wide_kernel(MassArgs a, AttnPlan p) {
  mass_run<D, KV4, true>(a, p);
}

template <int D, bool KV4>
__global__ __launch_bounds__(kThreads, 3) void mass_rows_kernel(MassArgs a, AttnPlan p) {
  constexpr int KSTEPS = D / 16, NCH = D / 8, TILE = 32 * D * 2;  // bytes of a column tile of Q
  constexpr int LOADS = TILE / 1024;
  __shared__ __attribute__((aligned(16))) char lds[kMassWaves * TILE + kMassWaves * 128 + kMassWaves * kMassRowKeys * 4];
  const MassItem it = mass_item(a, p, kMassRowKeys);
  const int tid = threadIdx.x, lane = tid & 63, lc = lane & 31, lh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  char* tile = lds + wave * TILE;
  const uint32_t tile_at = lds_place(tile);
  float* lse2 = reinterpret_cast<float*>(lds + kMassWaves * TILE) + wave * 32;
  float* sums = reinterpret_cast<float*>(lds + kMassWaves * TILE + kMassWaves * 128);

  // This wave's column tiles: every kMassWaves-th of those whose rows see a key.
  const int tiles = (it.M + 31) / 32;
  const int t0 = (int)((int64_t)max(0, it.kbeg - it.L) * a.g / 32) + wave;
  // A tile of Q in LDS: rows of D, 16-byte chunks c of row r at place c ^ (r % NCH).
  // Columns past the counted ones repeat the last: they weigh zero.
  const uint16_t* base = a.q + (size_t)it.q_start * a.hq * D;
  float ls_next = 0.f;
  // Byte of chunk i of the lane's in q, past the request's first row, its column
  // `col` of the tile's: rows of a request span less than 2^31 (host check).
  auto byte_at = [&](int i, int col) {
    const int row = (i * 64 + lane) / NCH, ch = (lane % NCH) ^ (row % NCH), tok = row_of(a, col);
    return ((uint32_t)(tok * a.hq + (col - tok * a.g) + it.hk * a.g) * D + 8 * ch) * 2;
  };
  // Where 16 columns are whole rows, the second half of a tile and a wave's next
  // tile, 32 kMassWaves columns on, lie at constant distances: only the base moves.
  const bool whole = 16 % a.g == 0;
  const size_t half = (size_t)(16 / a.g) * a.hq, stride = 2 * kMassWaves * half;
  const uint16_t* qt = base;
  const float* lt = a.lse + (size_t)it.q_start * a.hq;
  uint32_t at[LOADS / 2];
#pragma unroll
  for (int i = 0; i < LOADS / 2; ++i) at[i] = byte_at(i, 32 * t0 + (i * 64 + lane) / NCH);
  const uint32_t lse_at = (uint32_t)(column_row(a, it, 32 * t0 + lc) - (size_t)it.q_start * a.hq);
  auto load = [&](int t) {
    if (whole && 32 * t + 32 <= it.M) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i)
        load_to_lds(tile_at + i * 1024, qt + (i < LOADS / 2 ? 0 : half * D), at[i % (LOADS / 2)]);
      ls_next = lt[lse_at];
    } else {
      int first = 32 * t;
      asm volatile("" : "+v"(first));  // not for every tile
#pragma unroll
      for (int i = 0; i < LOADS; ++i)
        load_to_lds(tile_at + i * 1024, base, byte_at(i, min(first + (i * 64 + lane) / NCH, it.M - 1)));
      ls_next = first + lc < it.M ? a.lse[column_row(a, it, first + lc)] : -kNegInf;
    }
    qt += stride * D;
    lt += stride;
  };
  if (t0 < tiles) load(t0);

  bf16x8 kf[2][KSTEPS];
#pragma unroll
  for (int s = 0; s < 2; ++s) load_keys<D, KV4>(a, it, it.kbeg + 32 * s, kf[s]);

  float w[2] = {0.f, 0.f};
  for (int t = t0; t < tiles; t += kMassWaves) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (lh == 0) lse2[lc] = ls_next * kLog2e;  // the wave's own: no barrier
    bf16x8 qf[KSTEPS];
    const char* row = tile + lc * (2 * D);
#pragma unroll
    for (int ks = 0; ks < KSTEPS; ++ks) qf[ks] = *(const bf16x8*)(row + 16 * (q_chunk<KV4>(ks, lh) ^ (lc % NCH)));
    if (t + kMassWaves < tiles) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the tile is in registers
      load(t + kMassWaves);
    }
    f32x16 sc[2];
#pragma unroll
    for (int s = 0; s < 2; ++s)
      for (int i = 0; i < 16; ++i) sc[s][i] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KSTEPS; ++ks)
#pragma unroll
      for (int s = 0; s < 2; ++s) sc[s] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf[ks], kf[s][ks], sc[s], 0, 0, 0);
    float ls[16];
#pragma unroll
    for (int i4 = 0; i4 < 4; ++i4) {
      const float4 x = *(const float4*)(lse2 + 8 * i4 + 4 * lh);
      ls[4 * i4] = x.x, ls[4 * i4 + 1] = x.y, ls[4 * i4 + 2] = x.z, ls[4 * i4 + 3] = x.w;
    }
    // A tile's sum by itself: thousands of rows one by one would each round at the
    // size of the whole.
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      float sum = 0.f;
      add_weights(a, it, sc[s], ls, 32 * t, it.kbeg + 32 * s, sum);
      w[s] += sum;
    }
  }
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    w[s] += __shfl_xor(w[s], 32);
    if (lh == 0) sums[wave * kMassRowKeys + 32 * s + lc] = w[s];
  }
  lds_barrier();
  if (tid < kMassRowKeys && it.kbeg + tid < it.T) {
    float sum = sums[tid];
    for (int k = 1; k < kMassWaves; ++k) sum += sums[k * kMassRowKeys + tid];
    write_mass(a, it, it.kbeg + tid, sum);
  }
}

}  // namespace

hipError_t launch_mass(const MassArgs& a, const AttnPlan& p, int head_dim, bool kv4, bool wide, hipStream_t stream) {
  const dim3 grid(p.total_items), block(kThreads);
  auto launch = [&](auto narrow_kernel, auto wide_kernel) {
    hipLaunchKernelGGL((wide ? wide_kernel : narrow_kernel), grid, block, 0, stream, a, p);
  };
  if (head_dim == 128 && kv4) launch(mass_kernel<128, true>, mass_wide_kernel<128, true>);
  else if (head_dim == 128) launch(mass_kernel<128, false>, mass_wide_kernel<128, false>);
  else if (kv4) launch(mass_kernel<64, true>, mass_wide_kernel<64, true>);
  else launch(mass_kernel<64, false>, mass_wide_kernel<64, false>);
  return hipGetLastError();
}

hipError_t launch_mass_rows(const MassArgs& a, const AttnPlan& p, int head_dim, bool kv4, hipStream_t stream) {
  const dim3 grid(p.total_items), block(kThreads);
  if (head_dim == 128 && kv4) hipLaunchKernelGGL((mass_rows_kernel<128, true>), grid, block, 0, stream, a, p);
  else if (head_dim == 128) hipLaunchKernelGGL((mass_rows_kernel<128, false>), grid, block, 0, stream, a, p);
  else if (kv4) hipLaunchKernelGGL((mass_rows_kernel<64, true>), grid, block, 0, stream, a, p);
  else hipLaunchKernelGGL((mass_rows_kernel<64, false>), grid, block, 0, stream, a, p);
  return hipGetLastError();
}

}  // namespace rg
