// Attention over a sliding window on the sm_100a tensor cores.
//
// A CTA (one per SM, persistent) works on 256 query rows of a head at a time, two tiles of 128, which share the key and
// value tiles of 128 rows that they see: the first tokens' tiles, then the window's.  For each of the two and every key tile
//     S  = Q K^T           tcgen05.mma, Q and K in shared memory
//     P  = exp2(S c - m)   one query row per thread, so that its sum needs no other thread; P goes back over S in
//                          tensor memory as bf16, and its first three quarters are handed to the products before the last is computed
//     O += P V             tcgen05.mma, P from tensor memory
// and while four warps are at the softmax of one tile, the tensor core is at the products of the other.  Roles: warp 0 loads (TMA, 128-byte
// swizzle), one thread of warp 1 issues the products, warp 2 sets value rows behind the last key to zero, warp 3 hands out work,
// warps 4-7 and 8-11 are the softmax of the two query tiles.  All of them run ahead of one another across pieces of work.
//
// m is not the running maximum but a reference that keeps exp2 in range: the maximum of the first keys that a row sees, raised (by a
// whole number, at the next step) when a sum of 32 probabilities exceeded 2^32.  P is bf16, O and the sum are fp32, so
// that probabilities far above 1 cost no precision, and no pass over the scores for their maximum stands between S and P.
// Masks: only key tiles at a border of a row's window are masked, by selecting scores.  A masked P is 0, and
// 0 x infinity is not: rows whose result is not finite are marked and computed again on the CUDA cores, where
// what is masked takes no part and no P is above 1 (a launch of its own, which ends at once when no row is marked).
//
// What bounds it: a step (256 x 128 scores, d = 128) takes some 3,100 cycles.  The products take 2,650 of them, 2,048 if shared
// memory fed both operands of Q K^T without a pause (they need all of its 128 bytes a cycle, and the loads of the next tiles and V
// come on top); the exponentials 1,900 of the special-function unit's time.  Between the two lies the chain S -> P -> O of each
// query tile.  Calls in a row are bound by power: 40 heads of 32,760 rows, d = 128, two frames of 1,560 to either side and the first
// one take 4.1 ms by themselves and 4.6 in a row (1.07 PFLOP/s of visible pairs, 1.20 with the masked parts of tiles; plain
// products of 8,192^3 1.41 in a row).  384 threads leave 168 registers to each, of which 68 bytes go by way of local memory.  Tried and slower: 16 softmax warps with half of a row's columns each (4.40 ms), the
// issuing thread looking at barriers without a pause (5.27: its looks delay everybody's), a pass for the exact maximum (4.17),
// every eighth instead of every sixteenth pair of exponentials on the FMA units (4.26; none 4.09, but 476 us instead of 452 at d = 64,
// 8 heads of 18,944 rows), P handed over in halves (4.07) or in whole (4.19), steps of 64 keys with two score buffers to a query tile
// (6.42 in a row: the issuing thread is what they wait for).
#include <math.h>

#include "tc_ptx.cuh"
#include "window.cuh"

namespace ca {

using namespace ptx;

constexpr int kWtThreads = 384;
constexpr int kWtRows = kWindowBlock;      // query rows of a piece of work
constexpr int kWtKeys = 128;

constexpr int kWtEvery = 16;               // of every 16 columns, two take their exponentials from the FMA units
constexpr float kE1 = 0.693147004f, kE2 = 0.240222424f, kE3 = 0.0555073358f, kE4 = 0.00967151299f, kE5 = 0.00132647273f;
constexpr float kWtSumLimit = 4294967296.f;   // 2^32: a sum of 32 probabilities above it raises the reference

constexpr int kWtRing = 4;                 // pieces of work on their way

template <int D>
struct WtCfg {
  static constexpr int PANELS = D / 64;                       // 128-byte wide column panels of a tile
  static constexpr int PANEL_BYTES = 128 * 128;
  static constexpr int TILE_BYTES = PANELS * PANEL_BYTES;     // 128 rows
  static constexpr int NK = D == 128 ? 2 : 4, NV = D == 128 ? 3 : 4;
  static constexpr int OFF_Q = 0, OFF_K = 2 * TILE_BYTES, OFF_V = OFF_K + NK * TILE_BYTES;
  static constexpr int OFF_WORK = OFF_V + NV * TILE_BYTES;    // [kWtRing] Work
  static constexpr int OFF_BAR = OFF_WORK + kWtRing * 64;
  static constexpr int NUM_BARS = 17 + 2 * kWtRing + 2 * NK + 3 * NV;
  static constexpr int OFF_MISC = OFF_BAR + 8 * NUM_BARS;     // tensor memory base, abort flag
  static constexpr int SMEM = 1024 + OFF_MISC + 16;
  static_assert(SMEM <= 227 * 1024, "shared memory");
};

// 256 query rows, as the warps read them.  Key tiles: [0, sink_tiles), then from tile_lo on, `tiles` in all.
struct Work {
  int b, h, r0, len_q, len_k, tiles, sink_tiles, tile_lo;
  int lo[2], hi[2];                        // keys that the rows of a query tile see: [lo, hi) and those below sinks
  int pad[4];
  __device__ __forceinline__ int tile(int u) const { return u < sink_tiles ? u : tile_lo + u - sink_tiles; }
  // whether query tile i takes part in the step of key tile t
  __device__ __forceinline__ bool active(int i, int t, int sinks) const { return takes_part(lo[i], hi[i], t * kWtKeys, sinks); }
  __device__ __forceinline__ static bool takes_part(int lo, int hi, int k0, int sinks) {
    return k0 < hi && (k0 + kWtKeys > lo || k0 < sinks);
  }
};
static_assert(sizeof(Work) == 64, "a work slot");

struct WtParams {
  WindowParams w;
  int blocks, rows_first;                  // blocks of a head; order of the pieces
  long long wait_limit;
  int wide;                                // rows of O start at 32-byte boundaries
  int skip_key_load;                       // diagnostic hook: the loader leaves out the keys of the step with these 64 (-1: none)
};

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int w, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
      ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar)
      : "memory");
}

__device__ __forceinline__ f32x2 exp2_unit(f32x2 x) {
  float a, b;
  unpack2(x, a, b);
  return pack2(ex2_approx(a), ex2_approx(b));
}
// 2^x without the special-function unit, for part of the scores (kWtEvery): x = j + f with j the nearest whole number, 2^f by a
// polynomial of degree 5 (fitted to the smallest relative error on [-1/2, 1/2] with the constant term 1; 1.2e-7 with its roundings)
// and j added to the exponent.  x at or below -127 gives exactly 0 (there the polynomial is 1, whose exponent field is 127), from 128 on exactly
// infinity.  What is no number stays so up to the sum with the exponent, which makes the largest finite number of it (0x7fffffff +
// (0x7fffffff << 23)): in bf16 that is infinity, so that O is not finite and the row is computed again.
__device__ __forceinline__ float clamp_nan(float x) {
  float y;
  asm("{.reg .f32 t;\n\tmax.NaN.f32 t, %1, 0fC2FE0000;\n\tmin.NaN.f32 %0, t, 0f43000000;}" : "=f"(y) : "f"(x));       // -127, 128
  return y;
}
__device__ __forceinline__ f32x2 exp2_fma(f32x2 x) {
  float a, b;
  unpack2(x, a, b);
  x = pack2(clamp_nan(a), clamp_nan(b));
  const f32x2 magic = pack2(12582912.f, 12582912.f), magic_neg = pack2(-12582912.f, -12582912.f);   // 1.5 2^23: j in the low bits
  const f32x2 shifted = add2(x, magic);
  const f32x2 f = fma2(add2(shifted, magic_neg), pack2(-1.f, -1.f), x);
  f32x2 p = pack2(kE5, kE5);
  p = fma2(p, f, pack2(kE4, kE4));
  p = fma2(p, f, pack2(kE3, kE3));
  p = fma2(p, f, pack2(kE2, kE2));
  p = fma2(p, f, pack2(kE1, kE1));
  p = fma2(p, f, pack2(1.f, 1.f));
  float pa, pb, ja, jb;
  unpack2(p, pa, pb);
  unpack2(shifted, ja, jb);
  return pack2(__int_as_float(__float_as_int(pa) + (__float_as_int(ja) << 23)), __int_as_float(__float_as_int(pb) + (__float_as_int(jb) << 23)));
}

template <int D>
__global__ void __launch_bounds__(kWtThreads, 1)
window_tc_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                 const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ WtParams prm) {
  wait_for_previous();
  using C = WtCfg<D>;
  extern __shared__ unsigned char smem_unaligned[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_unaligned) + 1023) & ~uintptr_t(1023));
  const uint32_t s_base = smem_u32(smem);
  const uint32_t s_q = s_base + C::OFF_Q, s_k = s_base + C::OFF_K, s_v = s_base + C::OFF_V;
  volatile Work* work_ring = reinterpret_cast<volatile Work*>(smem + C::OFF_WORK);
  const uint32_t bar0 = s_base + C::OFF_BAR;
  auto b_q_full = [&](int i) { return bar0 + 8 * i; };
  auto b_q_empty = [&](int i) { return bar0 + 16 + 8 * i; };
  auto b_s_full = [&](int i) { return bar0 + 32 + 8 * i; };
  auto b_p_most = [&](int i) { return bar0 + 48 + 8 * i; };
  auto b_p_ready = [&](int i) { return bar0 + 64 + 8 * i; };
  auto b_pv_done = [&](int i) { return bar0 + 80 + 8 * i; };
  auto b_o_full = [&](int i) { return bar0 + 96 + 8 * i; };
  auto b_o_empty = [&](int i) { return bar0 + 112 + 8 * i; };
  auto b_work_full = [&](int n) { return bar0 + 128 + 8 * (n % kWtRing); };
  auto b_work_empty = [&](int n) { return bar0 + 128 + 8 * (kWtRing + n % kWtRing); };
  const uint32_t b_claim = bar0 + 128 + 16 * kWtRing;
  const uint32_t bar1 = b_claim + 8;
  auto b_k_full = [&](int s) { return bar1 + 8 * s; };
  auto b_k_empty = [&](int s) { return bar1 + 8 * (C::NK + s); };
  auto b_v_full = [&](int s) { return bar1 + 8 * (2 * C::NK + s); };
  auto b_v_ready = [&](int s) { return bar1 + 8 * (2 * C::NK + C::NV + s); };
  auto b_v_empty = [&](int s) { return bar1 + 8 * (2 * C::NK + 2 * C::NV + s); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + C::OFF_MISC);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + C::OFF_MISC + 4);
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const int sinks = prm.w.sinks;

  if (prm.w.one_each && blockIdx.x == 0) window_status(prm.w, kWtThreads);     // (a wait that gives up writes it a second later)
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(b_q_full(i), 1);
      mbar_init(b_q_empty(i), 1);
      mbar_init(b_s_full(i), 1);
      mbar_init(b_p_most(i), 4);
      mbar_init(b_p_ready(i), 4);
      mbar_init(b_pv_done(i), 1);
      mbar_init(b_o_full(i), 1);
      mbar_init(b_o_empty(i), 4);
    }
    for (int i = 0; i < kWtRing; ++i) { mbar_init(b_work_full(i), 1); mbar_init(b_work_empty(i), 11); }
    for (int s = 0; s < C::NK; ++s) { mbar_init(b_k_full(s), 1); mbar_init(b_k_empty(s), 1); }
    for (int s = 0; s < C::NV; ++s) { mbar_init(b_v_full(s), 1); mbar_init(b_v_ready(s), 1); mbar_init(b_v_empty(s), 1); }
    mbar_init(b_claim, 1);
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(tmem_slot), 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = __shfl_sync(0xffffffffu, *tmem_slot, 0);
  auto tmem_s = [&](int i) { return tmem_base + i * kWtKeys; };
  auto tmem_o = [&](int i) { return tmem_base + 2 * kWtKeys + i * 128; };

  auto wait = [&](uint32_t bar, uint32_t phase) { return mbar_wait(bar, phase & 1, abort_flag, prm.w.status, prm.wait_limit); };
  auto relaxed = [&](uint32_t bar, uint32_t phase) { return mbar_wait_relaxed(bar, phase & 1, abort_flag, prm.w.status, prm.wait_limit); };
  auto read_work = [&](int n, Work& w) {               // a thread's copy of piece n, which is there
    const volatile int* src = reinterpret_cast<const volatile int*>(work_ring + n % kWtRing);
    int* dst = reinterpret_cast<int*>(&w);
#pragma unroll
    for (int i = 0; i < 12; ++i) dst[i] = src[i];
  };

  if (warp == 3) {
    // ---------------------------------------------------------- work
    if (lane == 0) {
      const int all_blocks = prm.w.one_each ? prm.blocks * prm.w.batch : prm.w.pieces[prm.w.batch], n_work = all_blocks * prm.w.heads_q;
      int n = 0;
      for (int idx = blockIdx.x;; ++n) {
        // A piece is claimed when the one before is nearly loaded, not earlier: what a CTA has claimed another that is done cannot take
        // (with four claimed ahead SMs were at work for 77 % of a call of four pieces each).
        if (n > 0 && prm.w.one_each) {
          idx = n_work;
        } else if (n > 0) {
          if (!relaxed(b_claim, n - 1)) break;
          idx = (int)gridDim.x + atomicAdd(prm.w.status + kNextWord, 1);
        }
        Work w;
        w.b = -1;
        if (idx < n_work) {
          // the blocks of a head one after the other, or the last blocks of all heads first
          int block = idx % all_blocks;
          w.h = idx / all_blocks;
          if (prm.rows_first) {
            w.h = idx % prm.w.heads_q;
            block = all_blocks - 1 - idx / prm.w.heads_q;
          }
          if (prm.w.one_each) {
            w.b = block / prm.blocks;
            w.r0 = block % prm.blocks * kWtRows;
          } else {
            int lo = 0, hi = prm.w.batch - 1;            // the batch item of the block
            while (lo < hi) {
              const int mid = (lo + hi + 1) >> 1;
              if (prm.w.pieces[mid] <= block) lo = mid;
              else hi = mid - 1;
            }
            w.b = lo;
            w.r0 = (block - prm.w.pieces[lo]) * kWtRows;
          }
          const WindowItem it(prm.w, w.b);
          if (w.r0 >= it.len_q) {                        // (of one_each: a block behind its sequence)
            w.b = -1;
            idx = n_work;
          }
          w.len_q = it.len_q;
          w.len_k = it.len_k;
          const WindowSpan all(prm.w, it, w.r0, min(w.r0 + kWtRows, it.len_q), kWtKeys);
          w.tiles = all.tiles;
          w.sink_tiles = all.sink_tiles;
          w.tile_lo = all.tile_lo;
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int first = w.r0 + i * kWindowTile;
            w.lo[i] = w.hi[i] = 0;
            if (first < it.len_q) {
              const WindowSpan part(prm.w, it, first, min(first + kWindowTile, it.len_q), kWtKeys);
              w.lo[i] = part.lo;
              w.hi[i] = part.hi;
            }
          }
        }
        if (n >= kWtRing && !relaxed(b_work_empty(n), n / kWtRing - 1)) break;
        volatile int* dst = reinterpret_cast<volatile int*>(work_ring + n % kWtRing);
        const int* src = reinterpret_cast<const int*>(&w);
#pragma unroll
        for (int i = 0; i < 12; ++i) dst[i] = src[i];
        mbar_arrive(b_work_full(n));
        if (w.b < 0) break;
      }
    }
  } else if (warp == 0) {
    // ---------------------------------------------------------- loads
    if (lane == 0) {
      prefetch_tensormap(&tm_q);
      prefetch_tensormap(&tm_k);
      prefetch_tensormap(&tm_v);
      int q_used[2] = {0, 0}, k_slot = 0, v_slot = 0, steps = 0;
      uint32_t k_ph = 1, v_ph = 1;
      bool ok = true;
      for (int n = 0; ok; ++n) {
        if (!relaxed(b_work_full(n), n / kWtRing)) break;
        Work w;
        read_work(n, w);
        mbar_arrive(b_work_empty(n));
        if (w.b < 0) break;
        const int g = w.h / prm.w.group;
        bool q_there[2] = {false, false};
        if (w.tiles == 0) mbar_arrive(b_claim);
        for (int u = 0; u < w.tiles && ok; ++u) {
          const int t = w.tile(u);
          if (u == max(0, w.tiles - 4)) mbar_arrive(b_claim);
          // queries of the tiles that begin here: the first before the keys, which wait for less than the second
          auto queries = [&](int i) {
            if (q_there[i] || !w.active(i, t, sinks)) return;
            q_there[i] = true;
            if (q_used[i] > 0) ok = ok && relaxed(b_q_empty(i), q_used[i] - 1);
            if (!ok) return;
            ++q_used[i];
            mbar_expect_tx(b_q_full(i), C::TILE_BYTES);
#pragma unroll
            for (int pn = 0; pn < C::PANELS; ++pn)
              tma_load_4d(s_q + i * C::TILE_BYTES + pn * C::PANEL_BYTES, &tm_q, pn * 64, w.r0 + i * kWindowTile, w.h, w.b, b_q_full(i));
          };
          queries(0);
          if (!ok) break;
          if (steps >= C::NK && !relaxed(b_k_empty(k_slot), k_ph)) { ok = false; break; }
          if (steps != (prm.skip_key_load >> 1)) {           // diagnostic: this slot never fills, its waiters time out
            mbar_expect_tx(b_k_full(k_slot), C::TILE_BYTES);
#pragma unroll
            for (int pn = 0; pn < C::PANELS; ++pn)
              tma_load_4d(s_k + k_slot * C::TILE_BYTES + pn * C::PANEL_BYTES, &tm_k, pn * 64, t * kWtKeys, g, w.b, b_k_full(k_slot));
          }
          if (++k_slot == C::NK) { k_slot = 0; k_ph ^= 1; }
          queries(1);
          if (!ok) break;
          if (steps >= C::NV && !relaxed(b_v_empty(v_slot), v_ph)) { ok = false; break; }
          mbar_expect_tx(b_v_full(v_slot), C::TILE_BYTES);
#pragma unroll
          for (int pn = 0; pn < C::PANELS; ++pn)
            tma_load_4d(s_v + v_slot * C::TILE_BYTES + pn * C::PANEL_BYTES, &tm_v, pn * 64, t * kWtKeys, g, w.b, b_v_full(v_slot));
          if (++v_slot == C::NV) { v_slot = 0; v_ph ^= 1; }
          ++steps;
        }
      }
    }
  } else if (warp == 2) {
    // ---------------------------------------------------------- value rows behind the last key
    int slot = 0;
    uint32_t ph = 0;
    bool ok = true;
    for (int n = 0; ok; ++n) {
      ok = __all_sync(0xffffffffu, relaxed(b_work_full(n), n / kWtRing));
      if (!ok) break;
      Work w;
      read_work(n, w);
      __syncwarp();
      if (lane == 0) mbar_arrive(b_work_empty(n));
      if (w.b < 0) break;
      for (int u = 0; u < w.tiles; ++u) {
        ok = __all_sync(0xffffffffu, relaxed(b_v_full(slot), ph));
        if (!ok) break;
        const int from = w.len_k - w.tile(u) * kWtKeys;      // rows of the tile from here on are not keys
        if (from < kWtKeys) {
          unsigned char* tile = smem + C::OFF_V + slot * C::TILE_BYTES;
          for (int i = lane; i < C::PANELS * (kWtKeys - from) * 8; i += 32) {
            const int pn = i / ((kWtKeys - from) * 8), rest = i % ((kWtKeys - from) * 8);
            *reinterpret_cast<uint4*>(tile + pn * C::PANEL_BYTES + from * 128 + rest * 16) = make_uint4(0u, 0u, 0u, 0u);
          }
          fence_proxy_async();
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(b_v_ready(slot));
        if (++slot == C::NV) { slot = 0; ph ^= 1; }
      }
    }
  } else if (warp == 1) {
    // ---------------------------------------------------------- products
    if (elect_one()) {
      constexpr uint32_t idesc_qk = idesc_bf16_f32(kWindowTile, kWtKeys, 0, 0);
      constexpr uint32_t idesc_pv = idesc_bf16_f32(kWindowTile, D, 0, 1);
      const uint64_t q_desc0 = smem_desc_sw128(s_q, 16, 1024);
      const uint64_t k_desc0 = smem_desc_sw128(s_k, 16, 1024);
      const uint64_t v_desc0 = smem_desc_sw128(s_v, C::PANEL_BYTES, 1024);
      int n_pv[2] = {0, 0}, n_q[2] = {0, 0}, n_o[2] = {0, 0};   // steps, query tiles, results so far
      int k_slot = 0, v_slot = 0;
      uint32_t k_ph = 0, v_ph = 0;
      bool on[2] = {false, false};             // the step before: query tiles that take part, the first, the last of their steps
      bool was_first[2] = {false, false}, was_last[2] = {false, false};
      bool any_before = false;
      bool ok = true, more = true;
      Work w;
      w.tiles = 0;
      int u = 0, n = 0;
      bool begun[2] = {false, false};
      while (ok) {
        // the step that comes: the next key tile of this piece of work or the first one of the next
        while (more && u >= w.tiles) {
          if (!wait(b_work_full(n), n / kWtRing)) { ok = false; break; }
          read_work(n, w);
          mbar_arrive(b_work_empty(n));
          ++n;
          u = 0;
          begun[0] = begun[1] = false;
          if (w.b < 0) { more = false; w.tiles = 0; }
        }
        if (!ok || (!more && !any_before)) break;
        const int t = more ? w.tile(u) : 0;
        bool now[2], first[2], last[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          now[i] = more && w.active(i, t, sinks);
          first[i] = now[i] && !begun[i];
          begun[i] = begun[i] || now[i];
          last[i] = now[i] && (t + 1) * kWtKeys >= w.hi[i];  // a query tile's steps end with its window
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          // A look at a barrier takes some 200 cycles, done or not: all that is there early (loads, a free accumulator) is looked
          // at before P, whose softmax it overlaps with.
          if (i == 0) {
            if (any_before && !wait(b_v_ready(v_slot), v_ph)) { ok = false; break; }
            if (more && !wait(b_k_full(k_slot), k_ph)) { ok = false; break; }
          }
          if (first[i]) {
            if (!wait(b_q_full(i), n_q[i])) { ok = false; break; }
            ++n_q[i];
          }
          if (on[i]) {
            // O of query tile i += P V of the step before
            if (was_first[i]) {
              if (n_o[i] > 0 && !wait(b_o_empty(i), n_o[i] - 1)) { ok = false; break; }
              ++n_o[i];
            }
            if (!wait(b_p_most(i), n_pv[i])) { ok = false; break; }
            tc_fence_after();
            const uint64_t vd = v_desc0 + ((v_slot * C::TILE_BYTES) >> 4);
#pragma unroll
            for (int ks = 0; ks < 6; ++ks)
              mma_ts(tmem_o(i), tmem_s(i) + ks * 8, vd + (uint64_t)(ks * (2048 >> 4)), idesc_pv, (ks > 0 || !was_first[i]) ? 1u : 0u);
            if (!wait(b_p_ready(i), n_pv[i])) { ok = false; break; }
            tc_fence_after();
#pragma unroll
            for (int ks = 6; ks < 8; ++ks)
              mma_ts(tmem_o(i), tmem_s(i) + ks * 8, vd + (uint64_t)(ks * (2048 >> 4)), idesc_pv, 1u);
            ++n_pv[i];
          }
          if (now[i]) {
            tc_fence_after();
            const uint64_t qd = q_desc0 + ((i * C::TILE_BYTES) >> 4), kd = k_desc0 + ((k_slot * C::TILE_BYTES) >> 4);
            if (on[i]) {                                     // (commits behind the products of both: nothing waits for O alone unless the tile ends)
              mma_commit(b_pv_done(i));
              if (was_last[i]) mma_commit(b_o_full(i));
            }
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
              const uint32_t off = ((ks / 4) * C::PANEL_BYTES + (ks % 4) * 32) >> 4;
              mma_ss(tmem_s(i), qd + off, kd + off, idesc_qk, ks > 0 ? 1u : 0u);
            }
            mma_commit(b_s_full(i));
            if (last[i]) mma_commit(b_q_empty(i));
          } else if (on[i]) {
            mma_commit(b_pv_done(i));
            if (was_last[i]) mma_commit(b_o_full(i));
          }
          if (i == 1 && any_before) {
            mma_commit(b_v_empty(v_slot));
            if (++v_slot == C::NV) { v_slot = 0; v_ph ^= 1; }
          }
        }
        if (!ok) break;
        if (more) {
          mma_commit(b_k_empty(k_slot));
          if (++k_slot == C::NK) { k_slot = 0; k_ph ^= 1; }
          ++u;
        }
        any_before = more;
#pragma unroll
        for (int i = 0; i < 2; ++i) { on[i] = now[i]; was_first[i] = first[i]; was_last[i] = last[i]; }
      }
    }
    __syncwarp();
  } else {
    // ---------------------------------------------------------- softmax and results
    const int i = (warp >> 2) - 1, quarter = warp & 3;
    const int row = quarter * 32 + lane;
    const uint32_t lane_addr = (uint32_t)(quarter * 32) << 16;
    const uint32_t t_s = tmem_s(i) + lane_addr, t_o = tmem_o(i) + lane_addr;
    const float scale = prm.w.scale_log2;
    auto all_wait = [&](uint32_t bar, uint32_t phase) { return __all_sync(0xffffffffu, wait(bar, phase)); };
    int steps = 0, results = 0;
    bool ok = true;
    for (int n = 0; ok; ++n) {
      ok = all_wait(b_work_full(n), n / kWtRing);
      if (!ok) break;
      const volatile Work& w = work_ring[n % kWtRing];       // (read where it is needed: registers are few)
      if (w.b < 0) break;
      const int r = w.r0 + i * kWindowTile + row;            // query row
      if (w.r0 + i * kWindowTile >= w.len_q) {
        __syncwarp();
        if (lane == 0) mbar_arrive(b_work_empty(n));
        continue;
      }
      const WindowItem it(w.len_q, w.len_k);
      const WindowSpan span(prm.w, it, w.r0 + i * kWindowTile, min(w.r0 + (i + 1) * kWindowTile, it.len_q), kWtKeys);
      const WindowRow sees(prm.w, it, r);
      float m = r < it.len_q ? -INFINITY : 0.f, l = 0.f, pend = 0.f;      // (a row behind the last one needs no reference)
      bool begun = false;
#pragma unroll 1
      for (int u = 0; u < w.tiles; ++u) {
        const int j0 = (u < w.sink_tiles ? u : w.tile_lo + u - w.sink_tiles) * kWtKeys;
        if (!Work::takes_part(span.lo, span.hi, j0, sinks)) continue;
        ok = all_wait(b_s_full(i), steps);
        if (!ok) break;
        tc_fence_after();
        const bool masked = !span.whole(j0, j0 + kWtKeys);
        uint32_t sa[32], sb[32];
        tmem_ld32(t_s, sa);
        // what a row does not see of columns c .. c + 31: columns at or behind `end`, and those before `from` that are no first tokens
        auto mask = [&](uint32_t (&s)[32], int c) {
          auto below = [&](int x) {                          // bits of columns below x
            const int k = x - j0 - c;
            return k >= 32 ? 0xffffffffu : k <= 0 ? 0u : (1u << k) - 1u;
          };
          const unsigned seen = below(sees.end) & (~below(sees.from) | below(sinks));
#pragma unroll
          for (int e = 0; e < 32; ++e)
            if (!((seen >> e) & 1u)) s[e] = 0xff800000u;
        };
        // ---- reference
        if (__any_sync(0xffffffffu, m == -INFINITY || pend > 0.f)) {
          float up = m + pend;
          if (__any_sync(0xffffffffu, m == -INFINITY)) {
            float top = -INFINITY;
#pragma unroll 1
            for (int c = 0; c < kWtKeys; c += 32) {
              tmem_ld32(t_s + c, sa);
              tmem_wait_ld32(sa);
              if (masked) mask(sa, c);
              float x0 = -INFINITY, x1 = -INFINITY;
#pragma unroll
              for (int e = 0; e < 32; e += 4) {
                x0 = max3(x0, __uint_as_float(sa[e]), __uint_as_float(sa[e + 1]));
                x1 = max3(x1, __uint_as_float(sa[e + 2]), __uint_as_float(sa[e + 3]));
              }
              top = max3(top, x0, x1);
            }
            if (m == -INFINITY) up = top * scale;
            tmem_ld32(t_s, sa);
          }
          const float by = m == -INFINITY ? 0.f : ex2_approx(m - up);
          l *= by;
          m = up;
          pend = 0.f;
          if (begun) {
            // the products of the step before are complete; those of this step wait for this warp
            ok = all_wait(b_pv_done(i), steps - 1);
            if (!ok) break;
            tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < D / 16; ++c) {
              uint32_t o[16];
              tmem_ld16(t_o + c * 16, o);
              tmem_wait_ld();
#pragma unroll
              for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * by);
              tmem_st16(t_o + c * 16, o);
            }
          }
        }
        // ---- probabilities: column c to half a word
        const float ref = m == -INFINITY ? 0.f : -m;
        const f32x2 sc2 = pack2(scale, scale), nm2 = pack2(ref, ref);
        float big = 0.f;                                     // largest sum of 32
        auto exponentials = [&](uint32_t (&s)[32], int c) {
          if (masked) mask(s, c);
          uint32_t pk[16];
          f32x2 sum0 = pack2(0.f, 0.f), sum1 = sum0;
#pragma unroll
          for (int e = 0; e < 32; e += 4) {
            f32x2 x01 = fma2(pack2(__uint_as_float(s[e]), __uint_as_float(s[e + 1])), sc2, nm2);
            f32x2 x23 = fma2(pack2(__uint_as_float(s[e + 2]), __uint_as_float(s[e + 3])), sc2, nm2);
            x01 = e % kWtEvery == 0 ? exp2_fma(x01) : exp2_unit(x01);
            x23 = exp2_unit(x23);
            sum0 = add2(sum0, x01);
            sum1 = add2(sum1, x23);
            float x0, x1, x2, x3;
            unpack2(x01, x0, x1);
            unpack2(x23, x2, x3);
            pk[e / 2] = pack_bf16x2(x0, x1);
            pk[e / 2 + 1] = pack_bf16x2(x2, x3);
          }
          float a0, a1, a2, a3;
          unpack2(sum0, a0, a1);
          unpack2(sum1, a2, a3);
          const float sum = (a0 + a1) + (a2 + a3);
          l += sum;
          big = fmaxf(big, sum);
          tmem_st16(t_s + c / 2, pk);
        };
        tmem_wait_ld32(sa);
        tmem_ld32(t_s + 32, sb);
        exponentials(sa, 0);
        tmem_wait_ld32(sb);
        tmem_ld32(t_s + 64, sa);
        exponentials(sb, 32);
        tmem_wait_ld32(sa);
        tmem_ld32(t_s + 96, sb);
        exponentials(sa, 64);
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(b_p_most(i));             // the products of the first 96 keys need not wait for the others
        tmem_wait_ld32(sb);
        exponentials(sb, 96);
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(b_p_ready(i));
        if (big > kWtSumLimit) pend = fminf(ceilf(log2f(big)), 126.f);     // (2^-127 would be zero, and the sum so far lost)
        begun = true;
        ++steps;
      }
      if (!ok) break;
      // ---- O / l; a row that sees nothing: zeros, log-sum-exp -inf.  (By the mask: m and l of a row whose scores are no numbers can be
      // -inf and 0 too, since the sum so far is scaled by 0 while m is -inf; its O is not finite, and it is computed again.)
      const bool live = r < it.len_q, empty = sees.end == 0;
      const float inv = empty ? 0.f : 1.f / l;
      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(prm.w.o) + w.b * prm.w.o_b + w.h * prm.w.o_h + r * prm.w.o_n;
      if (begun) {
        ok = all_wait(b_o_full(i), results);
        if (!ok) break;
        ++results;
        tc_fence_after();
      }
      f32x2 any2 = pack2(0.f, 0.f);
      uint32_t o[32];
#pragma unroll 1
      for (int c = 0; c < D; c += 32) {
        if (begun) {
          tmem_ld32(t_o + c, o);
          tmem_wait_ld32(o);
        }
        uint32_t x[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const f32x2 y = mul2(pack2(__uint_as_float(o[2 * e]), __uint_as_float(o[2 * e + 1])), pack2(inv, inv));
          any2 = fma2(y, pack2(1.01f, 1.01f), any2);       // (what rounds beyond bf16's largest number counts as not finite)
          float y0, y1;
          unpack2(y, y0, y1);
          x[e] = empty ? 0u : pack_bf16x2(y0, y1);
        }
        if (live) {
#pragma unroll
          for (int e = 0; e < 16; e += 8) {
            __nv_bfloat16* dst = out + c + 2 * e;
            if (prm.wide) {                                  // whole sectors at a time
              asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst), "r"(x[e]), "r"(x[e + 1]), "r"(x[e + 2]),
                           "r"(x[e + 3]), "r"(x[e + 4]), "r"(x[e + 5]), "r"(x[e + 6]), "r"(x[e + 7]) : "memory");
            } else {
              reinterpret_cast<uint4*>(dst)[0] = make_uint4(x[e], x[e + 1], x[e + 2], x[e + 3]);
              reinterpret_cast<uint4*>(dst)[1] = make_uint4(x[e + 4], x[e + 5], x[e + 6], x[e + 7]);
            }
          }
        }
      }
      float any, any_odd;
      unpack2(any2, any, any_odd);
      any += any_odd;
      if (begun) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(b_o_empty(i));
      }
      if (live && prm.w.lse)
        prm.w.lse[((size_t)w.b * prm.w.heads_q + w.h) * prm.w.n_q + r] = empty ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
      // rows to be computed again: two words for 32 rows
      const bool again = __any_sync(0xffffffffu, live && !empty && !(fabsf(any) < INFINITY && l < INFINITY));
      if (lane == 0) {
        int32_t* mark = prm.w.redo + ((size_t)(w.b * prm.w.heads_q + w.h) * prm.blocks + w.r0 / kWtRows) * 16 + (i * 4 + quarter) * 2;
        mark[0] = mark[1] = again ? 1 : 0;
        if (again && !prm.w.one_each) atomicExch(prm.w.status + kRedoWord, 1);
        mbar_arrive(b_work_empty(n));
      }
    }
  }
  let_next_start();
  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {                       // a wait gave up: copies in flight land before the CTA's shared memory is another's
    const long long t0 = clock64();
    while (clock64() - t0 < 2000000) __nanosleep(1000);
  }
  if (warp == 1) tmem_dealloc(tmem_base, 512);
}

// ---- host side -------------------------------------------------------------------------------------------

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
static EncodeTiledFn encode_fn() {
  static EncodeTiledFn fn = [] {
    void* ptr = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess)
      ptr = nullptr;
    return reinterpret_cast<EncodeTiledFn>(ptr);
  }();
  return fn;
}

// [batch, heads, rows, D] by strides (elements), boxes of 128 rows by 64 columns
static bool rows_map(CUtensorMap* map, const void* base, int D, int n, int heads, int batch, long long s_n, long long s_h, long long s_b) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)n, (cuuint64_t)heads, (cuuint64_t)batch};
  const long long stride[3] = {n > 1 ? s_n : D, heads > 1 ? s_h : D, batch > 1 ? s_b : D};
  cuuint64_t strides[3];
  for (int i = 0; i < 3; ++i) {
    if (stride[i] <= 0 || stride[i] >= (1LL << 39)) return false;    // 40 bits of bytes; a broadcast dimension has none
    strides[i] = (cuuint64_t)stride[i] * 2;
  }
  const cuuint32_t box[4] = {64, 128, 1, 1}, step[4] = {1, 1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D>
static int launch_window_tc_d(const CUtensorMap* maps, const WtParams& prm, int n_work, LaunchStream st) {
  auto kernel = window_tc_kernel<D>;
  const int sms = multiprocessors();
  if (sms == 0) return CA_ERR_CUDA;
  CA_RETURN_IF_CUDA(allow_smem(kernel, WtCfg<D>::SMEM));
  launch_chained(kernel, n_work < sms ? n_work : sms, kWtThreads, WtCfg<D>::SMEM, st, maps[0], maps[1], maps[2], prm);
  CA_LAUNCH_CHECK();
  return CA_OK;
}

// CA_ERR_UNSUPPORTED: strides that a tensor map does not describe
int launch_window_tc(WindowParams& w, int D, LaunchStream st) {
  CUtensorMap maps[3];
  if (!rows_map(&maps[0], w.q, D, w.n_q, w.heads_q, w.batch, w.q_n, w.q_h, w.q_b) ||
      !rows_map(&maps[1], w.k, D, w.n_k, w.heads_kv, w.batch, w.k_n, w.k_h, w.k_b) ||
      !rows_map(&maps[2], w.v, D, w.n_k, w.heads_kv, w.batch, w.v_n, w.v_h, w.v_b))
    return CA_ERR_UNSUPPORTED;
  WtParams prm{};
  prm.w = w;
  prm.blocks = ceil_div(w.n_q, kWtRows);
  const long long n_work = (long long)prm.blocks * w.heads_q * w.batch;
  if (n_work > 0x3fffffffLL) return CA_ERR_UNSUPPORTED;
  // Pieces are handed out head by head, whose blocks read the same keys; or, where the keys and values that all heads' windows
  // reach at a time stay in L2 (126 MB; two thirds of it), last blocks of all heads first, so that the short ones at the start of a
  // causal sequence even out the end of the call.
  const double reach = (w.left < 0 ? w.n_k : fmin((double)w.n_k, (double)w.left + (w.right < 0 ? w.n_k : w.right) + 2.0 * kWtRows));
  prm.rows_first = (double)w.batch * w.heads_kv * reach * D * 4 < 80e6;
  // A wait for the next piece can be as long as a piece: 20 us for every step of one, which takes 2, on top of the usual limit.
  const DebugWait debug = debug_wait();
  prm.skip_key_load = debug.skip_key_load;
  prm.wait_limit = debug.limit + (long long)(fmin(reach + w.sinks, (double)w.n_k) / kWtKeys + 4) * 40000;
  prm.wide = (reinterpret_cast<uintptr_t>(w.o) % 32 == 0) && (w.batch == 1 || w.o_b % 16 == 0) && (w.heads_q == 1 || w.o_h % 16 == 0) &&
             (w.n_q == 1 || w.o_n % 16 == 0);
  const int sms = multiprocessors();
  if (sms == 0) return CA_ERR_CUDA;
  // A CTA for every piece: no counter, no list of pieces, and the marks are few enough to be looked at one by one; a launch less.
  prm.w.one_each = w.one_each = n_work <= sms;
  if (!w.one_each) {
    const int rc = launch_window_prepare(w, st);
    if (rc != CA_OK) return rc;
  }
  return D == 64 ? launch_window_tc_d<64>(maps, prm, (int)n_work, st) : launch_window_tc_d<128>(maps, prm, (int)n_work, st);
}

}  // namespace ca
