// Attention of one new token per sequence over a cache in pages, with an optional window and first tokens that stay
// visible:  O = sum_j p_j v_j / sum_j p_j,  p_j = exp(s q.k_j - m),  over the visible rows j of a sequence of n rows,
//     j >= n - 1 - left  or  j < sinks.
//
// What bounds it: reading every visible key and value row once, at 4 d bytes (bf16) and 4 d operations per row and
// query head; the query heads of a key head share the read.  So the rows of a tile are those heads (up to 16), and the products run
// as m16n8k16 (the tcgen05 tiles have 64 rows and more, three quarters of them empty here, and the tensor
// core is not what is waited for).
//
// Split: the visible rows of all sequences and key heads are one line of units, which the CTAs cut into equal
// parts: whatever the lengths, every CTA reads as much as any other.  A part begins and ends anywhere; where a sequence's rows lie in
// several parts, each leaves {O, m, l} in the workspace, and the CTA that is last to do so joins them, in the
// order of the rows, so that results do not depend on the order in which CTAs finish.
// A CTA's warps take the rows of a unit in turn and have their own rings of asynchronous copies: nothing but the end of
// a sequence makes them wait for one another, and copies run ahead across that.  Rows that are not visible are filled with
// zeros instead of being read, so what stands in them (in unused slots of a page, anything) is not seen.
#include <math.h>

#include <type_traits>

#include "kernels.h"
#include "tc_ptx.cuh"

namespace ca {

using namespace ptx;

constexpr int kPagedWarps = 4;
constexpr int kPagedThreads = kPagedWarps * 32;
constexpr int kPagedMaxCtas = 640;           // most CTAs of a launch: the workspace holds two partial results of each

struct PagedParams {
  const void* q;
  long long q_b, q_h;
  void* o;
  long long o_b, o_h;
  float* lse;
  const void *k_pages, *v_pages;
  const int32_t *lengths, *page_table;
  int* status;
  long long* units;              // [batch + 1] units of a (key head, row tile) of the sequences before
  int* arrived;                  // [batch * heads_kv * row_tiles]
  float* partial;                // [2 * CTAs][rows][D + 2]: O (not divided), m (log2 units), l
  int batch, heads_q, heads_kv, group, row_tiles, page_rows, pages, pages_per_sequence, appended, left, sinks;
  float scale_log2;
};

// The visible rows of a sequence as tiles of U rows: tiles of the first tokens, then tiles of the window.
struct Span {
  int n, lo, sink_end, sink_tiles, tile_lo, tiles;
  __device__ __forceinline__ Span(const PagedParams& prm, int b, int U) {
    const long long rows = (long long)prm.lengths[b] + prm.appended, most = (long long)prm.pages_per_sequence * prm.page_rows;
    n = (int)(rows < 0 ? 0 : rows > most ? most : rows);
    lo = prm.left < 0 ? 0 : max(0, n - 1 - prm.left);
    sink_end = min(min(prm.sinks, n), lo);
    tile_lo = lo / U;
    sink_tiles = min((sink_end + U - 1) / U, tile_lo);
    tiles = max(1, sink_tiles + (n + U - 1) / U - tile_lo);       // of no rows one tile without any
  }
  __device__ __forceinline__ int tile(int i) const { return i < sink_tiles ? i : tile_lo + i - sink_tiles; }
  __device__ __forceinline__ bool sees(int j) const { return j < n && (j >= lo || j < sink_end); }
};

// One CTA: units before each sequence, counters and status cleared, lengths looked at.
__global__ void __launch_bounds__(1024) paged_plan_kernel(const __grid_constant__ PagedParams prm, int U) {
  wait_for_previous();
  let_next_start();
  __shared__ long long warp_sum[32];
  __shared__ long long carry;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int segments = prm.batch * prm.heads_kv * prm.row_tiles;
  for (int i = tid; i < segments; i += blockDim.x) prm.arrived[i] = 0;
  int bad = 0;
  if (tid == 0) { carry = 0; prm.units[0] = 0; }
  __syncthreads();
  for (int base = 0; base < prm.batch; base += blockDim.x) {
    const int b = base + tid;
    long long v = 0;
    if (b < prm.batch) {
      const long long rows = (long long)prm.lengths[b] + prm.appended;
      bad |= rows < 0 || rows > (long long)prm.pages_per_sequence * prm.page_rows;
      v = Span(prm, b, U).tiles;
    }
    for (int d = 1; d < 32; d <<= 1) {
      const long long o = __shfl_up_sync(0xffffffffu, v, d);
      if (lane >= d) v += o;
    }
    if (lane == 31) warp_sum[warp] = v;
    __syncthreads();
    long long before = carry;
    for (int w = 0; w < warp; ++w) before += warp_sum[w];
    if (b < prm.batch) prm.units[b + 1] = before + v;
    __syncthreads();
    if (tid == (int)blockDim.x - 1) carry = before + v;
    __syncthreads();
  }
  bad = __syncthreads_or(bad);
  if (tid == 0) *prm.status = bad ? CA_ERR_BAD_INDEX : CA_OK;
}

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool in) {
  const int bytes = in ? 16 : 0;
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4t(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float max_of_keys(float x) {      // over the four lanes that hold a row's columns
  x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
  return fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
}
__device__ __forceinline__ float sum_of_keys(float x) {
  x += __shfl_xor_sync(0xffffffffu, x, 1);
  return x + __shfl_xor_sync(0xffffffffu, x, 2);
}

// Tensor-core products of a warp: 16 query rows against 16 keys at a time.  Accumulator layout of m16n8: a thread holds
// rows lane/4 and lane/4 + 8, columns 2 (lane % 4) and the next of every 8.
template <int D>
struct WarpMma {
  using T = __nv_bfloat16;
  static constexpr int ROWS = 16, KEYS = 16;
  static constexpr int ROW_BYTES = D * 2, CHUNKS = ROW_BYTES / 16;
  uint32_t q[D / 16][4];
  float o[D / 8][4];
  float m[2], l[2];

  __device__ __forceinline__ static int swizzle(int row, int chunk) { return chunk ^ (row & 7); }
  __device__ __forceinline__ void start(const T* qp, long long stride, int rows, int lane) {
    const int r0 = lane >> 2, c0 = (lane & 3) * 2;
#pragma unroll
    for (int k = 0; k < D / 16; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = r0 + (i & 1) * 8, c = k * 16 + c0 + (i >> 1) * 8;
        q[k][i] = r < rows ? *reinterpret_cast<const uint32_t*>(qp + r * stride + c) : 0u;
      }
#pragma unroll
    for (int n = 0; n < D / 8; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[n][i] = 0.f;
    m[0] = m[1] = -INFINITY;
    l[0] = l[1] = 0.f;
  }
  // keys j0 .. j0 + 15 of the sequence, in shared memory at ks and vs
  __device__ __forceinline__ void step(uint32_t ks, uint32_t vs, int j0, const Span& span, float scale, int lane) {
    float s[2][4] = {};
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      uint32_t b[4];
      const int row = (lane & 7) + ((lane >> 4) << 3), chunk = 2 * k + ((lane >> 3) & 1);
      ldmatrix4(ks + row * ROW_BYTES + swizzle(row, chunk) * 16, b);
      mma16816(s[0], q[k], b[0], b[1]);
      mma16816(s[1], q[k], b[2], b[3]);
    }
    const bool whole = j0 >= span.lo ? j0 + KEYS <= span.n : j0 + KEYS <= span.sink_end;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[t][i] *= scale;
        if (!whole && !span.sees(j0 + t * 8 + (lane & 3) * 2 + (i & 1))) s[t][i] = -INFINITY;
      }
    float top[2];
#pragma unroll
    for (int r = 0; r < 2; ++r)
      top[r] = max_of_keys(fmaxf(fmaxf(s[0][2 * r], s[0][2 * r + 1]), fmaxf(s[1][2 * r], s[1][2 * r + 1])));
    if (__any_sync(0xffffffffu, top[0] > m[0] || top[1] > m[1])) {
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const float up = fmaxf(m[r], top[r]);
        const float by = m[r] == -INFINITY ? 0.f : ex2_approx(m[r] - up);
        l[r] *= by;
        m[r] = up;
#pragma unroll
        for (int n = 0; n < D / 8; ++n) { o[n][2 * r] *= by; o[n][2 * r + 1] *= by; }
      }
    }
    // Probabilities in two bf16 parts, the upper bits and the rest: the products have time to spare, and the result the accuracy of
    // fp32.  The rest is kept above zero, so that an infinite value stays one (of a weight that is 1 at least 1e-30 is nothing).
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const float ref = m[r] == -INFINITY ? 0.f : m[r];
        const float p0 = ex2_approx(s[t][2 * r] - ref), p1 = ex2_approx(s[t][2 * r + 1] - ref);
        l[r] += p0 + p1;
        const uint32_t u0 = __float_as_uint(p0) & 0xffff0000u, u1 = __float_as_uint(p1) & 0xffff0000u;
        hi[2 * t + r] = __byte_perm(u0, u1, 0x7632);
        lo[2 * t + r] = pack_bf16x2(fmaxf(p0 - __uint_as_float(u0), 1e-30f), fmaxf(p1 - __uint_as_float(u1), 1e-30f));
      }
#pragma unroll
    for (int n = 0; n < D / 8; n += 2) {
      uint32_t b[4];
      const int row = lane & 15, chunk = n + (lane >> 4);
      ldmatrix4t(vs + row * ROW_BYTES + swizzle(row, chunk) * 16, b);
      mma16816(o[n], hi, b[0], b[1]);
      mma16816(o[n], lo, b[0], b[1]);
      mma16816(o[n + 1], hi, b[2], b[3]);
      mma16816(o[n + 1], lo, b[2], b[3]);
    }
  }
  __device__ __forceinline__ void finish(int) {
    l[0] = sum_of_keys(l[0]);
    l[1] = sum_of_keys(l[1]);
  }
  // rows of the result in fp32: [rows][D] and {m, l} behind them
  __device__ __forceinline__ void put(float* buf, float* ml, int rows, int lane) const {
    const int r0 = lane >> 2, c0 = (lane & 3) * 2;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int row = r0 + 8 * r;
      if (row >= rows) continue;
#pragma unroll
      for (int n = 0; n < D / 8; ++n) *reinterpret_cast<float2*>(buf + row * D + n * 8 + c0) = make_float2(o[n][2 * r], o[n][2 * r + 1]);
      if ((lane & 3) == 0) { ml[2 * row] = m[r]; ml[2 * row + 1] = l[r]; }
    }
  }
};

// fp32 storage: the same on the CUDA cores.  Scores: four lanes to a key, which divide d; values: a lane holds
// four columns (at d = 64 half a warp each takes every other key).  ROWS query rows are worked on.
template <int D, int R>
struct WarpFma {
  using T = float;
  static constexpr int ROWS = R, KEYS = 8;
  static constexpr int ROW_BYTES = D * 4, CHUNKS = ROW_BYTES / 16;
  static constexpr int SPLIT = 128 / D;      // keys that are worked on side by side in P V
  float o[R][4];
  float m[R], l[R];
  const float* qs;                           // [R][D] in shared memory, the warp's own copy
  float* ps;                                 // [KEYS][R] probabilities

  // eight lanes that read at a time are two keys by four chunks: chunks of neighbouring keys in different banks
  __device__ __forceinline__ static int swizzle(int row, int chunk) { return chunk ^ (((row & 1) << 2) | ((row >> 1) & 3)); }
  __device__ __forceinline__ void start(const T* qp, long long stride, int rows, int lane, float* scratch) {
    qs = scratch;
    ps = scratch + R * D;
    __syncwarp();
    for (int i = lane; i < R * D; i += 32) scratch[i] = i / D < rows ? qp[(i / D) * stride + i % D] : 0.f;
    __syncwarp();
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
      for (int i = 0; i < 4; ++i) o[r][i] = 0.f;
      m[r] = -INFINITY;
      l[r] = 0.f;
    }
  }
  __device__ __forceinline__ void step(const unsigned char* ks, const unsigned char* vs, int j0, const Span& span, float scale, int lane) {
    const int key = lane >> 2, quarter = lane & 3;
    float s[R];
#pragma unroll
    for (int r = 0; r < R; ++r) s[r] = 0.f;
#pragma unroll
    for (int i = 0; i < CHUNKS / 4; ++i) {
      const int chunk = quarter + 4 * i;
      const float4 k = *reinterpret_cast<const float4*>(ks + key * ROW_BYTES + swizzle(key, chunk) * 16);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float4 q = *reinterpret_cast<const float4*>(qs + r * D + chunk * 4);
        s[r] = fmaf(q.x, k.x, fmaf(q.y, k.y, fmaf(q.z, k.z, fmaf(q.w, k.w, s[r]))));
      }
    }
    const bool seen = span.sees(j0 + key);
    float p[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      s[r] += __shfl_xor_sync(0xffffffffu, s[r], 1);
      s[r] += __shfl_xor_sync(0xffffffffu, s[r], 2);
      s[r] = seen ? s[r] * scale : -INFINITY;
      float top = s[r];
#pragma unroll
      for (int x = 4; x < 32; x <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
      if (top > m[r]) {
        const float by = m[r] == -INFINITY ? 0.f : ex2_approx(m[r] - top);
        m[r] = top;
        l[r] *= by;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[r][i] *= by;
      }
      p[r] = ex2_approx(s[r] - (m[r] == -INFINITY ? 0.f : m[r]));
      if (quarter == 0) l[r] += p[r];
    }
    __syncwarp();
    if (quarter == 0) {
#pragma unroll
      for (int r = 0; r < R; ++r) ps[key * R + r] = p[r];
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < KEYS / SPLIT; ++i) {
      const int row = i * SPLIT + (SPLIT == 2 ? lane >> 4 : 0), chunk = lane & (CHUNKS - 1);
      const float4 v = *reinterpret_cast<const float4*>(vs + row * ROW_BYTES + swizzle(row, chunk) * 16);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float w = ps[row * R + r];
        o[r][0] = fmaf(w, v.x, o[r][0]);
        o[r][1] = fmaf(w, v.y, o[r][1]);
        o[r][2] = fmaf(w, v.z, o[r][2]);
        o[r][3] = fmaf(w, v.w, o[r][3]);
      }
    }
  }
  __device__ __forceinline__ void finish(int) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
      for (int x = 4; x < 32; x <<= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], x);
      l[r] = __shfl_sync(0xffffffffu, l[r], 0);
      if (SPLIT == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) o[r][i] += __shfl_xor_sync(0xffffffffu, o[r][i], 16);
      }
    }
  }
  __device__ __forceinline__ void put(float* buf, float* ml, int rows, int lane) const {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (r >= rows) break;
      if (lane < CHUNKS) *reinterpret_cast<float4*>(buf + r * D + lane * 4) = make_float4(o[r][0], o[r][1], o[r][2], o[r][3]);
      if (lane == 0) { ml[2 * r] = m[r]; ml[2 * r + 1] = l[r]; }
    }
  }
};

template <typename W, int D>
struct PagedCfg {
  static constexpr bool MMA = std::is_same<typename W::T, __nv_bfloat16>::value;
  static constexpr int U = kPagedWarps * W::KEYS;                  // rows of a unit
  static constexpr int STEP_BYTES = 2 * W::KEYS * W::ROW_BYTES;    // keys and values of a warp's step
  static constexpr int STAGES = 3;
  static constexpr int RING = STAGES * STEP_BYTES;
  static constexpr int SCRATCH = MMA ? 0 : (W::ROWS * D + W::KEYS * W::ROWS) * 4;
  static constexpr int OFF_SCRATCH = kPagedWarps * RING;
  static constexpr int OFF_FLAG = OFF_SCRATCH + kPagedWarps * SCRATCH;
  static constexpr int OFF_ML = OFF_FLAG + 16;                              // [kPagedWarps][ROWS]{m, l}
  static constexpr int OFF_JOIN = OFF_ML + kPagedWarps * W::ROWS * 8;       // [kPagedWarps][rows][D], as many rows as there are
  static_assert(OFF_JOIN % 16 == 0, "alignment");
  static int smem(int rows) { return OFF_JOIN + kPagedWarps * rows * D * 4; }
};

// Where a CTA or one of its warps stands on the line of units.
struct Place {
  int b, h, rt, tile;
  long long left;                // units from here to the end of the part
};

template <typename W, int D>
__global__ void __launch_bounds__(kPagedThreads) paged_kernel(const __grid_constant__ PagedParams prm) {
  using C = PagedCfg<W, D>;
  using T = typename W::T;
  extern __shared__ __align__(128) unsigned char smem[];
  wait_for_previous();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int per = prm.heads_kv * prm.row_tiles;              // (key head, row tile) pairs of a sequence
  const long long total = prm.units[prm.batch] * per;
  const long long parts = min((long long)gridDim.x, total);  // every part has a unit at least
  if (blockIdx.x >= parts) { let_next_start(); return; }
  const long long begin = total * blockIdx.x / parts, end = total * (blockIdx.x + 1) / parts;

  Place at;
  {
    int lo = 0, hi = prm.batch - 1;                          // last sequence whose units begin at or before `begin`
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (prm.units[mid] * per <= begin) lo = mid;
      else hi = mid - 1;
    }
    const long long off = begin - prm.units[lo] * per;
    const int tiles = (int)(prm.units[lo + 1] - prm.units[lo]);
    const int pair = (int)(off / tiles);
    at.b = lo;
    at.h = pair / prm.row_tiles;
    at.rt = pair % prm.row_tiles;
    at.tile = (int)(off % tiles);
    at.left = end - begin;
  }
  auto next_pair = [&](Place& p) {
    p.tile = 0;
    if (++p.rt == prm.row_tiles) {
      p.rt = 0;
      if (++p.h == prm.heads_kv) { p.h = 0; ++p.b; }
    }
  };

  unsigned char* ring = smem + warp * C::RING;
  const uint32_t s_ring = smem_u32(ring);
  // ---- copies: a unit's rows of this warp into the next stage; the page of a row is looked up a step ahead
  Place ld = at;
  Span ld_span(prm, ld.b, C::U);
  int ld_stage = 0;
  int page = 0;
  bool seen = false;
  constexpr int CH = W::CHUNKS, RPI = 32 / CH;               // 16-byte chunks of a row, rows of an instruction
  auto look_up = [&]() {                                     // page of row `lane` of the coming step
    seen = false;
    if (ld.left > 0 && lane < W::KEYS) {
      const int j = ld_span.tile(ld.tile) * C::U + warp * W::KEYS + lane;
      seen = ld_span.sees(j);
      if (seen) page = prm.page_table[(size_t)ld.b * prm.pages_per_sequence + j / prm.page_rows];
    }
  };
  auto load = [&]() {
    if (ld.left > 0) {
      const uint32_t dst = s_ring + ld_stage * C::STEP_BYTES + lane / CH * W::ROW_BYTES;
      int id = seen ? page : -1;
      if (seen && (unsigned)page >= (unsigned)prm.pages) {   // not a page: flagged, its rows read as zeros
        atomicCAS(prm.status, 0, CA_ERR_BAD_INDEX);
        id = -1;
      }
      const int j = ld_span.tile(ld.tile) * C::U + warp * W::KEYS + lane;
      const int slot = ld.h * prm.page_rows + j % prm.page_rows;
      const long long page_elements = (long long)prm.heads_kv * prm.page_rows * D;
#pragma unroll
      for (int i = 0; i < W::KEYS / RPI; ++i) {
        const int row = i * RPI + lane / CH, c = lane % CH;
        const int row_id = __shfl_sync(0xffffffffu, id, row), row_slot = __shfl_sync(0xffffffffu, slot, row);
        const long long off = row_id >= 0 ? row_id * page_elements + (long long)row_slot * D + c * (16 / (int)sizeof(T)) : 0;
        const uint32_t to = dst + i * RPI * W::ROW_BYTES + W::swizzle(row, c) * 16;
        cp_async16(to, static_cast<const T*>(prm.k_pages) + off, row_id >= 0);
        cp_async16(to + W::KEYS * W::ROW_BYTES, static_cast<const T*>(prm.v_pages) + off, row_id >= 0);
      }
      if (--ld.left > 0 && ++ld.tile == ld_span.tiles) {
        const int b = ld.b;
        next_pair(ld);
        if (ld.b != b) ld_span = Span(prm, ld.b, C::U);
      }
    }
    cp_async_commit();
    ld_stage = ld_stage + 1 == C::STAGES ? 0 : ld_stage + 1;
    look_up();
  };
  look_up();
#pragma unroll
  for (int i = 0; i < C::STAGES - 1; ++i) load();

  // an element of the result; a row that sees nothing: zero, log-sum-exp -inf
  auto finish_row = [&](int b, int head, int col, float o, float m, float l) {
    static_cast<T*>(prm.o)[b * prm.o_b + head * prm.o_h + col] = from_f32<T>(l == 0.f ? 0.f : o / l);
    if (col == 0 && prm.lse) prm.lse[(size_t)b * prm.heads_q + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
  };
  W w;
  int stage = 0;
  float* join = reinterpret_cast<float*>(smem + C::OFF_JOIN);
  float* ml = reinterpret_cast<float*>(smem + C::OFF_ML);
  volatile int* flag = reinterpret_cast<volatile int*>(smem + C::OFF_FLAG);
  while (at.left > 0) {
    // ---- one (sequence, key head, row tile): its units in this CTA's part
    const Span span(prm, at.b, C::U);
    const int rows = min(prm.group - at.rt * W::ROWS, W::ROWS);
    const int head0 = at.h * prm.group + at.rt * W::ROWS;    // query head of row 0
    const T* qp = static_cast<const T*>(prm.q) + at.b * prm.q_b + head0 * prm.q_h;
    if constexpr (C::MMA) w.start(qp, prm.q_h, rows, lane);
    else w.start(qp, prm.q_h, rows, lane, reinterpret_cast<float*>(smem + C::OFF_SCRATCH + warp * C::SCRATCH));
    const int first_tile = at.tile;
    const int last_tile = (int)min((long long)span.tiles, first_tile + at.left);      // behind the last
#pragma unroll 1
    for (int t = first_tile; t < last_tile; ++t) {
      cp_async_wait<C::STAGES - 2>();
      __syncwarp();
      const int j0 = span.tile(t) * C::U + warp * W::KEYS;
      const int off = stage * C::STEP_BYTES;
      load();                                                // into the stage that the step before has read
      if (j0 < span.n) {
        if constexpr (C::MMA) w.step(s_ring + off, s_ring + off + W::KEYS * W::ROW_BYTES, j0, span, prm.scale_log2, lane);
        else w.step(ring + off, ring + off + W::KEYS * W::ROW_BYTES, j0, span, prm.scale_log2, lane);
      }
      __syncwarp();
      stage = stage + 1 == C::STAGES ? 0 : stage + 1;
    }
    at.left -= last_tile - first_tile;
    w.finish(lane);
    // ---- the warps' results into one
    const bool whole = first_tile == 0 && last_tile == span.tiles;
    const int all_rows = min(prm.group, W::ROWS);            // rows of a hand-over buffer
    __syncthreads();                                         // the buffers have been read
    w.put(join + warp * all_rows * D, ml + warp * 2 * W::ROWS, rows, lane);
    __syncthreads();
    float* part = prm.partial + (size_t)(2 * blockIdx.x + (first_tile == 0 ? 1 : 0)) * W::ROWS * (D + 2);
    for (int i = threadIdx.x; i < rows * D; i += kPagedThreads) {
      const int r = i / D;
      float top = -INFINITY, o = 0.f, l = 0.f;
#pragma unroll
      for (int x = 0; x < kPagedWarps; ++x) top = fmaxf(top, ml[(x * W::ROWS + r) * 2]);
#pragma unroll
      for (int x = 0; x < kPagedWarps; ++x) {
        const float m = ml[(x * W::ROWS + r) * 2], by = m == -INFINITY ? 0.f : ex2_approx(m - top);
        o = fmaf(join[x * all_rows * D + i], by, o);
        l = fmaf(ml[(x * W::ROWS + r) * 2 + 1], by, l);
      }
      if (whole) {
        finish_row(at.b, head0 + r, i % D, o, top, l);
      } else {
        part[i] = o;
        if (i % D == 0) { part[W::ROWS * D + 2 * r] = top; part[W::ROWS * D + 2 * r + 1] = l; }
      }
    }
    if (!whole) {
      // ---- the last of the CTAs that share these rows joins their results, in the order of the rows
      const long long base = prm.units[at.b] * per + (long long)(at.h * prm.row_tiles + at.rt) * span.tiles;
      const int cta0 = (int)(((base + 1) * parts + total - 1) / total) - 1;
      const int cta1 = (int)(((base + span.tiles) * parts + total - 1) / total) - 1;
      __threadfence();
      __syncthreads();
      if (threadIdx.x == 0) *flag = atomicAdd(&prm.arrived[((long long)at.b * prm.heads_kv + at.h) * prm.row_tiles + at.rt], 1) == cta1 - cta0;
      __syncthreads();
      if (*flag) {
        __threadfence();
        for (int i = threadIdx.x; i < rows * D; i += kPagedThreads) {
          const int r = i / D;
          float top = -INFINITY, o = 0.f, l = 0.f;
          for (int c = cta0; c <= cta1; ++c) {
            const float* p = prm.partial + (size_t)(2 * c + (c == cta0 ? 1 : 0)) * W::ROWS * (D + 2);
            const float pm = __ldcg(p + W::ROWS * D + 2 * r), pl = __ldcg(p + W::ROWS * D + 2 * r + 1), po = __ldcg(p + i);
            const float up = fmaxf(top, pm);
            const float w0 = top == -INFINITY ? 0.f : ex2_approx(top - up), w1 = pm == -INFINITY ? 0.f : ex2_approx(pm - up);
            o = o * w0 + po * w1;
            l = l * w0 + pl * w1;
            top = up;
          }
          finish_row(at.b, head0 + r, i % D, o, top, l);
        }
      }
    }
    next_pair(at);
  }
  let_next_start();
  cp_async_wait<0>();
}

// ---- host side -------------------------------------------------------------------------------------------

static int row_tile(const ca_cache_t& c) {
  if (c.dtype == CA_DTYPE_BF16) return 16;
  const int group = c.heads_q / c.heads_kv;
  return group >= 5 ? 8 : group >= 3 ? 4 : group;
}

struct PagedWs {
  int* status;
  long long* units;
  int* arrived;
  float* partial;
  size_t bytes;
};
static PagedWs carve_paged(const ca_cache_t& c, void* base) {
  PagedWs w{};
  Carver k(base);
  const int rows = row_tile(c);
  w.status = k.take<int>(kStatusBytes / sizeof(int));
  w.units = k.take<long long>((size_t)c.batch + 1);
  w.arrived = k.take<int>((size_t)c.batch * c.heads_kv * ceil_div(c.heads_q / c.heads_kv, rows));
  w.partial = k.take<float>((size_t)2 * kPagedMaxCtas * rows * (c.head_dim + 2));
  w.bytes = k.used();
  return w;
}
size_t paged_workspace_bytes(const ca_cache_t& c) { return carve_paged(c, nullptr).bytes; }

template <typename W, int D>
static int launch_paged_d(PagedParams& prm, LaunchStream st) {
  using C = PagedCfg<W, D>;
  int dev = 0, sms = 0;
  CA_RETURN_IF_CUDA(cudaGetDevice(&dev));
  CA_RETURN_IF_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  prm.row_tiles = ceil_div(prm.group, W::ROWS);
  const int smem = C::smem(min(prm.group, W::ROWS));
  auto kernel = paged_kernel<W, D>;
  CA_RETURN_IF_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  launch_chained(paged_plan_kernel, 1, 1024, 0, st, prm, C::U);
  CA_LAUNCH_CHECK();
  const int per_sm = min(3, (227 * 1024) / (smem + 1024));
  launch_chained(kernel, min(kPagedMaxCtas, sms * per_sm), kPagedThreads, smem, st, prm);
  CA_LAUNCH_CHECK();
  return CA_OK;
}

int launch_paged(const ca_cache_t& c, const ca_rows_t* Q, const void* K_pages, const void* V_pages, const int32_t* lengths, int appended,
                 const int32_t* page_table, float scale, const ca_rows_t* O, float* lse, void* ws, LaunchStream st) {
  const PagedWs w = carve_paged(c, ws);
  PagedParams prm{};
  prm.q = Q->data; prm.q_b = Q->stride_b; prm.q_h = Q->stride_h;
  prm.o = O->data; prm.o_b = O->stride_b; prm.o_h = O->stride_h;
  prm.lse = lse;
  prm.k_pages = K_pages; prm.v_pages = V_pages;
  prm.lengths = lengths; prm.page_table = page_table;
  prm.status = w.status; prm.units = w.units; prm.arrived = w.arrived; prm.partial = w.partial;
  prm.batch = c.batch; prm.heads_q = c.heads_q; prm.heads_kv = c.heads_kv; prm.group = c.heads_q / c.heads_kv;
  prm.page_rows = c.page_rows; prm.pages = c.pages; prm.pages_per_sequence = c.pages_per_sequence;
  prm.appended = appended; prm.left = c.left; prm.sinks = c.sinks;
  prm.scale_log2 = scale * 1.4426950408889634f;
  if (c.dtype == CA_DTYPE_BF16)
    return c.head_dim == 64 ? launch_paged_d<WarpMma<64>, 64>(prm, st) : launch_paged_d<WarpMma<128>, 128>(prm, st);
  auto fp32 = [&](auto rows) {
    constexpr int R = decltype(rows)::value;
    return c.head_dim == 64 ? launch_paged_d<WarpFma<64, R>, 64>(prm, st) : launch_paged_d<WarpFma<128, R>, 128>(prm, st);
  };
  switch (row_tile(c)) {
    case 1: return fp32(std::integral_constant<int, 1>{});
    case 2: return fp32(std::integral_constant<int, 2>{});
    case 4: return fp32(std::integral_constant<int, 4>{});
    default: return fp32(std::integral_constant<int, 8>{});
  }
}

}  // namespace ca
