// Attention of one new token per sequence over a cache in pages, with an optional window and first tokens that stay
// visible:  O = sum_j p_j v_j / sum_j p_j,  p_j = exp(s q.k_j - m),  over the visible rows j of a sequence of n rows,
//     j >= n - 1 - left  or  j < sinks.
//
// What bounds it: reading every visible key and value row once, at 4 d bytes (bf16) and 4 d operations per row and
// query head; the query heads of a key head share the read.  So the rows of a tile are those heads, and the products run as m16n8k16
// (the tcgen05 tiles have 64 rows and more, nine tenths of them empty here, and the tensor core is not what is waited for).
// A warp's step is a chain of products, softmax and products: it is the length of that chain, and how many warps are on it, that
// costs bandwidth before memory does (with the query heads as the 16 rows of the product, half of them empty, 623 instructions a
// step: two sequences of 131,000 rows, 40 heads, 981 us; as its 8 columns 790, 6.8 TB/s).
//
// Split: the visible rows of all sequences and key heads are one line of units, which the CTAs cut into equal
// parts: whatever the lengths, every CTA has as much to do as any other.  A part begins and ends anywhere; where a sequence's rows lie in
// several parts, each leaves {O, m, l} in the workspace, and a last launch joins them in the order of the rows, so that results
// do not depend on the order in which CTAs finish.  (The last CTA of a sequence joining by itself, while its own part waits, took 59 us
// instead of 41 for four sequences of up to 60,000 rows and 16 query heads to a key head, and 85 instead of 51.5 for 64 short ones.)
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
// What the start and the end of a (sequence, key head, row tile) cost, in units of rows: without it the parts that hold many short
// sequences take longest (64 sequences of 1 to 8,192 rows, 8 key heads of 4 query heads, d = 128: 0 90 us, 1 61, 2 51.5, 4 53, 8 57).
constexpr int kPairUnits = 3;
// Caches of at most so many rows a sequence are not split: a CTA for every (sequence, key head, row tile), one launch instead of two or three
// (of 8, 64 and 256 sequences of up to 256 rows, 8 key heads of 4 query heads, d = 128, 7.0, 12.5 and 45 us instead of 10.0, 20 and 60; of
// up to 512 rows 10.1, 18 and 62 instead of 9.9, 24 and 75, one sequence alone 11.1 instead of 8.6; fp32 and d = 64 alike).
constexpr int kDirectRows = 256;
constexpr int kAddUp = 256;                    // sequences whose lengths every CTA adds up by itself; of more, a launch does
constexpr int kPagedMaxCtas = 640;           // most CTAs of a launch: the workspace holds two partial results of each

__host__ __device__ inline int ceil_div_device(int a, int b) { return (a + b - 1) / b; }

struct PagedParams {
  const void* q;
  long long q_b, q_h;
  void* o;
  long long o_b, o_h;
  float* lse;
  const void *k_pages, *v_pages;
  const int32_t *lengths, *page_table;
  int* status;
  long long* units;              // [batch + 1] units of a (key head, row tile) of the sequences before (planned calls)
  int* bad;                      // [CTAs] whether a CTA met a page that is none
  float* partial;                // [2 * CTAs] O [rows][D] (not divided), {m (log2 units), l} [rows]; rows (D + 4) floats apart
  int batch, heads_q, heads_kv, group, row_tiles, page_rows, pages, pages_per_sequence, appended, left, sinks;
  int planned;                   // units come from paged_plan_kernel, otherwise every CTA adds up the lengths itself
  int direct;                    // a CTA for every (sequence, key head, row tile): nothing is planned or joined
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

// One CTA: units before each sequence.
__global__ void __launch_bounds__(1024) paged_plan_kernel(const __grid_constant__ PagedParams prm, int U) {
  wait_for_previous();
  let_next_start();
  __shared__ long long warp_sum[32];
  __shared__ long long carry;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) { carry = 0; prm.units[0] = 0; }
  __syncthreads();
  for (int base = 0; base < prm.batch; base += blockDim.x) {
    const int b = base + tid;
    long long v = 0;
    if (b < prm.batch) v = Span(prm, b, U).tiles + kPairUnits;
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
}

// What the append before left out is missing here: its error stays until the next append.
__device__ __forceinline__ void write_status(const PagedParams& prm, int bad) {
  prm.status[0] = bad || prm.status[kAppendWord] == CA_ERR_BAD_INDEX ? CA_ERR_BAD_INDEX : CA_OK;
}

template <int THREADS>
__device__ __forceinline__ int bad_lengths(const PagedParams& prm) {
  int bad = 0;
  for (int b = threadIdx.x; b < prm.batch; b += THREADS) {
    const long long rows = (long long)prm.lengths[b] + prm.appended;
    bad |= rows < 0 || rows > (long long)prm.pages_per_sequence * prm.page_rows;
  }
  return bad;
}

// Units of all sequences, of those before sequence `b`, and of it, added up by the THREADS threads of a CTA.
struct Units {
  long long total, before;
  int own;
};
template <int THREADS>
__device__ __forceinline__ Units add_units(const PagedParams& prm, int b, int U) {
  __shared__ long long part[THREADS / 32][2];
  long long all = 0, before = 0;
  for (int i = threadIdx.x; i < prm.batch; i += THREADS) {
    const int v = Span(prm, i, U).tiles + kPairUnits;
    all += v;
    if (i < b) before += v;
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    all += __shfl_xor_sync(0xffffffffu, all, d);
    before += __shfl_xor_sync(0xffffffffu, before, d);
  }
  if ((threadIdx.x & 31) == 0) { part[threadIdx.x >> 5][0] = all; part[threadIdx.x >> 5][1] = before; }
  __syncthreads();
  Units r{0, 0, Span(prm, b, U).tiles + kPairUnits};
#pragma unroll
  for (int w = 0; w < THREADS / 32; ++w) { r.total += part[w][0]; r.before += part[w][1]; }
  return r;
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
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// Tensor-core products of a warp, 16 keys at a time, keys (then columns of V) as the rows of the m16n8k16 product and query
// rows as its columns: eight query heads to a key head are one column tile, and no half of the product is empty.
//     S^T = K Q^T      a thread holds keys lane/4 and lane/4 + 8, query rows 2 (lane % 4) and the next
//     O^T += V^T P^T   columns of V lane/4 and lane/4 + 8 of every 16, the same query rows
// (P^T changes hands inside the warp by 8 x 8 transposes.)
template <int D, int NT>
struct WarpMma {
  using T = __nv_bfloat16;
  static constexpr int ROWS = 8 * NT, KEYS = 16, STAGES = NT == 1 ? 3 : 2;
  static constexpr int CTAS = 5 - NT - D / 128;   // to an SM, by registers: 128, 168 or 255
  static constexpr int ROW_BYTES = D * 2, CHUNKS = ROW_BYTES / 16;
  uint32_t q[NT][D / 16][2], coming[NT][D / 16][2];
  float o[NT][D / 16][4];
  float m[NT][2], l[NT][2];

  __device__ __forceinline__ static int swizzle(int row, int chunk) { return chunk ^ (row & 7); }
  // query rows of the work behind the present one, on their way while that is worked on
  __device__ __forceinline__ void prefetch(const T* qp, long long stride, int rows, int lane) {
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int k = 0; k < D / 16; ++k)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int r = t * 8 + (lane >> 2), c = k * 16 + (lane & 3) * 2 + i * 8;
          coming[t][k][i] = r < rows ? *reinterpret_cast<const uint32_t*>(qp + r * stride + c) : 0u;
        }
  }
  __device__ __forceinline__ void start(int) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        q[t][k][0] = coming[t][k][0];
        q[t][k][1] = coming[t][k][1];
#pragma unroll
        for (int i = 0; i < 4; ++i) o[t][k][i] = 0.f;
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) { m[t][i] = -INFINITY; l[t][i] = 0.f; }
    }
  }
  // keys j0 .. j0 + 15 of the sequence, in shared memory at `keys` and `values`
  __device__ __forceinline__ void step(const unsigned char* keys, const unsigned char* values, int j0, const Span& span, float scale, int lane) {
    const uint32_t ks = smem_u32(keys), vs = smem_u32(values);
    float s[NT][4] = {};
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      uint32_t a[4];
      const int row = lane & 15, chunk = 2 * k + (lane >> 4);
      ldmatrix4(ks + row * ROW_BYTES + swizzle(row, chunk) * 16, a);
#pragma unroll
      for (int t = 0; t < NT; ++t) mma16816(s[t], a, q[t][k][0], q[t][k][1]);
    }
    const bool whole = j0 >= span.lo ? j0 + KEYS <= span.n : j0 + KEYS <= span.sink_end;
    if (!whole) {
      const bool first = span.sees(j0 + (lane >> 2)), second = span.sees(j0 + (lane >> 2) + 8);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        if (!first) s[t][0] = s[t][1] = -INFINITY;
        if (!second) s[t][2] = s[t][3] = -INFINITY;
      }
    }
    uint32_t hi[NT][2], lo[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      float top[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        top[i] = fmaxf(s[t][i], s[t][2 + i]);
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], x));
        top[i] *= scale;
      }
      if (__any_sync(0xffffffffu, top[0] > m[t][0] || top[1] > m[t][1])) {
        float by[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float up = fmaxf(m[t][i], top[i]);
          by[i] = m[t][i] == -INFINITY ? 0.f : ex2_approx(m[t][i] - up);
          l[t][i] *= by[i];
          m[t][i] = up;
        }
#pragma unroll
        for (int n = 0; n < D / 16; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[t][n][i] *= by[i & 1];
      }
      // Probabilities in two bf16 parts, the upper bits and the rest, since the products have time to spare: a weight is off by 2^-16 of
      // itself (the rest is below 2^-8 of it and rounded by 2^-8).  The rest is at least 2^-24 of the probability: where it is zero, 0 x
      // infinity would make an infinite value a NaN, and of a weight that is itself zero it stays zero, however large the value.
      const float ref0 = m[t][0] == -INFINITY ? 0.f : -m[t][0], ref1 = m[t][1] == -INFINITY ? 0.f : -m[t][1];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float p0 = ex2_approx(fmaf(s[t][2 * h], scale, ref0)) * kWeightScale, p1 = ex2_approx(fmaf(s[t][2 * h + 1], scale, ref1)) * kWeightScale;
        l[t][0] += p0;
        l[t][1] += p1;
        const uint32_t u0 = __float_as_uint(p0) & 0xffff0000u, u1 = __float_as_uint(p1) & 0xffff0000u;
        hi[t][h] = transpose8x8(__byte_perm(u0, u1, 0x7632));
        lo[t][h] = transpose8x8(pack_bf16x2(fmaxf(p0 - __uint_as_float(u0), p0 * 0x1p-24f), fmaxf(p1 - __uint_as_float(u1), p1 * 0x1p-24f)));
      }
    }
#pragma unroll
    for (int n = 0; n < D / 16; ++n) {
      uint32_t a[4];
      const int row = (lane & 7) + ((lane >> 4) << 3), chunk = 2 * n + ((lane >> 3) & 1);
      ldmatrix4t(vs + row * ROW_BYTES + swizzle(row, chunk) * 16, a);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        mma16816(o[t][n], a, hi[t][0], hi[t][1]);
        mma16816(o[t][n], a, lo[t][0], lo[t][1]);
      }
    }
  }
  // the result in fp32: [rows][D] by place(), and {m, l} of each row
  __device__ __forceinline__ void put(float* buf, float* ml, int rows, int lane) {
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) l[t][i] += __shfl_xor_sync(0xffffffffu, l[t][i], x);
        const int row = t * 8 + (lane & 3) * 2 + i;
        if (row >= rows) continue;
#pragma unroll
        for (int n = 0; n < D / 16; ++n) {
          const int col = n * 16 + (lane >> 2);
          buf[row * D + place(row, col)] = o[t][n][i];
          buf[row * D + place(row, col + 8)] = o[t][n][2 + i];
        }
        if (lane < 4) { ml[2 * row] = m[t][i]; ml[2 * row + 1] = l[t][i]; }
      }
  }
  // where column `col` of a row lies: the lanes that write at a time are four rows apart, in different banks
  __device__ __forceinline__ static int place(int row, int col) { return col ^ (((row >> 1) & 3) << 3); }
};

// fp32 storage: the same on the CUDA cores, two multiply-adds to an instruction.  Scores: four lanes to a key, which divide d; values: a
// lane holds four columns (at d = 64 half a warp each takes every other key).  R query rows are worked on.
template <int D, int R>
struct WarpFma {
  using T = float;
  static constexpr int ROWS = R, KEYS = 8, STAGES = 3;
  static constexpr int CTAS = D == 128 ? (R > 2 ? 1 : 2) : R > 1 ? 3 : 4;   // to an SM, by shared memory and by registers
  static constexpr int ROW_BYTES = D * 4, CHUNKS = ROW_BYTES / 16;
  static constexpr int SPLIT = 128 / D;      // keys that are worked on side by side in P V
  static constexpr bool HELD = R * D <= 256; // query rows in registers (a quarter of each: R D / 4), otherwise in shared memory
  static constexpr int SCRATCH = HELD ? KEYS * R : R * D + KEYS * R;
  f32x2 o[R][2];
  float m[R], l[R];
  float4 held[HELD ? R : 1][CHUNKS / 4];
  float coming[R * D / 32];
  float *qs, *ps;                            // the warp's own: [R][D] query rows, [KEYS][R] probabilities

  // eight lanes that read at a time are two keys by four chunks: chunks of neighbouring keys in different banks
  __device__ __forceinline__ static int swizzle(int row, int chunk) { return chunk ^ (((row & 1) << 2) | ((row >> 1) & 3)); }
  __device__ __forceinline__ void prefetch(const T* qp, long long stride, int rows, int lane) {
#pragma unroll
    for (int i = 0; i < R * D / 32; ++i) {
      const int e = i * 32 + lane;
      coming[i] = e / D < rows ? qp[e / D * stride + e % D] : 0.f;
    }
  }
  __device__ __forceinline__ void start(int lane, float* scratch, float* buf) {
    ps = scratch;
    qs = HELD ? buf : scratch + KEYS * R;    // (held rows only pass through the hand-over buffer)
    __syncwarp();
#pragma unroll
    for (int i = 0; i < R * D / 32; ++i) qs[i * 32 + lane] = coming[i];
    __syncwarp();
    if (HELD) {
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < CHUNKS / 4; ++i) held[r][i] = *reinterpret_cast<const float4*>(qs + r * D + ((lane & 3) + 4 * i) * 4);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      o[r][0] = o[r][1] = pack2(0.f, 0.f);
      m[r] = -INFINITY;
      l[r] = 0.f;
    }
  }
  __device__ __forceinline__ void step(const unsigned char* ks, const unsigned char* vs, int j0, const Span& span, float scale, int lane) {
    const int key = lane >> 2, quarter = lane & 3;
    f32x2 s2[R][2];
#pragma unroll
    for (int r = 0; r < R; ++r) s2[r][0] = s2[r][1] = pack2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < CHUNKS / 4; ++i) {
      const int chunk = quarter + 4 * i;
      const float4 k = *reinterpret_cast<const float4*>(ks + key * ROW_BYTES + swizzle(key, chunk) * 16);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float4 q = HELD ? held[HELD ? r : 0][i] : *reinterpret_cast<const float4*>(qs + r * D + chunk * 4);
        s2[r][0] = fma2(pack2(q.x, q.y), pack2(k.x, k.y), s2[r][0]);
        s2[r][1] = fma2(pack2(q.z, q.w), pack2(k.z, k.w), s2[r][1]);
      }
    }
    const bool seen = span.sees(j0 + key);
    float s[R], p[R];
    bool up = false;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float a, b, c, d;
      unpack2(s2[r][0], a, b);
      unpack2(s2[r][1], c, d);
      s[r] = (a + b) + (c + d);
      s[r] += __shfl_xor_sync(0xffffffffu, s[r], 1);
      s[r] += __shfl_xor_sync(0xffffffffu, s[r], 2);
      s[r] = seen ? s[r] * scale : -INFINITY;
      up = up || s[r] > m[r];
    }
    if (__any_sync(0xffffffffu, up)) {       // a new maximum of some row
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float top = fmaxf(m[r], s[r]);
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
        const float by = m[r] == -INFINITY ? 0.f : ex2_approx(m[r] - top);
        m[r] = top;
        l[r] *= by;
        o[r][0] = mul2(o[r][0], pack2(by, by));
        o[r][1] = mul2(o[r][1], pack2(by, by));
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      p[r] = ex2_approx(s[r] - (m[r] == -INFINITY ? 0.f : m[r])) * kWeightScale;
      if (quarter == 0) l[r] += p[r];
    }
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
        o[r][0] = fma2(pack2(w, w), pack2(v.x, v.y), o[r][0]);
        o[r][1] = fma2(pack2(w, w), pack2(v.z, v.w), o[r][1]);
      }
    }
    __syncwarp();                            // the probabilities have been read
  }
  __device__ __forceinline__ void put(float* buf, float* ml, int rows, int lane) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
      for (int x = 4; x < 32; x <<= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], x);
      float v[4];
      unpack2(o[r][0], v[0], v[1]);
      unpack2(o[r][1], v[2], v[3]);
      if (SPLIT == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], 16);
      }
      if (r >= rows) continue;
      if (lane < CHUNKS) *reinterpret_cast<float4*>(buf + r * D + lane * 4) = make_float4(v[0], v[1], v[2], v[3]);
      if (lane == 0) { ml[2 * r] = m[r]; ml[2 * r + 1] = l[r]; }
    }
  }
  __device__ __forceinline__ static int place(int, int col) { return col; }
};

template <typename W>
constexpr int scratch_floats() {
  if constexpr (std::is_same<typename W::T, float>::value) return W::SCRATCH;
  else return 0;
}

template <typename W, int D>
struct PagedCfg {
  static constexpr bool MMA = std::is_same<typename W::T, __nv_bfloat16>::value;
  static constexpr int U = kPagedWarps * W::KEYS;                  // rows of a unit
  static constexpr int STEP_BYTES = 2 * W::KEYS * W::ROW_BYTES;    // keys and values of a warp's step
  static constexpr int STAGES = W::STAGES;
  static constexpr int RING = STAGES * STEP_BYTES;
  static constexpr int SCRATCH = scratch_floats<W>() * 4;
  static constexpr int OFF_SCRATCH = kPagedWarps * RING;
  static constexpr int OFF_ML = OFF_SCRATCH + kPagedWarps * SCRATCH;        // [kPagedWarps][ROWS]{m, l}
  static constexpr int OFF_JOIN = OFF_ML + kPagedWarps * W::ROWS * 8;       // [kPagedWarps][rows][D], as many rows as there are
  static_assert(OFF_JOIN % 16 == 0 && SCRATCH % 16 == 0, "alignment");
  // rows of a hand-over buffer: as many as there are (query rows in fp32 pass through it in whole tiles)
  __host__ __device__ static int buffer_rows(int group) { return MMA && group < W::ROWS ? group : W::ROWS; }
  static int smem(int group) {
    return OFF_JOIN + kPagedWarps * buffer_rows(group) * D * 4;
  }
};

__device__ __forceinline__ void add_scaled(float4& o, float4 v, float by) {
  o.x = fmaf(v.x, by, o.x);
  o.y = fmaf(v.y, by, o.y);
  o.z = fmaf(v.z, by, o.z);
  o.w = fmaf(v.w, by, o.w);
}

// The line of units: of every (sequence, key head, row tile) kPairUnits and then its tiles.  Part c of `parts` is [total c / parts,
// total (c + 1) / parts); the part that holds position x:
__device__ __forceinline__ int part_of(long long x, long long parts, long long total) { return (int)(((x + 1) * parts + total - 1) / total) - 1; }

// Where a CTA or one of its warps stands in its part: tiles [tile, last) of a (sequence, key head, row tile).
struct Place {
  int b, h, rt, tile, last;
  long long pos, end;                        // where the next one begins on the line, where the part ends
  __device__ __forceinline__ bool there() const { return tile < last; }
  // tiles of the part in the one that begins at `base`, from position `from` on
  __device__ __forceinline__ void cut(long long base, long long from, int tiles) {
    const long long first = from - base - kPairUnits, behind = min(end, base + kPairUnits + tiles) - base - kPairUnits;
    tile = (int)max(0LL, first);
    last = (int)max(0LL, behind);
    pos = base + kPairUnits + tiles;
  }
  // position `begin` in sequence `seq`, which begins at `base` and has `each` units per (key head, row tile)
  __device__ __forceinline__ void place(int seq, long long base, int each, int row_tiles, long long begin) {
    const int pair = (int)((begin - base) / each);
    b = seq;
    h = pair / row_tiles;
    rt = pair % row_tiles;
    cut(base + (long long)pair * each, begin, each - kPairUnits);
  }
  // the next one; `span` follows the sequence
  __device__ __forceinline__ void next(const PagedParams& prm, Span& span, int U) {
    tile = last = 0;
    while (!there() && pos < end) {
      if (++rt == prm.row_tiles) {
        rt = 0;
        if (++h == prm.heads_kv) {
          h = 0;
          ++b;
          span = Span(prm, b, U);
        }
      }
      cut(pos, pos, span.tiles);
    }
  }
};

// four columns of the mean; of a row that sees nothing zeros
__device__ __forceinline__ float4 mean_of(float4 o, float l) {
  return l == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(o.x / l, o.y / l, o.z / l, o.w / l);
}
// whether they are to be taken again: not finite, though the weights are
__device__ __forceinline__ bool beyond(float4 mean, float l) {
  return l < INFINITY && !(fabsf(mean.x) < INFINITY && fabsf(mean.y) < INFINITY && fabsf(mean.z) < INFINITY && fabsf(mean.w) < INFINITY);
}
template <typename T>
__device__ __forceinline__ float4 replaced(float4 mean, float4 small, float l) {
  if (!(fabsf(mean.x) < INFINITY)) mean.x = mean_of_small<T>(small.x, l);
  if (!(fabsf(mean.y) < INFINITY)) mean.y = mean_of_small<T>(small.y, l);
  if (!(fabsf(mean.z) < INFINITY)) mean.z = mean_of_small<T>(small.z, l);
  if (!(fabsf(mean.w) < INFINITY)) mean.w = mean_of_small<T>(small.w, l);
  return mean;
}
// Sums of weighted small values of a query head, by a warp: of the visible rows, 32 at a time, groups first, first + step, ... .  A lane
// weighs one of the 32, then has columns lane D / 32 and the next.  Slow, and called only for sums beyond fp32 and where values in sight are
// infinite or NaN: with a NaN in each sequence, 64 of up to 8,192 rows, 8 key heads of 4 query heads, take 1.5 ms instead of 0.05, two of 131,000
// rows, 40 heads, 7.2 instead of 0.8.
template <typename T, int D>
__device__ __noinline__ float4 small_sums(const PagedParams& prm, int b, int h, int head, float m, int first, int step) {
  const int lane = threadIdx.x & 31;
  const Span span(prm, b, 32);
  const int count = span.sink_end + span.n - span.lo;
  const T* q = static_cast<const T*>(prm.q) + b * prm.q_b + head * prm.q_h;
  float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
  for (int c = first * 32; c < count; c += step * 32) {
    float weight = 0.f;
    long long at = -1;                         // (a row of a page that is none is zero, key and value)
    if (c + lane < count) {
      const int j = c + lane < span.sink_end ? c + lane : span.lo + (c + lane - span.sink_end);
      const int page = prm.page_table[(size_t)b * prm.pages_per_sequence + j / prm.page_rows];
      float s = 0.f;
      if ((unsigned)page < (unsigned)prm.pages) {
        at = (((long long)page * prm.heads_kv + h) * prm.page_rows + j % prm.page_rows) * D;
        const T* k = static_cast<const T*>(prm.k_pages) + at;
#pragma unroll 4
        for (int i = 0; i < D; i += 4) {
          const float4 x = load4(q + i), y = load4(k + i);
          s = fmaf(x.x, y.x, fmaf(x.y, y.y, fmaf(x.z, y.z, fmaf(x.w, y.w, s))));
        }
      }
      weight = ex2_approx(fmaf(s, prm.scale_log2, -m)) * kWeightScale;
    }
    const int rows = min(32, count - c);
#pragma unroll 1
    for (int i = 0; i < rows; i += 4) {        // (four rows on their way; of those that are not there weight and value are zero)
      struct __align__(D / 32 * sizeof(T)) Row { T e[D / 32]; } v[4];
      float w[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        w[k] = __shfl_sync(0xffffffffu, weight, i + k);
        const long long from = __shfl_sync(0xffffffffu, at, i + k);
#pragma unroll
        for (int e = 0; e < D / 32; ++e) v[k].e[e] = from_f32<T>(0.f);
        if (from >= 0) v[k] = *reinterpret_cast<const Row*>(static_cast<const T*>(prm.v_pages) + from + lane * (D / 32));
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        sum.x = fmaf(w[k], to_f32<T>(v[k].e[0]) * kValueScale, sum.x);
        sum.y = fmaf(w[k], to_f32<T>(v[k].e[1]) * kValueScale, sum.y);
        if (D == 128) {
          sum.z = fmaf(w[k], to_f32<T>(v[k].e[2 % (D / 32)]) * kValueScale, sum.z);
          sum.w = fmaf(w[k], to_f32<T>(v[k].e[3 % (D / 32)]) * kValueScale, sum.w);
        }
      }
    }
  }
  return sum;
}
// The means of a warp, four columns to a lane (at d = 64 of two query heads), where some are to be taken again.
template <typename T, int D>
__device__ __noinline__ float4 taken_again(const PagedParams& prm, int b, int h, int head, float4 mean, float m, float l) {
  constexpr int LANES = D / 4;
  const int lane = threadIdx.x & 31;
  const bool need = beyond(mean, l);
#pragma unroll 1
  for (int side = 0; side < 32 / LANES; ++side) {
    const bool mine = lane / LANES == side;
    if (!__any_sync(0xffffffffu, need && mine)) continue;
    float4 s = small_sums<T, D>(prm, b, h, __shfl_sync(0xffffffffu, head, side * LANES), __shfl_sync(0xffffffffu, m, side * LANES), 0, 1);
    if (D == 64) {                             // two lanes' columns are the four of one
      const int a = lane % LANES * 2;
      s = make_float4(__shfl_sync(0xffffffffu, s.x, a), __shfl_sync(0xffffffffu, s.y, a), __shfl_sync(0xffffffffu, s.x, a + 1), __shfl_sync(0xffffffffu, s.y, a + 1));
    }
    if (mine) mean = replaced<T>(mean, s, l);
  }
  return mean;
}

// four columns of the result; a row that sees nothing has a log-sum-exp of -inf
template <typename T>
__device__ __forceinline__ void finish_row(const PagedParams& prm, int b, int head, int col, float4 mean, float m, float l) {
  store4(static_cast<T*>(prm.o) + b * prm.o_b + head * prm.o_h + col, mean);
  if (col == 0 && prm.lse) prm.lse[(size_t)b * prm.heads_q + head] = l == 0.f ? -INFINITY : (m + log2f(l * kWeightBack)) * 0.6931471805599453f;
}

template <typename W, int D>
__global__ void __launch_bounds__(kPagedThreads, W::CTAS) paged_kernel(const __grid_constant__ PagedParams prm) {
  using C = PagedCfg<W, D>;
  using T = typename W::T;
  extern __shared__ __align__(128) unsigned char smem[];
  wait_for_previous();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int per = prm.heads_kv * prm.row_tiles;              // (key head, row tile) pairs of a sequence
  auto no_part = [&]() {
    if (threadIdx.x == 0) prm.bad[blockIdx.x] = 0;
    let_next_start();
  };
  int bad = 0;
  Place at;
  if (prm.direct) {
    at.b = blockIdx.x / per;
    at.h = blockIdx.x % per / prm.row_tiles;
    at.rt = blockIdx.x % prm.row_tiles;
    at.pos = at.end = 0;                                     // (none behind it)
    at.tile = 0;
    at.last = Span(prm, at.b, C::U).tiles;
  } else if (prm.planned) {
    const long long total = prm.units[prm.batch] * per;
    const long long parts = min((long long)gridDim.x, total);
    if (blockIdx.x >= parts) { no_part(); return; }
    const long long begin = total * blockIdx.x / parts;
    at.end = total * (blockIdx.x + 1) / parts;
    int lo = 0, hi = prm.batch - 1;                          // last sequence whose units begin at or before `begin`
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (prm.units[mid] * per <= begin) lo = mid;
      else hi = mid - 1;
    }
    at.place(lo, prm.units[lo] * per, (int)(prm.units[lo + 1] - prm.units[lo]), prm.row_tiles, begin);
  } else {
    // Every CTA adds up the lengths by itself: thread t has sequences 2 t and 2 t + 1.
    static_assert(kAddUp == 2 * kPagedThreads, "two sequences to a thread");
    long long* sums = reinterpret_cast<long long*>(smem);    // (the rings are not in use yet) [4] of warps, then what is found
    const int b0 = 2 * (int)threadIdx.x;
    const int v0 = b0 < prm.batch ? Span(prm, b0, C::U).tiles + kPairUnits : 0, v1 = b0 + 1 < prm.batch ? Span(prm, b0 + 1, C::U).tiles + kPairUnits : 0;
    long long behind = (long long)v0 + v1;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const long long o = __shfl_up_sync(0xffffffffu, behind, d);
      if (lane >= d) behind += o;
    }
    if (lane == 31) sums[warp] = behind;
    __syncthreads();
    long long total = 0;
#pragma unroll
    for (int w = 0; w < kPagedWarps; ++w) {
      if (w < warp) behind += sums[w];
      total += sums[w];
    }
    total *= per;
    const long long parts = min((long long)gridDim.x, total);
    if (blockIdx.x >= parts) { no_part(); return; }
    const long long begin = total * blockIdx.x / parts;
    at.end = total * (blockIdx.x + 1) / parts;
    const long long base1 = (behind - v1) * per, base0 = base1 - (long long)v0 * per;
    if (v0 && begin >= base0 && begin < base1) { sums[4] = b0; sums[5] = base0; sums[6] = v0; }
    if (v1 && begin >= base1 && begin < behind * per) { sums[4] = b0 + 1; sums[5] = base1; sums[6] = v1; }
    __syncthreads();
    at.place((int)sums[4], sums[5], (int)sums[6], prm.row_tiles, begin);
    __syncthreads();                                         // (read before the rings are filled)
  }
  Span span(prm, at.b, C::U);
  if (!at.there()) at.next(prm, span, C::U);

  unsigned char* ring = smem + warp * C::RING;
  const uint32_t s_ring = smem_u32(ring);
  // ---- copies: a unit's rows of this warp into the next stage; the page of a row is looked up a step ahead
  Place ld = at;
  Span ld_span = span;
  int ld_stage = 0;
  constexpr int CH = W::CHUNKS, RPI = 32 / CH;               // 16-byte chunks of a row, rows of an instruction
  const bool aligned = prm.page_rows % W::KEYS == 0;         // a step's rows are in one page, side by side
  const long long page_elements = (long long)prm.heads_kv * prm.page_rows * D;
  int page = 0;
  bool seen = false;
  auto look_up = [&]() {                                     // page of row `lane` of the coming step
    seen = false;
    if (ld.there() && lane < W::KEYS) {
      const int j = ld_span.tile(ld.tile) * C::U + warp * W::KEYS + lane;
      seen = ld_span.sees(j);
      if (seen) page = prm.page_table[(size_t)ld.b * prm.pages_per_sequence + j / prm.page_rows];
    }
  };
  auto load = [&]() {
    if (ld.there()) {
      const int row0 = lane / CH, c = lane % CH;
      const int j = ld_span.tile(ld.tile) * C::U + warp * W::KEYS;
      const uint32_t dst = s_ring + ld_stage * C::STEP_BYTES + row0 * W::ROW_BYTES;
      int id = seen ? page : -1;
      if (seen && (unsigned)page >= (unsigned)prm.pages) {   // not a page: flagged, its rows read as zeros
        bad = 1;
        id = -1;
      }
      if (aligned && __all_sync(0xffffffffu, id >= 0 || lane >= W::KEYS)) {
        const long long off = __shfl_sync(0xffffffffu, id, 0) * page_elements + (long long)(ld.h * prm.page_rows + j % prm.page_rows + row0) * D + c * (16 / (int)sizeof(T));
        const T* k = static_cast<const T*>(prm.k_pages) + off;
        const T* v = static_cast<const T*>(prm.v_pages) + off;
#pragma unroll
        for (int i = 0; i < W::KEYS / RPI; ++i) {
          const uint32_t to = dst + i * RPI * W::ROW_BYTES + W::swizzle(i * RPI + row0, c) * 16;
          cp_async16(to, k + i * RPI * D, true);
          cp_async16(to + W::KEYS * W::ROW_BYTES, v + i * RPI * D, true);
        }
      } else {
        const int slot = ld.h * prm.page_rows + (j + lane) % prm.page_rows;
#pragma unroll
        for (int i = 0; i < W::KEYS / RPI; ++i) {
          const int row = i * RPI + row0;
          const int row_id = __shfl_sync(0xffffffffu, id, row), row_slot = __shfl_sync(0xffffffffu, slot, row);
          const long long off = row_id >= 0 ? row_id * page_elements + (long long)row_slot * D + c * (16 / (int)sizeof(T)) : 0;
          const uint32_t to = dst + i * RPI * W::ROW_BYTES + W::swizzle(row, c) * 16;
          cp_async16(to, static_cast<const T*>(prm.k_pages) + off, row_id >= 0);
          cp_async16(to + W::KEYS * W::ROW_BYTES, static_cast<const T*>(prm.v_pages) + off, row_id >= 0);
        }
      }
      if (++ld.tile == ld.last) ld.next(prm, ld_span, C::U);
    }
    cp_async_commit();
    ld_stage = ld_stage + 1 == C::STAGES ? 0 : ld_stage + 1;
    look_up();
  };
  look_up();
#pragma unroll
  for (int i = 0; i < C::STAGES - 1; ++i) load();

  W w;
  int stage = 0;
  float* join = reinterpret_cast<float*>(smem + C::OFF_JOIN);
  float* ml = reinterpret_cast<float*>(smem + C::OFF_ML);
  auto head_of = [&](const Place& p) { return p.h * prm.group + p.rt * W::ROWS; };        // query head of row 0
  auto rows_of = [&](const Place& p) { return min(prm.group - p.rt * W::ROWS, W::ROWS); };
  auto prefetch_queries = [&](const Place& p) {
    w.prefetch(static_cast<const T*>(prm.q) + p.b * prm.q_b + head_of(p) * prm.q_h, prm.q_h, rows_of(p), lane);
  };
  if (at.there()) prefetch_queries(at);
  const int all_rows = C::buffer_rows(prm.group);
  float* mine = join + warp * all_rows * D;
  while (at.there()) {
    // ---- one (sequence, key head, row tile): its units in this CTA's part
    const int rows = rows_of(at), head0 = head_of(at);
    if constexpr (C::MMA) w.start(lane);
    else w.start(lane, reinterpret_cast<float*>(smem + C::OFF_SCRATCH + warp * C::SCRATCH), mine);
    const int first_tile = at.tile, last_tile = at.last;
    Place coming = at;
    Span coming_span = span;
    coming.next(prm, coming_span, C::U);
    if (coming.there()) prefetch_queries(coming);
#pragma unroll 1
    for (int t = first_tile; t < last_tile; ++t) {
      cp_async_wait<C::STAGES - 2>();
      __syncwarp();
      const int j0 = span.tile(t) * C::U + warp * W::KEYS;
      const unsigned char* keys = ring + stage * C::STEP_BYTES;
      load();                                                // into the stage that the step before has read
      if (j0 < span.n) w.step(keys, keys + W::KEYS * W::ROW_BYTES, j0, span, prm.scale_log2, lane);
      __syncwarp();
      stage = stage + 1 == C::STAGES ? 0 : stage + 1;
    }
    // ---- the warps' results into one
    const bool whole = first_tile == 0 && last_tile == span.tiles;
    w.put(mine, ml + warp * 2 * W::ROWS, rows, lane);
    __syncthreads();
    float* part = prm.partial + (size_t)(2 * blockIdx.x + (first_tile == 0 ? 1 : 0)) * W::ROWS * (D + 4);
    for (int first = warp * 32; first < rows * (D / 4); first += kPagedThreads) {      // (by whole warps)
      const int i = first + lane, r = min(i / (D / 4), rows - 1), col = i % (D / 4) * 4;
      const bool live = i < rows * (D / 4);
      float top = -INFINITY, l = 0.f;
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int x = 0; x < kPagedWarps; ++x) top = fmaxf(top, ml[(x * W::ROWS + r) * 2]);
#pragma unroll
      for (int x = 0; x < kPagedWarps; ++x) {
        const float m = ml[(x * W::ROWS + r) * 2], by = m == -INFINITY ? 0.f : ex2_approx(m - top);
        const float4 v = *reinterpret_cast<const float4*>(join + (x * all_rows + r) * D + W::place(r, col));
        add_scaled(o, v, by);
        l = fmaf(ml[(x * W::ROWS + r) * 2 + 1], by, l);
      }
      if (whole) {
        float4 mean = mean_of(o, l);
        if (__any_sync(0xffffffffu, beyond(mean, l))) mean = taken_again<T, D>(prm, at.b, at.h, head0 + r, mean, top, l);
        if (live) finish_row<T>(prm, at.b, head0 + r, col, mean, top, l);
      } else if (live) {
        *reinterpret_cast<float4*>(part + r * D + col) = o;
        if (col == 0) *reinterpret_cast<float2*>(part + W::ROWS * D + 2 * r) = make_float2(top, l);
      }
    }
    __syncthreads();                                         // the hand-over buffers have been read
    at = coming;
    span = coming_span;
  }
  let_next_start();
  cp_async_wait<0>();
  if (!prm.direct) {
    bad = __syncthreads_or(bad);
    if (threadIdx.x == 0) prm.bad[blockIdx.x] = bad;         // (the launch that joins makes the status of it)
  } else if (blockIdx.x == 0) {
    // This CTA looks at every index of the call and alone writes the status word, so that nothing has to clear it first.
    bad = bad_lengths<kPagedThreads>(prm);
    const unsigned entries = (unsigned)prm.batch * (unsigned)prm.pages_per_sequence;      // (few: kDirectRows of each sequence)
#pragma unroll 4
    for (unsigned e = threadIdx.x; e < entries; e += kPagedThreads) {
      const int b = (int)(e / (unsigned)prm.pages_per_sequence), first = (int)(e % (unsigned)prm.pages_per_sequence) * prm.page_rows;
      const Span s(prm, b, C::U);
      const bool read = first < s.n && (first + prm.page_rows > s.lo || first < s.sink_end);
      if (read) bad |= (unsigned)prm.page_table[e] >= (unsigned)prm.pages;
    }
    bad = __syncthreads_or(bad);
    if (threadIdx.x == 0) write_status(prm, bad);
  }
}

// Results of the parts that share a (sequence, key head, row tile) into one, in the order of the rows, whichever was
// finished first.  A CTA takes two query rows: 256 threads are a float4 of a row each, by groups of parts (part g, g + groups, ...), and
// have the loads of eight parts in flight; then the groups are joined in shared memory.
constexpr int kJoinThreads = 256, kJoinRows = 2;
template <typename W, int D>
__global__ void __launch_bounds__(kJoinThreads, 3) paged_join_kernel(const __grid_constant__ PagedParams prm, int ctas) {
  using C = PagedCfg<W, D>;
  wait_for_previous();
  let_next_start();
  const int chunks = ceil_div_device(min(prm.group, W::ROWS), kJoinRows);
  const int chunk = blockIdx.x % chunks, pair = blockIdx.x / chunks, per = prm.heads_kv * prm.row_tiles;
  const int b = pair / per, h = pair % per / prm.row_tiles, rt = pair % prm.row_tiles;
  if (blockIdx.x == 0) {
    // the status: this CTA alone writes it
    int bad = bad_lengths<kJoinThreads>(prm);
    for (int c = threadIdx.x; c < ctas; c += kJoinThreads) bad |= prm.bad[c];
    bad = __syncthreads_or(bad);
    if (threadIdx.x == 0) write_status(prm, bad);
  }
  Units u;
  if (prm.planned) u = Units{prm.units[prm.batch], prm.units[b], (int)(prm.units[b + 1] - prm.units[b])};
  else u = add_units<kJoinThreads>(prm, b, C::U);
  const int each = u.own;
  const long long total = u.total * per, parts = min((long long)ctas, total);
  const long long base = u.before * per + (long long)(pair % per) * each;
  const int cta0 = part_of(base + kPairUnits, parts, total), cta1 = part_of(base + each - 1, parts, total);
  const int row0 = chunk * kJoinRows, rows = min(min(prm.group - rt * W::ROWS, W::ROWS) - row0, kJoinRows);
  if (cta0 == cta1 || rows <= 0) return;
  constexpr int ITEMS = kJoinRows * D / 4, GROUPS = kJoinThreads / ITEMS;
  __shared__ float4 sum[GROUPS][ITEMS];
  __shared__ float2 ml[GROUPS][ITEMS];
  const int item = threadIdx.x % ITEMS, g = threadIdx.x / ITEMS, r = min(item / (D / 4), rows - 1), col = item % (D / 4) * 4;
  float top = -INFINITY, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
  for (int c = cta0 + g; c <= cta1; c += 8 * GROUPS) {
    float2 pml[8];
    float4 po[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int cc = c + k * GROUPS;
      pml[k] = make_float2(-INFINITY, 0.f);
      po[k] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (cc <= cta1) {
        const float* p = prm.partial + (size_t)(2 * cc + (cc == cta0 ? 1 : 0)) * W::ROWS * (D + 4);
        pml[k] = *reinterpret_cast<const float2*>(p + W::ROWS * D + 2 * (row0 + r));
        po[k] = *reinterpret_cast<const float4*>(p + (row0 + r) * D + col);
      }
    }
    float up = top;
#pragma unroll
    for (int k = 0; k < 8; ++k) up = fmaxf(up, pml[k].x);
    const float by = top == -INFINITY ? 0.f : ex2_approx(top - up);
    o.x *= by; o.y *= by; o.z *= by; o.w *= by;
    l *= by;
    top = up;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float wk = pml[k].x == -INFINITY ? 0.f : ex2_approx(pml[k].x - top);
      add_scaled(o, po[k], wk);
      l = fmaf(pml[k].y, wk, l);
    }
  }
  sum[g][item] = o;
  ml[g][item] = make_float2(top, l);
  __syncthreads();
  const int head0 = h * prm.group + rt * W::ROWS + row0;
  float4 mean = make_float4(0.f, 0.f, 0.f, 0.f);
  if (g == 0) {
#pragma unroll
    for (int k = 1; k < GROUPS; ++k) top = fmaxf(top, ml[k][item].x);
    const float own = ml[0][item].x == -INFINITY ? 0.f : ex2_approx(ml[0][item].x - top);
    o.x *= own; o.y *= own; o.z *= own; o.w *= own;
    l *= own;
#pragma unroll
    for (int k = 1; k < GROUPS; ++k) {
      const float wk = ml[k][item].x == -INFINITY ? 0.f : ex2_approx(ml[k][item].x - top);
      add_scaled(o, sum[k][item], wk);
      l = fmaf(ml[k][item].y, wk, l);
    }
    mean = mean_of(o, l);
    ml[0][item].x = top;
  }
  if (__syncthreads_or(g == 0 && beyond(mean, l))) {
    // again, by all warps; their sums by way of `sum`
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    float* all = reinterpret_cast<float*>(sum);
    static_assert(kJoinThreads / 32 * D <= GROUPS * ITEMS * 4, "a row of each warp");
#pragma unroll 1
    for (int x = 0; x < rows; ++x) {
      const float4 s = small_sums<typename W::T, D>(prm, b, h, head0 + x, ml[0][x * (D / 4)].x, warp, kJoinThreads / 32);
      float* to = all + warp * D + lane * (D / 32);
      to[0] = s.x;
      to[1] = s.y;
      if (D == 128) { to[2 % (D / 32)] = s.z; to[3 % (D / 32)] = s.w; }
      __syncthreads();
      if (g == 0 && item / (D / 4) == x && beyond(mean, l)) {
        float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kJoinThreads / 32; ++w) {
          const float4 y = *reinterpret_cast<const float4*>(all + w * D + col);
          t = make_float4(t.x + y.x, t.y + y.y, t.z + y.z, t.w + y.w);
        }
        mean = replaced<typename W::T>(mean, t, l);
      }
      __syncthreads();
    }
  }
  if (g == 0 && item / (D / 4) < rows) finish_row<typename W::T>(prm, b, head0 + r, col, mean, top, l);
}

// ---- host side -------------------------------------------------------------------------------------------

static int row_tile(const ca_cache_t& c) {
  const int group = c.heads_q / c.heads_kv;
  if (c.dtype == CA_DTYPE_BF16) return group > 8 ? 16 : 8;
  return group >= 5 ? 8 : group >= 3 ? 4 : group;
}

struct PagedWs {
  int* status;
  long long* units;
  int* bad;
  float* partial;
  size_t bytes;
};
static PagedWs carve_paged(const ca_cache_t& c, void* base) {
  PagedWs w{};
  Carver k(base);
  const int rows = row_tile(c);
  w.status = k.take<int>(kStatusBytes / sizeof(int));
  w.units = k.take<long long>((size_t)c.batch + 1);
  w.bad = k.take<int>(kPagedMaxCtas);
  w.partial = k.take<float>((size_t)2 * kPagedMaxCtas * rows * (c.head_dim + 4));
  w.bytes = k.used();
  return w;
}
size_t paged_workspace_bytes(const ca_cache_t& c) { return carve_paged(c, nullptr).bytes; }

template <typename W, int D>
static int launch_paged_d(PagedParams& prm, LaunchStream st) {
  using C = PagedCfg<W, D>;
  const int sms = multiprocessors();
  if (sms == 0) return CA_ERR_CUDA;
  prm.row_tiles = ceil_div(prm.group, W::ROWS);
  const int smem = C::smem(prm.group);
  auto kernel = paged_kernel<W, D>;
  CA_RETURN_IF_CUDA(allow_smem(kernel, smem));
  const long long pairs = (long long)prm.batch * prm.heads_kv * prm.row_tiles;
  prm.direct = (long long)prm.pages_per_sequence * prm.page_rows <= kDirectRows;
  if (prm.direct) {
    launch_chained(kernel, (unsigned)pairs, kPagedThreads, smem, st, prm);
    CA_LAUNCH_CHECK();
    return CA_OK;
  }
  prm.planned = prm.batch > kAddUp;
  if (prm.planned) {
    launch_chained(paged_plan_kernel, 1, 1024, 0, st, prm, C::U);
    CA_LAUNCH_CHECK();
  }
  const int per_sm = min(4, (228 * 1024) / (smem + 1024));
  const int ctas = min(kPagedMaxCtas, sms * per_sm);
  launch_chained(kernel, ctas, kPagedThreads, smem, st, prm);
  CA_LAUNCH_CHECK();
  const long long joins = pairs * ceil_div(min(prm.group, W::ROWS), kJoinRows);
  launch_chained(paged_join_kernel<W, D>, (unsigned)joins, kJoinThreads, 0, st, prm, ctas);
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
  prm.status = w.status; prm.units = w.units; prm.bad = w.bad; prm.partial = w.partial;
  prm.batch = c.batch; prm.heads_q = c.heads_q; prm.heads_kv = c.heads_kv; prm.group = c.heads_q / c.heads_kv;
  prm.page_rows = c.page_rows; prm.pages = c.pages; prm.pages_per_sequence = c.pages_per_sequence;
  prm.appended = appended; prm.left = c.left; prm.sinks = c.sinks;
  prm.scale_log2 = scale * 1.4426950408889634f;
  if (c.dtype == CA_DTYPE_BF16) {
    if (row_tile(c) == 8) return c.head_dim == 64 ? launch_paged_d<WarpMma<64, 1>, 64>(prm, st) : launch_paged_d<WarpMma<128, 1>, 128>(prm, st);
    return c.head_dim == 64 ? launch_paged_d<WarpMma<64, 2>, 64>(prm, st) : launch_paged_d<WarpMma<128, 2>, 128>(prm, st);
  }
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
