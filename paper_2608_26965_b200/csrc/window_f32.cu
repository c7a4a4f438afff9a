// Attention over a sliding window for fp32 storage, on m16n8k8 products of tf32 operands.
//
// tf32 has 11 significant bits, so each operand is split in two, x = hi + lo with hi = x rounded to tf32 and lo = the rest cut
// to tf32, and a product is lo hi + hi lo + hi hi: what is left out is 2^-22 of it.  The tensor core cuts its sums instead of rounding
// them, which over long chains loses more than that (2.7e-6 of the result with one accumulator for all); so chains of upper parts are two
// products long and are added up in fp32, and the small products have chains of their own: 3.2e-7 off where a plain fp32 form is
// 6.3e-7 (12 heads of 1,370 rows, d = 64, 148 rows to either side).
//
// Three products for one, at four times the rate of the CUDA cores' multiply-adds, and the operands come from shared memory a
// word per lane and product: the 1,370 rows take 48 us (window_ref.cu, which waits for vectors of shared memory, 80), 2 x 8 heads of 4,000
// rows, causal, d = 64, 500 rows before 221 us (351).  What bounds it is the chain of a warp's step (copy to registers, split,
// product, softmax, product): tensor pipe 43 % busy, an instruction every other cycle, with the eight warps that 255 registers allow (168
// registers and twelve warps: 55 us, 128 and sixteen: 76, for the registers that then go through memory).  Each of the four warps splits
// the tiles by itself, and the queries in every tile again; tf32 products of tcgen05 are not used.
//
// A warp has 16 query rows in registers, a CTA four warps; keys and values come 32 at a time by asynchronous copies, shared by the
// warps, while the 32 before are worked on.
//     S = Q K^T      a thread holds rows lane/4 and lane/4 + 8, keys 2 (lane % 4) and the next of every 8
//     O += P V       P as it is held: its keys 2 t and 2 t + 1 stand at columns t and t + 4 of the product, and V's rows likewise
// Masked probabilities are 0, and 0 x infinity is not: rows whose result is not finite are marked and computed again by the
// CUDA-core kernel (as those of the bf16 kernel are).  So are rows with a result below 2^-100 that is not zero: of a value below some 2^-112
// the lower half is below the normal range, where tf32 has only ten bits behind 2^-126.  (Scores lose as much where queries below 2^-116
// meet keys above 2^116, or keys such queries.)
#include <math.h>

#include "tc_ptx.cuh"
#include "window.cuh"

namespace ca {

using namespace ptx;

constexpr int kWfKeys = 32, kWfRows = 64, kWfThreads = 128;

template <int D>
struct WfCfg {
  static constexpr int PITCH = D + 4;                   // floats: lanes of a read are in different banks
  static constexpr int TILE = kWfKeys * PITCH;
  static constexpr int SMEM = 4 * TILE * 4;             // two stages of keys and values
};

struct Split {
  uint32_t hi, lo;
};
// In integers and one subtraction (the conversion instruction runs at an eighth of their rate).  The product looks at the upper 19 bits: of
// lo, which has 12 significant ones at most, it cuts the last, 2^-24 of x.  (Rounding lo in integers too would carry the mantissa of a
// number that is none, all ones, into its sign and make it zero, as it does for hi; so lo of what is no number, or infinite, is no
// number, and so is what comes of it.)
__device__ __forceinline__ Split split(float x) {
  Split s;
  s.hi = (__float_as_uint(x) + 0x1000u) & 0xffffe000u;
  s.lo = __float_as_uint(x - __uint_as_float(s.hi));
  return s;
}
__device__ __forceinline__ void mma1688(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

template <int D>
__global__ void __launch_bounds__(kWfThreads) window_f32_kernel(const __grid_constant__ WindowParams prm) {
  wait_for_previous();
  let_next_start();
  using C = WfCfg<D>;
  extern __shared__ __align__(16) float smf[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t4 = lane & 3;
  if (blockIdx.x == 0) window_status(prm, kWfThreads);
  const int blocks = (prm.n_q + kWfRows - 1) / kWfRows;
  // (the last rows of a causal sequence see most: first)
  const int r0 = (blocks - 1 - (int)(blockIdx.x % blocks)) * kWfRows, bh = blockIdx.x / blocks, b = bh / prm.heads_q, h = bh % prm.heads_q;
  const WindowItem it(prm, b);
  if (r0 >= it.len_q) return;
  const WindowSpan span(prm, it, r0, min(r0 + kWfRows, it.len_q), kWfKeys);
  const int kv = h / prm.group;
  const float* k = static_cast<const float*>(prm.k) + b * prm.k_b + kv * prm.k_h;
  const float* v = static_cast<const float*>(prm.v) + b * prm.v_b + kv * prm.v_h;
  auto fetch = [&](int t) {
    const int j0 = span.tile(t) * kWfKeys;
    const uint32_t to = smem_u32(smf + (t & 1) * 2 * C::TILE);
#pragma unroll
    for (int i = tid; i < kWfKeys * D / 4; i += kWfThreads) {
      const int r = i / (D / 4), c = i % (D / 4) * 4;
      const bool there = j0 + r < it.len_k;
      const uint32_t at = to + (r * C::PITCH + c) * 4;
      const float* ks = k + (there ? (j0 + r) * prm.k_n + c : 0);
      const float* vs = v + (there ? (j0 + r) * prm.v_n + c : 0);
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(at), "l"(ks), "r"(there ? 16 : 0) : "memory");
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(at + C::TILE * 4), "l"(vs), "r"(there ? 16 : 0) : "memory");
    }
  };
  if (span.tiles > 0) fetch(0);

  // ---- this warp's rows g and g + 8, columns t4 and t4 + 4 of every 8
  const int row0 = r0 + warp * 16 + g, row1 = row0 + 8;
  float q[D / 8][4];
  {
    const float* src = static_cast<const float*>(prm.q) + b * prm.q_b + h * prm.q_h;
#pragma unroll
    for (int c = 0; c < D / 8; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = i & 1 ? row1 : row0;
        q[c][i] = row < it.len_q ? src[row * prm.q_n + c * 8 + t4 + (i >> 1) * 4] : 0.f;
      }
  }
  const WindowRow sees0(prm, it, row0), sees1(prm, it, row1);
  float o[D / 8][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
  for (int n = 0; n < D / 8; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) o[n][i] = 0.f;

#pragma unroll 1
  for (int t = 0; t < span.tiles; ++t) {
    const int j0 = span.tile(t) * kWfKeys;
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();                                    // the tile is there, and the one before has been read
    if (t + 1 < span.tiles) fetch(t + 1);
    const float* ks = smf + (t & 1) * 2 * C::TILE;
    const float* vs = ks + C::TILE;
    // Sums of the tensor core are cut, not rounded: chains of two products of the upper parts, added up in fp32, and one chain of the
    // small ones.
    float s[kWfKeys / 8][4] = {}, small[kWfKeys / 8][4] = {};
#pragma unroll
    for (int c = 0; c < D / 8; c += 2) {
      uint32_t qh[2][4], ql[2][4];
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const Split x = split(q[c + e][i]);
          qh[e][i] = x.hi;
          ql[e][i] = x.lo;
        }
#pragma unroll
      for (int n = 0; n < kWfKeys / 8; ++n) {
        float big[4] = {};
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float* at = ks + (n * 8 + g) * C::PITCH + (c + e) * 8 + t4;
          const Split b0 = split(at[0]), b1 = split(at[4]);
          mma1688(small[n], ql[e], b0.hi, b1.hi);
          mma1688(small[n], qh[e], b0.lo, b1.lo);
          mma1688(big, qh[e], b0.hi, b1.hi);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) s[n][i] += big[i];
      }
    }
#pragma unroll
    for (int n = 0; n < kWfKeys / 8; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[n][i] += small[n][i];
    if (!span.whole(j0, j0 + kWfKeys)) {
#pragma unroll
      for (int n = 0; n < kWfKeys / 8; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (!(i < 2 ? sees0 : sees1).sees(j0 + n * 8 + 2 * t4 + (i & 1))) s[n][i] = -INFINITY;
    }
    float top[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      float x = -INFINITY;
#pragma unroll
      for (int n = 0; n < kWfKeys / 8; ++n) x = max3(x, s[n][2 * r], s[n][2 * r + 1]);
      x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
      top[r] = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2)) * prm.scale_log2;
    }
    if (__any_sync(0xffffffffu, top[0] > m[0] || top[1] > m[1])) {
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const float up = fmaxf(m[r], top[r]), by = m[r] == -INFINITY ? 0.f : ex2_approx(m[r] - up);
        m[r] = up;
        l[r] *= by;
#pragma unroll
        for (int n = 0; n < D / 8; ++n) { o[n][2 * r] *= by; o[n][2 * r + 1] *= by; }
      }
    }
    const float ref0 = m[0] == -INFINITY ? 0.f : -m[0], ref1 = m[1] == -INFINITY ? 0.f : -m[1];
    uint32_t ph[kWfKeys / 8][4], pl[kWfKeys / 8][4];
#pragma unroll
    for (int n = 0; n < kWfKeys / 8; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float p = ex2_approx(fmaf(s[n][i], prm.scale_log2, i < 2 ? ref0 : ref1)) * kWeightScale;
        l[i >> 1] += p;
        const Split x = split(p);
        const int at = (i >> 1) + (i & 1) * 2;          // (row, key) of the score -> place of the operand
        ph[n][at] = x.hi;
        pl[n][at] = x.lo;
      }
#pragma unroll
    for (int c = 0; c < D / 8; ++c) {
      float first[4] = {}, second[4] = {}, less[4] = {};
#pragma unroll
      for (int n = 0; n < kWfKeys / 8; ++n) {
        const float* at = vs + (n * 8 + 2 * t4) * C::PITCH + c * 8 + g;
        const Split b0 = split(at[0]), b1 = split(at[C::PITCH]);
        mma1688(less, pl[n], b0.hi, b1.hi);
        mma1688(less, ph[n], b0.lo, b1.lo);
        mma1688(n < kWfKeys / 16 ? first : second, ph[n], b0.hi, b1.hi);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) o[c][i] += (first[i] + second[i]) + less[i];
    }
  }
  // ---- O / l; a row that sees nothing: zeros, log-sum-exp -inf
  float any = 0.f;
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
    l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
    const int row = r ? row1 : row0;
    if (row >= it.len_q) continue;
    const bool empty = l[r] == 0.f;
    float* out = static_cast<float*>(prm.o) + b * prm.o_b + h * prm.o_h + row * prm.o_n + 2 * t4;
#pragma unroll
    for (int n = 0; n < D / 8; ++n) {
      const float x = empty ? 0.f : o[n][2 * r] / l[r], y = empty ? 0.f : o[n][2 * r + 1] / l[r];
      any += (x != 0.f && fabsf(x) < 0x1p-100f) || (y != 0.f && fabsf(y) < 0x1p-100f) ? INFINITY : fabsf(x) + fabsf(y);
      *reinterpret_cast<float2*>(out + n * 8) = make_float2(x, y);
    }
    any += empty ? 0.f : l[r];
    if (t4 == 0 && prm.lse)
      prm.lse[((size_t)b * prm.heads_q + h) * prm.n_q + row] = empty ? -INFINITY : (m[r] + log2f(l[r] * kWeightBack)) * 0.6931471805599453f;
  }
  const bool again = __any_sync(0xffffffffu, !(any < INFINITY));
  if (lane == 0) {
    const int first = r0 + warp * 16;
    if (first < prm.n_q) prm.redo[((size_t)bh * ((prm.n_q + kWindowBlock - 1) / kWindowBlock) + first / kWindowBlock) * 16 + first % kWindowBlock / 16] = again ? 1 : 0;
  }
}

template <int D>
static int launch_window_f32_d(const WindowParams& prm, LaunchStream st) {
  auto kernel = window_f32_kernel<D>;
  CA_RETURN_IF_CUDA(allow_smem(kernel, WfCfg<D>::SMEM));
  const long long n_work = (long long)ceil_div(prm.n_q, kWfRows) * prm.heads_q * prm.batch;
  if (n_work > 0x7fffffffLL) return CA_ERR_UNSUPPORTED;
  launch_chained(kernel, (unsigned)n_work, kWfThreads, WfCfg<D>::SMEM, st, prm);
  CA_LAUNCH_CHECK();
  return CA_OK;
}

int launch_window_f32(const WindowParams& prm, int D, LaunchStream st) {
  return D == 64 ? launch_window_f32_d<64>(prm, st) : launch_window_f32_d<128>(prm, st);
}

}  // namespace ca
