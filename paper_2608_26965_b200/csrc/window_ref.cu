// Attention over a sliding window on the CUDA cores, in fp32: fp32 storage, and the rows that the tensor-core kernel
// leaves to it.
//     S = Q K^T, P = exp2(s c - m) over the visible keys, O = P V / sum P,    m the running maximum of a row.
// A CTA takes 64 query rows and goes over the keys that they see, 64 at a time; a thread has 4 x 4 scores and 4 x D/16
// columns of the result in registers, so that shared memory is read 8 times (P V: 4 + D/16) for 64 (D) multiply-adds.
// Only tiles at a border of the window are masked: what a row does not see takes no part, whatever stands there
// (0 x infinity would).
#include <math.h>

#include "tc_ptx.cuh"
#include "window.cuh"

namespace ca {

constexpr int kWrRows = 64, kWrKeys = 64, kWrThreads = 256;

template <typename T, int D>
__device__ __forceinline__ void window_rows_to_smem(float* dst, const T* src, long long stride, int rows, int tid) {
  constexpr int V = D / 4;
#pragma unroll 4
  for (int i = tid; i < 64 * V; i += kWrThreads) {
    const int r = i / V, c = i % V * 4;
    const float4 x = r < rows ? load4(src + r * stride + c) : make_float4(0.f, 0.f, 0.f, 0.f);
    *reinterpret_cast<float4*>(dst + r * (D + 4) + c) = x;
  }
}

template <typename T, int D>
__global__ void __launch_bounds__(kWrThreads) window_ref_kernel(const __grid_constant__ WindowParams prm) {
  wait_for_previous();
  let_next_start();
  extern __shared__ __align__(16) float smf[];
  float* sq = smf;                              // [64][D + 4]: rows a vector apart from a multiple of the banks
  float* sk = sq + kWrRows * (D + 4);
  float* sv = sk + kWrKeys * (D + 4);
  float* sp = sv + kWrKeys * (D + 4);           // [64][68]
  const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
  if (prm.redo) {
    if (prm.status[kRedoWord] == 0) return;
  } else if (blockIdx.x == 0) {
    // the only one that writes the status word
    int bad = 0;
    for (int i = tid; i < prm.batch; i += kWrThreads)
      bad |= (prm.len_q && (unsigned)prm.len_q[i] > (unsigned)prm.n_q) || (prm.len_k && (unsigned)prm.len_k[i] > (unsigned)prm.n_k);
    bad = __syncthreads_or(bad);
    if (tid == 0) *prm.status = bad ? CA_ERR_BAD_INDEX : CA_OK;
  }
  const int blocks64 = (prm.n_q + kWrRows - 1) / kWrRows;
  const long long n_work = (long long)blocks64 * prm.heads_q * prm.batch;
#pragma unroll 1
  for (long long idx = blockIdx.x; idx < n_work; idx += gridDim.x) {
  const int r0 = (int)(idx % blocks64) * kWrRows, bh = (int)(idx / blocks64), b = bh / prm.heads_q, h = bh % prm.heads_q;
  const WindowItem it(prm, b);
  if (r0 >= it.len_q) continue;
  if (prm.redo) {
    const int32_t* marks = prm.redo + ((size_t)bh * ((prm.n_q + kWindowBlock - 1) / kWindowBlock) + r0 / kWindowBlock) * 8 + r0 % kWindowBlock / 32;
    if ((marks[0] | marks[1]) == 0) continue;
  }
  const int rows = min(kWrRows, it.len_q - r0);
  const WindowSpan span(prm, it, r0, r0 + rows, kWrKeys);
  const int g = h / prm.group;
  const T* q = static_cast<const T*>(prm.q) + b * prm.q_b + h * prm.q_h + r0 * prm.q_n;
  const T* k = static_cast<const T*>(prm.k) + b * prm.k_b + g * prm.k_h;
  const T* v = static_cast<const T*>(prm.v) + b * prm.v_b + g * prm.v_h;
  __syncthreads();                              // (the rows before have been worked off)
  window_rows_to_smem<T, D>(sq, q, prm.q_n, rows, tid);

  float o[4][D / 64][4], m[4], l[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int c = 0; c < D / 64; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[i][c][e] = 0.f;
  }
#pragma unroll 1
  for (int t = 0; t < span.tiles; ++t) {
    const int j0 = span.tile(t) * kWrKeys, keys = min(kWrKeys, it.len_k - j0);
    __syncthreads();
    window_rows_to_smem<T, D>(sk, k + j0 * prm.k_n, prm.k_n, keys, tid);
    window_rows_to_smem<T, D>(sv, v + j0 * prm.v_n, prm.v_n, keys, tid);
    __syncthreads();
    // ---- scores of rows 4 ty .. 4 ty + 3, keys tx, tx + 16, ...
    float s[4][4] = {};
#pragma unroll 4
    for (int c = 0; c < D; c += 4) {
      float4 a[4], x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = *reinterpret_cast<const float4*>(sq + (4 * ty + i) * (D + 4) + c);
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = *reinterpret_cast<const float4*>(sk + (tx + 16 * j) * (D + 4) + c);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[i][j] = fmaf(a[i].x, x[j].x, fmaf(a[i].y, x[j].y, fmaf(a[i].z, x[j].z, fmaf(a[i].w, x[j].w, s[i][j]))));
    }
    const bool whole = span.whole(j0, j0 + kWrKeys);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const WindowRow row(prm, it, r0 + 4 * ty + i);
      bool seen[4];
      float top = m[i];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        seen[j] = whole || row.sees(j0 + tx + 16 * j);
        s[i][j] = seen[j] ? s[i][j] * prm.scale_log2 : -INFINITY;
        top = fmaxf(top, s[i][j]);
      }
#pragma unroll
      for (int x = 1; x < 16; x <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
      const float by = m[i] == -INFINITY ? 0.f : ptx::ex2_approx(m[i] - top), ref = top == -INFINITY ? 0.f : top;
      m[i] = top;
      l[i] *= by;
#pragma unroll
      for (int c = 0; c < D / 64; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][c][e] *= by;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float p = ptx::ex2_approx(s[i][j] - ref);
        if (seen[j]) l[i] += p;
        sp[(4 * ty + i) * (kWrKeys + 4) + tx + 16 * j] = seen[j] ? p : -1.f;    // (no probability: takes no part)
      }
    }
    __syncwarp();                                          // the rows of a warp's probabilities are its own
    auto values = [&](auto masked) {
#pragma unroll 2
      for (int j = 0; j < kWrKeys; j += 4) {
        float p[4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<float4*>(p[i]) = *reinterpret_cast<const float4*>(sp + (4 * ty + i) * (kWrKeys + 4) + j);
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int c = 0; c < D / 64; ++c) {
            const float4 x = *reinterpret_cast<const float4*>(sv + (j + e) * (D + 4) + c * 64 + tx * 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if (decltype(masked)::value && p[i][e] == -1.f) continue;
              o[i][c][0] = fmaf(p[i][e], x.x, o[i][c][0]);
              o[i][c][1] = fmaf(p[i][e], x.y, o[i][c][1]);
              o[i][c][2] = fmaf(p[i][e], x.z, o[i][c][2]);
              o[i][c][3] = fmaf(p[i][e], x.w, o[i][c][3]);
            }
          }
      }
    };
    if (whole) values(std::false_type{});
    else values(std::true_type{});
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int x = 1; x < 16; x <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], x);
    const int row = r0 + 4 * ty + i;
    if (row >= it.len_q) continue;
    // a row that sees nothing: zeros, log-sum-exp -inf
    T* out = static_cast<T*>(prm.o) + b * prm.o_b + h * prm.o_h + row * prm.o_n;
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      if (l[i] != 0.f) x = make_float4(o[i][c][0] / l[i], o[i][c][1] / l[i], o[i][c][2] / l[i], o[i][c][3] / l[i]);
      store4(out + c * 64 + tx * 4, x);
    }
    if (tx == 0 && prm.lse)
      prm.lse[((size_t)b * prm.heads_q + h) * prm.n_q + row] = l[i] == 0.f ? -INFINITY : (m[i] + log2f(l[i])) * 0.6931471805599453f;
  }
  }
}

template <typename T, int D>
static int launch_window_ref_d(const WindowParams& prm, LaunchStream st) {
  constexpr int smem = (3 * 64 * (D + 4) + 64 * (kWrKeys + 4)) * 4;
  auto kernel = window_ref_kernel<T, D>;
  CA_RETURN_IF_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  const long long n_work = (long long)ceil_div(prm.n_q, kWrRows) * prm.heads_q * prm.batch;
  // a CTA for every 64 rows; to compute rows again, hardly ever any, as many as are on the GPU at a time
  const long long most = prm.redo ? 296 : 0x7fffffffLL;
  launch_chained(kernel, (unsigned)(n_work < most ? n_work : most), kWrThreads, smem, st, prm);
  CA_LAUNCH_CHECK();
  return CA_OK;
}

int launch_window_ref(const WindowParams& prm, int D, int dtype, LaunchStream st) {
  if (dtype == CA_DTYPE_BF16)
    return D == 64 ? launch_window_ref_d<__nv_bfloat16, 64>(prm, st) : launch_window_ref_d<__nv_bfloat16, 128>(prm, st);
  return D == 64 ? launch_window_ref_d<float, 64>(prm, st) : launch_window_ref_d<float, 128>(prm, st);
}

size_t window_workspace_bytes(const ca_window_t& p) {
  // status block, blocks of rows of every batch item, marks of the rows to compute again
  return kStatusBytes + align_up(((size_t)p.batch + 1) * sizeof(int32_t), 256) + align_up((size_t)p.batch * p.heads_q * ceil_div(p.n_q, kWindowBlock) * 8 * sizeof(int32_t), 256);
}

int launch_window(const ca_window_t& p, const ca_rows_t* Q, const ca_rows_t* K, const ca_rows_t* V, const int32_t* len_q,
                  const int32_t* len_k, float scale, const ca_rows_t* O, float* lse, void* ws, LaunchStream st) {
  WindowParams prm{};
  prm.q = Q->data; prm.q_b = Q->stride_b; prm.q_h = Q->stride_h; prm.q_n = Q->stride_n;
  prm.k = K->data; prm.k_b = K->stride_b; prm.k_h = K->stride_h; prm.k_n = K->stride_n;
  prm.v = V->data; prm.v_b = V->stride_b; prm.v_h = V->stride_h; prm.v_n = V->stride_n;
  prm.o = O->data; prm.o_b = O->stride_b; prm.o_h = O->stride_h; prm.o_n = O->stride_n;
  prm.lse = lse;
  prm.len_q = len_q; prm.len_k = len_k;
  prm.status = static_cast<int*>(ws);
  prm.batch = p.batch; prm.heads_q = p.heads_q; prm.heads_kv = p.heads_kv; prm.group = p.heads_q / p.heads_kv;
  prm.n_q = p.n_q; prm.n_k = p.n_k; prm.left = p.left; prm.right = p.right; prm.sinks = p.sinks;
  prm.scale_log2 = scale * 1.4426950408889634f;
  if (p.dtype == CA_DTYPE_BF16 && !(p.flags & CA_ATTN_FP32)) {
    Carver c(ws);
    c.take<int>(kStatusBytes / sizeof(int));
    prm.pieces = c.take<int32_t>((size_t)p.batch + 1);
    prm.redo = c.take<int32_t>((size_t)p.batch * p.heads_q * ceil_div(p.n_q, kWindowBlock) * 8);
    const int rc = launch_window_tc(prm, p.head_dim, st);
    if (rc == CA_OK) return launch_window_ref(prm, p.head_dim, p.dtype, st);
    if (rc != CA_ERR_UNSUPPORTED) return rc;
    prm.redo = nullptr;                         // strides of a broadcast: on the CUDA cores
  }
  return launch_window_ref(prm, p.head_dim, p.dtype, st);
}

}  // namespace ca
