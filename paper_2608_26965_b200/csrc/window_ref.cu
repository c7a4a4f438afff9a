// Attention over a sliding window on the CUDA cores, in fp32: the rows that the tensor-core kernels leave to it, strides that they do not
// take, and CA_ATTN_FP32.
//     S = Q K^T, P = exp2(S c - m) over the visible keys, O = P V / sum P,    m the running maximum of a row.
// A CTA takes M query rows and goes over the keys that they see, 32 at a time, which arrive while the 32 before are worked on (fp32
// storage).  A thread has R x 4 scores and R x D/8 columns of the result in registers.  What bounds it is reading shared memory, not the
// multiply-adds (two to an instruction): a vector of 16 bytes per lane takes 3.6 cycles whether lanes read the same
// one or not, so 8 vectors for 32 instructions (R = 4) keep the reads of four warps at it for 115 cycles and the multiply-adds
// for 64.  2 x 8 heads of 4,000 rows, causal, d = 128: 2.2 ms, 30 TFLOP/s of visible pairs (R = 2 2.9 ms; R = 8 3.2, for want of
// registers and warps).  M = 64 with R = 4; M = 32 with R = 2 where tiles of 64 rows would be fewer than one to an SM (100 rows, one
// head, fp32: 11.8 us instead of 20.9 at d = 64, 19.3 instead of 29.4 at d = 128; 12 heads of 400 rows 38.8 instead of 46.4).
// Only tiles at a border of the window are masked: what a row does not see takes no part, whatever stands there
// (0 x infinity would).  Rows with a mean that is not finite are gone over a second time, with small values (kernels.h).
#include <math.h>

#include <type_traits>

#include "tc_ptx.cuh"
#include "window.cuh"

namespace ca {

using namespace ptx;

constexpr int kWrKeys = 32;

template <int D, int M>
struct WrCfg {
  static constexpr int R = M == 32 ? 2 : 4;           // query rows of a thread
  static constexpr int THREADS = M / R * 8;
  static constexpr int PITCH = D + 4;           // floats: rows a vector apart from a multiple of the banks
  static constexpr int P_PITCH = kWrKeys + 4;
  static constexpr int KV = kWrKeys * PITCH;    // a tile of keys, of values
  static constexpr int OFF_KV = M * PITCH, OFF_P = OFF_KV + 4 * KV;
  static constexpr int SMEM = (OFF_P + M * P_PITCH) * 4;
};

// rows of [.., D] into shared memory as fp32; rows from `there` on as zeros
template <typename T, int D, int THREADS, int ROWS>
__device__ __forceinline__ void window_rows_to_smem(float* dst, const T* src, long long stride, int there, int tid) {
  constexpr int V = D / 4;
#pragma unroll
  for (int i = tid; i < ROWS * V; i += THREADS) {
    const int r = i / V, c = i % V * 4;
    float* to = dst + r * (D + 4) + c;
    if constexpr (std::is_same<T, float>::value) {
      const int bytes = r < there ? 16 : 0;
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(to)), "l"(src + (r < there ? r * stride + c : 0)), "r"(bytes) : "memory");
    } else {
      *reinterpret_cast<float4*>(to) = r < there ? load4(src + r * stride + c) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
  }
}

template <typename T, int D, int M>
__global__ void __launch_bounds__(WrCfg<D, M>::THREADS) window_ref_kernel(const __grid_constant__ WindowParams prm) {
  wait_for_previous();
  let_next_start();
  using C = WrCfg<D, M>;
  constexpr int R = C::R;
  extern __shared__ __align__(16) float smf[];
  float* sq = smf;
  float* sp = smf + C::OFF_P;
  const int tid = threadIdx.x, ty = tid >> 3, tx = tid & 7;
  const int blocks = (prm.n_q + M - 1) / M;
  const long long n_work = (long long)blocks * prm.heads_q * prm.batch;
  auto marked = [&](int bh, int r0, int part, int len_q) {         // rows r0 + 16 part .. of a tile
    const int r = r0 + 16 * part;
    return r < len_q && prm.redo[((size_t)bh * ((prm.n_q + kWindowBlock - 1) / kWindowBlock) + r / kWindowBlock) * 16 + r % kWindowBlock / 16] != 0;
  };
  if (prm.redo) {
    // hardly ever anything: all marks of this CTA's tiles at once
    if (!prm.one_each && prm.status[kRedoWord] == 0) return;
    int any = 0;
    for (long long i = tid;; i += C::THREADS) {
      const long long idx = blockIdx.x + i / (M / 16) * gridDim.x;
      if (idx >= n_work) break;
      const int bh = (int)(idx / blocks), r0 = (blocks - 1 - (int)(idx % blocks)) * M;
      any |= marked(bh, r0, (int)(i % (M / 16)), WindowItem(prm, bh / prm.heads_q).len_q);
    }
    if (!__syncthreads_or(any)) return;
  } else if (blockIdx.x == 0) {
    window_status(prm, C::THREADS);
  }
#pragma unroll 1
  for (long long idx = blockIdx.x; idx < n_work; idx += gridDim.x) {
    // (the last rows of a causal sequence see most: first)
    const int r0 = (blocks - 1 - (int)(idx % blocks)) * M, bh = (int)(idx / blocks), b = bh / prm.heads_q, h = bh % prm.heads_q;
    const WindowItem it(prm, b);
    if (r0 >= it.len_q) continue;
    if (prm.redo) {
      bool any = false;
#pragma unroll
      for (int i = 0; i < M / 16; ++i) any = any || marked(bh, r0, i, it.len_q);
      if (!any) continue;
    }
    const int rows = min(M, it.len_q - r0);
    const WindowSpan span(prm, it, r0, r0 + rows, kWrKeys);
    const int g = h / prm.group;
    const T* q = static_cast<const T*>(prm.q) + b * prm.q_b + h * prm.q_h + r0 * prm.q_n;
    const T* k = static_cast<const T*>(prm.k) + b * prm.k_b + g * prm.k_h;
    const T* v = static_cast<const T*>(prm.v) + b * prm.v_b + g * prm.v_h;
    auto fetch = [&](int t) {
      const int j0 = span.tile(t) * kWrKeys, keys = it.len_k - j0;
      float* to = smf + C::OFF_KV + (t & 1) * 2 * C::KV;
      window_rows_to_smem<T, D, C::THREADS, kWrKeys>(to, k + j0 * prm.k_n, prm.k_n, keys, tid);
      window_rows_to_smem<T, D, C::THREADS, kWrKeys>(to + C::KV, v + j0 * prm.v_n, prm.v_n, keys, tid);
    };
    auto arrived = [&]() {
      if (std::is_same<T, float>::value) asm volatile("cp.async.wait_all;" ::: "memory");
      __syncthreads();
    };
    __syncthreads();                            // the rows before have been worked off
    window_rows_to_smem<T, D, C::THREADS, M>(sq, q, prm.q_n, rows, tid);

    unsigned again[R] = {};                     // bits of this thread's columns that are to be taken again
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {
      if (span.tiles > 0) fetch(0);
      f32x2 o[R][D / 32][2];
      float m[R], l[R];
#pragma unroll
      for (int i = 0; i < R; ++i) {
        m[i] = -INFINITY;
        l[i] = 0.f;
#pragma unroll
        for (int c = 0; c < D / 32; ++c) o[i][c][0] = o[i][c][1] = pack2(0.f, 0.f);
      }
#pragma unroll 1
      for (int t = 0; t < span.tiles; ++t) {
        const int j0 = span.tile(t) * kWrKeys;
        arrived();                                // and the tile before has been read
        if (t + 1 < span.tiles) fetch(t + 1);
        const float* sk = smf + C::OFF_KV + (t & 1) * 2 * C::KV;
        const float* sv = sk + C::KV;
        // ---- scores of rows R ty .. R ty + R - 1, keys tx, tx + 8, ...
        f32x2 s2[R][4];
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) s2[i][j] = pack2(0.f, 0.f);
#pragma unroll 4
        for (int c = 0; c < D; c += 4) {
          float4 a[R], x[4];
#pragma unroll
          for (int i = 0; i < R; ++i) a[i] = *reinterpret_cast<const float4*>(sq + (R * ty + i) * C::PITCH + c);
#pragma unroll
          for (int j = 0; j < 4; ++j) x[j] = *reinterpret_cast<const float4*>(sk + (tx + 8 * j) * C::PITCH + c);
#pragma unroll
          for (int i = 0; i < R; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
              s2[i][j] = fma2(pack2(a[i].z, a[i].w), pack2(x[j].z, x[j].w), fma2(pack2(a[i].x, a[i].y), pack2(x[j].x, x[j].y), s2[i][j]));
        }
        const bool whole = span.whole(j0, j0 + kWrKeys);
#pragma unroll
        for (int i = 0; i < R; ++i) {
          const WindowRow row(prm, it, r0 + R * ty + i);
          bool seen[4];
          float s[4], top = m[i];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float even, odd;
            unpack2(s2[i][j], even, odd);
            seen[j] = whole || row.sees(j0 + tx + 8 * j);
            s[j] = seen[j] ? (even + odd) * prm.scale_log2 : -INFINITY;
            top = fmaxf(top, s[j]);
          }
#pragma unroll
          for (int x = 1; x < 8; x <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
          const float by = m[i] == -INFINITY ? 0.f : ex2_approx(m[i] - top), ref = top == -INFINITY ? 0.f : top;
          m[i] = top;
          l[i] *= by;
#pragma unroll
          for (int c = 0; c < D / 32; ++c) {
            o[i][c][0] = mul2(o[i][c][0], pack2(by, by));
            o[i][c][1] = mul2(o[i][c][1], pack2(by, by));
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float p = ex2_approx(s[j] - ref) * kWeightScale;
            if (seen[j]) l[i] += p;
            sp[(R * ty + i) * C::P_PITCH + tx + 8 * j] = seen[j] ? p : -1.f;      // (no probability: takes no part)
          }
        }
        __syncwarp();                             // the rows of a warp's probabilities are its own
        auto values = [&](auto masked, auto small) {
#pragma unroll 2
          for (int j = 0; j < kWrKeys; j += 4) {
            float p[R][4];
#pragma unroll
            for (int i = 0; i < R; ++i) *reinterpret_cast<float4*>(p[i]) = *reinterpret_cast<const float4*>(sp + (R * ty + i) * C::P_PITCH + j);
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
              for (int c = 0; c < D / 32; ++c) {
                float4 x = *reinterpret_cast<const float4*>(sv + (j + e) * C::PITCH + c * 32 + tx * 4);
                if (decltype(small)::value) x = make_float4(x.x * kValueScale, x.y * kValueScale, x.z * kValueScale, x.w * kValueScale);
#pragma unroll
                for (int i = 0; i < R; ++i) {
                  if (decltype(masked)::value && p[i][e] == -1.f) continue;
                  o[i][c][0] = fma2(pack2(p[i][e], p[i][e]), pack2(x.x, x.y), o[i][c][0]);
                  o[i][c][1] = fma2(pack2(p[i][e], p[i][e]), pack2(x.z, x.w), o[i][c][1]);
                }
              }
          }
        };
        if (pass == 1) values(std::true_type{}, std::true_type{});
        else if (whole) values(std::false_type{}, std::false_type{});
        else values(std::true_type{}, std::false_type{});
      }
      if (std::is_same<T, float>::value) asm volatile("cp.async.wait_all;" ::: "memory");
      bool any = false;
#pragma unroll
      for (int i = 0; i < R; ++i) {
#pragma unroll
        for (int x = 1; x < 8; x <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], x);
        const int row = r0 + R * ty + i;
        if (row >= it.len_q) continue;
        // a row that sees nothing: zeros, log-sum-exp -inf
        T* out = static_cast<T*>(prm.o) + b * prm.o_b + h * prm.o_h + row * prm.o_n;
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          float x[4] = {0.f, 0.f, 0.f, 0.f};
          if (l[i] != 0.f) {
            unpack2(o[i][c][0], x[0], x[1]);
            unpack2(o[i][c][1], x[2], x[3]);
          }
          if (pass == 1) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (again[i] >> (4 * c + e) & 1u) out[c * 32 + tx * 4 + e] = from_f32<T>(mean_of_small<T>(x[e], l[i]));
            continue;
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (l[i] != 0.f) x[e] = x[e] / l[i];
            if (l[i] < INFINITY && !(fabsf(x[e]) < INFINITY)) again[i] |= 1u << (4 * c + e);
          }
          store4(out + c * 32 + tx * 4, make_float4(x[0], x[1], x[2], x[3]));
        }
        any = any || again[i] != 0;
        if (tx == 0 && prm.lse && pass == 0)
          prm.lse[((size_t)b * prm.heads_q + h) * prm.n_q + row] = l[i] == 0.f ? -INFINITY : (m[i] + log2f(l[i] * kWeightBack)) * 0.6931471805599453f;
      }
      if (pass == 0 && !__syncthreads_or(any)) break;      // (a barrier before the keys are fetched again, too)
    }
  }
}

template <typename T, int D, int M>
static int launch_window_ref_m(const WindowParams& prm, LaunchStream st) {
  using C = WrCfg<D, M>;
  auto kernel = window_ref_kernel<T, D, M>;
  CA_RETURN_IF_CUDA(allow_smem(kernel, C::SMEM));
  const long long n_work = (long long)ceil_div(prm.n_q, M) * prm.heads_q * prm.batch;
  // a CTA for every tile of rows; to compute rows again, hardly ever any, one to an SM
  const long long most = prm.redo ? multiprocessors() : 0x7fffffffLL;
  if (most == 0) return CA_ERR_CUDA;
  launch_chained(kernel, (unsigned)(n_work < most ? n_work : most), C::THREADS, C::SMEM, st, prm);
  CA_LAUNCH_CHECK();
  return CA_OK;
}

template <typename T, int D>
static int launch_window_ref_d(const WindowParams& prm, LaunchStream st) {
  if (!prm.redo && (long long)ceil_div(prm.n_q, 64) * prm.heads_q * prm.batch < multiprocessors()) return launch_window_ref_m<T, D, 32>(prm, st);
  return launch_window_ref_m<T, D, 64>(prm, st);
}

int launch_window_ref(const WindowParams& prm, int D, int dtype, LaunchStream st) {
  if (dtype == CA_DTYPE_BF16)
    return D == 64 ? launch_window_ref_d<__nv_bfloat16, 64>(prm, st) : launch_window_ref_d<__nv_bfloat16, 128>(prm, st);
  return D == 64 ? launch_window_ref_d<float, 64>(prm, st) : launch_window_ref_d<float, 128>(prm, st);
}

// Blocks of rows before each batch item, counters and status: one CTA.
__global__ void __launch_bounds__(256) window_prepare_kernel(const __grid_constant__ WindowParams prm) {
  wait_for_previous();
  let_next_start();
  __shared__ int warp_sum[8];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int bad = 0, before = 0;
  for (int base = 0; base < prm.batch; base += 256) {
    const int b = base + tid;
    int v = 0;
    if (b < prm.batch) {
      bad |= (prm.len_q && (unsigned)prm.len_q[b] > (unsigned)prm.n_q) || (prm.len_k && (unsigned)prm.len_k[b] > (unsigned)prm.n_k);
      v = (WindowItem(prm, b).len_q + kWindowBlock - 1) / kWindowBlock;
    }
    for (int d = 1; d < 32; d <<= 1) {
      const int o = __shfl_up_sync(0xffffffffu, v, d);
      if (lane >= d) v += o;
    }
    if (lane == 31) warp_sum[warp] = v;
    __syncthreads();
    int all = 0;
    for (int w = 0; w < 8; ++w) {
      if (w < warp) v += warp_sum[w];
      all += warp_sum[w];
    }
    if (b < prm.batch) prm.pieces[b + 1] = before + v;
    before += all;
    __syncthreads();
  }
  bad = __syncthreads_or(bad);
  if (tid == 0) {
    prm.pieces[0] = 0;
    prm.status[0] = bad ? CA_ERR_BAD_INDEX : CA_OK;
    prm.status[kNextWord] = 0;
    prm.status[kRedoWord] = 0;
  }
}

int launch_window_prepare(const WindowParams& prm, LaunchStream st) {
  launch_chained(window_prepare_kernel, 1, 256, 0, st, prm);
  CA_LAUNCH_CHECK();
  return CA_OK;
}

size_t window_workspace_bytes(const ca_window_t& p) {
  // status block, blocks of rows of every batch item, marks of the rows to compute again
  return kStatusBytes + align_up(((size_t)p.batch + 1) * sizeof(int32_t), 256) + align_up((size_t)p.batch * p.heads_q * ceil_div(p.n_q, kWindowBlock) * 16 * sizeof(int32_t), 256);
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
  if (!(p.flags & CA_ATTN_FP32)) {
    Carver c(ws);
    c.take<int>(kStatusBytes / sizeof(int));
    prm.pieces = c.take<int32_t>((size_t)p.batch + 1);
    prm.redo = c.take<int32_t>((size_t)p.batch * p.heads_q * ceil_div(p.n_q, kWindowBlock) * 16);
    int rc;
    if (p.dtype == CA_DTYPE_BF16) {
      rc = launch_window_tc(prm, p.head_dim, st);
    } else {
      prm.one_each = 1;
      rc = launch_window_f32(prm, p.head_dim, st);
    }
    if (rc == CA_OK) return launch_window_ref(prm, p.head_dim, p.dtype, st);
    if (rc != CA_ERR_UNSUPPORTED) return rc;
    prm.one_each = 0;
    prm.redo = nullptr;                         // strides of a broadcast, or too many pieces: on the CUDA cores
  }
  return launch_window_ref(prm, p.head_dim, p.dtype, st);
}

}  // namespace ca
