// Rotary positions with several axes, on the way from the projections' layout to rows, and rows put into the
// pages of a cache (keys rotated on the way).
//
// A pair of channels (x, y) of axis a turns by t = position[a] * frequency:
//     (x, y) -> (x cos t - y sin t, x sin t + y cos t),          the inverse by -t.
// Positions are whole numbers, so t / (2 pi) is only needed modulo 1: the host turns a frequency into a 64-bit
// fraction of a turn, and the product with the position modulo 2^64 is the phase, to 2^-64 of a turn per step at any
// distance, without a double in the kernel.  The nearest quarter turn is taken off in whole numbers and the remainder rounded to fp32 once,
// so that sines and cosines next to zero are as accurate as the others.
//
// What bounds it: memory.  Every element is read and written once in 16-byte vectors; a thread keeps the sines
// and cosines of its channels and goes through heads with them, which share the positions of a row.
#include <math.h>
#include <string.h>

#include <type_traits>

#include "kernels.h"

namespace ca {

constexpr int kMaxPairs = 64;

struct RotaryTable {
  unsigned long long turns[kMaxPairs];       // 2^64 frequency / (2 pi) modulo 2^64
  unsigned char axis[kMaxPairs];
  int pairs, axes;
};

// A set of heads that is read and written: [batch, heads, rows, head_dim] by strides in elements.
struct RowSet {
  const void* in;
  void* out;
  long long in_b, in_h, in_n, out_b, out_h, out_n;
  int heads;
};

struct RotaryParams {
  RowSet set[2];
  const int32_t* positions;
  long long pos_b;
  int n, rows_per_block, items, heads_per_thread, inverse;
  // pages (kPaged): out is a pool [pages][heads][page_rows][D]
  const int32_t *lengths, *count, *page_table;
  int page_rows, pages, pages_per_sequence, batch;
  long long lines;                           // rows of all batch items
  int* status;
};

// how pairs lie: none, neighbours, halves a vector at a time, halves an element at a time (where the half does not start at a vector)
enum { kNoPairs = 0, kAdjacent = 1, kHalves = 2, kHalvesScalar = 3 };

template <typename T, int W>
struct Vec;
template <>
struct Vec<float, 4> { using type = uint4; };
template <>
struct Vec<__nv_bfloat16, 8> { using type = uint4; };
template <>
struct Vec<float, 1> { using type = uint32_t; };
template <>
struct Vec<__nv_bfloat16, 1> { using type = uint16_t; };

template <typename T, int W>
union Pack {
  typename Vec<T, W>::type raw;
  T e[W];
  __device__ __forceinline__ Pack() {}
};

// Sine and cosine of a phase (2^64: a turn).  The quarter turn next to it is taken off; of the remainder r half turns, |r| <= 1/4,
//     sin(pi r) = r (pi + t S(t)),  cos(pi r) = 1 + t C(t),  t = r^2
// with polynomials fitted to the smallest relative error (of sine 0.06 u, of cosine 0.001 u, u = 2^-24), pi in two parts: with their roundings
// 1.2 u and 1.4 u.  (sincospif of the remainder, which looks for the quarter again, cost 6 %: a video layer of 2 x 40 heads by 32,760 rows
// 218 us instead of 205.)
__device__ __forceinline__ void sine_cosine(unsigned long long phase, float* sine, float* cosine) {
  const unsigned top = (unsigned)(phase >> 32), quarter = (top + 0x20000000u) >> 30;
  const float r = fmaf((float)(unsigned)phase, 0x1p-63f, (float)(int)(top - (quarter << 30)) * 0x1p-31f), t = r * r;
  const float S = fmaf(fmaf(-0.58947957f, t, 2.5498104f), t, -5.1677094f);
  const float C = fmaf(fmaf(fmaf(0.23136422f, t, -1.3350506f), t, 4.0587077f), t, -4.934802f);
  const float s = fmaf(r, 3.1415927f, r * fmaf(S, t, -8.7422777e-8f)), c = fmaf(C, t, 1.f);
  const float x = quarter & 1 ? c : s, y = quarter & 1 ? s : c;
  *sine = quarter & 2 ? -x : x;
  *cosine = (quarter + 1) & 2 ? -y : y;
}

template <typename T>
__device__ __forceinline__ void turn(T& x, T& y, float c, float s) {
  const float a = to_f32<T>(x), b = to_f32<T>(y);
  x = from_f32<T>(fmaf(a, c, -(b * s)));
  y = from_f32<T>(fmaf(a, s, b * c));
}

// An item of a row: a vector of it, or with halves a vector of the first half and its partner.  Threads of a
// block: rows_per_block rows by the items of a row; blockIdx.y: heads.
template <typename T, int D, int PAIRS, bool PAGED>
__device__ __forceinline__ void rotary_rows(const unsigned long long* s_turns, const unsigned char* s_axis, int pairs, int axes,
                                            const RotaryParams& prm) {
  constexpr int W = PAIRS == kHalvesScalar ? 1 : 16 / (int)sizeof(T);
  constexpr bool HALVES = PAIRS == kHalves || PAIRS == kHalvesScalar;
  constexpr int ANGLES = PAIRS == kNoPairs ? 1 : HALVES ? W : W / 2;
  const int item = threadIdx.x % prm.items, sub = threadIdx.x / prm.items;
  const long long line = (long long)blockIdx.x * prm.rows_per_block + sub;     // of all batch items
  if (sub >= prm.rows_per_block || line >= prm.lines) return;
  const int b = prm.lines <= 0xffffffffLL ? (int)((unsigned)line / (unsigned)prm.n) : (int)(line / prm.n);
  const long long row = line - (long long)b * prm.n;

  long long slot = 0;                                    // first element of the row's place in a pool, of head 0
  if (PAGED) {
    const int start = prm.lengths[b], count = prm.count ? prm.count[b] : prm.n;
    if (start < 0 || row >= count) return;               // (a row that is not there)
    const unsigned at = (unsigned)start + (unsigned)row, page = at / (unsigned)prm.page_rows;
    if (page >= (unsigned)prm.pages_per_sequence) return;
    const int id = prm.page_table[(size_t)b * prm.pages_per_sequence + page];
    if ((unsigned)id >= (unsigned)prm.pages) return;
    slot = ((long long)id * prm.set[0].heads * prm.page_rows + at % (unsigned)prm.page_rows) * D;
  }

  const int R = PAIRS == kNoPairs ? 0 : pairs;
  const int lead = HALVES ? R / W : 0;                   // items with a partner
  const bool both = HALVES && item < lead;
  const int first = !HALVES ? item * W : both ? item * W : 2 * R + (item - lead) * W;
  const int begin = blockIdx.y * prm.heads_per_thread, heads0 = prm.set[0].heads;
  const int end = min(begin + prm.heads_per_thread, heads0 + prm.set[1].heads);

  // ---- heads, four at a time
  using V = typename Vec<T, W>::type;
  constexpr int N = 4;
  Pack<T, W> x[N], y[N];
  auto load = [&](int h) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if (h + j >= end) break;
      const RowSet& set = prm.set[h + j < heads0 ? 0 : 1];
      const T* in = static_cast<const T*>(set.in) + b * set.in_b + row * set.in_n + (h + j - (h + j < heads0 ? 0 : heads0)) * set.in_h + first;
      x[j].raw = *reinterpret_cast<const V*>(in);
      if (both) y[j].raw = *reinterpret_cast<const V*>(in + R);
    }
  };
  load(begin);                                           // on their way while the angles are computed

  // ---- sines and cosines of this thread's pairs; a pair behind the last one stays as it is
  float cs[ANGLES], sn[ANGLES];
  int turned = 0;
  if (PAIRS != kNoPairs) {
    const int32_t* pos = prm.positions + b * prm.pos_b + row * axes;
    const int pair0 = HALVES ? item * W : item * (W / 2);
#pragma unroll
    for (int i = 0; i < ANGLES; ++i) {
      const int pair = pair0 + i;
      cs[i] = 1.f;
      sn[i] = 0.f;
      if (pair < R) {
        const unsigned long long phase = (unsigned long long)(long long)pos[s_axis[pair]] * s_turns[pair];
        sine_cosine(phase, &sn[i], &cs[i]);
        if (prm.inverse) sn[i] = -sn[i];
        turned = i + 1;
      }
    }
  }
  for (int h = begin; h < end; h += N) {
    if (h > begin) load(h);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if (h + j >= end) break;
      const int which = h + j < heads0 ? 0 : 1, head = h + j - (which ? heads0 : 0);
      const RowSet& set = prm.set[which];
      if (PAIRS != kNoPairs && (!PAGED || which == 0)) { // (of rows for a cache the second set are values)
        if (HALVES) {
          if (both) {
#pragma unroll
            for (int i = 0; i < ANGLES; ++i) turn(x[j].e[i], y[j].e[i], cs[i], sn[i]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < ANGLES; ++i)
            if (i < turned) turn(x[j].e[2 * i % W], x[j].e[(2 * i + 1) % W], cs[i], sn[i]);
        }
      }
      T* out = static_cast<T*>(set.out) + first + (PAGED ? slot + (long long)head * prm.page_rows * D : b * set.out_b + row * set.out_n + head * set.out_h);
      *reinterpret_cast<V*>(out) = x[j].raw;
      if (both) *reinterpret_cast<V*>(out + R) = y[j].raw;
    }
  }
}

template <typename T, int D, int PAIRS, bool PAGED>
__global__ void __launch_bounds__(256) rotary_kernel(const __grid_constant__ RotaryTable table,
                                                     const __grid_constant__ RotaryParams prm) {
  wait_for_previous();
  __shared__ unsigned long long s_turns[kMaxPairs];
  __shared__ unsigned char s_axis[kMaxPairs];
  if (PAIRS != kNoPairs) {
    if (threadIdx.x < kMaxPairs) {
      s_turns[threadIdx.x] = table.turns[threadIdx.x];
      s_axis[threadIdx.x] = table.axis[threadIdx.x];
    }
    __syncthreads();
  }
  let_next_start();
  rotary_rows<T, D, PAIRS, PAGED>(s_turns, s_axis, table.pairs, table.axes, prm);
  if (PAGED && blockIdx.x == 0 && blockIdx.y == 0) {
    // This block looks at every index of the call and writes the status word, so that nothing has to clear it first.
    int bad = 0;
    const unsigned most = (unsigned)(prm.n / prm.page_rows + 2);
#pragma unroll 4
    for (unsigned long long e = threadIdx.x; e < (unsigned long long)prm.batch * most; e += blockDim.x) {
      const unsigned s = e <= 0xffffffffULL ? (unsigned)e / most : (unsigned)(e / most), part = (unsigned)(e - (unsigned long long)s * most);
      const int start = prm.lengths[s], count = prm.count ? prm.count[s] : prm.n;
      bad |= start < 0 || count < 0 || count > prm.n;
      const int rows = min(max(count, 0), prm.n);
      const unsigned first = (unsigned)max(start, 0), page = first / (unsigned)prm.page_rows + part;
      if (rows == 0 || page > (first + (unsigned)rows - 1u) / (unsigned)prm.page_rows) continue;
      if (page >= (unsigned)prm.pages_per_sequence) bad = 1;
      else bad |= (unsigned)prm.page_table[(size_t)s * prm.pages_per_sequence + page] >= (unsigned)prm.pages;
    }
    bad = __syncthreads_or(bad);
    if (threadIdx.x == 0) prm.status[0] = prm.status[kAppendWord] = bad ? CA_ERR_BAD_INDEX : CA_OK;
  }
}

// ---- host side -------------------------------------------------------------------------------------------

// frequency / (2 pi) modulo 1 as a 64-bit fraction, rounded: the frequency's 53-bit mantissa times 128 bits of 1 / (2 pi), so that the
// fraction is right to its last bit up to 2^32 radians per step.
static unsigned long long turn_fraction(double freq) {
  constexpr unsigned long long kHi = 0x28BE60DB9391054Aull, kLo = 0x7F09D5F47D4D3770ull;   // 2^128 / (2 pi)
  unsigned long long bits;
  memcpy(&bits, &freq, sizeof(bits));
  const int field = (int)(bits >> 52) & 0x7ff;
  const unsigned long long M = (bits & 0xfffffffffffffULL) | (field ? 1ULL << 52 : 0);   // |freq| = M 2^(exponent - 53)
  const int exponent = (field ? field : 1) - 1022;
  const unsigned __int128 low = (unsigned __int128)M * kLo, high = (unsigned __int128)M * kHi + (low >> 64);
  // the product is (high, low's lower word) 2^(exponent - 53 - 128) turns; word `shift` bits up is the fraction
  const unsigned long long w[4] = {(unsigned long long)low, (unsigned long long)high, (unsigned long long)(high >> 64), 0ull};
  const int shift = 64 - (exponent - 53);
  unsigned long long r = 0;
  if (shift < 193) {
    const int word = (shift - 1) / 64, bit = (shift - 1) % 64;         // one bit more, to round
    auto at = [&](int i) { return i < 3 ? w[i] : 0ull; };
    const unsigned __int128 two = ((unsigned __int128)at(word + 1) << 64) | at(word);
    const unsigned long long below = (unsigned long long)(two >> bit);
    const unsigned long long top = (unsigned long long)(((((unsigned __int128)at(word + 2) << 64) | at(word + 1)) >> bit) & 1u);
    r = (below >> 1) + (top << 63) + (below & 1u);
  }
  return freq < 0 ? 0ull - r : r;
}

static int make_table(const ca_rotary_t& rot, int D, RotaryTable* table) {
  if (rot.axes < 1 || rot.axes > 4 || !rot.freq) return CA_ERR_INVALID_ARG;
  table->axes = rot.axes;
  int n = 0;
  for (int a = 0; a < rot.axes; ++a) {
    if (rot.pairs[a] < 0 || rot.pairs[a] > D / 2 - n) return CA_ERR_INVALID_ARG;
    for (int i = 0; i < rot.pairs[a]; ++i, ++n) {
      if (!(fabs(rot.freq[n]) <= 4294967296.0)) return CA_ERR_INVALID_ARG;
      table->turns[n] = turn_fraction(rot.freq[n]);
      table->axis[n] = (unsigned char)a;
    }
  }
  if (n < 1) return CA_ERR_INVALID_ARG;
  table->pairs = n;
  return CA_OK;
}

template <typename T, int D, bool PAGED>
static int launch_rotary_d(const RotaryTable& table, RotaryParams& prm, int pairs_mode, int batch, LaunchStream st) {
  constexpr int W = 16 / (int)sizeof(T);
  const int R = table.pairs;
  // (an element at a time it is the number of accesses that counts: 2 x 12 heads of 16,385 rows, bf16, d = 64, 29 pairs 51.8 us, 32 pairs 17.8)
  if (pairs_mode == kHalves && R % W != 0) pairs_mode = kHalvesScalar;
  const int w = pairs_mode == kHalvesScalar ? 1 : W;
  prm.items = pairs_mode == kHalves || pairs_mode == kHalvesScalar ? D / w - R / w : D / W;
  prm.rows_per_block = 256 / prm.items;
  const int heads = prm.set[0].heads + prm.set[1].heads;
  prm.batch = batch;
  prm.lines = (long long)prm.n * batch;
  const long long blocks_n = (prm.lines + prm.rows_per_block - 1) / prm.rows_per_block;
  // heads per thread: its sines and cosines serve 8, fewer where that leaves SMs without blocks
  const int sms = multiprocessors();
  if (sms == 0) return CA_ERR_CUDA;
  int per = 8;
  while (per > 1 && blocks_n * ((heads + per - 1) / per) < 2 * sms) per /= 2;
  prm.heads_per_thread = per;
  const dim3 grid((unsigned)blocks_n, (unsigned)((heads + per - 1) / per));
  if (blocks_n > 0x7fffffffLL || grid.y > 65535u) return CA_ERR_UNSUPPORTED;
  auto go = [&](auto mode) -> int {
    launch_chained(rotary_kernel<T, D, decltype(mode)::value, PAGED>, grid, 256, 0, st, table, prm);
    CA_LAUNCH_CHECK();
    return CA_OK;
  };
  switch (pairs_mode) {
    case kNoPairs: return go(std::integral_constant<int, kNoPairs>{});
    case kAdjacent: return go(std::integral_constant<int, kAdjacent>{});
    case kHalves: return go(std::integral_constant<int, kHalves>{});
    default: return go(std::integral_constant<int, kHalvesScalar>{});
  }
}

template <bool PAGED>
static int launch_rotary(const RotaryTable& table, RotaryParams& prm, int mode, int batch, int D, int dtype, LaunchStream st) {
  if (dtype == CA_DTYPE_BF16)
    return D == 64 ? launch_rotary_d<__nv_bfloat16, 64, PAGED>(table, prm, mode, batch, st)
                   : launch_rotary_d<__nv_bfloat16, 128, PAGED>(table, prm, mode, batch, st);
  return D == 64 ? launch_rotary_d<float, 64, PAGED>(table, prm, mode, batch, st)
                 : launch_rotary_d<float, 128, PAGED>(table, prm, mode, batch, st);
}

int check_rows(const ca_rows_t* x, int batch, int heads, int n, int D, int dtype, bool written) {
  if (!x || !x->data || (reinterpret_cast<uintptr_t>(x->data) & 15u)) return CA_ERR_INVALID_ARG;
  const long long vec = dtype == CA_DTYPE_BF16 ? 8 : 4;
  const long long stride[3] = {x->stride_b, x->stride_h, x->stride_n};
  const int extent[3] = {batch, heads, n};
  for (int i = 0; i < 3; ++i) {
    if (extent[i] <= 1) continue;                          // a stride that nothing is multiplied with
    if (stride[i] % vec != 0) return CA_ERR_INVALID_ARG;
    if (written && stride[i] < D) return CA_ERR_INVALID_ARG;   // rows of an output do not overlap
  }
  return CA_OK;
}

static RowSet row_set(const ca_rows_t* in, const ca_rows_t* out, int heads) {
  RowSet s{};
  s.in = in->data;
  s.in_b = in->stride_b; s.in_h = in->stride_h; s.in_n = in->stride_n;
  if (out) {
    s.out = out->data;
    s.out_b = out->stride_b; s.out_h = out->stride_h; s.out_n = out->stride_n;
  }
  s.heads = heads;
  return s;
}

int launch_rotary_axes(const ca_rotary_t& rot, int batch, int heads_q, int heads_k, int n, int D, int dtype, int inverse,
                       const ca_rows_t* Q, const ca_rows_t* K, const int32_t* positions, long long pos_b, const ca_rows_t* Qo,
                       const ca_rows_t* Ko, LaunchStream st) {
  RotaryTable table{};
  const int rc = make_table(rot, D, &table);
  if (rc != CA_OK) return rc;
  RotaryParams prm{};
  if (heads_q) prm.set[0] = row_set(Q, Qo, heads_q);
  if (heads_k) prm.set[1] = row_set(K, Ko, heads_k);
  prm.positions = positions;
  prm.pos_b = pos_b;
  prm.n = n;
  prm.inverse = inverse;
  return launch_rotary<false>(table, prm, rot.adjacent ? kAdjacent : kHalves, batch, D, dtype, st);
}

int launch_cache_append(const ca_cache_t& c, int n, const ca_rows_t* K, const ca_rows_t* V, const int32_t* lengths,
                        const int32_t* count, const int32_t* page_table, const ca_rotary_t* rot, const int32_t* positions,
                        long long pos_b, void* K_pages, void* V_pages, int* status, LaunchStream st) {
  RotaryTable table{};
  if (rot) {
    const int rc = make_table(*rot, c.head_dim, &table);
    if (rc != CA_OK) return rc;
  }
  RotaryParams prm{};
  prm.set[0] = row_set(K, nullptr, c.heads_kv);
  prm.set[1] = row_set(V, nullptr, c.heads_kv);
  prm.set[0].out = K_pages;
  prm.set[1].out = V_pages;
  prm.positions = positions;
  prm.pos_b = pos_b;
  prm.n = n;
  prm.lengths = lengths;
  prm.count = count;
  prm.page_table = page_table;
  prm.page_rows = c.page_rows;
  prm.pages = c.pages;
  prm.pages_per_sequence = c.pages_per_sequence;
  prm.batch = c.batch;
  prm.status = status;
  return launch_rotary<true>(table, prm, !rot ? kNoPairs : rot->adjacent ? kAdjacent : kHalves, c.batch, c.head_dim, c.dtype, st);
}

}  // namespace ca
