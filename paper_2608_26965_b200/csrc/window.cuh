// What the kernels of attention over a sliding window share: the call's arguments and which keys a run of rows sees.
#pragma once
#include "kernels.h"

namespace ca {

struct WindowParams {
  const void *q, *k, *v;
  void* o;
  long long q_b, q_h, q_n, k_b, k_h, k_n, v_b, v_h, v_n, o_b, o_h, o_n;     // strides in elements
  float* lse;                       // [batch][heads_q][n_q] or null
  const int32_t *len_q, *len_k;     // [batch] or null
  int* status;
  int32_t* pieces;                  // [batch + 1] blocks of kWindowBlock rows of the batch items before
  int32_t* redo;                    // [batch * heads_q][blocks of kWindowBlock rows][16]: 16 rows each, to be computed again (null: all)
  int batch, heads_q, heads_kv, group, n_q, n_k, left, right, sinks;
  int one_each;                     // a CTA of the tensor-core kernel for every block of rows: nothing is prepared for it, marks are looked at one by one
  float scale_log2;
};

constexpr int kWindowTile = 128;    // query rows of a tensor-core tile
constexpr int kWindowBlock = 256;   // two of them: what a CTA works on at a time
// words of the status block behind the status: a counter that hands out work, whether rows are to be computed again
constexpr int kNextWord = kTileWord, kRedoWord = kTileWord + 1;

// Lengths of a batch item, kept in range (what is out of it is flagged by window_status, or by the launch that prepares the bf16 kernel's).
struct WindowItem {
  int len_q, len_k, shift;          // the last query stands at the last key: query i at key i + shift
  __device__ __forceinline__ WindowItem(const WindowParams& prm, int b) {
    len_q = prm.len_q ? min(max(prm.len_q[b], 0), prm.n_q) : prm.n_q;
    len_k = prm.len_k ? min(max(prm.len_k[b], 0), prm.n_k) : prm.n_k;
    shift = len_k - len_q;
  }
  __device__ __forceinline__ WindowItem(int q, int k) : len_q(q), len_k(k), shift(k - q) {}
};

// Key tiles of U keys that rows [r0, r1) see: first tokens, then the window.
struct WindowSpan {
  int lo, hi, sink_end, sink_tiles, tile_lo, tiles;
  int all_lo, all_hi, all_sink;     // keys in [all_lo, all_hi) or below all_sink (and all_hi) are seen by every row
  __device__ __forceinline__ WindowSpan(const WindowParams& prm, const WindowItem& it, int r0, int r1, int U) {
    const long long p0 = (long long)r0 + it.shift, p1 = (long long)r1 - 1 + it.shift;
    hi = (int)(prm.right < 0 ? it.len_k : max(0LL, min((long long)it.len_k, p1 + prm.right + 1)));
    lo = (int)(prm.left < 0 ? 0 : min((long long)hi, max(0LL, p0 - prm.left)));
    sink_end = min(min(prm.sinks, hi), lo);
    tile_lo = lo / U;
    sink_tiles = min((sink_end + U - 1) / U, tile_lo);
    // (where hi > 0, lo < hi: a query stands at len_k - 1 at most)
    tiles = hi > 0 ? sink_tiles + (hi + U - 1) / U - tile_lo : 0;
    all_lo = (int)(prm.left < 0 ? 0 : max(0LL, min((long long)it.len_k, p1 - prm.left)));
    all_hi = (int)(prm.right < 0 ? it.len_k : max(0LL, min((long long)it.len_k, p0 + prm.right + 1)));
    all_sink = min(prm.sinks, all_hi);
  }
  __device__ __forceinline__ int tile(int i) const { return i < sink_tiles ? i : tile_lo + i - sink_tiles; }
  // every row sees keys [j0, j1)
  __device__ __forceinline__ bool whole(int j0, int j1) const { return j1 <= all_hi && (j0 >= all_lo || j1 <= all_sink); }
};

// Keys that a row sees: below `end`, and from `from` on or below `sinks`.
struct WindowRow {
  int from, end, sinks;
  __device__ __forceinline__ WindowRow(const WindowParams& prm, const WindowItem& it, int row) {
    const long long p = (long long)row + it.shift;
    end = (int)(prm.right < 0 ? it.len_k : max(0LL, min((long long)it.len_k, p + prm.right + 1)));
    from = (int)(prm.left < 0 ? 0 : max(0LL, min((long long)it.len_k, p - prm.left)));
    sinks = prm.sinks;
  }
  __device__ __forceinline__ bool sees(int j) const { return j < end && (j >= from || j < sinks); }
};

// Lengths looked at, by the threads of one block, which alone writes the status word.
__device__ __forceinline__ void window_status(const WindowParams& prm, int threads) {
  int bad = 0;
  for (int i = threadIdx.x; i < prm.batch; i += threads)
    bad |= (prm.len_q && (unsigned)prm.len_q[i] > (unsigned)prm.n_q) || (prm.len_k && (unsigned)prm.len_k[i] > (unsigned)prm.n_k);
  bad = __syncthreads_or(bad);
  if (threadIdx.x == 0) *prm.status = bad ? CA_ERR_BAD_INDEX : CA_OK;
}

// window_ref, with `redo` set, belongs behind the tensor-core kernels, for the rows that they marked.
int launch_window_prepare(const WindowParams& prm, LaunchStream st);     // (the bf16 kernel's: pieces, counters, status)
int launch_window_f32(const WindowParams& prm, int D, LaunchStream st);
int launch_window_ref(const WindowParams& prm, int D, int dtype, LaunchStream st);
int launch_window_tc(WindowParams& prm, int D, LaunchStream st);    // CA_ERR_UNSUPPORTED: strides that it does not take

}  // namespace ca
