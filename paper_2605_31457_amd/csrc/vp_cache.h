// Host/device interface of the bounded-cache calls (vp_window_decode_attn, vp_evict)
// between the C ABI (vp_api.hip) and their kernels.
#pragma once

#include "vp_internal.h"

namespace vp {

// ---------------------------------------------------------------------------
// vp_window_decode_attn
// ---------------------------------------------------------------------------
// Work decomposition and workspace carving, a pure function of shape and window.
struct WindowPlan {
  int tiles;     // 32-row tiles that any sequence's queries see, at most
  int groups;    // work-groups that the walks of the batch are dealt to; 0: one per (sequence, KV head)
  int gp;        // floats per spilled row of logits: the query rows padded to 1, 2, 4, 8 or 16
  size_t stats;  // float [groups][T*G][2]          (max, sum) of each work-group's part of a walk
  size_t acc;    // float [groups][T*G][d]          its value partials
  size_t pieces; // int32 [B*Hkv][2]                where a pair's pieces begin, and how many there are
  size_t zs;     // float [B][Hkv][tiles * 32][gp]  products q.K by row of the walk
  size_t total;
};
WindowPlan make_window_plan(const vp_shape& s, const vp_window& w, bool sums);

struct WindowArgs {
  const void* q;
  const void* K;
  const void* V;
  void* out;
  float* attn_sum;             // [B][Hkv][max_seq_len] or null
  int64_t sb, sh, ss;          // KV strides (elements); paged caches: sb is the block stride
  const int32_t* block_table;  // paged caches: [B][nblk] physical blocks (else null)
  int bs_log2;                 // paged caches: log2 of the rows per block; -1: contiguous
  int nblk;                    // row stride of block_table
  const int32_t* seq_len;
  int B, Hq, Hkv, G, T, max_seq_len;
  int window, n_sink;
  uint32_t over_g;             // r / G = r * over_g >> 16 for query rows r < 16
  float zscale;                // sm_scale * log2(e)
  float raise;                 // a running maximum is raised when a product exceeds it by more
  int tiles, groups, gp;
  float* stats;
  float* acc;
  int2* pieces;
  float* zs;
};
hipError_t launch_window(const WindowArgs& a, int dtype, int head_dim, hipStream_t st);

// Pieces of the above that attention over 4-bit caches shares: the tiles of the longest walk,
// the workspace's parts for a plan of so many work-groups, and the launch that joins the pieces.
int window_tiles(const vp_shape& s, const vp_window& w);
void carve_window_plan(WindowPlan& p, const vp_shape& s, bool sums);
hipError_t launch_window_join(const WindowArgs& a, int dtype, int head_dim, hipStream_t st);

// The rows that the queries of one sequence see, as a walk over 32-row tiles of
// positions: the tiles of the first n_sink rows, then those of the window. Query t is
// the token at position L - T + t and sees the positions j <= L - T + t with j < n_sink
// or j > L - T + t - window (window 0: all of them).
struct WindowWalk {
  int L, T, W, S;
  int lo;      // first position in the first query's window
  int sinks;   // tiles of the sinks
  int first;   // tile of the window's first row; the tiles in between are not walked
  int n;       // tiles walked
  __host__ __device__ WindowWalk(int L_, int T_, int W_, int S_) : L(L_), T(T_), W(W_) {
    S = S_ < L ? S_ : L;
    const long l = static_cast<long>(L) - T - W + 1;
    lo = W > 0 && l > 0 ? static_cast<int>(l) : 0;
    sinks = (S + 31) / 32;
    first = lo / 32 > sinks ? lo / 32 : sinks;
    n = sinks + (L + 31) / 32 - first;
  }
  __host__ __device__ int t0(int k) const { return 32 * (k < sinks ? k : k - sinks + first); }
  // tiles lie between the sinks' and the window's: then a sink tile's rows end at the
  // last sink, and the window's first tile begins at its first row
  __host__ __device__ bool apart() const { return lo / 32 >= sinks; }
  __host__ __device__ int row_begin(int k) const {
    const int p = t0(k);
    return apart() && k >= sinks && p < lo ? lo : p;
  }
  __host__ __device__ int row_end(int k) const {
    const int p = t0(k) + 32;
    const int end = apart() && k < sinks ? S : L;
    return p < end ? p : end;
  }
};

// ---------------------------------------------------------------------------
// vp_evict
// ---------------------------------------------------------------------------
struct EvictPlan {
  size_t meta;   // int32 [B*U][2]           rows kept, clamped length (of each kept list)
  size_t keys;   // uint32 [B*U][max_seq_len] sort keys, for caches of more rows than registers hold
  size_t turns;  // uint32 [B*Hkv][turn_words] per KV head: the work-groups that have begun, and one
                 // word per work-group, set when its rows are read
  int rows;      // rows per work-group of the move
  int chunks;    // work-groups that move the rows of a KV head
  int turn_words;
  size_t total;
};
EvictPlan make_evict_plan(const vp_shape& s, const vp_evict_params& p);

struct EvictArgs {
  const int32_t* seq_len;
  const int32_t* seg_off;
  const int32_t* seg;          // (seg_out may be the same array)
  const int32_t* block_table;  // paged caches: [B][nblk] physical blocks (else null)
  int bs_log2, nblk;
  int B, Hkv, U, max_seq_len;  // U: kept lists per sequence, 1 or Hkv
  int budget, n_sink, n_recent;
  int64_t sb, sh, ss;          // KV strides in BYTES; paged caches: sb is the block stride
  const float* sum;            // [B][Hkv][max_seq_len]
  float* sum_out;              // (may be sum)
  void* K;
  void* V;
  int32_t* kept;               // [B*U][budget]
  int32_t* seg_out;            // or null
  int32_t* new_len;            // [B] (may be seq_len)
  int32_t* meta;
  uint32_t* keys;
  uint32_t* turns;
  int rows, chunks, turn_words;
};
hipError_t launch_evict(const EvictArgs& a, int row_bytes, hipStream_t st);

}  // namespace vp
