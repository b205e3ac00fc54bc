// Eviction from a cache by accumulated attention weight (vp_evict).
//
// Of a sequence of L > budget rows the first n_sink, the last n_recent and, of the
// rows in between, the budget - n_sink - n_recent with the largest score stay (ties to
// the lower position); they move to the rows 0 .. budget - 1 in their order. The score
// of row j is its sum (VP_SCOPE_KV_GROUP: every KV head keeps its own rows) or, per
// sequence, the sum over the KV heads, added in 64 bits and rounded once to 32, so that
// it does not depend on the order of the heads.
//
// Two launches:
//   evict_select_kernel  one 1024-thread work-group per kept list: sort keys of the rows
//                        in between (registers up to 32768 rows, the workspace beyond),
//                        radix select and ordered compaction of vp_blocks.h;
//   evict_move_kernel    the rows. Bound: HBM, every moved row read and written once.
// Row i comes from kept[i] >= i, so a row is read before it is written over if the
// rows of lower i are read first: a work-group walks its rows upwards, a step's rows all
// read before any is written.
#include "vp_blocks.h"
#include "vp_cache.h"

namespace vp {
namespace {

// order key of a sum: NaN above every number, -0 as 0
__device__ __forceinline__ uint32_t sum_key(float f) {
  return f != f ? 0xffffffffu : order_key(f + 0.f);
}

// score of row j of kept list u of sequence b
__device__ __forceinline__ float row_score(const EvictArgs& a, int b, int u, int j) {
  const float* s = a.sum + (static_cast<size_t>(b) * a.Hkv + u) * a.max_seq_len + j;
  if (a.U == a.Hkv) return *s;
  double t = 0.0;
  for (int g = 0; g < a.Hkv; ++g) t += static_cast<double>(s[static_cast<size_t>(g) * a.max_seq_len]);
  return static_cast<float>(t);
}

// KPT > 0: the keys in registers (max_seq_len <= KPT * kSelThreads); 0: in the workspace
template <int KPT>
__global__ __launch_bounds__(kSelThreads) void evict_select_kernel(const EvictArgs a) {
  __shared__ SelectShared sh;
  __shared__ SegTable tab;
  const int row = blockIdx.x;
  const int b = row / a.U, u = row % a.U;
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wid = tid >> 6;
  const int L = clamp_len(a.seq_len[b], a.max_seq_len);
  int32_t* kept = a.kept + static_cast<size_t>(row) * a.budget;
  const int C = a.budget, S = a.n_sink, R = a.n_recent;
  if (tid == 0) {
    a.meta[2 * row] = min(L, C);
    a.meta[2 * row + 1] = L;
  }
  if (L <= C) {
    for (int i = tid; i < C; i += kSelThreads) kept[i] = i < L ? i : -1;
    return;
  }
  const int n = L - S - R;  // candidates S .. L - R - 1
  const int k = C - S - R;  // 0 <= k < n
  for (int i = tid; i < S; i += kSelThreads) kept[i] = i;
  for (int i = tid; i < R; i += kSelThreads) kept[C - R + i] = L - R + i;
  if (k == 0) return;
  if (tid == 0) {
    // one segment: candidate r is row S + r
    tab.st[0] = S;
    tab.en[0] = S + n;
    tab.rk[0] = 0;
    tab.rk[1] = n;
    tab.n = 1;
  }
  for (int i = tid; i < kHistWords; i += kSelThreads) sh.hist[i] = 0;
  uint32_t kmin = 0xffffffffu, kmax = 0u;
  if constexpr (KPT > 0) {
    RegKeys<KPT> keys;
    keys.r0 = wid * 64 * KPT + lane;
    keys.n = n;
#pragma unroll
    for (int j = 0; j < KPT; ++j) {  // slots past n hold the last key: no change of the range
      keys.u[j] = sum_key(row_score(a, b, u, S + min(keys.rank(j), n - 1)));
      kmin = min(kmin, keys.u[j]);
      kmax = max(kmax, keys.u[j]);
    }
    block_key_range(sh, kmin, kmax, lane, wid);
    select_from_registers(sh, tab, keys, k, false, kmin, kmax, kept + S, tid, lane, wid);
  } else {
    uint32_t* keys = a.keys + static_cast<size_t>(row) * a.max_seq_len;
    for (int i = tid; i < n; i += kSelThreads) {
      const uint32_t x = sum_key(row_score(a, b, u, S + i));
      keys[i] = x;
      kmin = min(kmin, x);
      kmax = max(kmax, x);
    }
    __threadfence_block();
    block_key_range(sh, kmin, kmax, lane, wid);  // (its barrier puts the keys before the reads)
    int need = k;
    const uint32_t T = radix_select(
        sh,
        [&](auto visit) {
          for (int i = tid; i < n; i += kSelThreads) visit(keys[i]);
        },
        need, kmin, kmax, tid, lane, wid);
    ordered_compaction(sh, tab, [&](int i) -> uint32_t { return keys[i]; }, n, k, need, T, false, kept + S, lane, wid);
  }
}

constexpr int kMoveThreads = 256;

// Grid (2 + 1, Hkv, B): the K rows, the V rows, and the sums with (KV head 0) the new
// length and the segments.
template <int ROWB>
__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(const EvictArgs a) {
  const int what = blockIdx.x, g = blockIdx.y, b = blockIdx.z;
  const int tid = threadIdx.x;
  const int row = b * a.U + (a.U == 1 ? 0 : g);
  const int n = a.meta[2 * row], L = a.meta[2 * row + 1];
  const int32_t* kept = a.kept + static_cast<size_t>(row) * a.budget;
  if (what == 2) {
    const float* src = a.sum + (static_cast<size_t>(b) * a.Hkv + g) * a.max_seq_len;
    float* dst = a.sum_out + (static_cast<size_t>(b) * a.Hkv + g) * a.max_seq_len;
    for (int i0 = 0; i0 < n; i0 += kMoveThreads) {
      const int i = i0 + tid;
      const float v = i < n ? src[kept[i]] : 0.f;
      __syncthreads();
      if (i < n) dst[i] = v;
    }
    if (g != 0) return;
    if (tid == 0) a.new_len[b] = n;
    if (!a.seg_out) return;
    __shared__ SegTable tab;
    const int o0 = a.seg_off[b];
    if (tid < 64) load_segments(tab, a.seg + 2 * static_cast<long>(o0), a.seg_off[b + 1] - o0, L, tid);
    __syncthreads();
    // rows kept before position p
    auto before = [&](int p) {
      int lo = 0, hi = n;
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (kept[mid] < p) lo = mid + 1;
        else hi = mid;
      }
      return lo;
    };
    for (int s = tid; s < tab.n; s += kMoveThreads) {
      const int st = before(tab.st[s]), en = before(tab.en[s]);
      a.seg_out[2 * (static_cast<long>(o0) + s)] = st;
      a.seg_out[2 * (static_cast<long>(o0) + s) + 1] = en - st;
    }
    return;
  }
  constexpr int PIECES = ROWB / 16;
  constexpr int RPS = kMoveThreads / PIECES;  // rows per round of loads
  constexpr int U = 8;                        // rounds per step
  char* base = static_cast<char*>(what == 0 ? a.K : a.V);
  const int32_t* bt = a.block_table ? a.block_table + static_cast<size_t>(b) * a.nblk : nullptr;
  const int bmask = (1 << a.bs_log2) - 1;
  auto at = [&](int j) -> uint4* {
    const size_t off = bt ? static_cast<size_t>(bt[j >> a.bs_log2]) * a.sb + static_cast<size_t>(j & bmask) * a.ss
                          : static_cast<size_t>(b) * a.sb + static_cast<size_t>(j) * a.ss;
    return reinterpret_cast<uint4*>(base + off + static_cast<size_t>(g) * a.sh) + tid % PIECES;
  };
  for (int i0 = 0; i0 < n; i0 += RPS * U) {
    uint4 v[U];
    int src[U];
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int i = i0 + j * RPS + tid / PIECES;
      src[j] = i < n ? kept[i] : -1;
      if (src[j] != i && i < n) v[j] = *at(src[j]);
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int i = i0 + j * RPS + tid / PIECES;
      if (src[j] != i && i < n) *at(i) = v[j];
    }
    __syncthreads();
  }
}

template <int KPT>
void launch_select_keys(const EvictArgs& a, hipStream_t st) {
  hipLaunchKernelGGL((evict_select_kernel<KPT>), dim3(a.B * a.U), dim3(kSelThreads), 0, st, a);
}

template <int ROWB>
void launch_move(const EvictArgs& a, hipStream_t st) {
  hipLaunchKernelGGL((evict_move_kernel<ROWB>), dim3(3, a.Hkv, a.B), dim3(kMoveThreads), 0, st, a);
}

}  // namespace

EvictPlan make_evict_plan(const vp_shape& s) {
  auto align = [](size_t x) { return (x + 255) & ~static_cast<size_t>(255); };
  EvictPlan p{};
  const size_t rows = static_cast<size_t>(s.batch) * rows_per_query(s);
  size_t off = 0;
  p.meta = off;
  off = align(off + rows * 2 * 4);
  p.keys = off;
  if (reg_keys(s.max_seq_len) == 0) off = align(off + rows * s.max_seq_len * 4);
  p.total = off;
  return p;
}

hipError_t launch_evict(const EvictArgs& a, int row_bytes, hipStream_t st) {
  switch (reg_keys(a.max_seq_len)) {
    case 2: launch_select_keys<2>(a, st); break;
    case 4: launch_select_keys<4>(a, st); break;
    case 8: launch_select_keys<8>(a, st); break;
    case 16: launch_select_keys<16>(a, st); break;
    case 32: launch_select_keys<32>(a, st); break;
    default: launch_select_keys<0>(a, st); break;
  }
  if (hipError_t e = hipGetLastError()) return e;
  switch (row_bytes) {
    case 128: launch_move<128>(a, st); break;
    case 256: launch_move<256>(a, st); break;
    case 512: launch_move<512>(a, st); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace vp
