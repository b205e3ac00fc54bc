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
//                        the radix select of vp_blocks.h, the kept rows in order;
//   evict_move_kernel    the rows. Bound: HBM, K and V of every moved row read and
//                        written once.
// Row i comes from kept[i] >= i, in place: it may be written over once the rows that are
// read from there have been read, and those have lower indices. A work-group reads all of
// its rows, says so, waits until the work-groups of lower rows have said so and then
// writes. The work-groups of a KV head take their rows in the order in which they begin
// (a counter), so what a work-group waits for has begun and waits for nothing before it
// reads: every wait ends, in whatever order the GPU starts them. 32 x 32k tokens of 4 KV
// heads of 128 to half: 400 us, 5.3 TB/s read and written (one work-group per KV head and
// cache that walks its rows upwards, without waits: 1500).
#include "vp_blocks.h"
#include "vp_cache.h"
#include "vp_tile.h"

namespace vp {
namespace {

// order key of a sum: NaN above every number, -0 as 0
__device__ __forceinline__ uint32_t sum_key(float f) {
  return f != f ? 0xffffffffu : order_key(f + 0.f);
}

// scores of rows j0, j0 + STEP, ... (at most last) of kept list u, the heads outermost:
// every head's loads are issued together (heads innermost: the selection of 16 sequences
// of 12k rows, 4 KV heads, 40 us instead of 17)
template <int KPT, int STEP = 64>
__device__ __forceinline__ void row_scores(const EvictArgs& a, int b, int u, int j0, int last, float (&score)[KPT]) {
  const float* s = a.sum + (static_cast<size_t>(b) * a.Hkv + u) * a.max_seq_len;
  if (a.U == a.Hkv) {
#pragma unroll
    for (int j = 0; j < KPT; ++j) score[j] = s[min(j0 + STEP * j, last)];
    return;
  }
  constexpr int N = KPT < 16 ? KPT : 16;  // rows in flight
#pragma unroll
  for (int c = 0; c < KPT; c += N) {
    double t[N];
#pragma unroll
    for (int j = 0; j < N; ++j) t[j] = 0.0;
    const float* sg = s;
    for (int g = 0; g < a.Hkv; ++g, sg += a.max_seq_len) {
      float v[N];
#pragma unroll
      for (int j = 0; j < N; ++j) v[j] = sg[min(j0 + STEP * (c + j), last)];
#pragma unroll
      for (int j = 0; j < N; ++j) t[j] += static_cast<double>(v[j]);
    }
#pragma unroll
    for (int j = 0; j < N; ++j) score[c + j] = static_cast<float>(t[j]);
  }
}

// Writes first + rank of the kept ranks (every key > T and the first `need` keys == T) in
// ascending order to out, from keys in registers; keys of slots past the last rank are 0
// (no sum has that key). Eviction keeps a good part of its rows, so every slot is a
// compare, whose mask the lanes count themselves in, and a store of consecutive words.
// Bound by instruction issue (a SIMD runs four of the block's waves): lanes that walk only
// their own kept slots, as the sparse selection of vp_blocks.h has them, take 9.7 us for
// 16k of 32k rows, this 4.5. One barrier.
template <int KPT>
__device__ __forceinline__ void dense_compaction(SelectShared& sh, const RegKeys<KPT>& keys, int need, uint32_t T,
                                                 int32_t* out, int first, int lane, int wid) {
  int gt = 0, eq = 0;  // of the wave
#pragma unroll
  for (int j = 0; j < KPT; ++j) gt += __popcll(__ballot(keys.u[j] > T));
  if (need > 0) {
#pragma unroll
    for (int j = 0; j < KPT; ++j) eq += __popcll(__ballot(keys.u[j] == T));
  }
  if (lane == 0) {
    sh.gt[wid] = gt;
    sh.eq[wid] = eq;
  }
  __syncthreads();
  gt = __builtin_amdgcn_readfirstlane(waves_below(sh.gt, wid));
  const int rank0 = first + keys.r0;
  if (need == 0) {
#pragma unroll
    for (int j = 0; j < KPT; ++j) {
      const bool mine = keys.u[j] > T;
      const uint64_t mask = __ballot(mine);
      if (mine) out[gt + lanes_below(mask)] = rank0 + 64 * j;
      gt += __popcll(mask);
    }
    return;
  }
  eq = __builtin_amdgcn_readfirstlane(waves_below(sh.eq, wid));
#pragma unroll
  for (int j = 0; j < KPT; ++j) {
    const bool over = keys.u[j] > T, tied = keys.u[j] == T;
    const uint64_t bgt = __ballot(over), beq = __ballot(tied);
    const int e = eq + lanes_below(beq);  // equal keys before this lane's
    if (over || (tied && e < need)) out[gt + lanes_below(bgt) + min(need, e)] = rank0 + 64 * j;
    gt += __popcll(bgt);
    eq += __popcll(beq);
  }
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
  // the move kernel's counters of this list's KV heads
  {
    const int heads = a.U == 1 ? a.Hkv : 1;
    uint32_t* turns = a.turns + (static_cast<size_t>(b) * a.Hkv + u) * a.turn_words;
    for (int i = tid; i < heads * a.turn_words; i += kSelThreads) turns[i] = 0u;
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
  for (int i = tid; i < kHistWords; i += kSelThreads) sh.hist[i] = 0;
  uint32_t kmin = 0xffffffffu, kmax = 0u;
  if constexpr (KPT > 0) {
    RegKeys<KPT> keys;
    keys.r0 = wid * 64 * KPT + lane;
    keys.n = n;
    float score[KPT];
    row_scores<KPT>(a, b, u, S + keys.r0, S + n - 1, score);
#pragma unroll
    for (int j = 0; j < KPT; ++j) {  // slots past n hold the last key: no change of the range
      keys.u[j] = sum_key(score[j]);
      kmin = min(kmin, keys.u[j]);
      kmax = max(kmax, keys.u[j]);
    }
    block_key_range(sh, kmin, kmax, lane, wid);
    // slots past n: a key below every other
#pragma unroll
    for (int j = 0; j < KPT; ++j) keys.u[j] = keys.rank(j) < n ? keys.u[j] : 0u;
    int need = k;
    const uint32_t T = radix_select(
        sh,
        [&](auto visit) {
#pragma unroll
          for (int j = 0; j < KPT; ++j) visit(keys.u[j]);
        },
        need, kmin, kmax, tid, lane, wid);
    dense_compaction(sh, keys, need, T, kept + S, S, lane, wid);
  } else {
    uint32_t* keys = a.keys + static_cast<size_t>(row) * a.max_seq_len;
    constexpr int kBatch = 8;  // rows in flight per thread
    for (int base = 0; base < n; base += kBatch * kSelThreads) {
      float score[kBatch];
      row_scores<kBatch, kSelThreads>(a, b, u, S + base + tid, S + n - 1, score);
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int i = base + j * kSelThreads + tid;
        if (i < n) {
          const uint32_t x = sum_key(score[j]);
          keys[i] = x;
          kmin = min(kmin, x);
          kmax = max(kmax, x);
        }
      }
    }
    if (tid == 0) {
      // one segment: candidate r is row S + r
      tab.st[0] = S;
      tab.en[0] = S + n;
      tab.rk[0] = 0;
      tab.rk[1] = n;
      tab.n = 1;
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
// Rows per work-group: 128 KB of K and V of 256- and 512-byte rows (32 x 32k tokens: 64 rows
// of 256 bytes 627 us per call, 128 494, 256 441), 32 KB where that would leave CUs idle
// (1 x 8k tokens: 18.1 us, with 256 rows 19.7). Rows of 128 bytes: as many as of 256, half
// the bytes, as a work-group has a thread for each row.
constexpr int large_rows(int row_bytes) { return row_bytes > 256 ? 128 : 256; }
constexpr int small_rows(int row_bytes) { return row_bytes > 256 ? 32 : 64; }

// set, or wait for, a word that work-groups of this launch share (device scope: the
// XCDs' L2 caches are not coherent with each other)
__device__ __forceinline__ void set_word(uint32_t* p) {
  __hip_atomic_store(p, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void await_word(const uint32_t* p) {
  while (__hip_atomic_load(const_cast<uint32_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == 0u)
    __builtin_amdgcn_s_sleep(1);
}

// 16 bytes of a row that moves: its old place is not read again (cached: 513 us,
// read past the caches 494, 32 x 32k tokens at 128 rows per work-group)
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint4 load_row(const char* p) {
  const u32x4 x = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
  return make_uint4(x.x, x.y, x.z, x.w);
}

// the visual segments of sequence b in the numbering of its n kept rows (L before)
__device__ __forceinline__ void move_segments(const EvictArgs& a, int b, const int32_t* kept, int n, int L, int tid) {
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
}

// Grid (chunks, Hkv, B), and one more work-group per KV head when segments are wanted.
template <int ROWB, int ROWS>
__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(const EvictArgs a) {
  constexpr int PIECES = ROWB / 16;
  constexpr int RPR = kMoveThreads / PIECES;  // rows per round of loads
  constexpr int U = ROWS / RPR;               // rounds
  static_assert(U * RPR == ROWS && ROWS <= kMoveThreads, "rows of a work-group");
  __shared__ int s_turn;
  __shared__ int s_src[ROWS];  // position each row comes from (its own: it stays; -1: no row)
  __shared__ size_t s_from[ROWS], s_to[ROWS];
  const int g = blockIdx.y, b = blockIdx.z;
  const int tid = threadIdx.x;
  const int row = b * a.U + (a.U == 1 ? 0 : g);
  uint32_t* turns = a.turns + (static_cast<size_t>(b) * a.Hkv + g) * a.turn_words;
  if (tid == 0 && static_cast<int>(blockIdx.x) < a.chunks)
    s_turn = static_cast<int>(__hip_atomic_fetch_add(turns, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
  const int n = a.meta[2 * row], L = a.meta[2 * row + 1];
  const int32_t* kept = a.kept + static_cast<size_t>(row) * a.budget;
  if (static_cast<int>(blockIdx.x) == a.chunks) {
    if (g == 0) move_segments(a, b, kept, n, L, tid);
    return;
  }
  __syncthreads();
  const int c = s_turn;
  if (c == 0 && g == 0 && tid == 0) a.new_len[b] = n;
  const int i0 = c * ROWS;
  if (i0 >= n) return;  // (rows past the end are nobody's source)
  const int64_t head = static_cast<int64_t>(g) * a.sh;
  float sum = 0.f;
  const size_t sums = (static_cast<size_t>(b) * a.Hkv + g) * a.max_seq_len;
  if (tid < ROWS) {
    const int i = i0 + tid;
    const int src = i < n ? kept[i] : -1;
    const int from = src < 0 ? 0 : src, to = i < n ? i : 0;
    if (a.block_table) {
      const int32_t* bt = a.block_table + static_cast<size_t>(b) * a.nblk;
      const int mask = (1 << a.bs_log2) - 1;
      s_from[tid] = static_cast<size_t>(bt[from >> a.bs_log2]) * a.sb + static_cast<size_t>(from & mask) * a.ss + head;
      s_to[tid] = static_cast<size_t>(bt[to >> a.bs_log2]) * a.sb + static_cast<size_t>(to & mask) * a.ss + head;
    } else {
      s_from[tid] = static_cast<size_t>(b) * a.sb + static_cast<size_t>(from) * a.ss + head;
      s_to[tid] = static_cast<size_t>(b) * a.sb + static_cast<size_t>(to) * a.ss + head;
    }
    s_src[tid] = src;
    if (src >= 0) sum = a.sum[sums + src];
  }
  __syncthreads();
  const int r0 = tid / PIECES;
  const size_t piece = 16 * static_cast<size_t>(tid % PIECES);
  uint4 k[U], v[U];
#pragma unroll
  for (int j = 0; j < U; ++j) {
    const int r = j * RPR + r0;
    k[j] = v[j] = make_uint4(0u, 0u, 0u, 0u);
    if (s_src[r] > i0 + r) {
      k[j] = load_row(static_cast<const char*>(a.K) + s_from[r] + piece);
      v[j] = load_row(static_cast<const char*>(a.V) + s_from[r] + piece);
    }
  }
  // the rows and the sums are in registers: what follows waits for every load
#pragma unroll
  for (int j = 0; j < U; ++j) {
    unhoist_vector(k[j].x);
    unhoist_vector(v[j].x);
  }
  unhoist_vector(sum);
  __syncthreads();
  if (tid == 0) set_word(turns + 1 + c);
  // Rows of this chunk may be the source of chunks that began earlier: at most L - n
  // rows further down. Each of those has begun, and sets its word without waiting for
  // anything, so the wait ends.
  const int lowest = max(0, i0 - (L - n)) / ROWS;
  for (int w = lowest + tid; w < c; w += kMoveThreads) await_word(turns + 1 + w);
  __syncthreads();
#pragma unroll
  for (int j = 0; j < U; ++j) {
    const int r = j * RPR + r0;
    if (s_src[r] > i0 + r) {
      *reinterpret_cast<uint4*>(static_cast<char*>(a.K) + s_to[r] + piece) = k[j];
      *reinterpret_cast<uint4*>(static_cast<char*>(a.V) + s_to[r] + piece) = v[j];
    }
  }
  if (tid < ROWS && i0 + tid < n) a.sum_out[sums + i0 + tid] = sum;
}

template <int KPT>
void launch_select_keys(const EvictArgs& a, hipStream_t st) {
  hipLaunchKernelGGL((evict_select_kernel<KPT>), dim3(a.B * a.U), dim3(kSelThreads), 0, st, a);
}

template <int ROWB>
void launch_move(const EvictArgs& a, hipStream_t st) {
  const dim3 grid(a.chunks + (a.seg_out ? 1 : 0), a.Hkv, a.B);
  if (a.rows == large_rows(ROWB))
    hipLaunchKernelGGL((evict_move_kernel<ROWB, large_rows(ROWB)>), grid, dim3(kMoveThreads), 0, st, a);
  else
    hipLaunchKernelGGL((evict_move_kernel<ROWB, small_rows(ROWB)>), grid, dim3(kMoveThreads), 0, st, a);
}

}  // namespace

EvictPlan make_evict_plan(const vp_shape& s, const vp_evict_params& e) {
  auto align = [](size_t x) { return (x + 255) & ~static_cast<size_t>(255); };
  EvictPlan p{};
  const size_t rows = static_cast<size_t>(s.batch) * rows_per_query(s);
  size_t off = 0;
  p.meta = off;
  off = align(off + rows * 2 * 4);
  p.keys = off;
  if (reg_keys(s.max_seq_len) == 0) off = align(off + rows * s.max_seq_len * 4);
  p.turns = off;
  const int most = e.budget < s.max_seq_len ? e.budget : s.max_seq_len;  // rows a sequence holds afterwards
  const int row_bytes = s.head_dim * (s.dtype == VP_BF16 ? 2 : 4);
  p.rows = large_rows(row_bytes);
  if (static_cast<int64_t>(s.batch) * s.n_kv_heads * ((most + p.rows - 1) / p.rows) < 256) p.rows = small_rows(row_bytes);
  p.chunks = (most + p.rows - 1) / p.rows;
  p.turn_words = (1 + p.chunks + 31) / 32 * 32;  // (KV heads on cache lines of their own)
  off = align(off + static_cast<size_t>(s.batch) * s.n_kv_heads * p.turn_words * 4);
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
