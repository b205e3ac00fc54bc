// Attention of a step's queries over a sliding window and the first tokens
// (vp_window_decode_attn), optionally adding every row's attention weight to a
// running sum.
//
//   z_j = sm_scale <q_h, K_j>,  A_j = 2^(z_j - M) / l over the rows j that query t sees,
//   out = sum_j A_j V_j,        attn_sum_j += sum over the KV head's query rows of A_j
//
// Bound: the K and V rows that any query sees, read once from HBM (the sums add 8 bytes
// per row and KV head to its 4 * d (bf16) or 8 * d); short walks: launches and
// dependent loads.
//
// Two kernels:
//   window_kernel  one pass over the rows with a running maximum and sum. Grid (parts,
//                  Hkv, B); the four waves of a work-group take 32-row tiles of the
//                  walk (WindowWalk) in turn, part p's wave w the tiles p + parts * w,
//                  p + parts * (w + 4), ...: consecutive work-groups, so all XCDs, read
//                  consecutive tiles. The T*G <= 16 query rows of the KV head share
//                  every tile. The waves' partials meet in LDS; a KV head with one part
//                  is finished there. With sums the logits leave as rows of gp floats
//                  (32 bytes per row at 7 heads, beside 512 bytes of K and V), since a
//                  weight is known only when the whole walk is.
//   finish_kernel  joins the parts of each head, and turns the logits into weights:
//                  one thread per row, the query rows in order, so the sums do not
//                  depend on the partition of the walk or on arrival.
//
// A masked row weighs nothing whatever it holds: its logit is not looked at, and in
// the tiles where some query does not see some row (the ends of the window, of the
// sinks and of the sequence) each query's value product has the rows it does not see
// replaced by zeros, so that a NaN or infinity there stays out of its output.
#include <algorithm>

#include "vp_cache.h"
#include "vp_tile.h"

namespace vp {
namespace {

constexpr int kWinWaves = 4;
constexpr int kWinThreads = 64 * kWinWaves;

size_t align256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

// A running maximum is raised only when a logit exceeds it by more than this (log2
// units): weights stay below 2^64, and rescaling is rare
constexpr float kRaise = 64.f;

template <int DT, int D, bool SUMS>
struct WinLds {
  using C = Cfg<DT, D>;
  static constexpr int STAGE = SUMS ? C::STAGE_BYTES : 0;
  static constexpr int BYTES = 2 * C::SUB_ROWS_BYTES + STAGE;  // per wave: a K block, a V block, a logit stage
};

// (max, sum) of the query rows, per wave
struct WinStats {
  float m[kWinWaves][16];
  float l[kWinWaves][16];
};

template <int DT>
__device__ __forceinline__ void store_out(void* out, size_t row, int D, int col4, float4 v) {
  if constexpr (DT == VP_BF16) {
    uint2 o;
    o.x = f32_to_bf16_bits(v.x) | (static_cast<uint32_t>(f32_to_bf16_bits(v.y)) << 16);
    o.y = f32_to_bf16_bits(v.z) | (static_cast<uint32_t>(f32_to_bf16_bits(v.w)) << 16);
    reinterpret_cast<uint2*>(static_cast<uint16_t*>(out) + row * D)[col4] = o;
  } else {
    reinterpret_cast<float4*>(static_cast<float*>(out) + row * D)[col4] = v;
  }
}

// row of out [B][T][Hq] for query row r (query t = r / G, head g*G + r % G)
__device__ __forceinline__ size_t out_row(const WindowArgs& a, int b, int g, int r) {
  return (static_cast<size_t>(b) * a.T + r / a.G) * a.Hq + g * a.G + r % a.G;
}

template <int DT, int D, bool PAGED, bool SUMS>
__global__ __launch_bounds__(kWinThreads) __attribute__((amdgpu_waves_per_eu(DT == VP_BF16 ? 2 : 1))) void
window_kernel(const WindowArgs a) {
  using C = Cfg<DT, D>;
  using Q = WinLds<DT, D, SUMS>;
  __shared__ __attribute__((aligned(1024))) unsigned char lds_block[kWinWaves * Q::BYTES];
  __shared__ WinStats ws;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const int lane = threadIdx.x & 63;
  const int n16 = lane & 15;
  const int a4 = lane >> 4;
  const int part = blockIdx.x, g = blockIdx.y, b = blockIdx.z;
  const int TG = a.T * a.G;
  unsigned char* lds = lds_block + wave * Q::BYTES;
  lds_byte* dma = (lds_byte*)lds;
  float* stage = reinterpret_cast<float*>(lds + 2 * C::SUB_ROWS_BYTES);

  // the query rows load while the length arrives
  const bool hv = n16 < TG;
  const int tq = hv ? n16 / a.G : 0;
  QFrag<DT, D> qf;
  load_q<DT, D>(qf, static_cast<const char*>(a.q) + (hv ? out_row(a, b, g, n16) : 0) * C::ROWB, hv, a4);
  const WindowWalk w(clamp_len(a.seq_len[b], a.max_seq_len), a.T, a.window, a.n_sink);
  const int hi = w.L - a.T + tq;                           // this lane's query sees j <= hi
  const int below = a.window > 0 ? hi - a.window : -1;     // and j > below or j < n_sink

  const size_t seq_off = PAGED ? 0 : static_cast<size_t>(b) * a.sb;
  const char* Kb = static_cast<const char*>(a.K) + (seq_off + static_cast<size_t>(g) * a.sh) * C::ESZ;
  const char* Vb = static_cast<const char*>(a.V) + (seq_off + static_cast<size_t>(g) * a.sh) * C::ESZ;
  const size_t rstride = static_cast<size_t>(a.ss) * C::ESZ;
  const size_t bstride = static_cast<size_t>(a.sb) * C::ESZ;
  const int32_t* bt = PAGED ? a.block_table + static_cast<size_t>(b) * a.nblk : nullptr;
  const int bmask = PAGED ? (1 << a.bs_log2) - 1 : 0;
  float* zplane = SUMS ? a.zs + (static_cast<size_t>(b) * a.Hkv + g) * a.tiles * 32 * static_cast<size_t>(a.gp) : nullptr;

  float m = kNoLogit, l = 0.f;  // shared by the four lanes of a query row; l is lane-local
  f32x4 acc[C::ACC_N];
#pragma unroll
  for (int i = 0; i < C::ACC_N; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};

  const int step = a.parts * kWinWaves;
  for (int k = part + a.parts * wave; k < w.n; k += step) {
    const int t0 = w.t0(k);
    const int r0 = w.row_begin(k), r1 = w.row_end(k);  // rows that some query sees, r0 < r1
    // LDS reads of the previous tile have returned before the copies overwrite it
    __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
    {
      // row r of the tile, the others' places take the nearest row that is read anyway
      const int rr = lane / C::PIECES, slot = lane % C::PIECES;
      size_t off[C::COPIES];
#pragma unroll
      for (int j = 0; j < C::COPIES; ++j) {
        const int r = j * C::RPI + rr;
        const int pos = min(max(t0 + r, r0), r1 - 1);
        const int piece = 16 * (slot ^ (r & (C::PIECES - 1)));
        if constexpr (PAGED)
          off[j] = static_cast<size_t>(bt[pos >> a.bs_log2]) * bstride + static_cast<size_t>(pos & bmask) * rstride + piece;
        else
          off[j] = static_cast<size_t>(pos) * rstride + piece;
      }
#pragma unroll
      for (int j = 0; j < C::COPIES; ++j)
        __builtin_amdgcn_global_load_lds((global_void*)(Kb + off[j]), (lds_void*)(dma + 1024 * j), 16, 0, kCopyPolicy);
#pragma unroll
      for (int j = 0; j < C::COPIES; ++j)
        __builtin_amdgcn_global_load_lds((global_void*)(Vb + off[j]), (lds_void*)(dma + C::SUB_ROWS_BYTES + 1024 * j), 16,
                                         0, kCopyPolicy);
    }
    __builtin_amdgcn_s_waitcnt(kWaitVm0);

    float z[8];
    {
      const f32x4 c0 = score_half<DT, D>(lds, 0, qf, a4, n16);
      const f32x4 c1 = score_half<DT, D>(lds, 1, qf, a4, n16);
#pragma unroll
      for (int i = 0; i < 8; ++i) z[i] = (i < 4 ? c0[i & 3] : c1[i & 3]) * a.zscale;
    }
    // value i of this lane is row t0 + pv_token(a4, i). Does every query see every row?
    const int last0 = w.L - a.T;                                     // the first query's own position
    const int hidden = a.window > 0 ? w.L - 1 - a.window : -1;       // the last query sees no row from n_sink to here
    const bool edge = t0 + 31 > last0 || max(t0, w.S) <= min(t0 + 31, hidden);
    unsigned seen = 0xffu;
    if (edge) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int j = t0 + pv_token(a4, i);
        if (j > hi || (j <= below && j >= w.S)) seen &= ~(1u << i);
      }
    }
    if constexpr (SUMS) {
      // the tile's logits as 32 rows of gp floats, -inf where a query does not see the row
      const int gp = a.gp;
      if (n16 < gp) {
#pragma unroll
        for (int i = 0; i < 8; ++i) stage[pv_token(a4, i) * gp + n16] = (seen >> i) & 1u ? z[i] : kNegInf;
      }
      const float4* src = reinterpret_cast<const float4*>(stage);
      float4* dst = reinterpret_cast<float4*>(zplane + static_cast<size_t>(k) * 32 * gp);
      for (int i = lane; i < 8 * gp; i += 64) dst[i] = src[i];
    }
    float lmax = kNegInf;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if ((seen >> i) & 1u) lmax = fmaxf(lmax, z[i]);
    if (__builtin_amdgcn_ballot_w64(lmax > m + kRaise)) {
      // the four lanes of a query row share the reference (their weights meet in one MFMA)
      const float tm = max_over_quads(lmax);
      const bool up = tm > m + kRaise;
      const float al = up ? fast_exp2(m - tm) : 1.f;
      l *= al;
#pragma unroll
      for (int i = 0; i < C::ACC_N; ++i) acc[i] *= al;
      m = up ? tm : m;
    }
    float p[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      p[i] = (seen >> i) & 1u ? fast_exp2(z[i] - m) : 0.f;
      l += p[i];
    }
    const unsigned char* vb = lds + C::SUB_ROWS_BYTES;
    if (!edge) {
      value_product<DT, D, C::ACC_N, true>(acc, vb, p, a4, n16);
    } else {
      // one query at a time, with the rows that it sees
#pragma unroll 1
      for (int t = 0; t < a.T; ++t) {
        const int h = w.L - a.T + t;
        const int lo = a.window > 0 ? h - a.window : -1;
        unsigned rows = 0u;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int j = t0 + pv_token(a4, i);
          if (j <= h && (j > lo || j < w.S)) rows |= 1u << i;
        }
        // (a lane's accumulators are its own query row's: those of other queries are dropped)
        f32x4 sum[C::ACC_N];
#pragma unroll
        for (int i = 0; i < C::ACC_N; ++i) sum[i] = acc[i];
        value_product<DT, D, C::ACC_N, true, true>(sum, vb, p, a4, n16, rows);
#pragma unroll
        for (int i = 0; i < C::ACC_N; ++i) acc[i] = tq == t ? sum[i] : acc[i];
      }
    }
  }
  l = sum_over_quads(l);

  // ---- join the four waves ----
  constexpr int PITCH = D + 4;  // accumulator rows start on different banks
  static_assert(16 * PITCH * 4 <= Q::BYTES, "accumulator rows of a wave");
  __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
  if (a4 == 0) {
    ws.m[wave][n16] = m;
    ws.l[wave][n16] = l;
  }
  store_acc<DT, D, C::ACC_N>(reinterpret_cast<float*>(lds) + n16 * PITCH, acc, a4);
  __syncthreads();
  const size_t pair = static_cast<size_t>(b) * a.Hkv + g;
  constexpr int COLS = D / 4;
  for (int i = threadIdx.x; i < TG * COLS; i += kWinThreads) {
    const int h = i / COLS, c = i % COLS;
    float M = ws.m[0][h];
#pragma unroll
    for (int v = 1; v < kWinWaves; ++v) M = fmaxf(M, ws.m[v][h]);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    float den = 0.f;
#pragma unroll
    for (int v = 0; v < kWinWaves; ++v) {
      const float f = fast_exp2(ws.m[v][h] - M);
      const float4 x = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(lds_block + v * Q::BYTES) + h * PITCH)[c];
      den = fmaf(f, ws.l[v][h], den);
      o.x = fmaf(f, x.x, o.x);
      o.y = fmaf(f, x.y, o.y);
      o.z = fmaf(f, x.z, o.z);
      o.w = fmaf(f, x.w, o.w);
    }
    const size_t row = (pair * TG + h) * a.parts + part;
    if (a.parts == 1) {
      const float inv = 1.0f / den;
      const float4 r = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
      store_out<DT>(a.out, out_row(a, b, g, h), D, c, den == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : r);
    } else {
      reinterpret_cast<float4*>(a.acc + row * D)[c] = o;
    }
    if ((SUMS || a.parts > 1) && c == 0) *reinterpret_cast<float2*>(a.stats + row * 2) = make_float2(M, den);
  }
}

// Grid (heads + row groups, Hkv, B): with more than one part, the first T*G
// work-groups of a KV head join the parts of one query row each; the others (sums)
// take kFinishRows rows of the walk each.
constexpr int kFinishThreads = 256;
constexpr int kFinishRows = kFinishThreads;

// (max, 1 / sum) of query row r over the parts, by the 16 lanes that share it
__device__ __forceinline__ float2 row_norm(const WindowArgs& a, size_t pair, int r, int sub) {
  const float2* st = reinterpret_cast<const float2*>(a.stats) + (pair * a.T * a.G + r) * a.parts;
  float M = kNoLogit;
  for (int i = sub; i < a.parts; i += 16) M = fmaxf(M, st[i].x);
  M = group_max_f32(M, 16);
  float l = 0.f;
  for (int i = sub; i < a.parts; i += 16) l = fmaf(fast_exp2(st[i].x - M), st[i].y, l);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) l += __shfl_xor(l, o, 16);
  return make_float2(M, l == 0.f ? 0.f : 1.0f / l);
}

template <int DT, int D>
__global__ __launch_bounds__(kFinishThreads) void finish_kernel(const WindowArgs a, int heads) {
  constexpr int COLS = D / 4;
  constexpr int R = kFinishThreads / COLS;
  const int g = blockIdx.y, b = blockIdx.z;
  const int tid = threadIdx.x;
  const size_t pair = static_cast<size_t>(b) * a.Hkv + g;
  const int TG = a.T * a.G;
  __shared__ float2 norm[16];
  __shared__ float4 part_sum[R][COLS];
  if (static_cast<int>(blockIdx.x) < heads) {
    const int h = blockIdx.x;
    if (tid < 16) norm[tid] = row_norm(a, pair, h, tid);
    __syncthreads();
    const float2 mn = norm[0];
    const int col = tid % COLS, r = tid / COLS;
    const size_t row0 = (pair * TG + h) * a.parts;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = r; i < a.parts; i += R) {
      const float f = fast_exp2(a.stats[(row0 + i) * 2] - mn.x);
      const float4 x = reinterpret_cast<const float4*>(a.acc + (row0 + i) * D)[col];
      o.x = fmaf(f, x.x, o.x);
      o.y = fmaf(f, x.y, o.y);
      o.z = fmaf(f, x.z, o.z);
      o.w = fmaf(f, x.w, o.w);
    }
    part_sum[r][col] = o;
    __syncthreads();
    if (r == 0) {
#pragma unroll
      for (int v = 1; v < R; ++v) {
        const float4 x = part_sum[v][col];
        o.x += x.x;
        o.y += x.y;
        o.z += x.z;
        o.w += x.w;
      }
      // (an empty context, or one of logits -inf: zeros)
      const float4 z = make_float4(0.f, 0.f, 0.f, 0.f);
      const float4 v = make_float4(o.x * mn.y, o.y * mn.y, o.z * mn.y, o.w * mn.y);
      store_out<DT>(a.out, out_row(a, b, g, h), D, col, mn.y == 0.f ? z : v);
    }
    return;
  }
  const WindowWalk w(clamp_len(a.seq_len[b], a.max_seq_len), a.T, a.window, a.n_sink);
  const int i0 = (static_cast<int>(blockIdx.x) - heads) * kFinishRows;
  if (i0 >= 32 * w.n) return;
  if (tid < 16 * TG) {
    const float2 mn = row_norm(a, pair, tid >> 4, tid & 15);
    if ((tid & 15) == 0) norm[tid >> 4] = mn;
  }
  __syncthreads();
  const int i = i0 + tid;
  const int k = i >> 5;
  if (k >= w.n) return;
  const int j = w.t0(k) + (i & 31);
  if (j < w.row_begin(k) || j >= w.row_end(k)) return;
  const float* z = a.zs + (pair * a.tiles * 32 + i) * a.gp;
  float s = 0.f;
  for (int h = 0; h < TG; ++h) s = fmaf(fast_exp2(z[h] - norm[h].x), norm[h].y, s);
  float* dst = a.attn_sum + pair * a.max_seq_len + j;
  *dst = j >= w.L - a.T ? s : *dst + s;
}

template <int DT, int D>
hipError_t launch_dd(const WindowArgs& a, hipStream_t st) {
  const dim3 grid(a.parts, a.Hkv, a.B);
  const bool paged = a.bs_log2 >= 0, sums = a.attn_sum != nullptr;
  if (paged && sums) hipLaunchKernelGGL((window_kernel<DT, D, true, true>), grid, dim3(kWinThreads), 0, st, a);
  else if (paged) hipLaunchKernelGGL((window_kernel<DT, D, true, false>), grid, dim3(kWinThreads), 0, st, a);
  else if (sums) hipLaunchKernelGGL((window_kernel<DT, D, false, true>), grid, dim3(kWinThreads), 0, st, a);
  else hipLaunchKernelGGL((window_kernel<DT, D, false, false>), grid, dim3(kWinThreads), 0, st, a);
  if (hipError_t e = hipGetLastError()) return e;
  const int heads = a.parts > 1 ? a.T * a.G : 0;
  const int rows = sums ? (a.tiles * 32 + kFinishRows - 1) / kFinishRows : 0;
  if (heads + rows > 0)
    hipLaunchKernelGGL((finish_kernel<DT, D>), dim3(heads + rows, a.Hkv, a.B), dim3(kFinishThreads), 0, st, a, heads);
  return hipGetLastError();
}

}  // namespace

WindowPlan make_window_plan(const vp_shape& s, const vp_window& w, bool sums) {
  WindowPlan p{};
  const int64_t T = queries(s), cap = (static_cast<int64_t>(s.max_seq_len) + 31) / 32;
  int64_t tiles = cap;
  if (w.window > 0)  // the window's rows may begin anywhere in a tile
    tiles = std::min(cap, (static_cast<int64_t>(w.n_sink) + 31) / 32 + (w.window + T - 1 + 30) / 32 + 1);
  p.tiles = static_cast<int>(tiles);
  const int64_t pairs = static_cast<int64_t>(s.batch) * s.n_kv_heads;
  // one resident round of work-groups, a tile per wave at least
  const int64_t parts = std::min<int64_t>(resident_groups(s.dtype, s.head_dim) / pairs, (tiles + kWinWaves - 1) / kWinWaves);
  p.parts = static_cast<int>(std::max<int64_t>(1, parts));
  const int rows = static_cast<int>(T) * (s.n_q_heads / s.n_kv_heads);
  p.gp = 1;
  while (p.gp < rows) p.gp *= 2;
  size_t off = 0;
  p.stats = off;
  off = align256(off + static_cast<size_t>(pairs) * rows * p.parts * 2 * 4);
  p.acc = off;
  if (p.parts > 1) off = align256(off + static_cast<size_t>(pairs) * rows * p.parts * s.head_dim * 4);
  p.zs = off;
  if (sums) off = align256(off + static_cast<size_t>(pairs) * p.tiles * 32 * p.gp * 4);
  p.total = off;
  return p;
}

hipError_t launch_window(const WindowArgs& a, int dtype, int head_dim, hipStream_t st) {
  if (dtype == VP_BF16) {
    if (head_dim == 128) return launch_dd<VP_BF16, 128>(a, st);
    if (head_dim == 64) return launch_dd<VP_BF16, 64>(a, st);
  } else if (dtype == VP_F32) {
    if (head_dim == 128) return launch_dd<VP_F32, 128>(a, st);
    if (head_dim == 64) return launch_dd<VP_F32, 64>(a, st);
  }
  return hipErrorInvalidValue;
}

}  // namespace vp
