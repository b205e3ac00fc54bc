// Attention of a step's queries over a sliding window and the first tokens
// (vp_window_decode_attn), optionally adding every row's attention weight to a
// running sum.
//
//   z_j = <q_h, K_j>,  A_j = 2^(c (z_j - M)) / l over the rows j that query t sees, c = sm_scale log2(e),
//   out = sum_j A_j V_j,        attn_sum_j += sum over the KV head's query rows of A_j
//
// Bound: the K and V rows that any query sees, read once from HBM (the sums add 8 bytes
// per row and KV head to its 4 * d (bf16) or 8 * d); short walks: launches and
// dependent loads.
//
// Two kernels:
//   window_kernel  one pass over the rows with a running maximum and sum. Every (sequence,
//                  KV head) pair has work-groups in proportion to the 32-row tiles of its
//                  walk (WindowWalk), as many as are resident at a time in all, so that
//                  ragged lengths leave no CU idle; every work-group finds its pair and part
//                  from the lengths (Deal). A part is a run of consecutive tiles, which
//                  its four waves take in turn (dealt out cyclically, the parts of 16
//                  contexts of 32k tokens walk their caches in step, 8 MB apart: 200 us
//                  where runs take 157); the T*G <= 16 query rows of the KV head share
//                  every tile. A wave asks for a tile's K as soon as the products of the
//                  one before are done and for its V when that one's values are in: asked
//                  for together, after the values, fp32 rows wait for the matrix
//                  instructions (fp32, 8 paged caches of 4k to 9k tokens, 4 KV heads of 128
//                  for 28, with sums: 252 MB in 69 us, now 60; 4 of 1k to 2.5k with 32 KV
//                  heads: 245 MB in 57, now 51; bf16, 64 windows of 8k, 1083 MB: 161, now
//                  159). The waves' partials meet in LDS. With sums the logits
//                  leave as rows of gp floats (32 bytes per row at 7 heads, beside 512 of
//                  K and V), since a weight is known only when the whole walk is. That
//                  is what sums cost: any stores in a stream of reads slow the reads (16
//                  contexts of 32k tokens 157 us without, 204 with them; the same whether
//                  they are issued tile by tile, four tiles together or behind the next
//                  tile's copies, 187 with a quarter of them, and no less with any cache
//                  policy).
//   finish_kernel  joins the pieces of each query row, and turns the logits into weights:
//                  one thread per row, the query rows in order, so the sums do not
//                  depend on the partition of the walk or on arrival.
// Short walks, and those of many pairs, have one work-group per pair, which does both
// (make_window_plan).
//
// A masked row weighs nothing whatever it holds: its logit is not looked at, and in
// the tiles where some query does not see some row (the ends of the window, of the
// sinks and of the sequence) each query's value product has the rows it does not see
// replaced by zeros, so that a NaN or infinity there stays out of its output.
#include <algorithm>
#include <type_traits>

#include "vp_blocks.h"
#include "vp_cache.h"
#include "vp_tile.h"
#include "vp_walk.h"

namespace vp {
namespace {

template <int DT, int D, bool SUMS>
struct WinLds {
  using C = Cfg<DT, D>;
  // per wave: a K block (after the walk its accumulator rows), a V block, a logit stage
  static constexpr int PITCH = D + 4;  // accumulator rows start on different banks
  static constexpr int K_BYTES = C::SUB_ROWS_BYTES > 16 * PITCH * 4 ? C::SUB_ROWS_BYTES : 16 * PITCH * 4;
  static constexpr int V_BYTES = C::SUB_ROWS_BYTES;
  static constexpr int STAGE_BYTES = SUMS ? C::STAGE_BYTES : 16;
};

// Scores of half a tile. fp32: four sums of a quarter of the products each, added in
// pairs; as one chain of d / 4 matrix instructions the logits, and with them the outputs,
// are up to twice as far from 64 bits as those of a blocked product.
template <int DT, int D>
__device__ __forceinline__ f32x4 score_rows(const unsigned char* kb, int hf, const QFrag<DT, D>& q, int a4, int n16) {
  if constexpr (DT == VP_BF16) {
    return score_half<DT, D>(kb, hf, q, a4, n16);
  } else {
    using C = Cfg<DT, D>;
    f32x4 c[4] = {};
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      const float4 k = *reinterpret_cast<const float4*>(kb + C::at(16 * hf + n16, (D / 16) * a4 + s));
      c[0] = __builtin_amdgcn_mfma_f32_16x16x4f32(k.x, q.v[4 * s + 0], c[0], 0, 0, 0);
      c[1] = __builtin_amdgcn_mfma_f32_16x16x4f32(k.y, q.v[4 * s + 1], c[1], 0, 0, 0);
      c[2] = __builtin_amdgcn_mfma_f32_16x16x4f32(k.z, q.v[4 * s + 2], c[2], 0, 0, 0);
      c[3] = __builtin_amdgcn_mfma_f32_16x16x4f32(k.w, q.v[4 * s + 3], c[3], 0, 0, 0);
    }
    return (c[0] + c[1]) + (c[2] + c[3]);
  }
}

// 32 rows at equal steps into an LDS block: those of the tile's lower half from `lower`,
// the upper half's (TWO; else the same address) from `upper`, both as seen from row 0;
// row_step holds the lane's offsets of the copies after which they repeat
template <typename C, int STEPS, bool TWO>
struct EvenCopy {
  static __device__ __forceinline__ void rows(const char* lower, const char* upper, const uint32_t (&row_step)[STEPS],
                                              int rstride, lds_byte* block) {
    const __amdgpu_buffer_rsrc_t rl =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(lower), 0, 0x7fffffff, kRawBufferWord3);
    const __amdgpu_buffer_rsrc_t ru =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(upper), 0, 0x7fffffff, kRawBufferWord3);
#pragma unroll
    for (int j = 0; j < C::COPIES; ++j)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(TWO && j >= C::COPIES / 2 ? ru : rl, (lds_void*)(block + 1024 * j), 16,
                                               row_step[j % STEPS], j / STEPS * (STEPS * C::RPI) * rstride, 0,
                                               kCopyPolicy);
  }
};

// a tile's logits, 32 rows of gp floats, from the stage to the plane
struct StoreLogits {
  static __device__ __forceinline__ void tile(float* dst, const float* stage, int gp, int lane) {
    typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
    const u32x4* src = reinterpret_cast<const u32x4*>(stage);
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(dst, 0, 128 * gp, kRawBufferWord3);
    // (lanes past 128 * gp bytes store nothing)
    __builtin_amdgcn_raw_buffer_store_b128(src[lane], rs, lane * 16, 0, 0);
    if (gp > 8) __builtin_amdgcn_raw_buffer_store_b128(src[64 + lane], rs, 1024 + lane * 16, 0, 0);
  }
};

// One row of the walk on its way to its weight: row i is row i % 32 of tile i / 32.
// Only the queries that see the row add to it, by its position: a query with a NaN or
// +inf logit has a NaN for 1 / sum, which a weight of 0 would not keep out.
template <int GP>
struct RowWeight {
  float z[GP];  // its products q.K
  float old;    // its sum so far
  float* dst;   // null: no row that a query sees
  int h0, h1;   // query rows that see it
  __device__ __forceinline__ RowWeight(const WindowArgs& a, const WindowWalk& w, size_t pair, int i) : dst(nullptr) {
    const int k = i >> 5;
    const int j = w.t0(k) + (i & 31);
    if (k >= w.n || j < w.row_begin(k) || j >= w.row_end(k)) return;
    // (where the sinks' and the window's tiles meet, rows that no query sees lie between)
    const int own = j - (w.L - a.T);  // the query whose position it is
    const int t0 = max(0, own), t1 = a.window == 0 || j < w.S ? a.T : min(a.T, own + a.window);
    if (t0 >= t1) return;
    h0 = t0 * a.G;
    h1 = t1 * a.G;
    const float* src = a.zs + (pair * a.tiles * 32 + i) * GP;
    if constexpr (GP >= 4) {
#pragma unroll
      for (int c = 0; c < GP / 4; ++c) {
        const float4 v = reinterpret_cast<const float4*>(src)[c];
        z[4 * c] = v.x;
        z[4 * c + 1] = v.y;
        z[4 * c + 2] = v.z;
        z[4 * c + 3] = v.w;
      }
    } else {
#pragma unroll
      for (int c = 0; c < GP; ++c) z[c] = src[c];
    }
    dst = a.attn_sum + pair * a.max_seq_len + j;
    old = j >= w.L - a.T ? 0.f : *dst;
  }
  // adds the weights of the query rows, in order: norm holds their (max, 1 / sum)
  __device__ __forceinline__ void add(const WindowArgs& a, const float2* norm) const {
    if (!dst) return;
    float s = 0.f;
#pragma unroll
    for (int h = 0; h < GP; ++h)
      if (h >= h0 && h < h1) s = fmaf(weight_of(a, z[h], norm[h].x), norm[h].y, s);
    *dst = old + s;
  }
};

// Rows i0 + threadIdx.x, + step, ... of the walk get their weights; the first row's
// logits are requested before `ready` (which ends in a barrier) makes norm.
template <int GP, typename Ready>
__device__ __forceinline__ void add_weights_gp(const WindowArgs& a, const WindowWalk& w, size_t pair, int i0, int step,
                                               const float2* norm, Ready ready) {
  int i = i0 + static_cast<int>(threadIdx.x);
  RowWeight<GP> row(a, w, pair, i);
  ready();
  for (;;) {
    row.add(a, norm);
    i += step;
    if (i >= 32 * w.n) return;
    row = RowWeight<GP>(a, w, pair, i);
  }
}
template <typename Ready>
__device__ __forceinline__ void add_weights(const WindowArgs& a, const WindowWalk& w, size_t pair, int i0, int step,
                                            const float2* norm, Ready ready) {
  switch (a.gp) {
    case 1: add_weights_gp<1>(a, w, pair, i0, step, norm, ready); break;
    case 2: add_weights_gp<2>(a, w, pair, i0, step, norm, ready); break;
    case 4: add_weights_gp<4>(a, w, pair, i0, step, norm, ready); break;
    case 8: add_weights_gp<8>(a, w, pair, i0, step, norm, ready); break;
    default: add_weights_gp<16>(a, w, pair, i0, step, norm, ready); break;
  }
}

template <int DT, int D, bool PAGED, bool SUMS>
__global__ __launch_bounds__(kWinThreads) __attribute__((amdgpu_waves_per_eu(DT == VP_BF16 ? 2 : 1))) void
window_kernel(const WindowArgs a) {
  using C = Cfg<DT, D>;
  using Q = WinLds<DT, D, SUMS>;
  // (three arrays: in one, the compiler would have reads of V wait for the copies into K)
  __shared__ __attribute__((aligned(1024))) unsigned char lds_k[kWinWaves * Q::K_BYTES];
  __shared__ __attribute__((aligned(1024))) unsigned char lds_v[kWinWaves * Q::V_BYTES];
  __shared__ __attribute__((aligned(1024))) unsigned char lds_stage[kWinWaves * Q::STAGE_BYTES];
  __shared__ WinStats ws;
  __shared__ float2 norm[16];
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const int lane = threadIdx.x & 63;
  const int n16 = lane & 15;
  const int a4 = lane >> 4;
  const int TG = a.T * a.G;
  const unsigned char* kb = lds_k + wave * Q::K_BYTES;
  const unsigned char* vb = lds_v + wave * Q::V_BYTES;
  float* stage = reinterpret_cast<float*>(lds_stage + wave * Q::STAGE_BYTES);
  const bool hv = n16 < TG;
  const int tq = hv ? query_of(a, n16) : 0;

  const bool dealt = a.groups > 0;
  int g = blockIdx.y, b = blockIdx.z, part = 0, parts = 1, L;
  if (dealt) {
    const Deal deal(a, lane, blockIdx.x);
    if (deal.b < 0) return;
    b = deal.b;
    g = deal.g;
    part = deal.part;
    parts = deal.parts;
    L = deal.L;
  } else {
    L = clamp_len(a.seq_len[b], a.max_seq_len);
  }
  // the query rows load while the length arrives
  QFrag<DT, D> qf;
  load_q<DT, D>(qf, static_cast<const char*>(a.q) + (hv ? out_row(a, b, g, n16) : 0) * C::ROWB, hv, a4);
  const WindowWalk w(L, a.T, a.window, a.n_sink);
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

  // Copies of a tile whose 32 rows are all read: rows at equal steps from one address
  // (paged caches: from one for each half), so lane offsets that never change. `even`:
  // the offsets fit 32 bits, and no half of a tile crosses a block.
  constexpr int STEPS = C::PIECES / C::RPI < C::COPIES ? max_i(C::PIECES / C::RPI, 1) : C::COPIES;
  const bool even = rstride < (1u << 25) && (!PAGED || bmask >= 15);
  const int rr = lane / C::PIECES, slot = lane % C::PIECES;
  uint32_t row_step[STEPS];
#pragma unroll
  for (int j = 0; j < STEPS; ++j) {
    const int r = j * C::RPI + rr;
    row_step[j] = static_cast<uint32_t>(r) * static_cast<uint32_t>(rstride) + 16 * (slot ^ (r & (C::PIECES - 1)));
  }
  // the position read in place of row r of a tile: rows that no query sees are not
  // read, their places take the nearest row that is read anyway
  auto row_pos = [&](int t0, int r0, int r1, int r) { return min(max(t0 + r, r0), r1 - 1); };
  // this part's tiles, and this wave's first one
  int k = static_cast<int>(static_cast<int64_t>(part) * w.n / parts) + wave;
  const int k1 = static_cast<int>(static_cast<int64_t>(part + 1) * w.n / parts);
  // paged caches: lane r < 32 holds the block of row r, loaded two tiles ahead
  auto blocks_of = [&](int k) -> int {
    int blk = 0;
    if constexpr (PAGED) {
      if (k < k1 && lane < 32) blk = bt[row_pos(w.t0(k), w.row_begin(k), w.row_end(k), lane) >> a.bs_log2];
    }
    return blk;
  };

  float m = kNoLogit, l = 0.f;  // m shared by the four lanes of a query row; l lane-local
  f32x4 acc[C::ACC_N];
#pragma unroll
  for (int i = 0; i < C::ACC_N; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};

  // the copies of tile k of K, of V or of both
  lds_byte* const k_block = (lds_byte*)(lds_k + wave * Q::K_BYTES);
  lds_byte* const v_block = (lds_byte*)(lds_v + wave * Q::V_BYTES);
  int blk = blocks_of(k), blk_next = 0;  // of the tile that is requested, and of the next one
  auto request = [&](int k, auto keys, auto values) {
    const int t0 = w.t0(k);
    const int r0 = w.row_begin(k), r1 = w.row_end(k);  // rows that some query sees, r0 < r1
    if (even && r0 == t0 && r1 == t0 + 32) {
      size_t lo, up;
      if constexpr (PAGED) {
        lo = static_cast<size_t>(__builtin_amdgcn_readlane(blk, 0)) * bstride + static_cast<size_t>(t0 & bmask) * rstride;
        up = static_cast<size_t>(__builtin_amdgcn_readlane(blk, 16)) * bstride +
             static_cast<size_t>((t0 + 16) & bmask) * rstride - 16 * rstride;
      } else {
        lo = up = static_cast<size_t>(t0) * rstride;
      }
      if constexpr (keys.value)
        EvenCopy<C, STEPS, PAGED>::rows(Kb + lo, Kb + up, row_step, static_cast<int>(rstride), k_block);
      if constexpr (values.value)
        EvenCopy<C, STEPS, PAGED>::rows(Vb + lo, Vb + up, row_step, static_cast<int>(rstride), v_block);
    } else {
      // (addresses computed here, not kept in registers through the loop)
      int ln = lane;
      unhoist_vector(ln);
      size_t off[C::COPIES];
#pragma unroll
      for (int j = 0; j < C::COPIES; ++j) {
        const int r = j * C::RPI + ln / C::PIECES;
        const int pos = row_pos(t0, r0, r1, r);
        const int piece = 16 * (ln % C::PIECES ^ (r & (C::PIECES - 1)));
        if constexpr (PAGED)
          off[j] = static_cast<size_t>(__shfl(blk, r)) * bstride + static_cast<size_t>(pos & bmask) * rstride + piece;
        else
          off[j] = static_cast<size_t>(pos) * rstride + piece;
      }
      if constexpr (keys.value) {
#pragma unroll
        for (int j = 0; j < C::COPIES; ++j)
          __builtin_amdgcn_global_load_lds((global_void*)(Kb + off[j]), (lds_void*)(k_block + 1024 * j), 16, 0, kCopyPolicy);
      }
      if constexpr (values.value) {
#pragma unroll
        for (int j = 0; j < C::COPIES; ++j)
          __builtin_amdgcn_global_load_lds((global_void*)(Vb + off[j]), (lds_void*)(v_block + 1024 * j), 16, 0, kCopyPolicy);
      }
    }
  };
  constexpr std::true_type yes;
  constexpr std::false_type no;
  // Memory operations of this wave complete in the order of their issue: K's copies, the
  // block ids, the logits of the tile before, V's copies. A wait names how many issued
  // after what it waits for may be left; block ids are not counted, as not every tile
  // loads them.
  constexpr int LEFT = C::COPIES + (SUMS ? 1 : 0);
  if (k < k1) {
    blk_next = blocks_of(k + kWinWaves);
    request(k, yes, yes);
    __builtin_amdgcn_s_waitcnt(wait_vm(C::COPIES));
  }
  while (k < k1) {
    const int t0 = w.t0(k);
    __builtin_amdgcn_s_waitcnt(wait_vm(LEFT));  // K

    // the products q.K, unscaled
    float z[8];
    {
      const f32x4 c0 = score_rows<DT, D>(kb, 0, qf, a4, n16);
      const f32x4 c1 = score_rows<DT, D>(kb, 1, qf, a4, n16);
#pragma unroll
      for (int i = 0; i < 8; ++i) z[i] = i < 4 ? c0[i & 3] : c1[i & 3];
    }
    const bool more = k + kWinWaves < k1;
    // LDS reads of K have returned before the next tile's copies overwrite it
    __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
    if (more) {
      blk = blk_next;
      request(k + kWinWaves, yes, no);
      blk_next = blocks_of(k + 2 * kWinWaves);
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
      // the tile's products as 32 rows of gp floats, -inf where a query does not see the row
      const int gp = a.gp;
      if (n16 < gp) {
#pragma unroll
        for (int i = 0; i < 8; ++i) stage_store(stage + pv_token(a4, i) * gp + n16, (seen >> i) & 1u ? z[i] : kNegInf);
      }
      StoreLogits::tile(zplane + static_cast<size_t>(k) * 32 * gp, stage, gp, lane);
    }
    float lmax = kNegInf;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if ((seen >> i) & 1u) lmax = fmaxf(lmax, z[i]);
    if (__builtin_amdgcn_ballot_w64(lmax > m + a.raise)) {
      // the four lanes of a query row share the reference (their weights meet in one MFMA)
      const float tm = max_over_quads(lmax);
      const bool up = tm > m + a.raise;
      const float al = up ? weight_of(a, m, tm) : 1.f;
      l *= al;
#pragma unroll
      for (int i = 0; i < C::ACC_N; ++i) acc[i] *= al;
      m = up ? tm : m;
    }
    float p[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      p[i] = (seen >> i) & 1u ? weight_of(a, z[i], m) : 0.f;
      l += p[i];
    }
    if (more) __builtin_amdgcn_s_waitcnt(wait_vm(LEFT));  // V
    else __builtin_amdgcn_s_waitcnt(kWaitVm0);
    if (!edge) {
      value_product<DT, D, C::ACC_N, true>(acc, vb, p, a4, n16);
    } else {
      // one query at a time, with the rows that it sees
      int e4 = a4, e16 = n16;
      unhoist_vector(e4);
      unhoist_vector(e16);
#pragma unroll 1
      for (int t = 0; t < a.T; ++t) {
        const int h = w.L - a.T + t;
        const int lo = a.window > 0 ? h - a.window : -1;
        unsigned rows = 0u;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int j = t0 + pv_token(e4, i);
          if (j <= h && (j > lo || j < w.S)) rows |= 1u << i;
        }
        // (a lane's accumulators are its own query row's: those of other queries are dropped)
        f32x4 sum[C::ACC_N];
#pragma unroll
        for (int i = 0; i < C::ACC_N; ++i) sum[i] = acc[i];
        value_product<DT, D, C::ACC_N, true, true>(sum, vb, p, e4, e16, rows);
#pragma unroll
        for (int i = 0; i < C::ACC_N; ++i) acc[i] = tq == t ? sum[i] : acc[i];
      }
    }
    k += kWinWaves;
    __builtin_amdgcn_s_waitcnt(kWaitLgkm0);  // (V likewise)
    if (more) request(k, no, yes);
  }
  l = sum_over_quads(l);

  // ---- join the four waves ----
  constexpr int PITCH = Q::PITCH;
  __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
  if (a4 == 0) {
    ws.m[wave][n16] = m;
    ws.l[wave][n16] = l;
  }
  store_acc<DT, D, C::ACC_N>(reinterpret_cast<float*>(lds_k + wave * Q::K_BYTES) + n16 * PITCH, acc, a4);
  __syncthreads();
  const size_t pair = static_cast<size_t>(b) * a.Hkv + g;
  const size_t piece0 = static_cast<size_t>(blockIdx.x) * TG;
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
      const float f = weight_of(a, ws.m[v][h], M);
      const float4 x = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(lds_k + v * Q::K_BYTES) + h * PITCH)[c];
      den = fmaf(f, ws.l[v][h], den);
      o.x = fmaf(f, x.x, o.x);
      o.y = fmaf(f, x.y, o.y);
      o.z = fmaf(f, x.z, o.z);
      o.w = fmaf(f, x.w, o.w);
    }
    if (dealt) {
      reinterpret_cast<float4*>(a.acc + (piece0 + h) * D)[c] = o;
      if (c == 0) *reinterpret_cast<float2*>(a.stats + (piece0 + h) * 2) = make_float2(M, den);
    } else {
      const float inv = den == 0.f ? 0.f : 1.0f / den;
      const float4 r = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
      // (nothing seen, or logits of -inf alone: zeros)
      store_out<DT>(a.out, out_row(a, b, g, h), D, c, den == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : r);
      if (SUMS && c == 0) norm[h] = make_float2(M, inv);
    }
  }
  if (dealt) {
    if (part == 0 && threadIdx.x == 0) a.pieces[pair] = make_int2(blockIdx.x, parts);
    return;
  }
  if constexpr (SUMS) {
    // the whole walk is here: its logits, which the waves have stored, become weights
    __builtin_amdgcn_s_waitcnt(kWaitVm0);
    __syncthreads();
    add_weights(a, w, pair, 0, kWinThreads, norm, [] {});
  }
}

// Grid (heads + row groups, Hkv, B): the first T*G work-groups of a KV head join the
// pieces of one query row each; the others (sums) take
// kFinishThreads rows of the walk at a time.
constexpr int kFinishThreads = 256;

// (max, 1 / sum) of query row r over the pieces, by the 16 lanes that share it
__device__ __forceinline__ float2 row_norm(const WindowArgs& a, int2 p, int r, int sub) {
  const int TG = a.T * a.G;
  const float2* st = reinterpret_cast<const float2*>(a.stats) + static_cast<size_t>(p.x) * TG + r;
  float M = kNoLogit;
  for (int i = sub; i < p.y; i += 16) M = fmaxf(M, st[static_cast<size_t>(i) * TG].x);
  M = group_max_f32(M, 16);
  float l = 0.f;
  for (int i = sub; i < p.y; i += 16) {
    const float2 v = st[static_cast<size_t>(i) * TG];
    l = fmaf(weight_of(a, v.x, M), v.y, l);
  }
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) l += __shfl_xor(l, o, 16);
  return make_float2(M, l == 0.f ? 0.f : 1.0f / l);
}

template <int DT, int D>
__global__ __launch_bounds__(kFinishThreads) void finish_kernel(const WindowArgs a, int heads) {
  constexpr int COLS = D / 4;
  constexpr int R = kFinishThreads / COLS;
  read_early(a.out, a.seq_len, a.stats, heads);
  const int g = blockIdx.y, b = blockIdx.z;
  const int tid = threadIdx.x;
  const size_t pair = static_cast<size_t>(b) * a.Hkv + g;
  const int TG = a.T * a.G;
  __shared__ float2 norm[16];
  __shared__ float4 part_sum[R][COLS];
  const int2 pieces = a.pieces[pair];
  const WindowWalk w = walk_of(a, b);
  const int i0 = (static_cast<int>(blockIdx.x) - heads) * kFinishThreads;
  if (i0 >= 32 * w.n) return;  // (no rows of the walk left for this work-group)
  const int2 p = w.n > 0 ? pieces : make_int2(0, 0);  // first piece, number of pieces
  if (i0 < 0) {
    const int h = blockIdx.x;
    const int col = tid % COLS, r = tid / COLS;
    // the first pieces' partials are requested together with all pieces' statistics
    constexpr int HELD = 4;
    float4 x[HELD];
    float mx[HELD];
#pragma unroll
    for (int j = 0; j < HELD; ++j) {
      const int i = r + j * R;
      const size_t row = static_cast<size_t>(p.x + (i < p.y ? i : 0)) * TG + h;  // past the end: not used
      x[j] = reinterpret_cast<const float4*>(a.acc + row * D)[col];
      mx[j] = a.stats[row * 2];
    }
    if (tid < 16) {
      const float2 mn = row_norm(a, p, h, tid);
      if (tid == 0) norm[0] = mn;
    }
    __syncthreads();
    const float2 mn = norm[0];
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](float m, const float4& v) {
      const float f = weight_of(a, m, mn.x);
      o.x = fmaf(f, v.x, o.x);
      o.y = fmaf(f, v.y, o.y);
      o.z = fmaf(f, v.z, o.z);
      o.w = fmaf(f, v.w, o.w);
    };
#pragma unroll
    for (int j = 0; j < HELD; ++j)
      if (r + j * R < p.y) add(mx[j], x[j]);
    for (int i = r + HELD * R; i < p.y; i += R) {
      const size_t row = static_cast<size_t>(p.x + i) * TG + h;
      add(a.stats[row * 2], reinterpret_cast<const float4*>(a.acc + row * D)[col]);
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
  const int step = (static_cast<int>(gridDim.x) - heads) * kFinishThreads;
  add_weights(a, w, pair, i0, step, norm, [&] {
    if (tid < 16 * TG) {
      const float2 mn = row_norm(a, p, tid >> 4, tid & 15);
      if ((tid & 15) == 0) norm[tid >> 4] = mn;
    }
    __syncthreads();
  });
}

template <int DT, int D>
hipError_t launch_dd(const WindowArgs& a, hipStream_t st) {
  const dim3 grid = a.groups > 0 ? dim3(a.groups) : dim3(1, a.Hkv, a.B);
  const bool paged = a.bs_log2 >= 0, sums = a.attn_sum != nullptr;
  if (paged && sums) hipLaunchKernelGGL((window_kernel<DT, D, true, true>), grid, dim3(kWinThreads), 0, st, a);
  else if (paged) hipLaunchKernelGGL((window_kernel<DT, D, true, false>), grid, dim3(kWinThreads), 0, st, a);
  else if (sums) hipLaunchKernelGGL((window_kernel<DT, D, false, true>), grid, dim3(kWinThreads), 0, st, a);
  else hipLaunchKernelGGL((window_kernel<DT, D, false, false>), grid, dim3(kWinThreads), 0, st, a);
  if (hipError_t e = hipGetLastError()) return e;
  if (a.groups == 0) return hipSuccess;
  // (a capacity far above the lengths costs no more work-groups than a full GPU needs)
  const int64_t pairs = static_cast<int64_t>(a.B) * a.Hkv;
  const int64_t most = std::max<int64_t>(1, 8192 / pairs);
  const int rows = sums ? static_cast<int>(std::min<int64_t>(most, (a.tiles * 32ll + kFinishThreads - 1) / kFinishThreads)) : 0;
  const int heads = a.T * a.G;
  hipLaunchKernelGGL((finish_kernel<DT, D>), dim3(heads + rows, a.Hkv, a.B), dim3(kFinishThreads), 0, st, a, heads);
  return hipGetLastError();
}

template <int DT, int D>
hipError_t join_dd(const WindowArgs& a, hipStream_t st) {
  const int heads = a.T * a.G;
  hipLaunchKernelGGL((finish_kernel<DT, D>), dim3(heads, a.Hkv, a.B), dim3(kFinishThreads), 0, st, a, heads);
  return hipGetLastError();
}

}  // namespace

int window_tiles(const vp_shape& s, const vp_window& w) {
  const int64_t T = queries(s), cap = (static_cast<int64_t>(s.max_seq_len) + 31) / 32;
  if (w.window == 0) return static_cast<int>(cap);
  // the window's rows may begin anywhere in a tile
  return static_cast<int>(std::min(cap, (static_cast<int64_t>(w.n_sink) + 31) / 32 + (w.window + T - 1 + 30) / 32 + 1));
}

WindowPlan make_window_plan(const vp_shape& s, const vp_window& w, bool sums) {
  WindowPlan p{};
  const int64_t cap = (static_cast<int64_t>(s.max_seq_len) + 31) / 32;
  const int64_t tiles = p.tiles = window_tiles(s, w);
  const int64_t pairs = static_cast<int64_t>(s.batch) * s.n_kv_heads;
  // One work-group per pair, and no second launch, where
  // * the walks are short: up to 16 tiles, 12 with sums (bf16; 8 KV heads of 128, 16 tiles:
  //   9.2 us and, dealt, 10.0; with sums 11.2 and 10.7, 32 pairs 12.9 and 10.9; 32 tiles
  //   13.8 and 10.2), 8 in fp32 (32 pairs of 128: 13.5 and 14.1, 16 tiles 19.7 and 14.5);
  // * the longest walk is short beside what dealing costs. A full sequence alone among short
  //   ones holds the call for 0.3 us a tile; dealing takes pairs (350 + sequences) / 40000 us,
  //   as every work-group reads all lengths before its rows. Dealt from five times that on.
  //   bf16 of 128, no window, all full / 100 to 1500 rows / one full among those, whole and dealt:
  //   192 pairs of 48 sequences, 32 tiles 18.2 and 23.7 / 16.3, 17.8 / 14.0, 14.4, 64 tiles
  //   33, 40 / 27, 25 / 24, 18; 1024 of 128, 128 tiles 311, 336 / 72, 88 / 93, 109, 256 tiles 616,
  //   644 / 72, 88 / 123, 111, 1024 tiles - / 71, 87 / 338, 129 (with sums 105, 120 / 599, 174);
  //   2048 of 512, 1024 tiles - / 146, 186 / 541, 200; 4096 of 1024 - / 281, 423 / 600, 431; 4096
  //   of 4096 - / 267, 726 / 583, 732;
  // * a window cuts the walks of the capacity to half or less, so that long sequences' are
  //   much the same, and the pairs nearly fill the CUs: 192 pairs (16 tiles: 11.3 and 16.3,
  //   256 tiles: 115 and 130; 128 pairs, 64 tiles: 27.5 and 27.1), 384 with rows of 128 bytes
  //   (64 tiles: 35.1 and 37.7; 256 pairs: 29.3 and 27.5), 512 with their sums (64 tiles: 50.8
  //   and 64.2; 384 pairs 47.2 and 45.1, 256 tiles 181 and 158). Where nearly all sequences
  //   are shorter than such a window this loses: window 8192, 256 pairs, one context of 32k
  //   among some of 1k 82 us and, dealt, 34; of 1k to 32k 144 and 151. A window that the
  //   capacity hardly exceeds, or does not, cuts nothing (24 contexts of 1k to 32k, 8 KV heads,
  //   window 32768: 328 us and, dealt, 233).
  const bool bf16 = s.dtype == VP_BF16;
  const int64_t few = bf16 ? (sums ? 12 : 16) : 8;
  const int64_t many = !bf16 || s.head_dim != 64 ? 192 : sums ? 512 : 384;
  const bool cut = w.window > 0 && 2 * tiles <= cap;
  const bool brief = 2400 * tiles <= pairs * (350 + s.batch);
  const bool one_each = tiles <= few || brief || (cut && pairs >= many) || pairs * tiles > 0x3fffffff;
  // Otherwise one resident round of work-groups, a tile per wave at least; twice as many
  // as pairs where those are more (24 ragged sequences of 16 heads of 64: 51.5 us, four
  // times as many 53.1)
  const int64_t most = std::max<int64_t>(resident_groups(s.dtype, s.head_dim), 2 * pairs);
  p.groups = one_each ? 0 : static_cast<int>(std::min(most, pairs * ((tiles + kWinWaves - 1) / kWinWaves)));
  carve_window_plan(p, s, sums);
  return p;
}

void carve_window_plan(WindowPlan& p, const vp_shape& s, bool sums) {
  const int64_t pairs = static_cast<int64_t>(s.batch) * s.n_kv_heads;
  const int rows = queries(s) * (s.n_q_heads / s.n_kv_heads);
  p.gp = 1;
  while (p.gp < rows) p.gp *= 2;
  const size_t pieces = p.groups;
  size_t off = 0;
  p.stats = off;
  off = align256(off + pieces * rows * 2 * 4);
  p.acc = off;
  off = align256(off + pieces * rows * s.head_dim * 4);
  p.pieces = off;
  if (p.groups > 0) off = align256(off + static_cast<size_t>(pairs) * 2 * 4);
  p.zs = off;
  if (sums) off = align256(off + static_cast<size_t>(pairs) * p.tiles * 32 * p.gp * 4);
  p.total = off;
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

hipError_t launch_window_join(const WindowArgs& a, int dtype, int head_dim, hipStream_t st) {
  if (dtype == VP_BF16) return head_dim == 128 ? join_dd<VP_BF16, 128>(a, st) : join_dd<VP_BF16, 64>(a, st);
  return head_dim == 128 ? join_dd<VP_F32, 128>(a, st) : join_dd<VP_F32, 64>(a, st);
}

}  // namespace vp
