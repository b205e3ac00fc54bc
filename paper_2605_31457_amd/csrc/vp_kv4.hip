// Rows of 4-bit caches back in 16 or 32 bits (vp_kv4_read), and attention of a step's queries
// over a 4-bit cache (vp_kv4_decode_attn).
//
//   z_j = <q_h, K_j>,  A_j = 2^(c (z_j - M)) / l over the rows j that query t sees, c = sm_scale log2(e),
//   out = sum_j A_j V_j,     K and V elements: code * 2^e, one e per 32 of them
//
// Bound: the codes and scales of the rows that any query sees, d + d/16 bytes per row and KV
// head, read once from HBM. A quarter of the bytes of 16-bit rows with the same products to
// form, so the vector units come next: an element's code becomes a bf16 number (exact: three
// significant bits at most, and a power of two), two an instruction, and is then an operand
// of the same matrix instructions as a 16-bit cache's rows. Scores: bf16 queries times keys,
// exact products; fp32 queries enter as three bf16 numbers, all 24 bits of them. Values: the
// weights as three bf16 numbers (as in value_product).
//
// The walk, its masks, its running maximum and its parts are those of window_kernel. The
// rows go to registers, not through LDS: a lane's 16 bytes of a key are one block of 32
// elements with one scale, which is what its slots of the products take, and the 4 bytes that
// it takes of a value row are 8 elements, for the 8 products that it takes part in.
#include <algorithm>
#include <type_traits>

#include "vp_kv4.h"
#include "vp_tile.h"
#include "vp_walk.h"

namespace vp {
namespace {

typedef __bf16 bf16x2 __attribute__((__vector_size__(2 * sizeof(__bf16))));

// the scale byte as a float (the mark of a block that is all NaN: NaN)
__device__ __forceinline__ float scale_of(uint32_t byte) {
  return __uint_as_float(byte == kScaleNan ? 0x7fc00000u : byte << 23);
}

// elements 2 B and 2 B + 1 of 8 codes, times the scale, as two bf16
template <int B>
__device__ __forceinline__ uint32_t two_of(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, B));
}

// ---------------------------------------------------------------------------
// vp_kv4_read
// ---------------------------------------------------------------------------
constexpr int kReadThreads = 256;

// Grid (chunks, Hkv, 2 B: K and V): a work-group takes 64 rows of 128 (128 of 64) at a time. A
// lane has 8 elements: stores of a wave are whole rows.
template <int DT, int D>
__global__ __launch_bounds__(kReadThreads) void read_kernel(const ReadArgs a) {
  constexpr int ESZ = DT == VP_BF16 ? 2 : 4;
  constexpr int LANES = D / 8;
  constexpr int ROWS = kReadThreads / LANES;
  constexpr int BATCH = 4;
  const int g = blockIdx.y, b = blockIdx.z >> 1;
  const bool value = blockIdx.z & 1;
  const int octet = threadIdx.x % LANES;
  const int L = clamp_len(a.seq_len[b], a.max_seq_len);
  const int first = a.first ? max(a.first[b], 0) : 0;
  const uint8_t* codes = (value ? a.four.vc : a.four.kc) + g * a.four.ch + octet * 4;
  const uint8_t* scales = (value ? a.four.vs : a.four.ks) + g * a.four.sh + (octet >> 2);
  char* out = static_cast<char*>(value ? a.V : a.K) + g * a.sh + octet * (8 * ESZ);
  const int mask = a.block_table ? (1 << a.bs_log2) - 1 : -1;
  for (int64_t r0 = first + static_cast<int64_t>(blockIdx.x) * (BATCH * ROWS); r0 < L;
       r0 += static_cast<int64_t>(gridDim.x) * (BATCH * ROWS)) {
    int64_t at[BATCH];
    int in[BATCH];
    uint32_t c[BATCH], s[BATCH];
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
      const int row = static_cast<int>(min(r0 + j * ROWS + static_cast<int>(threadIdx.x) / LANES, static_cast<int64_t>(L - 1)));
      at[j] = a.block_table ? a.block_table[static_cast<int64_t>(b) * a.nblk + (row >> a.bs_log2)] : b;
      in[j] = row & mask;
    }
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
      c[j] = *reinterpret_cast<const uint32_t*>(codes + at[j] * a.four.cb + static_cast<int64_t>(in[j]) * (D / 2));
      s[j] = scales[at[j] * a.four.sb + static_cast<int64_t>(in[j]) * (D / 32)];
    }
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
      if (r0 + j * ROWS + static_cast<int>(threadIdx.x) / LANES >= L) continue;
      const float scale = scale_of(s[j]);
      uint32_t w[4] = {two_of<0>(c[j], scale), two_of<1>(c[j], scale), two_of<2>(c[j], scale), two_of<3>(c[j], scale)};
      if (s[j] == kScaleNan) w[0] = w[1] = w[2] = w[3] = 0x7fc07fc0u;
      char* dst = out + at[j] * a.sb + in[j] * a.ss;
      if constexpr (DT == VP_BF16) {
        *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
      } else {
#pragma unroll
        for (int i = 0; i < 2; ++i)
          reinterpret_cast<float4*>(dst)[i] =
              make_float4(__uint_as_float(w[2 * i] << 16), __uint_as_float(w[2 * i] & 0xffff0000u),
                          __uint_as_float(w[2 * i + 1] << 16), __uint_as_float(w[2 * i + 1] & 0xffff0000u));
      }
    }
  }
}

template <int DT, int D>
hipError_t read_dd(const ReadArgs& a, hipStream_t st) {
  // (a capacity far above the lengths costs no more work-groups than a full GPU needs)
  const int64_t per = 4 * (kReadThreads / (D / 8));
  const int64_t pairs = static_cast<int64_t>(a.B) * a.Hkv * 2;
  const int64_t chunks = std::min((a.max_seq_len + per - 1) / per, std::max<int64_t>(1, 8192 / pairs));
  for (int b0 = 0; b0 < a.B; b0 += 32767) {  // (the grid's third dimension ends at 65535)
    ReadArgs x = a;
    x.B = std::min(32767, a.B - b0);
    x.seq_len += b0;
    if (x.first) x.first += b0;
    if (x.block_table) {
      x.block_table += static_cast<int64_t>(b0) * x.nblk;
    } else {
      x.four.kc += b0 * x.four.cb;
      x.four.vc += b0 * x.four.cb;
      x.four.ks += b0 * x.four.sb;
      x.four.vs += b0 * x.four.sb;
      x.K = static_cast<char*>(x.K) + b0 * x.sb;
      x.V = static_cast<char*>(x.V) + b0 * x.sb;
    }
    hipLaunchKernelGGL((read_kernel<DT, D>), dim3(static_cast<unsigned>(chunks), x.Hkv, 2 * x.B), dim3(kReadThreads), 0, st, x);
    if (hipError_t e = hipGetLastError()) return e;
  }
  return hipSuccess;
}

// ---------------------------------------------------------------------------
// vp_kv4_decode_attn
// ---------------------------------------------------------------------------

// query rows as bf16 operands: slot (a4, i) of step s <-> dim (D/4) a4 + 8 s + i
template <int DT, int D>
struct Queries {
  static constexpr int N = DT == VP_BF16 ? 1 : 3;
  bf16x8 v[N][D / 32];
  __device__ __forceinline__ void load(const char* row, bool valid, int a4) {
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
      if constexpr (DT == VP_BF16) {
        const uint4 u = valid ? reinterpret_cast<const uint4*>(row)[(D / 32) * a4 + s] : make_uint4(0, 0, 0, 0);
        v[0][s] = __builtin_bit_cast(bf16x8, u);
      } else {
        float x[8];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float4 u = valid ? reinterpret_cast<const float4*>(row)[2 * ((D / 32) * a4 + s) + i] : make_float4(0.f, 0.f, 0.f, 0.f);
          x[4 * i] = u.x;
          x[4 * i + 1] = u.y;
          x[4 * i + 2] = u.z;
          x[4 * i + 3] = u.w;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          // (an infinity leaves no rest)
          const uint32_t hi = __float_as_uint(x[i]) & 0xffff0000u;
          const float r = fabsf(x[i]) < __builtin_inff() ? x[i] - __uint_as_float(hi) : 0.f;
          const uint32_t mid = __float_as_uint(r) & 0xffff0000u;
          v[0][s][i] = x[i] == x[i] ? __builtin_bit_cast(__bf16, static_cast<uint16_t>(hi >> 16)) : static_cast<__bf16>(x[i]);
          v[1][s][i] = __builtin_bit_cast(__bf16, static_cast<uint16_t>(mid >> 16));
          v[2][s][i] = static_cast<__bf16>(r - __uint_as_float(mid));
        }
      }
    }
  }
};

// what a lane holds of a tile of 32 rows
template <int D>
struct Tile {
  static constexpr int KW = D / 32;          // dwords of a key row's piece, its dims (D/4) a4 ..
  uint32_t k[2][KW];                         // rows 16 half + n16
  uint32_t ks[2];                            // their scale bytes
  uint32_t v[8];                             // rows pv_token(a4, i): elements (D/16) n16 ..
  uint32_t vs[8];                            // their scale bytes
};

template <int D, int N>
__device__ __forceinline__ void scores(f32x4 (&c)[2], const Tile<D>& t, const bf16x8 (&q)[N][D / 32]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float scale = scale_of(t.ks[h]);
    c[h] = f32x4{0.f, 0.f, 0.f, 0.f};
    bf16x8 k[D / 32];
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
      const uint32_t u = t.k[h][s];
      k[s] = __builtin_bit_cast(bf16x8, make_uint4(two_of<0>(u, scale), two_of<1>(u, scale), two_of<2>(u, scale), two_of<3>(u, scale)));
    }
#pragma unroll
    for (int p = N - 1; p >= 0; --p)
#pragma unroll
      for (int s = 0; s < D / 32; ++s) c[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[s], q[p][s], c[h], 0, 0, 0);
  }
}

// acc[e][r] (dim (D/16) (4 a4 + r) + e of head n16) += V^T P^T over the tile's 32 rows. The
// weights enter as the sum of three bf16 numbers, all 24 bits of them.
template <int D>
__device__ __forceinline__ void values(f32x4 (&acc)[D / 16], const Tile<D>& t, const float (&p)[8]) {
  uint32_t pf[4], pm[4], pl[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    uint32_t a[2], b[2], c[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      a[i] = __float_as_uint(p[2 * j + i]);
      const float r = p[2 * j + i] - __uint_as_float(a[i] & 0xffff0000u);
      b[i] = __float_as_uint(r);
      c[i] = __float_as_uint(r - __uint_as_float(b[i] & 0xffff0000u));
    }
    // the leading halves of two floats as a pair
    pf[j] = __builtin_amdgcn_perm(a[1], a[0], 0x07060302u);
    pm[j] = __builtin_amdgcn_perm(b[1], b[0], 0x07060302u);
    pl[j] = __builtin_amdgcn_perm(c[1], c[0], 0x07060302u);  // (at most 8 bits: exact)
  }
  const bf16x8 w0 = __builtin_bit_cast(bf16x8, make_uint4(pf[0], pf[1], pf[2], pf[3]));
  const bf16x8 w1 = __builtin_bit_cast(bf16x8, make_uint4(pm[0], pm[1], pm[2], pm[3]));
  const bf16x8 w2 = __builtin_bit_cast(bf16x8, make_uint4(pl[0], pl[1], pl[2], pl[3]));
  float scale[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) scale[i] = scale_of(t.vs[i]);
  auto two_dims = [&](auto byte) {
    constexpr int B = decltype(byte)::value;
    uint32_t lo[4], hi[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t x = two_of<B>(t.v[2 * j], scale[2 * j]), y = two_of<B>(t.v[2 * j + 1], scale[2 * j + 1]);
      lo[j] = __builtin_amdgcn_perm(y, x, 0x05040100u);
      hi[j] = __builtin_amdgcn_perm(y, x, 0x07060302u);
    }
    const bf16x8 a0 = __builtin_bit_cast(bf16x8, make_uint4(lo[0], lo[1], lo[2], lo[3]));
    const bf16x8 a1 = __builtin_bit_cast(bf16x8, make_uint4(hi[0], hi[1], hi[2], hi[3]));
    acc[2 * B] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a0, w0, acc[2 * B], 0, 0, 0);
    acc[2 * B + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a1, w0, acc[2 * B + 1], 0, 0, 0);
    acc[2 * B] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a0, w1, acc[2 * B], 0, 0, 0);
    acc[2 * B + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a1, w1, acc[2 * B + 1], 0, 0, 0);
    acc[2 * B] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a0, w2, acc[2 * B], 0, 0, 0);
    acc[2 * B + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a1, w2, acc[2 * B + 1], 0, 0, 0);
  };
  two_dims(std::integral_constant<int, 0>());
  two_dims(std::integral_constant<int, 1>());
  if constexpr (D == 128) {
    two_dims(std::integral_constant<int, 2>());
    two_dims(std::integral_constant<int, 3>());
  }
}

template <int DT, int D, bool PAGED>
__global__ __launch_bounds__(kWinThreads) void kv4_kernel(const WindowArgs a, const Kv4Cache four) {
  constexpr int PITCH = D + 4;  // accumulator rows start on different banks
  constexpr int ROWB = D / 2, SROW = D / 32;
  __shared__ __attribute__((aligned(16))) float lds_acc[kWinWaves][16 * PITCH];
  __shared__ WinStats ws;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const int lane = threadIdx.x & 63;
  const int n16 = lane & 15;
  const int a4 = lane >> 4;
  const int TG = a.T * a.G;
  const bool hv = n16 < TG;
  const int tq = hv ? n16 / a.G : 0;

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
  Queries<DT, D> q;
  q.load(static_cast<const char*>(a.q) + (hv ? out_row(a, b, g, n16) : 0) * (D * (DT == VP_BF16 ? 2 : 4)), hv, a4);
  const WindowWalk w(L, a.T, a.window, a.n_sink);
  const int hi = w.L - a.T + tq;                        // this lane's query sees j <= hi
  const int below = a.window > 0 ? hi - a.window : -1;  // and j > below or j < n_sink

  const int64_t seq_c = (PAGED ? 0 : b * four.cb) + g * four.ch, seq_s = (PAGED ? 0 : b * four.sb) + g * four.sh;
  const uint8_t* const Kc = four.kc + seq_c;
  const uint8_t* const Vc = four.vc + seq_c;
  const uint8_t* const Ks = four.ks + seq_s;
  const uint8_t* const Vs = four.vs + seq_s;
  const int32_t* bt = PAGED ? a.block_table + static_cast<int64_t>(b) * a.nblk : nullptr;
  const int bmask = PAGED ? (1 << a.bs_log2) - 1 : 0;

  // this part's tiles, and this wave's first one
  int k = static_cast<int>(static_cast<int64_t>(part) * w.n / parts) + wave;
  const int k1 = static_cast<int>(static_cast<int64_t>(part + 1) * w.n / parts);
  // the position read in place of row r of a tile: rows that no query sees are not
  // read, their places take the nearest row that is read anyway
  auto row_pos = [&](int t0, int r0, int r1, int r) { return min(max(t0 + r, r0), r1 - 1); };
  // paged caches: lane r < 32 holds the block of row r
  auto blocks_of = [&](int k) -> int {
    int blk = 0;
    if constexpr (PAGED) {
      if (k < k1 && lane < 32) blk = bt[row_pos(w.t0(k), w.row_begin(k), w.row_end(k), lane) >> a.bs_log2];
    }
    return blk;
  };
  auto load = [&](Tile<D>& t, int k, int blk) {
    const int t0 = w.t0(k);
    const int r0 = w.row_begin(k), r1 = w.row_end(k);  // rows that some query sees, r0 < r1
    auto key = [&](int h, const uint8_t* c, const uint8_t* s) {
      if constexpr (D == 128) {
        const uint4 u = *reinterpret_cast<const uint4*>(c + 16 * a4);
        t.k[h][0] = u.x;
        t.k[h][1] = u.y;
        t.k[h][2] = u.z;
        t.k[h][3] = u.w;
        t.ks[h] = s[a4];
      } else {
        const uint2 u = *reinterpret_cast<const uint2*>(c + 8 * a4);
        t.k[h][0] = u.x;
        t.k[h][1] = u.y;
        t.ks[h] = s[a4 >> 1];
      }
    };
    auto value = [&](int i, const uint8_t* c, const uint8_t* s) {
      if constexpr (D == 128) {
        t.v[i] = reinterpret_cast<const uint32_t*>(c)[n16];
        t.vs[i] = s[n16 >> 2];
      } else {
        t.v[i] = reinterpret_cast<const uint16_t*>(c)[n16];
        t.vs[i] = s[n16 >> 3];
      }
    };
    // row r of the tile: (offset of its codes, of its scales)
    const bool whole = r0 == t0 && r1 == t0 + 32;
    if (whole) {
      // rows of a half follow each other (blocks hold at least 16)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        int64_t c, s;
        if constexpr (PAGED) {
          const int64_t at = __builtin_amdgcn_readlane(blk, 16 * h);
          const int in = (t0 + 16 * h) & bmask;
          c = at * four.cb + static_cast<int64_t>(in) * ROWB;
          s = at * four.sb + static_cast<int64_t>(in) * SROW;
        } else {
          c = static_cast<int64_t>(t0 + 16 * h) * ROWB;
          s = static_cast<int64_t>(t0 + 16 * h) * SROW;
        }
        key(h, Kc + c + n16 * ROWB, Ks + s + n16 * SROW);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          value(4 * h + i, Vc + c + (4 * a4 + i) * ROWB, Vs + s + (4 * a4 + i) * SROW);
      }
    } else {
      auto at = [&](int r, int64_t& c, int64_t& s) {
        const int pos = row_pos(t0, r0, r1, r);
        int64_t base = 0;
        int in = pos;
        if constexpr (PAGED) {
          base = __shfl(blk, r);
          in = pos & bmask;
        }
        c = base * four.cb + static_cast<int64_t>(in) * ROWB;
        s = base * four.sb + static_cast<int64_t>(in) * SROW;
      };
      int64_t c, s;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        at(16 * h + n16, c, s);
        key(h, Kc + c, Ks + s);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        at(pv_token(a4, i), c, s);
        value(i, Vc + c, Vs + s);
      }
    }
  };

  float m = kNoLogit, l = 0.f;  // m shared by the four lanes of a query row; l lane-local
  f32x4 acc[D / 16];
#pragma unroll
  for (int i = 0; i < D / 16; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};

  Tile<D> tile, next;
  int blk = blocks_of(k);
  if (k < k1) load(tile, k, blk);
  blk = blocks_of(k + kWinWaves);
  while (k < k1) {
    const int t0 = w.t0(k);
    const bool more = k + kWinWaves < k1;
    if (more) load(next, k + kWinWaves, blk);
    blk = blocks_of(k + 2 * kWinWaves);

    // the products q.K, unscaled; value i of this lane is row t0 + pv_token(a4, i)
    float z[8];
    {
      f32x4 c[2];
      scores<D>(c, tile, q.v);
#pragma unroll
      for (int i = 0; i < 8; ++i) z[i] = c[i >> 2][i & 3];
    }
    // Does every query see every row?
    const int last0 = w.L - a.T;                                // the first query's own position
    const int hidden = a.window > 0 ? w.L - 1 - a.window : -1;  // the last query sees no row from n_sink to here
    const bool edge = t0 + 31 > last0 || max(t0, w.S) <= min(t0 + 31, hidden);
    unsigned seen = 0xffu;
    if (edge) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int j = t0 + pv_token(a4, i);
        if (j > hi || (j <= below && j >= w.S)) seen &= ~(1u << i);
      }
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
      for (int i = 0; i < D / 16; ++i) acc[i] *= al;
      m = up ? tm : m;
    }
    float p[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      p[i] = (seen >> i) & 1u ? weight_of(a, z[i], m) : 0.f;
      l += p[i];
    }
    if (!edge) {
      values<D>(acc, tile, p);
    } else {
      // one query at a time, with the rows that it sees: the others count as zeros
      // whatever they hold
#pragma unroll 1
      for (int t = 0; t < a.T; ++t) {
        const int h = w.L - a.T + t;
        const int lo = a.window > 0 ? h - a.window : -1;
        Tile<D> own = tile;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int j = t0 + pv_token(a4, i);
          if (!(j <= h && (j > lo || j < w.S))) {
            own.v[i] = 0u;
            own.vs[i] = kScaleMin;
          }
        }
        // (a lane's accumulators are its own query row's: those of other queries are dropped)
        f32x4 sum[D / 16];
#pragma unroll
        for (int i = 0; i < D / 16; ++i) sum[i] = acc[i];
        values<D>(sum, own, p);
#pragma unroll
        for (int i = 0; i < D / 16; ++i) acc[i] = tq == t ? sum[i] : acc[i];
      }
    }
    k += kWinWaves;
    if (more) tile = next;
  }
  l = sum_over_quads(l);

  // ---- join the four waves ----
  if (a4 == 0) {
    ws.m[wave][n16] = m;
    ws.l[wave][n16] = l;
  }
  // acc[e][r] holds dim (D/16) (4 a4 + r) + e
  float* mine = lds_acc[wave] + n16 * PITCH;
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int e = 0; e < D / 16; e += 4)
      *reinterpret_cast<float4*>(mine + (D / 16) * (4 * a4 + r) + e) = make_float4(acc[e][r], acc[e + 1][r], acc[e + 2][r], acc[e + 3][r]);
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
      const float4 x = reinterpret_cast<const float4*>(lds_acc[v] + h * PITCH)[c];
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
      // (nothing seen, or logits of -inf alone: zeros)
      const float inv = den == 0.f ? 0.f : 1.0f / den;
      const float4 r = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
      store_out<DT>(a.out, out_row(a, b, g, h), D, c, den == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : r);
    }
  }
  if (dealt && part == 0 && threadIdx.x == 0) a.pieces[pair] = make_int2(blockIdx.x, parts);
}

template <int DT, int D>
hipError_t attention_dd(const WindowArgs& a, const Kv4Cache& four, hipStream_t st) {
  const dim3 grid = a.groups > 0 ? dim3(a.groups) : dim3(1, a.Hkv, a.B);
  if (a.bs_log2 >= 0) hipLaunchKernelGGL((kv4_kernel<DT, D, true>), grid, dim3(kWinThreads), 0, st, a, four);
  else hipLaunchKernelGGL((kv4_kernel<DT, D, false>), grid, dim3(kWinThreads), 0, st, a, four);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv4_read(const ReadArgs& a, int dtype, int head_dim, hipStream_t st) {
  if (dtype == VP_BF16) return head_dim == 128 ? read_dd<VP_BF16, 128>(a, st) : read_dd<VP_BF16, 64>(a, st);
  return head_dim == 128 ? read_dd<VP_F32, 128>(a, st) : read_dd<VP_F32, 64>(a, st);
}

WindowPlan make_kv4_plan(const vp_shape& s, const vp_window& w) {
  WindowPlan p{};
  const int64_t cap = (static_cast<int64_t>(s.max_seq_len) + 31) / 32;
  const int64_t tiles = p.tiles = window_tiles(s, w);
  const int64_t pairs = static_cast<int64_t>(s.batch) * s.n_kv_heads;
  const bool cut = w.window > 0 && 2 * tiles <= cap;
  const bool brief = 2400 * tiles <= pairs * (350 + s.batch);
  const bool one_each = tiles <= 16 || brief || (cut && pairs >= 512) || pairs * tiles > 0x3fffffff;
  const int64_t most = std::max<int64_t>(1024, 2 * pairs);
  p.groups = one_each ? 0 : static_cast<int>(std::min(most, pairs * ((tiles + kWinWaves - 1) / kWinWaves)));
  carve_window_plan(p, s, false);
  return p;
}

hipError_t launch_kv4_attention(const WindowArgs& a, const Kv4Cache& four, int dtype, int head_dim, hipStream_t st) {
  hipError_t e;
  if (dtype == VP_BF16) e = head_dim == 128 ? attention_dd<VP_BF16, 128>(a, four, st) : attention_dd<VP_BF16, 64>(a, four, st);
  else e = head_dim == 128 ? attention_dd<VP_F32, 128>(a, four, st) : attention_dd<VP_F32, 64>(a, four, st);
  if (e != hipSuccess || a.groups == 0) return e;
  return launch_window_join(a, dtype, head_dim, st);
}

}  // namespace vp
