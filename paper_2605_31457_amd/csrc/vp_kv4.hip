// Rows of 4-bit caches back in 16 or 32 bits (vp_kv4_read), and attention of a step's queries
// over a 4-bit cache (vp_kv4_decode_attn).
//
//   z_j = <q_h, K_j>,  A_j = 2^(c (z_j - M)) / l over the rows j that query t sees, c = sm_scale log2(e),
//   out = sum_j A_j V_j,     K and V elements: code * 2^e, one e per 32 of them
//
// Bound: the codes and scales of the rows that any query sees, d + d/16 bytes per row and KV
// head, read once from HBM (64 contexts of 32k tokens, 28/4 heads of 128: 1142 MB in 190 us, 6.0
// TB/s; the copies alone take 173). A quarter of the bytes of 16-bit rows with the same products
// to form, so the vector and matrix units, which do not overlap here, come next (157 us of that
// call with its tiles in the L2): an element's code becomes a bf16 number (exact: two
// significant bits, and a power of two), two an instruction, and is then an operand of the same
// matrix instructions as a 16-bit cache's rows. Scores: bf16 queries times keys, exact products;
// fp32 queries enter as three bf16 numbers, all 24 bits of them. Values: the weights as
// three bf16 numbers (as in value_product; two take 186 us).
//
// The walk, its masks, its running maximum and its parts are those of window_kernel. A
// wave has places for three tiles of 32 rows in LDS: while one is worked on, the next two
// tiles' copies are on their way.
#include <algorithm>
#include <type_traits>

#include "vp_kv4.h"
#include "vp_tile.h"
#include "vp_walk.h"

namespace vp {
namespace {

typedef __bf16 bf16x2 __attribute__((__vector_size__(2 * sizeof(__bf16))));

// The conversions take a scale's exponent bits alone (23 to 30; sign and mantissa do not
// count; 0 is 2^-127, 255 makes NaN).
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

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
  read_early(a.four.kc, a.K, a.block_table, a.first);
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
      const uint32_t w[4] = {two_of<0>(c[j], scale), two_of<1>(c[j], scale), two_of<2>(c[j], scale), two_of<3>(c[j], scale)};
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
  // Work-groups enough to fill the GPU many times over where whole contexts are read (16 of 5k
  // to 12k rows, 4 KV heads: 72 us, with a quarter of them 77, with a sixteenth 84). Where `first`
  // leaves a few rows of each they find nothing to do: fewer then (64 sequences, 2 rows each: 5 us
  // and 8 with four times as many).
  const int64_t per = 4 * (kReadThreads / (D / 8));
  const int64_t pairs = static_cast<int64_t>(a.B) * a.Hkv * 2;
  const int64_t chunks = std::min((a.max_seq_len + per - 1) / per, std::max<int64_t>(1, (a.first ? 2048 : 32768) / pairs));
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

// query rows as bf16 operands: slot (a4, i) of step s <-> dim (D/4) a4 + 8 s + i. fp32 rows
// are fetched first and taken apart once the first tiles are requested.
template <int DT, int D>
struct Queries {
  static constexpr int N = DT == VP_BF16 ? 1 : 3;
  bf16x8 v[N][D / 32];
  float4 raw[DT == VP_BF16 ? 1 : D / 16];
  __device__ __forceinline__ void fetch(const char* row, bool valid, int a4) {
    if constexpr (DT == VP_BF16) {
#pragma unroll
      for (int s = 0; s < D / 32; ++s) {
        const uint4 u = valid ? reinterpret_cast<const uint4*>(row)[(D / 32) * a4 + s] : make_uint4(0, 0, 0, 0);
        v[0][s] = __builtin_bit_cast(bf16x8, u);
      }
    } else {
#pragma unroll
      for (int s = 0; s < D / 16; ++s)
        raw[s] = valid ? reinterpret_cast<const float4*>(row)[(D / 16) * a4 + s] : make_float4(0.f, 0.f, 0.f, 0.f);
    }
  }
  __device__ __forceinline__ void split() {
    if constexpr (DT == VP_F32) {
#pragma unroll
      for (int s = 0; s < D / 32; ++s) {
        const float x[8] = {raw[2 * s].x,     raw[2 * s].y,     raw[2 * s].z,     raw[2 * s].w,
                            raw[2 * s + 1].x, raw[2 * s + 1].y, raw[2 * s + 1].z, raw[2 * s + 1].w};
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

// A tile of 32 rows in LDS: K codes and V codes, rows one after another as in memory, but for
// the 16-byte pieces of a key row of 64 bytes, which change places (at), so that the 16 rows that
// a product's operand takes do not meet on the same banks; then the scales.
template <int D>
struct Tile4 {
  static constexpr int ROWB = D / 2, SROW = D / 32;
  static constexpr int BYTES = 32 * ROWB;          // of K or V
  static constexpr int COPIES = BYTES / 1024;      // copy instructions of K or V
  static constexpr int REQUESTS = 2 * COPIES + 1;  // of a tile, that of its scales among them
  static __device__ __forceinline__ int at(int row, int piece) {
    return row * ROWB + 16 * (D == 128 ? piece ^ (row >> 2 & 3) : piece);
  }
};

// The row in a lane's slot i of the products: a key operand's row n16 of half h is the tile's
// row 16 h + 4 (n16 % 4) + n16 / 4, so that its score ends up where the lane's four values of
// an instruction are 4 neighbouring rows over the four lanes.
__device__ __forceinline__ int slot_row(int a4, int i) { return 16 * (i >> 2) + 4 * (i & 3) + a4; }

// The scales' places in LDS, a dword per row: those of a lane's slots side by side
__device__ __forceinline__ int scale_place(int row) { return (row & 16) + 4 * (row & 3) + ((row >> 2) & 3); }

// byte `b` of a row's scales, at bits 23 to 30
__device__ __forceinline__ float scale_at(uint32_t scales, int b) {
  return __uint_as_float(__builtin_amdgcn_alignbit(scales, scales, (8 * b + 9) & 31));
}

// What a lane holds of a tile: its pieces of the key rows of its operand row (dims (D/4) a4 ..)
// and of the value rows of its slots (elements (D/16) n16 ..), and all these rows' scales
template <int D>
struct Rows4 {
  typedef unsigned pieces __attribute__((ext_vector_type(D / 32)));
  typedef unsigned pair __attribute__((ext_vector_type(2)));
  typedef unsigned quad __attribute__((ext_vector_type(4)));
  pieces k[2];
  pair ks;
  uint32_t v[8];
  quad vs[2];
  // One wait for all of them. Written by hand, because the compiler has the reads of one of
  // the three places wait for all copies in flight.
  __device__ __forceinline__ void load(const unsigned char* kb, const unsigned char* vb, int a4, int n16) {
#ifdef __HIP_DEVICE_COMPILE__
    const int row = 4 * (n16 & 3) + (n16 >> 2);
    const uint32_t at_k = (uint32_t)(uintptr_t)(lds_byte*)(kb + (D == 128 ? Tile4<D>::at(row, a4) : row * 32 + 8 * a4));
    const uint32_t at_v = (uint32_t)(uintptr_t)(lds_byte*)(vb + a4 * Tile4<D>::ROWB + (D / 32) * n16);
    const uint32_t at_ks = (uint32_t)(uintptr_t)(lds_byte*)(vb + Tile4<D>::BYTES + 4 * n16);
    const uint32_t at_vs = (uint32_t)(uintptr_t)(lds_byte*)(vb + Tile4<D>::BYTES + 128 + 16 * a4);
    if constexpr (D == 128) {
      pair v0, v1, v2, v3;
      asm volatile(
          "ds_read_b128 %0, %9\n\t"
          "ds_read_b128 %1, %9 offset:1024\n\t"
          "ds_read2_b32 %2, %11 offset1:16\n\t"
          "ds_read2st64_b32 %3, %10 offset0:0 offset1:4\n\t"
          "ds_read2st64_b32 %4, %10 offset0:1 offset1:5\n\t"
          "ds_read2st64_b32 %5, %10 offset0:2 offset1:6\n\t"
          "ds_read2st64_b32 %6, %10 offset0:3 offset1:7\n\t"
          "ds_read_b128 %7, %12\n\t"
          "ds_read_b128 %8, %12 offset:64\n\t"
          "s_waitcnt lgkmcnt(0)"
          : "=&v"(k[0]), "=&v"(k[1]), "=&v"(ks), "=&v"(v0), "=&v"(v1), "=&v"(v2), "=&v"(v3), "=&v"(vs[0]), "=&v"(vs[1])
          : "v"(at_k), "v"(at_v), "v"(at_ks), "v"(at_vs)
          : "memory");
      v[0] = v0[0];
      v[4] = v0[1];
      v[1] = v1[0];
      v[5] = v1[1];
      v[2] = v2[0];
      v[6] = v2[1];
      v[3] = v3[0];
      v[7] = v3[1];
    } else {
      asm volatile(
          "ds_read_b64 %0, %13\n\t"
          "ds_read_b64 %1, %13 offset:512\n\t"
          "ds_read2_b32 %2, %15 offset1:16\n\t"
          "ds_read_u16 %3, %14\n\t"
          "ds_read_u16 %4, %14 offset:128\n\t"
          "ds_read_u16 %5, %14 offset:256\n\t"
          "ds_read_u16 %6, %14 offset:384\n\t"
          "ds_read_u16 %7, %14 offset:512\n\t"
          "ds_read_u16 %8, %14 offset:640\n\t"
          "ds_read_u16 %9, %14 offset:768\n\t"
          "ds_read_u16 %10, %14 offset:896\n\t"
          "ds_read_b128 %11, %16\n\t"
          "ds_read_b128 %12, %16 offset:64\n\t"
          "s_waitcnt lgkmcnt(0)"
          : "=&v"(k[0]), "=&v"(k[1]), "=&v"(ks), "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]), "=&v"(v[4]), "=&v"(v[5]),
            "=&v"(v[6]), "=&v"(v[7]), "=&v"(vs[0]), "=&v"(vs[1])
          : "v"(at_k), "v"(at_v), "v"(at_ks), "v"(at_vs)
          : "memory");
    }
#endif
  }
  // a value row's scale (a lane's elements lie in one block of 32)
  __device__ __forceinline__ float value_scale(int i, int n16) const { return scale_at(vs[i >> 2][i & 3], D == 128 ? n16 >> 2 : n16 >> 3); }
  // Tiles where some query does not see some row: blocks of NaN would reach the outputs of
  // the queries that do not see them as 0 NaN. They are taken out (bit i of the result: this
  // lane's block of row i is one), ...
  __device__ __forceinline__ unsigned take_nan(int n16) {
    unsigned bad = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool b = (__float_as_uint(value_scale(i, n16)) & 0x7f800000u) == 0x7f800000u;
      bad |= b ? 1u << i : 0u;
      v[i] = b ? 0u : v[i];
      vs[i >> 2][i & 3] = b ? 0x7f7f7f7fu : vs[i >> 2][i & 3];  // (all of this lane's copy: 2^0)
    }
    return bad;
  }
};

template <int D, int N>
__device__ __forceinline__ void scores(float (&z)[8], const Rows4<D>& t, const bf16x8 (&q)[N][D / 32], int a4) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float scale = scale_at(t.ks[h], D == 128 ? a4 : a4 >> 1);
    f32x4 c = {0.f, 0.f, 0.f, 0.f};
    bf16x8 k[D / 32];
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
      const uint32_t u = t.k[h][s];
      k[s] = __builtin_bit_cast(bf16x8, make_uint4(two_of<0>(u, scale), two_of<1>(u, scale), two_of<2>(u, scale), two_of<3>(u, scale)));
    }
#pragma unroll
    for (int p = N - 1; p >= 0; --p)
#pragma unroll
      for (int s = 0; s < D / 32; ++s) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[s], q[p][s], c, 0, 0, 0);
#pragma unroll
    for (int r = 0; r < 4; ++r) z[4 * h + r] = c[r];
  }
}

// The value product. The weights enter as the sum of three bf16 numbers, all 24 bits of
// them (truncated one after another: exact).
//
// FOLD, up to 8 query rows: a matrix product's 16 columns are 8 query rows for the elements
// of even number and the same 8 for those of odd number, and its 32 slots are 16 rows of V times
// the two elements of a code byte: the weights of the other parity are zeros. So a
// byte's conversion is an operand as it stands, nothing is sorted, and the accumulators have
// no idle columns. acc[byte][r]: element (D/16) (4 a4 + r) + 2 byte + (n16 >> 3) of query row n16 & 7.
// Else: acc[e][r]: element (D/16) (4 a4 + r) + e of query row n16, slots are 32 rows of V, and
// pairs of conversions are sorted by element.
template <int D, bool FOLD>
struct Values {
  static constexpr int N = FOLD ? D / 32 : D / 16;
  f32x4 acc[N];

  __device__ __forceinline__ static float rest(float p) {
    return p - __uint_as_float(__float_as_uint(p) & 0xffff0000u);
  }
  template <int B>
  __device__ __forceinline__ void byte(const Rows4<D>& t, const float (&scale)[8], const bf16x8 (&w)[FOLD ? 6 : 3]) {
    if constexpr (FOLD) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = two_of<B>(t.v[4 * h + j], scale[4 * h + j]);
        const bf16x8 a = __builtin_bit_cast(bf16x8, make_uint4(x[0], x[1], x[2], x[3]));
#pragma unroll
        for (int i = 0; i < 3; ++i) acc[B] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, w[3 * h + i], acc[B], 0, 0, 0);
      }
    } else {
      uint32_t lo[4], hi[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t x = two_of<B>(t.v[2 * j], scale[2 * j]), y = two_of<B>(t.v[2 * j + 1], scale[2 * j + 1]);
        lo[j] = __builtin_amdgcn_perm(y, x, 0x05040100u);
        hi[j] = __builtin_amdgcn_perm(y, x, 0x07060302u);
      }
      const bf16x8 a0 = __builtin_bit_cast(bf16x8, make_uint4(lo[0], lo[1], lo[2], lo[3]));
      const bf16x8 a1 = __builtin_bit_cast(bf16x8, make_uint4(hi[0], hi[1], hi[2], hi[3]));
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        acc[2 * B] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a0, w[i], acc[2 * B], 0, 0, 0);
        acc[2 * B + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a1, w[i], acc[2 * B + 1], 0, 0, 0);
      }
    }
  }
  // p: the weights of the lane's rows
  __device__ __forceinline__ void add(const Rows4<D>& t, const float (&p)[8], int n16) {
    bf16x8 w[FOLD ? 6 : 3];
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = p[i];
    // a weight's upper half in the lower or the upper half of a dword
    const uint32_t place = n16 < 8 ? 0x0c0c0302u : 0x03020c0cu;
#pragma unroll
    for (int part = 0; part < 3; ++part) {
      uint32_t u[8];
      if constexpr (FOLD) {
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = __builtin_amdgcn_perm(0u, __float_as_uint(x[i]), place);
        w[part] = __builtin_bit_cast(bf16x8, make_uint4(u[0], u[1], u[2], u[3]));
        w[3 + part] = __builtin_bit_cast(bf16x8, make_uint4(u[4], u[5], u[6], u[7]));
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) u[j] = __builtin_amdgcn_perm(__float_as_uint(x[2 * j + 1]), __float_as_uint(x[2 * j]), 0x07060302u);
        w[part] = __builtin_bit_cast(bf16x8, make_uint4(u[0], u[1], u[2], u[3]));
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = rest(x[i]);
    }
    float scale[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) scale[i] = t.value_scale(i, n16);
    byte<0>(t, scale, w);
    byte<1>(t, scale, w);
    if constexpr (D == 128) {
      byte<2>(t, scale, w);
      byte<3>(t, scale, w);
    }
  }
  // ... (Rows4::take_nan) and the queries that do see one get NaN: by the number of such rows, a product of
  // zeros and ones
  __device__ __forceinline__ void put_nan(unsigned bad, unsigned seen) {
    f32x4 count = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t x[4], y[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[j] = (bad >> (4 * h + j)) & 1u ? 0x3f803f80u : 0u;
        y[j] = (seen >> (4 * h + j)) & 1u ? 0x3f803f80u : 0u;
      }
      count = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, make_uint4(x[0], x[1], x[2], x[3])),
                                                      __builtin_bit_cast(bf16x8, make_uint4(y[0], y[1], y[2], y[3])), count, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[i][r] = count[r] > 0.f ? __builtin_nanf("") : acc[i][r];
  }
};

// work-groups that a CU's registers hold (a wave of each per SIMD)
constexpr int kv4_groups_per_cu(int dtype, int head_dim, bool fold) {
  return (dtype == VP_F32 && head_dim == 128) || !fold ? 2 : 3;
}

// The tiles of a walk all of whose rows every query sees, and the others, the outer ones: those at
// the end of the sinks, at the beginning of the windows, and around the queries' own rows.
struct Interior {
  int a1;        // inner tiles 0 .. a1 - 1
  int b0, b1;    // and b0 .. b1 - 1
  int n, outer;  // how many inner and outer ones
  __device__ __forceinline__ Interior(const WindowWalk& w, int T, int window) {
    const int past = max(w.L - T + 1, 0);              // rows that lie before every query but the first's own, and that one
    const int hidden = window > 0 ? w.L - window : 0;  // the last query sees no row from n_sink up to here
    a1 = min(window > 0 ? w.S / 32 : w.sinks, past / 32);
    b0 = max(w.sinks, w.sinks - w.first + (max(hidden, 0) + 31) / 32);
    b0 = min(b0, w.n);
    b1 = min(max(w.sinks - w.first + past / 32, b0), w.n);
    n = a1 + (b1 - b0);
    outer = w.n - n;
  }
  __device__ __forceinline__ int tile(int i) const { return i < a1 ? i : i - a1 + b0; }
  __device__ __forceinline__ int outer_tile(int e) const { return e < b0 - a1 ? a1 + e : e - (b0 - a1) + b1; }
};

template <int DT, int D, bool PAGED, bool FOLD>
__global__ __launch_bounds__(kWinThreads) __attribute__((amdgpu_waves_per_eu(kv4_groups_per_cu(DT, D, FOLD)))) void
kv4_kernel(const WindowArgs a, const Kv4Cache four) {
  using Q = Tile4<D>;
  constexpr int COLUMNS = FOLD ? 8 : 16;
  // Per wave: places for the K codes, and for the V codes and scales, of three tiles (after the
  // walk the first tile's make room for half of the accumulator rows each). Arrays of their
  // own: in one, the compiler would have reads of a tile wait for the copies of another (it
  // tells up to 8 arrays apart).
  constexpr int FIRST = max_i(Q::BYTES, COLUMNS / 2 * D * 4), SCALES = 64 * 4;
  __shared__ __attribute__((aligned(1024))) unsigned char lds_k0[kWinWaves * FIRST];
  __shared__ __attribute__((aligned(1024))) unsigned char lds_v0[kWinWaves * (FIRST + SCALES)];
  __shared__ __attribute__((aligned(1024))) unsigned char lds_k1[kWinWaves * Q::BYTES];
  __shared__ __attribute__((aligned(1024))) unsigned char lds_v1[kWinWaves * (Q::BYTES + SCALES)];
  __shared__ __attribute__((aligned(1024))) unsigned char lds_k2[kWinWaves * Q::BYTES];
  __shared__ __attribute__((aligned(1024))) unsigned char lds_v2[kWinWaves * (Q::BYTES + SCALES)];
  __shared__ WinStats ws;
  read_early(a.q, a.seq_len, a.zscale, four.vs);
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const int lane = threadIdx.x & 63;
  const int n16 = lane & 15;
  const int a4 = lane >> 4;
  const int col = n16 & (COLUMNS - 1);  // this lane's query row
  const int TG = a.T * a.G;
  const bool hv = col < TG;
  const int tq = hv ? query_of(a, col) : 0;

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
  q.fetch(static_cast<const char*>(a.q) + (hv ? out_row(a, b, g, col) : 0) * (D * (DT == VP_BF16 ? 2 : 4)), hv, a4);
  const WindowWalk w(L, a.T, a.window, a.n_sink);
  const int hi = w.L - a.T + tq;                        // this lane's query sees j <= hi
  const int below = a.window > 0 ? hi - a.window : -1;  // and j > below or j < n_sink

  const int64_t seq_c = (PAGED ? 0 : b * four.cb) + g * four.ch, seq_s = (PAGED ? 0 : b * four.sb) + g * four.sh;
  const uint8_t* const Kc = four.kc + seq_c;
  const uint8_t* const Vc = four.vc + seq_c;
  const int32_t* bt = PAGED ? a.block_table + static_cast<int64_t>(b) * a.nblk : nullptr;
  const int bmask = PAGED ? (1 << a.bs_log2) - 1 : 0;
  const Interior in(w, a.T, a.window);
  unsigned char* const k0 = lds_k0 + wave * FIRST;
  unsigned char* const v0 = lds_v0 + wave * (FIRST + SCALES);
  unsigned char* const k1 = lds_k1 + wave * Q::BYTES;
  unsigned char* const v1 = lds_v1 + wave * (Q::BYTES + SCALES);
  unsigned char* const k2 = lds_k2 + wave * Q::BYTES;
  unsigned char* const v2 = lds_v2 + wave * (Q::BYTES + SCALES);

  // Copies: lane i of an instruction fills bytes 16 i .. of 1 KB, so it takes one piece of
  // one row. Scales: a dword per row (of 64: their two bytes), key rows by lanes 0 to 31, value
  // rows by the others.
  const int copy_row = lane / (Q::ROWB / 16);
  const int copy_piece = (Q::at(copy_row, lane % (Q::ROWB / 16)) - copy_row * Q::ROWB) / 16;
  const uint32_t key_off = copy_row * Q::ROWB + 16 * copy_piece, value_off = 16 * lane;
  const int scale_row = scale_place(lane & 31);  // (its own inverse)
  const uint8_t* const scale_src = (lane < 32 ? four.ks : four.vs) + seq_s;
  auto copy = [&](const uint8_t* src, unsigned char* dst) {
    __builtin_amdgcn_global_load_lds((global_void*)src, (lds_void*)(lds_byte*)dst, 16, 0, kCopyPolicy);
  };
  auto copy_scales = [&](const uint8_t* src, unsigned char* dst) {
    __builtin_amdgcn_global_load_lds((global_void*)src, (lds_void*)(lds_byte*)dst, Q::SROW, 0, kCopyPolicy);
  };
  // Paged caches: the blocks of a tile's halves (a half's rows follow each other: blocks
  // hold at least 16). Scalar loads, so that no wait for one is a wait for copies.
  typedef __attribute__((address_space(4))) const int32_t table_entry;
  auto blocks_of = [&](int t0) -> int2 {
    if constexpr (PAGED) {
      const table_entry* t = (const table_entry*)bt;
      return make_int2(t[t0 >> a.bs_log2], t[(t0 + 16) >> a.bs_log2]);
    } else {
      return make_int2(0, 0);
    }
  };
  // Requests the tile at row t0, all of whose rows are read
  auto request = [&](int t0, int2 blk, unsigned char* kb, unsigned char* vb) {
    if constexpr (PAGED) {
      const int r0 = t0 & bmask, r1 = (t0 + 16) & bmask;
      const int64_t c0 = blk.x * four.cb + static_cast<int64_t>(r0) * Q::ROWB, c1 = blk.y * four.cb + static_cast<int64_t>(r1) * Q::ROWB;
      if constexpr (D == 128) {
        copy(Kc + c0 + key_off, kb);
        copy(Kc + c1 + key_off, kb + 1024);
        copy(Vc + c0 + value_off, vb);
        copy(Vc + c1 + value_off, vb + 1024);
      } else {
        const int64_t c = (lane < 32 ? c0 : c1 - 16 * Q::ROWB) + value_off;
        copy(Kc + c, kb);
        copy(Vc + c, vb);
      }
      const int64_t at0 = blk.x * four.sb + static_cast<int64_t>(r0) * Q::SROW, at1 = blk.y * four.sb + static_cast<int64_t>(r1 - 16) * Q::SROW;
      copy_scales(scale_src + ((lane & 16) == 0 ? at0 : at1) + scale_row * Q::SROW, vb + Q::BYTES);
    } else {
      const int64_t c = static_cast<int64_t>(t0) * Q::ROWB;
#pragma unroll
      for (int j = 0; j < Q::COPIES; ++j) copy(Kc + c + (key_off + 1024 * j), kb + 1024 * j);
#pragma unroll
      for (int j = 0; j < Q::COPIES; ++j) copy(Vc + c + (value_off + 1024 * j), vb + 1024 * j);
      copy_scales(scale_src + static_cast<int64_t>(t0) * Q::SROW + scale_row * Q::SROW, vb + Q::BYTES);
    }
  };
  // Requests any tile. Rows that no query sees are not read, their places take the nearest
  // row that is read anyway.
  auto request_any = [&](int k, unsigned char* kb, unsigned char* vb) {
    const int t0 = w.t0(k);
    const int r0 = w.row_begin(k), r1 = w.row_end(k);  // rows that some query sees, r0 < r1
    auto place = [&](int r, int64_t& block) {
      const int pos = min(max(t0 + r, r0), r1 - 1);
      block = PAGED ? bt[pos >> a.bs_log2] : 0;
      return PAGED ? pos & bmask : pos;
    };
    int64_t block;
#pragma unroll
    for (int j = 0; j < Q::COPIES; ++j) {
      const int row = place(1024 / Q::ROWB * j + copy_row, block);
      const int64_t c = block * four.cb + static_cast<int64_t>(row) * Q::ROWB;
      copy(Kc + c + 16 * copy_piece, kb + 1024 * j);
      copy(Vc + c + 16 * (lane % (Q::ROWB / 16)), vb + 1024 * j);
    }
    const int row = place(scale_row, block);
    copy_scales(scale_src + block * four.sb + static_cast<int64_t>(row) * Q::SROW, vb + Q::BYTES);
  };

  float m = kNoLogit, l = 0.f;  // m shared by the four lanes of a query row; l lane-local
  Values<D, FOLD> out;
#pragma unroll
  for (int i = 0; i < out.N; ++i) out.acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};

  // the products of a tile's rows, unscaled (value i of this lane is row slot_row(a4, i)),
  // become weights, and the values are added
  auto weigh = [&](float (&z)[8]) {
    float lmax = z[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) lmax = fmaxf(lmax, z[i]);
    if (__builtin_amdgcn_ballot_w64(lmax > m + a.raise)) {
      // the four lanes of a query row share the reference (their weights meet in one MFMA)
      const float tm = max_over_quads(lmax);
      const bool up = tm > m + a.raise;
      const float al = up ? weight_of(a, m, tm) : 1.f;
      l *= al;
      m = up ? tm : m;
#pragma unroll
      for (int i = 0; i < out.N; ++i) out.acc[i] *= al;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = weight_of(a, z[i], m);
    l += ((z[0] + z[1]) + (z[2] + z[3])) + ((z[4] + z[5]) + (z[6] + z[7]));
  };

  // this part's run of inner tiles, and this wave's first one
  const int each = in.n / parts, rest = in.n - each * parts;
  int i = part * each + min(part, rest);
  const int i1 = i + each + (part < rest ? 1 : 0);
  i += wave;
  auto first_row = [&](int i) { return w.t0(in.tile(i)); };
  auto own_row = [&](int n) { return first_row(min(i + n * kWinWaves, i1 - 1)); };  // the wave's n-th tile from here, or the last
  int2 blk{};  // of the next tile to be requested
  if (i < i1) {
    request(own_row(0), blocks_of(own_row(0)), k0, v0);
    if (i + kWinWaves < i1) request(own_row(1), blocks_of(own_row(1)), k1, v1);
    blk = blocks_of(own_row(2));
  }
  q.split();
  // The outer tiles, a few at the ends of what is seen, go round the parts
#pragma unroll 1
  for (int e = part + wave * parts; e < in.outer; e += kWinWaves * parts) {
    const int k = in.outer_tile(e);
    __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
    request_any(k, k2, v2);
    __builtin_amdgcn_s_waitcnt(kWaitVm0);
    Rows4<D> rows;
    rows.load(k2, v2, a4, n16);
    float z[8];
    scores<D>(z, rows, q.v, a4);
    unsigned seen = 0xffu;
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      const int j = w.t0(k) + slot_row(a4, r);
      if (j > hi || (j <= below && j >= w.S)) {
        seen &= ~(1u << r);
        z[r] = kNegInf;
      }
    }
    weigh(z);
    const unsigned bad = rows.take_nan(n16);
    out.add(rows, z, n16);
    if (__builtin_amdgcn_ballot_w64(bad != 0)) out.put_nan(bad, seen);
  }
  // Tile i is at (kb, vb), or on its way there, and so is the wave's next one at places of
  // its own; the one after is requested into the third. Memory operations of a wave complete
  // in the order of their issue: a wait names how many issued after what it waits for may be
  // left.
  auto step = [&](unsigned char* kb, unsigned char* vb, unsigned char* k_next, unsigned char* v_next) {
    __builtin_amdgcn_s_waitcnt(kWaitLgkm0);  // reads of the third place have returned
    if (i + 2 * kWinWaves < i1) {
      request(own_row(2), blk, k_next, v_next);
      blk = blocks_of(own_row(3));
      __builtin_amdgcn_s_waitcnt(wait_vm(2 * Q::REQUESTS));
    } else if (i + kWinWaves < i1) {
      __builtin_amdgcn_s_waitcnt(wait_vm(Q::REQUESTS));
    } else {
      __builtin_amdgcn_s_waitcnt(kWaitVm0);
    }
    Rows4<D> rows;
    rows.load(kb, vb, a4, n16);
    float z[8];
    scores<D>(z, rows, q.v, a4);
    weigh(z);
    out.add(rows, z, n16);
    i += kWinWaves;
  };
#pragma unroll 1
  while (i < i1) {
    step(k0, v0, k2, v2);
    if (i >= i1) break;
    step(k1, v1, k0, v0);
    if (i >= i1) break;
    step(k2, v2, k1, v1);
  }
  l = sum_over_quads(l);

  // ---- join the four waves ----
  if (a4 == 0 && n16 < COLUMNS) {
    ws.m[wave][n16] = m;
    ws.l[wave][n16] = l;
  }
  __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
  // (the 16-byte pieces of a row change places by its column, so that columns do not meet on
  // the same banks)
  auto piece = [](int column, int c) { return 4 * (c ^ (column & 7)); };
  float* mine = reinterpret_cast<float*>(col < COLUMNS / 2 ? k0 : v0) + col % (COLUMNS / 2) * D;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int dim = (D / 16) * (4 * a4 + r);
    if constexpr (FOLD) {
#pragma unroll
      for (int i = 0; i < out.N; ++i) mine[piece(col, (dim + 2 * i) / 4) + 2 * (i & 1) + (n16 >> 3)] = out.acc[i][r];
    } else {
#pragma unroll
      for (int e = 0; e < out.N; e += 4)
        *reinterpret_cast<float4*>(mine + piece(col, (dim + e) / 4)) =
            make_float4(out.acc[e][r], out.acc[e + 1][r], out.acc[e + 2][r], out.acc[e + 3][r]);
    }
  }
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
      const unsigned char* place = h < COLUMNS / 2 ? lds_k0 + v * FIRST : lds_v0 + v * (FIRST + SCALES);
      const float4 x = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(place) + h % (COLUMNS / 2) * D + piece(h, c));
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
  const bool paged = a.bs_log2 >= 0, fold = a.T * a.G <= 8;
  if (paged && fold) hipLaunchKernelGGL((kv4_kernel<DT, D, true, true>), grid, dim3(kWinThreads), 0, st, a, four);
  else if (paged) hipLaunchKernelGGL((kv4_kernel<DT, D, true, false>), grid, dim3(kWinThreads), 0, st, a, four);
  else if (fold) hipLaunchKernelGGL((kv4_kernel<DT, D, false, true>), grid, dim3(kWinThreads), 0, st, a, four);
  else hipLaunchKernelGGL((kv4_kernel<DT, D, false, false>), grid, dim3(kWinThreads), 0, st, a, four);
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
  // One work-group per pair, and no second launch, as make_window_plan has it (a tile takes
  // half as long here: 0.16 us), where (us whole and dealt; bf16, d = 128)
  // * the walks are short: up to 28 tiles (4 KV heads; 1 sequence: 16 tiles 7.1 and 9.4, 32
  //   tiles 10.0 and 9.5; 16 sequences: 16 tiles 7.4 and 9.9, 32 tiles 10.5 and 11.1, 64 tiles
  //   15.8 and 13.4);
  // * the longest walk is short beside what dealing costs (64 sequences, 256 pairs: 16 tiles
  //   8.3 and 15.4, 32 tiles 11.1 and 17.9, 128 tiles 29.2 and 34.7, lengths from a tenth of
  //   that 27.8 and 27.8, 256 tiles 55.6 and 57.1, 48.1 and 41.2; 128 sequences, 64 tiles 28.8
  //   and 37.7);
  // * a window cuts the walks of the capacity to half or less, and the pairs nearly fill the
  //   CUs (64 sequences, window 8192 of 32k: 56.4 and 58.1, lengths from 1k on 55.0 and 55.5; it
  //   loses where most have not filled the window, one of 32k among 1k: 46.9 and 23.6).
  const bool brief = 1200 * tiles <= pairs * (350 + s.batch);
  const bool cut = w.window > 0 && 2 * tiles <= cap;
  const bool one_each = tiles <= 28 || brief || (cut && pairs >= 192) || pairs * tiles > 0x3fffffff;
  // Otherwise two work-groups per CU (three or four, where registers allow them: 64 x 32k
  // 190 and 190, 16 x 12k ragged 21.3 and 22.3 to 24.2), twice as many as pairs where those are
  // more, a tile per wave at least; and no more than 32 for a walk, or one per 16 tiles, as the second
  // launch joins the pieces (1 sequence of 8k: 32 each 11.0, 64 each 12.1; of 32k: 64 each 14.6, 128
  // each 19.2)
  const int64_t most = std::min<int64_t>(std::max<int64_t>(512, 2 * pairs), pairs * std::max<int64_t>(32, tiles / 16));
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
