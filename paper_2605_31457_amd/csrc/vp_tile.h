// Tile primitives shared by the passes over a KV cache (gfx950, wave64): the LDS
// layout of a 32-row tile, the query operand, the scores of a tile and its value
// product on the matrix cores.
#pragma once

#include "vp_common.h"
#include "vp_internal.h"

typedef __attribute__((address_space(1))) void global_void;
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) unsigned char lds_byte;

// Cache policy of the K/V row copies: non-temporal (the "nt" bit). Every row is
// used once per step, and streaming it without cache allocation measured ~13%
// faster on the text pass (5.4 -> 6.1 TB/s on the 64 x 32k batch).
constexpr int kCopyPolicy = 2;

// s_waitcnt immediates (gfx9 encoding: vmcnt [3:0]+[15:14], expcnt [6:4], lgkmcnt [11:8])
constexpr int kWaitLgkm0 = 0xC07F;  // lgkmcnt(0), others unconstrained
constexpr int kWaitVm0 = 0x0F70;    // vmcnt(0), others unconstrained
// buffer resource word 3 for raw (untyped) dword access: 32-bit data format
constexpr int kRawBufferWord3 = 0x00020000;

namespace vp {

constexpr int max_i(int x, int y) { return x > y ? x : y; }

// Make a value unknown to the optimiser at this point, so that what is computed
// from it stays where it is instead of being kept in registers through a loop
// (device code only: the constraints name scalar and vector registers)
template <typename X>
__device__ __forceinline__ void unhoist_scalar(X& x) {
#ifdef __HIP_DEVICE_COMPILE__
  asm volatile("" : "+s"(x));
#endif
}
template <typename X>
__device__ __forceinline__ void unhoist_vector(X& x) {
#ifdef __HIP_DEVICE_COMPILE__
  asm volatile("" : "+v"(x));
#endif
}

template <int DT, int D>
struct Cfg {
  static constexpr bool BF = DT == VP_BF16;
  static constexpr int ESZ = BF ? 2 : 4;
  static constexpr int ROWB = D * ESZ;                      // bytes per K/V row
  static constexpr int PIECES = ROWB / 16;                  // 16-byte pieces per row
  static constexpr int RPI = 64 / PIECES;                   // rows per 1 KB copy instruction
  static constexpr int SUB_ROWS_BYTES = 32 * ROWB;          // one 32-row block of K or V
  static constexpr int STAGE_BYTES = 16 * 32 * 4;           // logits of 16 heads x 32 rows
  static constexpr int COPIES = 32 / RPI;                   // copy instructions per block
  static constexpr int ACC_N = BF ? (D / 64) * 4 : D / 16;  // f32x4 accumulators
  // LDS byte offset of 16-byte piece p of row r inside a block
  static __device__ __forceinline__ int at(int r, int p) { return r * ROWB + 16 * (p ^ (r & (PIECES - 1))); }
};

template <int DT, int D>
struct QFrag;

template <int D>
struct QFrag<VP_BF16, D> {
  bf16x8 v[D / 32];
};
template <int D>
struct QFrag<VP_F32, D> {
  float v[D / 4];
};

// q row of head h as the B operand (k-slot (a4, i) of step s <-> dim s*32 + 8*a4 + i
// for bf16; dim (D/4)*a4 + s for fp32)
template <int DT, int D>
__device__ __forceinline__ void load_q(QFrag<DT, D>& f, const void* qrow, bool valid, int a4) {
  if constexpr (DT == VP_BF16) {
    const uint4* p = reinterpret_cast<const uint4*>(qrow);
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
      uint4 u = valid ? p[4 * s + a4] : make_uint4(0, 0, 0, 0);
      f.v[s] = __builtin_bit_cast(bf16x8, u);
    }
  } else {
    const float4* p = reinterpret_cast<const float4*>(qrow);
#pragma unroll
    for (int s4 = 0; s4 < D / 16; ++s4) {
      float4 u = valid ? p[(D / 16) * a4 + s4] : make_float4(0.f, 0.f, 0.f, 0.f);
      f.v[4 * s4 + 0] = u.x;
      f.v[4 * s4 + 1] = u.y;
      f.v[4 * s4 + 2] = u.z;
      f.v[4 * s4 + 3] = u.w;
    }
  }
}

// C'[token n16 of 16-row half hf][head] from the key block in LDS (same dim
// mapping as load_q)
template <int DT, int D>
__device__ __forceinline__ f32x4 score_half(const unsigned char* kb, int hf, const QFrag<DT, D>& q, int a4,
                                            int n16) {
  using C = Cfg<DT, D>;
  const int r = 16 * hf + n16;
  f32x4 c = {0.f, 0.f, 0.f, 0.f};
  if constexpr (DT == VP_BF16) {
    uint4 k[D / 32];
#pragma unroll
    for (int s = 0; s < D / 32; ++s) k[s] = *reinterpret_cast<const uint4*>(kb + C::at(r, 4 * s + a4));
#pragma unroll
    for (int s = 0; s < D / 32; ++s)
      c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[s]), q.v[s], c, 0, 0, 0);
  } else {
    float4 k[D / 16];
#pragma unroll
    for (int s4 = 0; s4 < D / 16; ++s4) k[s4] = *reinterpret_cast<const float4*>(kb + C::at(r, (D / 16) * a4 + s4));
#pragma unroll
    for (int s4 = 0; s4 < D / 16; ++s4) {
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(k[s4].x, q.v[4 * s4 + 0], c, 0, 0, 0);
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(k[s4].y, q.v[4 * s4 + 1], c, 0, 0, 0);
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(k[s4].z, q.v[4 * s4 + 2], c, 0, 0, 0);
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(k[s4].w, q.v[4 * s4 + 3], c, 0, 0, 0);
    }
  }
  return c;
}

// sub-tile-relative token held by lane slot (a4, i) of the value product: the
// score registers of lane l hold tokens 4*a4 + r (half 0) and 16 + 4*a4 + r (half 1)
__device__ __forceinline__ int pv_token(int a4, int i) { return i < 4 ? 4 * a4 + i : 16 + 4 * a4 + (i - 4); }

// acc += V^T P^T over the tile's 32 rows. SPLIT (bf16): the weights enter as the sum
// of three bf16 numbers, all 24 bits of them, instead of one of 8: the leading two
// truncated, the rests positive where the weight is, so that an infinite value stays an
// infinity of its sign. (Two, 16 bits, cost 0.3 to 1.5% less, 64 windows of 8k 159.0 us
// and 159.6, and put 3 to 4 in 1000 bf16 outputs on the other side of a rounding than a
// product in float32, mostly the wrong one; with three it is 5 to 17 in 10000, mostly the
// right one.) Bit i of `rows` (masked tiles): the row in this lane's slot i takes part; the
// others count as zeros whatever they hold.
template <int DT, int D, int N, bool SPLIT = false, bool MASKED = false>
__device__ __forceinline__ void value_product(f32x4 (&acc)[N], const unsigned char* vb, const float (&p)[8],
                                              int a4, int n16, unsigned rows = 0xffu) {
  using C = Cfg<DT, D>;
  if constexpr (DT == VP_BF16) {
    // P^T operand: slot (a4, i) <-> token pv_token(a4, i), head n16
    bf16x8 pf, pm, pl;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (SPLIT) {
        const uint32_t u = __float_as_uint(p[i]);
        const float rest = fminf(fmaxf(p[i] - __uint_as_float(u & 0xffff0000u), 0x1p-100f), p[i]);
        const uint32_t v = __float_as_uint(rest);
        pf[i] = __builtin_bit_cast(__bf16, static_cast<uint16_t>(u >> 16));
        pm[i] = __builtin_bit_cast(__bf16, static_cast<uint16_t>(v >> 16));
        pl[i] = static_cast<__bf16>(fminf(fmaxf(rest - __uint_as_float(v & 0xffff0000u), 0x1p-100f), rest));
      } else {
        pf[i] = static_cast<__bf16>(p[i]);
      }
    }
#pragma unroll
    for (int u = 0; u < D / 64; ++u) {
      // lane n16 takes dims 64u + 4*n16 .. +3 = 8 bytes in piece 8u + n16/2
      uint2 w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        w[i] = *reinterpret_cast<const uint2*>(vb + C::at(pv_token(a4, i), 8 * u + (n16 >> 1)) + 8 * (n16 & 1));
      if constexpr (MASKED) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (!((rows >> i) & 1u)) w[i] = make_uint2(0u, 0u);
      }
      // A operand of MFMA (u, e): row n16 <-> dim 64u + 4*n16 + e, slot i <-> token pv_token(a4, i)
      uint32_t lo0[4], hi0[4], lo1[4], hi1[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        lo0[j] = __builtin_amdgcn_perm(w[2 * j + 1].x, w[2 * j].x, 0x05040100u);
        hi0[j] = __builtin_amdgcn_perm(w[2 * j + 1].x, w[2 * j].x, 0x07060302u);
        lo1[j] = __builtin_amdgcn_perm(w[2 * j + 1].y, w[2 * j].y, 0x05040100u);
        hi1[j] = __builtin_amdgcn_perm(w[2 * j + 1].y, w[2 * j].y, 0x07060302u);
      }
      const bf16x8 a0 = __builtin_bit_cast(bf16x8, make_uint4(lo0[0], lo0[1], lo0[2], lo0[3]));
      const bf16x8 a1 = __builtin_bit_cast(bf16x8, make_uint4(hi0[0], hi0[1], hi0[2], hi0[3]));
      const bf16x8 a2 = __builtin_bit_cast(bf16x8, make_uint4(lo1[0], lo1[1], lo1[2], lo1[3]));
      const bf16x8 a3 = __builtin_bit_cast(bf16x8, make_uint4(hi1[0], hi1[1], hi1[2], hi1[3]));
      acc[4 * u + 0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a0, pf, acc[4 * u + 0], 0, 0, 0);
      acc[4 * u + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a1, pf, acc[4 * u + 1], 0, 0, 0);
      acc[4 * u + 2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a2, pf, acc[4 * u + 2], 0, 0, 0);
      acc[4 * u + 3] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a3, pf, acc[4 * u + 3], 0, 0, 0);
      if constexpr (SPLIT) {
        acc[4 * u + 0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a0, pm, acc[4 * u + 0], 0, 0, 0);
        acc[4 * u + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a1, pm, acc[4 * u + 1], 0, 0, 0);
        acc[4 * u + 2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a2, pm, acc[4 * u + 2], 0, 0, 0);
        acc[4 * u + 3] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a3, pm, acc[4 * u + 3], 0, 0, 0);
        acc[4 * u + 0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a0, pl, acc[4 * u + 0], 0, 0, 0);
        acc[4 * u + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a1, pl, acc[4 * u + 1], 0, 0, 0);
        acc[4 * u + 2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a2, pl, acc[4 * u + 2], 0, 0, 0);
        acc[4 * u + 3] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a3, pl, acc[4 * u + 3], 0, 0, 0);
      }
    }
  } else {
    // k-step s covers tokens pv_token(a4, s) (one per lane group); row n16 <-> dim 16*dt + n16
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      const int t = pv_token(a4, s);
#pragma unroll
      for (int dt = 0; dt < D / 16; ++dt) {
        const int dim = 16 * dt + n16;
        float v = *reinterpret_cast<const float*>(vb + C::at(t, dim >> 2) + 4 * (dim & 3));
        if constexpr (MASKED) v = (rows >> s) & 1u ? v : 0.f;
        acc[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, p[s], acc[dt], 0, 0, 0);
      }
    }
  }
}

// store the lane's accumulator slice (head n16) of a (D)-float partial row
template <int DT, int D, int N>
__device__ __forceinline__ void store_acc(float* dst, const f32x4 (&acc)[N], int a4) {
  if constexpr (DT == VP_BF16) {
    // acc[4u + e][r] holds dim 64u + 16*a4 + 4r + e
#pragma unroll
    for (int u = 0; u < D / 64; ++u)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float4 o = make_float4(acc[4 * u + 0][r], acc[4 * u + 1][r], acc[4 * u + 2][r], acc[4 * u + 3][r]);
        *reinterpret_cast<float4*>(dst + 64 * u + 16 * a4 + 4 * r) = o;
      }
  } else {
    // acc[dt][r] holds dim 16*dt + 4*a4 + r
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt)
      *reinterpret_cast<float4*>(dst + 16 * dt + 4 * a4) = make_float4(acc[dt][0], acc[dt][1], acc[dt][2], acc[dt][3]);
  }
}

// A running maximum before any finite logit: the least float, not -inf, so that rows
// of logit -inf weigh 2^-inf = 0 until then (relative to -inf they would be NaN).
// Written out as -inf (an empty partial).
constexpr float kNoLogit = -3.402823466e38f;

}  // namespace vp
