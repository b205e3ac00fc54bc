// New tokens into caches (vp_append_kv, vp_append_kv4): queries and keys are rotated by their
// positions, keys and values go to the last rows of their sequences, as they are or in 4 bits.
//
//   a' = a cos - b sin,  b' = b cos + a sin      (pairs (a, b) of a head's first `rot` elements)
//   4 bits, per 32 elements: 2^e, e the least with max <= 7 2^e; codes nearest to x / 2^e, ties to even
//
// The rotation is done in 64 bits, where the products of 16- and 32-bit numbers are exact and
// the sum is rounded once; what is stored is that, rounded once more (to 16 bits through 32:
// off by at most half a step and 2^-16 of it). So a value does not depend on how the
// arithmetic is arranged, and 4-bit codes next to a border fall on the right side of it. In 16
// bits it costs little: 10k tokens of 72B-class heads (64/8 of 128) take 84 to 86 us in 16 bits, 5.0 TB/s
// read and written (a large copy: 5.2), 166 in 32. Into 4 bits 12.5k tokens of 28/4 heads take 50
// to 53, 4.1 to 4.3 TB/s (45 where the same rows come again and lie in the caches).
//
// Bound: HBM, every row read and written once; a few tokens: one launch of dependent loads
// (offsets, length, block id; position, cosines; the rows beside them: 2.6 us for one token). A
// lane holds 8 consecutive elements of a row and loads their 8 partners too, which another
// lane of the wave loads as its own (the second load is the first-level cache's); a wave holds
// 4 rows of 128 or 8 of 64, three times over. A token's rows (queries, keys, values) are taken
// by as few waves as fill the GPU (launch_append), whose cosines stay in registers.
#include <algorithm>

#include "vp_common.h"
#include "vp_kv4.h"

namespace vp {
namespace {

constexpr int kAppendWaves = 4;

// the float nearest to d whose last bit is set unless d is a float: rounded again to fewer
// bits it gives what d gives
__device__ __forceinline__ float to_odd(double d) {
  const float f = static_cast<float>(d);
  const double back = static_cast<double>(f);
  uint32_t u = __float_as_uint(f);
  if (back != d && d == d) {
    if (fabs(back) > fabs(d)) --u;
    u |= 1u;
  }
  return __uint_as_float(u);
}

template <int DT>
struct Octet;  // 8 consecutive elements as they lie in memory
template <>
struct Octet<VP_BF16> {
  uint4 u;
  __device__ __forceinline__ void load(const char* p) { u = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void store(char* p) const { *reinterpret_cast<uint4*>(p) = u; }
  __device__ __forceinline__ float get(int i) const {
    const uint32_t w = i < 2 ? u.x : i < 4 ? u.y : i < 6 ? u.z : u.w;
    return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
  }
  __device__ __forceinline__ void set(const float (&x)[8]) {
    auto two = [&](int i) { return f32_to_bf16_bits(x[i]) | static_cast<uint32_t>(f32_to_bf16_bits(x[i + 1])) << 16; };
    u = make_uint4(two(0), two(2), two(4), two(6));
  }
};
template <>
struct Octet<VP_F32> {
  float4 a, b;
  __device__ __forceinline__ void load(const char* p) {
    a = reinterpret_cast<const float4*>(p)[0];
    b = reinterpret_cast<const float4*>(p)[1];
  }
  __device__ __forceinline__ void store(char* p) const {
    reinterpret_cast<float4*>(p)[0] = a;
    reinterpret_cast<float4*>(p)[1] = b;
  }
  __device__ __forceinline__ float get(int i) const {
    switch (i) {
      case 0: return a.x;
      case 1: return a.y;
      case 2: return a.z;
      case 3: return a.w;
      case 4: return b.x;
      case 5: return b.y;
      case 6: return b.z;
      default: return b.w;
    }
  }
  __device__ __forceinline__ void set(const float (&x)[8]) {
    a = make_float4(x[0], x[1], x[2], x[3]);
    b = make_float4(x[4], x[5], x[6], x[7]);
  }
};

// The sequence whose tokens the offsets off[0 .. B] put `token` in: the number of entries
// off[1 ..] that are not above it (found by all lanes of a wave, 64 probes a round); >= B: none.
__device__ __forceinline__ int sequence_of(const int32_t* off, int B, int token, int lane) {
  int lo = 0, n = B;  // entries off[1 .. lo] are not above it, one of the next n may be
  while (n > 64) {
    const int step = (n + 63) / 64;
    const int i = (lane + 1) * step;
    const int c = __builtin_popcountll(__builtin_amdgcn_ballot_w64(i <= n && off[lo + i] <= token));
    lo += c * step;
    n = min(step, n - c * step);
  }
  return lo + __builtin_popcountll(__builtin_amdgcn_ballot_w64(lane < n && off[lo + 1 + lane] <= token));
}

// cosines and sines of a lane's elements: those of its 8 pairs, or (neighbours paired) 4 pairs,
// in two parts of 4 pairs, which have one axis each
struct Turn {
  float c[8], s[8];
};

__device__ __forceinline__ int pair_of(const AppendArgs& a, int octet, int part) {
  const int half = a.rot >> 1;
  if (a.interleaved) return 4 * octet;  // (both parts the same)
  return (8 * octet >= half ? 8 * octet - half : 8 * octet) + 4 * part;
}

__device__ __forceinline__ int position_of(const AppendArgs& a, int octet, int part, int token) {
  const int pair = pair_of(a, octet, part);
  int axis = 0;
  for (int x = 0; x + 1 < a.axes; ++x) axis += pair >= a.section_end[x];
  return a.pos[static_cast<int64_t>(axis) * a.n_tokens + token];
}

__device__ __forceinline__ void load_turn(const AppendArgs& a, Turn& t, int octet, const int (&pos)[2]) {
  const int half = a.rot >> 1;
#pragma unroll
  for (int part = 0; part < 2; ++part) {
    const int p = min(max(pos[part], 0), a.n_pos - 1);
    const float* src = a.cos_sin + static_cast<int64_t>(p) * a.rot + pair_of(a, octet, part);
    const float4 c = *reinterpret_cast<const float4*>(src);
    const float4 s = *reinterpret_cast<const float4*>(src + half);
    t.c[4 * part + 0] = c.x;
    t.c[4 * part + 1] = c.y;
    t.c[4 * part + 2] = c.z;
    t.c[4 * part + 3] = c.w;
    t.s[4 * part + 0] = s.x;
    t.s[4 * part + 1] = s.y;
    t.s[4 * part + 2] = s.z;
    t.s[4 * part + 3] = s.w;
  }
}

// Element i of a lane's 8, rotated. x: its elements, y: their partners' (halves paired: a
// lane of the upper half adds, one of the lower half subtracts).
template <int DT>
__device__ __forceinline__ double turned(const AppendArgs& a, const Turn& t, const Octet<DT>& x, const Octet<DT>& y,
                                         bool upper, int i) {
  double p, q, c, s;
  if (a.interleaved) {
    p = x.get(i);
    q = x.get(i ^ 1);
    c = t.c[i >> 1];
    s = i & 1 ? t.s[i >> 1] : -t.s[i >> 1];
  } else {
    p = x.get(i);
    q = y.get(i);
    c = t.c[i];
    s = upper ? t.s[i] : -t.s[i];
  }
  return fma(q, s, p * c);
}

// 8 elements (those of 4 neighbouring lanes make a block) as 8 codes; byte: the block's scale
__device__ __forceinline__ uint32_t to_4bit(const float (&x)[8], uint32_t& byte) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
  top = group_allreduce_u32(top, 4, [](uint32_t p, uint32_t q) { return max(p, q); });
  if (top >= 0x7f800000u) {
    byte = kScaleNan;
    return 0;
  }
  // max = 1.m 2^E <= 7 2^e = 1.75 2^(e + 2)
  const int e = static_cast<int>(top >> 23) - 2 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
  byte = static_cast<uint32_t>(min(max(e, kScaleMin), kScaleMax));
  const float scale = __uint_as_float(byte << 23);
  uint32_t u = 0;
  u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, x[0], x[1], scale, 0);
  u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, x[2], x[3], scale, 1);
  u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, x[4], x[5], scale, 2);
  u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, x[6], x[7], scale, 3);
  return u;
}

template <int DT, int D, bool FOUR>
__global__ __launch_bounds__(64 * kAppendWaves) void append_kernel(const AppendArgs a) {
  constexpr int ESZ = DT == VP_BF16 ? 2 : 4;
  constexpr int LANES = D / 8;      // lanes of a row
  constexpr int ROWS = 64 / LANES;  // rows of a wave
  constexpr int BATCH = 3;  // rows of a lane whose loads are in flight together
  read_early(a.k, a.four.vc, a.block_table, a.cos_sin);
  const int lane = threadIdx.x & 63;
  const int64_t id = static_cast<int64_t>(blockIdx.x) * kAppendWaves + __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  if (id >= static_cast<int64_t>(a.n_tokens) * a.waves) return;
  const int token = static_cast<int>(id / a.waves);
  const int first = static_cast<int>(id - static_cast<int64_t>(token) * a.waves) * ROWS;

  const int octet = lane % LANES;
  const bool turns = 8 * octet < a.rot;
  const int half = a.rot >> 1;
  const bool upper = 8 * octet >= half;
  const int partner = !turns || a.interleaved ? octet : upper ? octet - half / 8 : octet + half / 8;
  const int Hq = a.q ? a.Hq : 0;
  const int rows = Hq + 2 * a.Hkv;
  const int step = a.waves * ROWS;
  const char* const qs = static_cast<const char*>(a.q) + token * a.qs;
  const char* const ks = static_cast<const char*>(a.k) + token * a.ks;
  const char* const vs = static_cast<const char*>(a.v) + token * a.vs;
  Octet<DT> x[BATCH], y[BATCH];
  auto load = [&](int r0) {
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
      const int r = min(r0 + j * step, rows - 1);
      const bool key = r < Hq + a.Hkv;
      const char* src = r < Hq ? qs + r * (D * ESZ) : key ? ks + (r - Hq) * (D * ESZ) : vs + (r - Hq - a.Hkv) * (D * ESZ);
      x[j].load(src + octet * (8 * ESZ));
      y[j].load(src + (key ? partner : octet) * (8 * ESZ));
    }
  };
  // Requested together, in the order of their use: the offsets (up to 64 sequences: one of
  // each lane), the positions, the first rows
  const bool few = a.B <= 64;
  int end = 0x7fffffff;
  if (a.new_off && few && lane < a.B) end = a.new_off[1 + lane];
  int pos[2] = {0, 0};
  if (turns && a.pos) {
    pos[0] = position_of(a, octet, 0, token);
    pos[1] = position_of(a, octet, 1, token);
  }
  load(first + lane / LANES);

  // the token's sequence and row
  int b, i, n;
  if (a.new_off) {
    b = few ? __builtin_popcountll(__builtin_amdgcn_ballot_w64(end <= token)) : sequence_of(a.new_off, a.B, token, lane);
    if (b >= a.B) return;  // (behind the last sequence)
    const int64_t o = a.new_off[b];
    const int64_t len = a.new_off[b + 1] - o;
    if (token < o || token - o >= len || len > a.n_tokens) return;
    i = static_cast<int>(token - o);
    n = static_cast<int>(len);
  } else {
    b = token / a.T;
    i = token - b * a.T;
    n = a.T;
  }
  const int row = clamp_len(a.seq_len[b], a.max_seq_len) - n + i;
  if (row < 0) return;
  int64_t at = b;  // sequence, or block
  int in = row;    // row in it
  if (a.block_table) {
    at = a.block_table[static_cast<int64_t>(b) * a.nblk + (row >> a.bs_log2)];
    in = row & ((1 << a.bs_log2) - 1);
  }
  if (!a.pos) pos[0] = pos[1] = row;
  Turn turn{};
  if (turns) load_turn(a, turn, octet, pos);

  for (int r0 = first + lane / LANES;;) {
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
      const int r = r0 + j * step;
      if (r >= rows) break;
      const bool value = r >= Hq + a.Hkv;
      const int h = r < Hq ? r : value ? r - Hq - a.Hkv : r - Hq;
      const bool turn_it = turns && !value;
      if (FOUR && r >= Hq) {
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = turn_it ? to_odd(turned<DT>(a, turn, x[j], y[j], upper, i)) : x[j].get(i);
        uint32_t byte;
        const uint32_t codes = to_4bit(f, byte);
        // the row's scales meet in its first lane
        uint32_t all = byte << 8 * (octet >> 2);
        all |= static_cast<uint32_t>(__shfl_xor(static_cast<int>(all), 4));
        if constexpr (D == 128) all |= static_cast<uint32_t>(__shfl_xor(static_cast<int>(all), 8));
        uint8_t* cd = (value ? a.four.vc : a.four.kc) + at * a.four.cb + h * a.four.ch + static_cast<int64_t>(in) * (D / 2);
        uint8_t* sd = (value ? a.four.vs : a.four.ks) + at * a.four.sb + h * a.four.sh + static_cast<int64_t>(in) * (D / 32);
        reinterpret_cast<uint32_t*>(cd)[octet] = codes;
        if (octet == 0) {
          if constexpr (D == 128) *reinterpret_cast<uint32_t*>(sd) = all;
          else *reinterpret_cast<uint16_t*>(sd) = static_cast<uint16_t>(all);
        }
      } else {
        if (turn_it) {
          float f[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) f[i] = static_cast<float>(turned<DT>(a, turn, x[j], y[j], upper, i));
          x[j].set(f);
        }
        char* dst;
        if (r < Hq) dst = static_cast<char*>(a.q_out) + (static_cast<int64_t>(token) * Hq + h) * (D * ESZ);
        else dst = static_cast<char*>(value ? a.V : a.K) + at * a.sb + h * a.sh + in * a.ss;
        x[j].store(dst + octet * (8 * ESZ));
      }
    }
    r0 += BATCH * step;
    if (r0 - lane / LANES >= rows) break;
    load(r0);
  }
}

template <int DT, int D>
hipError_t launch_dd(const AppendArgs& a, bool four, hipStream_t st) {
  const int64_t waves = static_cast<int64_t>(a.n_tokens) * a.waves;
  const dim3 grid(static_cast<unsigned>((waves + kAppendWaves - 1) / kAppendWaves));
  if (four) hipLaunchKernelGGL((append_kernel<DT, D, true>), grid, dim3(64 * kAppendWaves), 0, st, a);
  else hipLaunchKernelGGL((append_kernel<DT, D, false>), grid, dim3(64 * kAppendWaves), 0, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_append(const AppendArgs& in, bool four, int dtype, int head_dim, hipStream_t st) {
  AppendArgs a = in;
  if (a.n_tokens == 0) return hipSuccess;
  // A token's rows go to as many waves as fill the GPU, up to one per 512 elements (a batch), and
  // with many tokens to one wave per 6 batches, rounded down (two to four rounds of the loop,
  // 3 batches each). 10k tokens of 72B-class heads in bf16, 20 batches: 3 waves 85.6 us, 4 (rounded
  // up) 84.8, 7 101, one 88; in fp32 166, 162, 162, 172. 12.5k of 28/4 heads into 4 bits, 9
  // batches: one wave 50.4, 2 (rounded up) 55.7, 3 57.6. At most 2^26 waves in all.
  const int batches = ((a.q ? a.Hq : 0) + 2 * a.Hkv + 512 / head_dim - 1) / (512 / head_dim);
  const int64_t fill = std::max<int64_t>(8192 / a.n_tokens, batches / 6);
  a.waves = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({batches, fill, (1 << 26) / a.n_tokens})));
  if (dtype == VP_BF16) return head_dim == 128 ? launch_dd<VP_BF16, 128>(a, four, st) : launch_dd<VP_BF16, 64>(a, four, st);
  return head_dim == 128 ? launch_dd<VP_F32, 128>(a, four, st) : launch_dd<VP_F32, 64>(a, four, st);
}

}  // namespace vp
