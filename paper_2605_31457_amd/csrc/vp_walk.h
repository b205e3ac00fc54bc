// What the attention calls over a walk of 32-row tiles share (vp_window.hip, vp_kv4.hip):
// how the walks of a batch are dealt to work-groups, weights, rows of the output.
#pragma once

#include "vp_blocks.h"
#include "vp_cache.h"
#include "vp_common.h"
#include "vp_tile.h"

namespace vp {

constexpr int kWinWaves = 4;
constexpr int kWinThreads = 64 * kWinWaves;

// s_waitcnt operand: at most n vector memory operations left (n < 64), others unconstrained
constexpr int wait_vm(int n) { return kWaitVm0 | (n & 15) | (n >> 4) << 14; }

// A float to the stage. Written by hand, because the compiler may have any LDS store wait
// for all copies in flight (fp32 rows of 128, 8 x 16k with sums: 111 us, so 108). A wave's LDS
// accesses happen in order, so its reads of the stage need nothing else.
__device__ __forceinline__ void stage_store(float* p, float x) {
#ifdef __HIP_DEVICE_COMPILE__
  typedef __attribute__((address_space(3))) float lds_float;
  asm volatile("ds_write_b32 %0, %1" ::"v"((uint32_t)(uintptr_t)(lds_float*)p), "v"(x) : "memory");
#endif
}

inline size_t align256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

// 2^(c (z - m)) of products z and m, m at most a.raise below z: the difference first, so
// that the weight of the largest product is what it should be however large it is (in one
// fma, with m scaled and rounded, it is off by 2^(c m 2^-25): from 2^31 on out of range)
__device__ __forceinline__ float weight_of(const WindowArgs& a, float z, float m) { return fast_exp2((z - m) * a.zscale); }

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
__device__ __forceinline__ int query_of(const WindowArgs& a, int r) { return static_cast<int>(r * a.over_g >> 16); }
__device__ __forceinline__ size_t out_row(const WindowArgs& a, int b, int g, int r) {
  const int t = query_of(a, r);
  return (static_cast<size_t>(b) * a.T + t) * a.Hq + g * a.G + (r - t * a.G);
}

__device__ __forceinline__ WindowWalk walk_of(const WindowArgs& a, int b) {
  return WindowWalk(clamp_len(a.seq_len[b], a.max_seq_len), a.T, a.window, a.n_sink);
}

// How the walks of a batch are dealt to `groups` work-groups, found by every wave from
// the lengths (no barrier): a work-group takes about `share` tiles of one pair, so a pair
// of n tiles has ceil(n / share) of them, its parts. Up to 64 sequences have a lane each,
// one load of the lengths is all that is read, and share is about the least whose
// work-groups are not too many; more sequences have consecutive ones in every lane, and
// share is what always fits.
struct Deal {
  int b, g, part, parts;  // this work-group's sequence, KV head and part of parts; b < 0: none
  int L;                  // the sequence's length
  __device__ __forceinline__ Deal(const WindowArgs& a, int lane, int group) {
    const int per = (a.B + 63) / 64;
    const int i0 = lane * per, i1 = min(a.B, i0 + per);
    int len = 0, mine = 0;  // of a lane's sequences: the (one) length, their tiles
    if (per == 1) {
      len = i0 < i1 ? clamp_len(a.seq_len[i0], a.max_seq_len) : 0;
      mine = tiles(a, len);
    } else {
      mine = sum(a, i0, i1, [](int n) { return n; });
    }
    const int total = a.Hkv * __builtin_amdgcn_readlane(wave_incl_sum(mine), 63);
    const int pairs = a.Hkv * a.B;
    int share = (total + a.groups - 1) / a.groups, count = 0;
    share = max(share, kWinWaves);  // a tile per wave at least
    if (per == 1) {
      // (ends: a share of the longest walk gives every pair one part, and there are as many groups)
      for (;; share += max(1, share / 32)) {
        count = wave_incl_sum(split(mine, share));
        if (a.Hkv * __builtin_amdgcn_readlane(count, 63) <= a.groups) break;
      }
      mine = split(mine, share);
    } else {
      share = max(share, (total + a.groups - pairs - 1) / (a.groups - pairs));
      mine = sum(a, i0, i1, [&](int n) { return split(n, share); });
      count = wave_incl_sum(mine);
    }
    // count: parts of this lane's sequences and those before, for one KV head
    const bool here = a.Hkv * (count - mine) <= group && group < a.Hkv * count;
    const uint64_t found = __builtin_amdgcn_ballot_w64(here);
    b = -1;
    if (found == 0) return;
    const int src = __builtin_ctzll(found);
    int before = count - mine, at = i0, own = mine;
    if (per > 1 && here) {
      for (own = split(walk_of(a, at).n, share); group >= a.Hkv * (before + own); own = split(walk_of(a, at).n, share)) {
        before += own;
        ++at;
      }
    }
    b = __builtin_amdgcn_readlane(at, src);
    parts = __builtin_amdgcn_readlane(own, src);
    const int i = group - a.Hkv * __builtin_amdgcn_readlane(before, src);
    g = i / parts;
    part = i - g * parts;
    L = per == 1 ? __builtin_amdgcn_readlane(len, src) : clamp_len(a.seq_len[b], a.max_seq_len);
  }

 private:
  static __device__ __forceinline__ int tiles(const WindowArgs& a, int len) {
    return WindowWalk(len, a.T, a.window, a.n_sink).n;
  }
  static __device__ __forceinline__ int split(int n, int share) {
    return static_cast<int>((static_cast<unsigned>(n) + share - 1) / static_cast<unsigned>(share));
  }
  // f(tiles) over sequences i0 .. i1 - 1, four loads in flight
  template <typename F>
  static __device__ __forceinline__ int sum(const WindowArgs& a, int i0, int i1, F f) {
    int s = 0;
    for (int i = i0; i < i1; i += 4) {
      int n[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) n[j] = walk_of(a, min(i + j, a.B - 1)).n;
#pragma unroll
      for (int j = 0; j < 4; ++j) s += i + j < i1 ? f(n[j]) : 0;
    }
    return s;
  }
};

}  // namespace vp
