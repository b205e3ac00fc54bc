// 4-bit caches and the calls that fill caches (vp_append_kv, vp_append_kv4, vp_kv4_read,
// vp_kv4_decode_attn): host/device interface between the C ABI (vp_api.hip) and their kernels.
//
// A 4-bit row of d elements is d/2 bytes of codes (two elements a byte, the lower-numbered
// one in the low half; sign, two exponent bits, one mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6)
// and d/32 scale bytes, one for 32 elements: value = code * 2^(scale - 127).
#pragma once

#include "vp_cache.h"
#include "vp_internal.h"

namespace vp {

constexpr int kMaxAxes = 4;
// scales that are written: 2^-125 (smaller blocks' elements count in its steps) to 2^125
// (a block whose largest element exceeds 7 * 2^125 saturates at 6 * 2^125), so that every
// value of a row is zero or a normal number of 16 and 32 bits; and the mark of a block that
// held an infinity or NaN, all of whose elements read as NaN
constexpr int kScaleMin = 2, kScaleMax = 252, kScaleNan = 255;

// a 4-bit cache in device memory; strides in bytes, rows of a head one after another
struct Kv4Cache {
  uint8_t* kc;
  uint8_t* ks;
  uint8_t* vc;
  uint8_t* vs;
  int64_t cb, ch;  // codes: between sequences (paged caches: blocks), between KV heads
  int64_t sb, sh;  // scales
};

struct AppendArgs {
  const void* q;  // or null
  const void* k;
  const void* v;
  void* q_out;
  void* K;                     // caches of 16 or 32 bits, or
  void* V;
  Kv4Cache four;               // ... a 4-bit cache
  int64_t qs, ks, vs;          // bytes between tokens
  int64_t sb, sh, ss;          // KV strides in BYTES; paged caches: sb is the block stride
  const int32_t* block_table;  // paged caches: [B][nblk] physical blocks (else null)
  int bs_log2, nblk;
  const int32_t* seq_len;
  const int32_t* new_off;      // [B+1], or null: T tokens per sequence
  int B, Hq, Hkv, T, max_seq_len, n_tokens;
  // rotation
  const float* cos_sin;        // [n_pos][rot], or null: none
  const int32_t* pos;          // [axes][n_tokens], or null: the token's row
  int n_pos, rot, interleaved, axes;
  int section_end[kMaxAxes];   // pairs of axis a: section_end[a - 1] .. section_end[a] - 1
  int waves;                   // waves that share a token's rows
};
hipError_t launch_append(const AppendArgs& a, bool four, int dtype, int head_dim, hipStream_t st);

struct ReadArgs {
  Kv4Cache four;
  void* K;
  void* V;
  int64_t sb, sh, ss;          // KV strides in BYTES; paged caches: sb is the block stride
  const int32_t* block_table;  // paged caches: [B][nblk] physical blocks (else null)
  int bs_log2, nblk;
  const int32_t* seq_len;
  const int32_t* first;        // [B], or null: 0
  int B, Hkv, max_seq_len;
};
hipError_t launch_kv4_read(const ReadArgs& a, int dtype, int head_dim, hipStream_t st);

WindowPlan make_kv4_plan(const vp_shape& s, const vp_window& w);
// a: as for window attention (K, V, their strides and attn_sum are not used)
hipError_t launch_kv4_attention(const WindowArgs& a, const Kv4Cache& four, int dtype, int head_dim, hipStream_t st);

}  // namespace vp
