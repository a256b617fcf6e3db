// Rows in 4 bits (include/wkv.h, WKV_KV4): how they lie in a page, how a row becomes codes and what a code stands for.
//
// 32 neighbouring channels of a row share a scale s and a zero point z; a code n in 0..15 stands for s (n - z).  The scale has four
// significant bits and is held as the upper eight of the fifteen magnitude bits of an fp16 number, so that s (n - z), 4 + 4 bits, is a
// bf16 and an fp16 number as it stands: prompts that attend to spread-out rows see what a decode step sees.
#pragma once
#include <cuda_fp16.h>

#include "wkv_paged.cuh"

namespace wkv {

constexpr int kKv4Group = 32;
constexpr float kKv4Least = 0x1p-17f, kKv4Most = 4096.f;   // scales

// A chunk (one kv head's rows of one page): page rows of codes, then page rows of (scale byte, zero byte) pairs.
template <int D>
struct Kv4Row {
  static constexpr int kCodes = D / 2;                     // bytes
  static constexpr int kGroups = D / kKv4Group;
  static constexpr int kPairs = 2 * kGroups;               // bytes
  static constexpr int kBytes = kCodes + kPairs;
  // Keys: a group's 16 bytes are a piece; word w of it holds channels 8w .. 8w+7, the even ones in its low half (4 bits each, lowest
  // first), the odd ones in its high half: a masked word is two fp16 lanes of neighbouring channels.  Pieces are exchanged so that
  // eight rows' pieces of one group lie on different banks.
  __device__ __forceinline__ static int k_piece(int row, int g) {
    return row * kCodes + ((g ^ (D == 128 ? (row >> 1) & 3 : (row >> 2) & 1)) << 4);
  }
  // Values: 16-bit units of four neighbouring channels, unit r of every group side by side: the four channels of all groups that one
  // lane of a matrix instruction owns are one load.  Halves of a row are exchanged so that four rows' loads lie on different banks.
  __device__ __forceinline__ static int v_unit(int row, int g, int r) {
    return row * kCodes + ((r * 2 * kGroups + 2 * g) ^ (D == 128 ? ((row >> 1) & 1) << 5 : 0));
  }
  __device__ __forceinline__ static int pairs(int page, int row) { return page * kCodes + row * kPairs; }
};

__device__ __forceinline__ float kv4_scale(uint32_t byte) { return __half2float(__ushort_as_half((unsigned short)(byte << 7))); }

// Scale and zero point of a group with least value lo <= 0 and largest hi >= 0.
struct Kv4Scale {
  uint32_t byte, zero;
  float s, inv, z;
};
__device__ __forceinline__ Kv4Scale kv4_scale_of(float lo, float hi) {
  Kv4Scale q;
  const float r = __fmul_rn(__fsub_rn(hi, lo), 1.f / 15.f);
  // up to the next number of four significant bits, or below 2^-14 the next multiple of 2^-17; a NaN ends at the largest scale
  float s = r < 0x1p-14f ? ceilf(r * 0x1p17f) * 0x1p-17f : __uint_as_float((__float_as_uint(r) + 0xfffffu) & 0xfff00000u);
  s = fminf(fmaxf(s, kKv4Least), kKv4Most);
  if (!(r < kKv4Most)) s = kKv4Most;
  q.s = s;
  q.byte = s < 0x1p-14f ? (uint32_t)(s * 0x1p17f) : (__float_as_uint(s) >> 20) - (112u << 3);
  q.inv = __frcp_rn(s);
  q.z = fminf(fmaxf(rintf(__fmul_rn(-lo, q.inv)), 0.f), 15.f);
  q.zero = (uint32_t)q.z;
  return q;
}
__device__ __forceinline__ uint32_t kv4_code(float x, const Kv4Scale& q) {
  return (uint32_t)fminf(fmaxf(__fadd_rn(rintf(__fmul_rn(x, q.inv)), q.z), 0.f), 15.f);
}

}  // namespace wkv
