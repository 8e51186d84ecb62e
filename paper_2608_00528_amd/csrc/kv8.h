// The 8-bit KV cache: blocks of 64 tokens of one (sequence, KV head) with one
// fp32 scale per block and side, in the order the attention kernel's MFMA
// operands take them.
//
// A block is 64 * d_h contiguous bytes; 1 KiB pieces, one 16-byte load per lane.
//   keys    (t / 16, d / 64, (d % 64) / 16, t % 16, d % 16): lane l of a piece
//           holds token l % 16 and 16 dims of k-group l / 16;
//   values  (d / 16, (t % 16) / 4, d % 16, t % 4, t / 16): lane l holds dim
//           l % 16 and 16 tokens of k-group l / 16, the tokens 16 i + 4 (l / 16) + v
//           at byte 4 v + i, which is how the logits' MFMA leaves the softmax
//           weights in the lanes (row l % 16, tokens 4 (l / 16) + v of subtile i).
#pragma once

#include "s4r_device.h"
#include "s4r_internal.h"

namespace s4r {

// the smallest block maximum that is stored; below it the block holds zeros (its
// scale and the scale's reciprocal stay normal fp32 numbers)
constexpr uint32_t kKv8MinBits = 0x12800000u;      // 2^-90

__device__ __forceinline__ int key_offset(int t, int d, int dh) {
  return (t >> 4) * (16 * dh) + (d >> 6) * 1024 + ((d & 63) >> 4) * 256 + (t & 15) * 16 + (d & 15);
}
__device__ __forceinline__ int value_offset(int t, int d) {
  return (d >> 4) * 1024 + ((t & 15) >> 2) * 256 + (d & 15) * 16 + (t & 3) * 4 + (t >> 4);
}

// scale of a block whose largest |value| has these bits (NaN where a value is
// not finite): int8 amax / 127 correctly rounded, e4m3 the smallest power of two
// with amax <= 448 * scale (a power of two leaves x / scale exact)
template <int FMT>
__device__ __forceinline__ float kv8_scale(uint32_t amax_bits) {
  if (amax_bits >= 0x7F800000u) return __uint_as_float(0x7FC00000u);
  if (amax_bits < kKv8MinBits) return 0.f;
  if (FMT == S4R_KV_INT8) return __fdiv_rn(__uint_as_float(amax_bits), 127.f);
  // 448 = 1.75 * 2^8: exponent of amax less 8, one more where the mantissa is above 1.75
  const uint32_t e = (amax_bits >> 23) - 8u + ((amax_bits & 0x7FFFFFu) > 0x600000u ? 1u : 0u);
  return __uint_as_float(e << 23);
}
// reciprocal used by the codes (0 where the block holds no values)
template <int FMT>
__device__ __forceinline__ float kv8_inverse(float s) {
  if (!(s > 0.f)) return 0.f;
  if (FMT == S4R_KV_INT8) return __fdiv_rn(1.f, s);
  return __uint_as_float((254u << 23) - __float_as_uint(s));   // 2^-e
}

// int8 codes of four numbers, little endian: the nearest integers to x / s, ties to
// even, exactly.  fma(x, 1 / s, 1.5 * 2^23) rounds to an integer n in one step (its low
// byte is the code) and is off by at most one, next to a tie only; the remainder
// x - n s is exact in one fma (a multiple of ulp(s) / 2 no larger than s), so `worst`,
// the largest |remainder|, says whether any of the numbers has to be looked at again:
// about one in 10^5 does.
constexpr float kKv8Round = 12582912.f;
typedef uint32_t kv8_u4 __attribute__((ext_vector_type(4)));
typedef uint32_t kv8_u2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t kv8_low_bytes(float a, float b, float c, float d) {
  const uint32_t ab = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x0C0C0400u);
  const uint32_t cd = __builtin_amdgcn_perm(__float_as_uint(d), __float_as_uint(c), 0x04000C0Cu);
  return ab | cd;
}
__device__ __forceinline__ uint32_t kv8_int8x4(float a, float b, float c, float d, float s, float inv, float& worst) {
  const float x[4] = {a, b, c, d};
  float n[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    n[i] = fmaf(x[i], inv, kKv8Round);
    worst = fmaxf(worst, fabsf(fmaf(kKv8Round - n[i], s, x[i])));
  }
  return kv8_low_bytes(n[0], n[1], n[2], n[3]);
}
// the same with every remainder looked at: past the middle, or on it with n odd,
// the neighbour is the nearest (or the even one)
__device__ __forceinline__ uint32_t kv8_int8x4_exact(float a, float b, float c, float d, float s, float inv) {
  const float x[4] = {a, b, c, d};
  float n[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    n[i] = fmaf(x[i], inv, kKv8Round);
    const float e = fmaf(kKv8Round - n[i], s, x[i]), h = 0.5f * s;
    if (fabsf(e) > h || (fabsf(e) == h && (__float_as_uint(n[i]) & 1u))) n[i] += e > 0.f ? 1.f : -1.f;
  }
  return kv8_low_bytes(n[0], n[1], n[2], n[3]);
}
__device__ __forceinline__ uint32_t kv8_e4m3x4(float a, float b, float c, float d, float inv) {
  const int v = __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, v, true);
}
// 4 x 4 bytes turned: byte i of r[j] from byte j of w[i]
__device__ __forceinline__ void kv8_turn4(const uint32_t* w, uint32_t* r) {
  const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), b = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u),
                 c = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u), d = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
  r[0] = __builtin_amdgcn_perm(c, a, 0x05040100u);
  r[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
  r[2] = __builtin_amdgcn_perm(d, b, 0x05040100u);
  r[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
}
// the four numbers that a dword of codes stands for, before the scale
typedef float kv8_f2 __attribute__((ext_vector_type(2)));
template <int FMT>
__device__ __forceinline__ void kv8_numbers(uint32_t w, float (&x)[4]) {
  if (FMT == S4R_KV_INT8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (float)(int)(int8_t)(w >> (8 * i));
  } else {
    const kv8_f2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    x[0] = lo[0];
    x[1] = lo[1];
    x[2] = hi[0];
    x[3] = hi[1];
  }
}

// rows a call writes to or reads from sequence b: [start, start + count), none (and
// start 0, so no block lies before the first row) where there are none or they do not
// lie inside the cache
__device__ __forceinline__ void kv8_rows(const int32_t* starts, const int32_t* counts, int b, int64_t row0, int n_rows,
                                         int64_t cap, int64_t& start, int& count) {
  start = starts ? (int64_t)starts[b] : row0;
  count = counts ? min(max(counts[b], 0), n_rows) : n_rows;
  if (count == 0 || start < 0 || start + count > cap) start = 0, count = 0;
}

}  // namespace s4r
