// The K/V cache held in 4 bits: layout, scales and codes.
//
// 32 consecutive dims of a head at one position are a group: one scale and 32
// codes.  A code is a sign and one of 0, 1/2, 1, 3/2, 2, 3, 4, 6 (E2M1, which
// this GPU converts two at a time in one instruction); a value is code times
// scale.  A scale has at most 6 significant bits, is a multiple of 2^-23 and at
// most 10,752: every value then has 8 significant bits, is a multiple of 2^-24
// and at most 64,512, so it is exact in fp32, bf16 and fp16 alike, and a product
// of a code and a 16-bit operand is exact in an MFMA with the scale left out.
//
// A block of 64 positions of a KV head is 72 hd bytes, J = hd / 32 groups a row:
//   K codes   [64][hd / 2]      byte 4 J i + 4 j + b of a row holds dims 32 j + 8 i
//                               + 2 b (low half) and the next, i, b < 4, j < J
//   K scales  [64][J]           fp16
//   V codes   [16][hd / 8][4]   words: of positions 4 n .. 4 n + 3 the words w = 0 ..,
//                               each of the four positions side by side.  Byte J r + j
//                               of a position's hd / 2 bytes holds dims 32 j + 2 r and
//                               the next, r < 16
//   V scales  [J][64]           fp16
// A position's K and V are whole words and halves of its own, so that a row is
// written without reading what is beside it.  The orders are those of the matrix
// operands: a lane's piece of a K row is 8 dims of each group (MFMA j is group
// j's product), its words of V hold the same two dims of each group.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device.hpp"

namespace lp {

template <int HD>
struct Kv4 {
  static constexpr int J = HD / 32;
  static constexpr int K_SCALES = 32 * HD, V_CODES = 36 * HD, V_SCALES = 68 * HD, BYTES = 72 * HD;
  // byte offsets inside a block's head
  static __host__ __device__ constexpr int k_row(int p) { return p * (HD / 2); }
  static __host__ __device__ constexpr int k_scale(int p, int j) { return K_SCALES + (p * J + j) * 2; }
  static __host__ __device__ constexpr int v_word(int p, int w) {
    return V_CODES + ((p / 4 * (HD / 8) + w) * 4 + p % 4) * 4;
  }
  static __host__ __device__ constexpr int v_scale(int p, int j) { return V_SCALES + (j * 64 + p) * 2; }
};

// A group's scale from the bits of its largest magnitude: the least number of 6
// significant bits and steps of 2^-23 that is not below a sixth of it; NaN for
// an infinity or NaN.  The division is the correctly rounded one, which reaches
// a number of 6 bits only where the quotient is one; where it is 0 but the magnitude
// is not, 2^-149 stands for it, whose scale is the same.
__device__ __forceinline__ float kv4_scale(uint32_t amax) {
  if (amax >= 0x7F800000u) return __uint_as_float(0x7FC00000u);
  const float t = __uint_as_float(max(__float_as_uint(__uint_as_float(amax) / 6.0f), min(amax, 1u)));
  const float s = t < 0x1p-18f ? ceilf(t * 0x1p23f) * 0x1p-23f
                               : __uint_as_float((__float_as_uint(t) + 0x3FFFFu) & ~0x3FFFFu);
  return fminf(s, 10752.f);
}

// The code of x under the scale s: the nearest magnitude, of two equally near
// ones the even code; past 6 s, 6.  The borders are products of 6 and 3 bits, so
// the comparisons decide exactly.  A NaN scale, and one of 0 (its group is all
// zeros), leaves the sign alone.
__device__ __forceinline__ uint32_t kv4_code(float x, float s) {
  const float a = s > 0.f ? fabsf(x) : 0.f;
  const bool b2 = a >= 1.75f * s;
  const bool b1 = a >= (b2 ? 3.5f : 0.75f) * s;
  const float mid = b1 ? (b2 ? 5.f : 1.25f) : (b2 ? 2.5f : 0.25f);
  const uint32_t c = (b2 ? 4u : 0u) | (b1 ? 2u : 0u) | (a > mid * s ? 1u : 0u);
  return (s > 0.f ? c : 0u) | (__float_as_uint(x) >> 31 << 3);
}

// Two codes (byte B of w, the low half first) as two numbers.
template <typename T, int B>
__device__ __forceinline__ uint32_t kv4_pair16(uint32_t w) {
  if constexpr (std::is_same_v<T, bf16_t>)
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, B));
  else
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, B));
}
typedef float f32x2_t __attribute__((ext_vector_type(2)));
template <int B>
__device__ __forceinline__ f32x2_t kv4_pair32(uint32_t w) {
  return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, B);
}

}  // namespace lp
