// The 8-bit forms of a K or V row (the s numbers of one token and key/value head), shared by the kernels that write pages
// of them, read them back and attend over them.  With a = max |x_d| over the row:
//   e4m3  scale c = 2^e, e the least integer >= -100 with a <= 448 2^e;   values RNE(x_d / c)
//   int8  scale c = the least bf16 >= a / 127, at least 2^-100;           values RNE(x_d / c), |.| <= 127
// a = 0: c = 1.  An infinity or a NaN in the row: c = NaN, values 0; the row stands for NaN throughout.
// A value has at most 7, a scale at most 8 significant bits, so what a row stands for (value * c) is exact in fp32 (but for the
// e4m3 numbers from 248 2^120 on, which round to 256 2^120 = 2^128).
// (The least scale keeps every product above the numbers that bf16 and fp32 hold with fewer bits.)
//
// Pages: K [num_blocks, n_kv, 16, s] as the bf16 cache has them; V [num_blocks, n_kv, s, 16], a feature's 16 tokens
// together: the attention's second product contracts over tokens, and a lane's operand for it is then one 16-byte load.
// (With V as K is, that operand has to be turned through LDS for each step; here it is turned once, when written.)
// Scales [num_blocks, n_kv, 16] bf16.
#pragma once
#include "common.h"
#include "kernels.h"

namespace ds {

constexpr int kKvPage = 16;
constexpr uint32_t kBf16NaN = 0x7fc0u;

// a's bf16 bits without the sign (0x7f80 and above: not finite) -> the scale's bf16 bits
template <int T>
__device__ __forceinline__ uint32_t scale_bits(uint32_t a) {
  uint32_t c;
  if constexpr (T == kKvE4m3) {
    // a = (1 + m / 128) 2^(f - 127) and 448 = 1.75 2^8: e + 127 = f - 8, one more if m / 128 > 3/4
    const int f = (int)(a >> 7) - 8 + ((a & 0x7fu) > 0x60u ? 1 : 0);
    c = (uint32_t)max(f, 127 - 100) << 7;
  } else {
    // rounded up: bits of the fp32 quotient behind the bf16 ones are 0 only if it is a bf16 itself (a / 127 with 8
    // significant bits in a is either one or at least 2^-15 of itself away from all of them)
    const uint32_t q = __float_as_uint(__uint_as_float(a << 16) / 127.f);
    c = max((q >> 16) + ((q & 0xffffu) ? 1u : 0u), (uint32_t)(127 - 100) << 7);
  }
  if (a == 0) c = 0x3f80u;
  return a >= 0x7f80u ? kBf16NaN : c;
}

// 1 / c for quantise4 (0 for a row that stands for NaN: its values are 0)
__device__ __forceinline__ float scale_inverse(uint32_t c) { return c == kBf16NaN ? 0.f : 1.f / __uint_as_float(c << 16); }

// Four bf16 (two packed pairs) -> four 8-bit values, the first in bits 0..7.
// int8: x / c has to be rounded as the exact quotient is.  q = x (1/c) is off by two units in the last place at most; the
// remainder x - q c, exact in one fma, corrects it, so that a quotient that lies on a half stays there (ties go to even),
// and one that does not is 2^-10 away from it (numbers of 8 significant bits).  Adding 1.5 2^23 rounds to whole numbers and
// leaves them in the low byte.
template <int T>
__device__ __forceinline__ uint32_t quantise4(uint32_t x01, uint32_t x23, uint32_t c, float inv) {
  const float x[4] = {bf16_lo(x01), bf16_hi(x01), bf16_lo(x23), bf16_hi(x23)};
  if (c == kBf16NaN) return 0;
  if constexpr (T == kKvE4m3) {  // (1 / c is a power of two: the products are exact)
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * inv, x[1] * inv, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2] * inv, x[3] * inv, w, true);
  } else {
    const float cf = __uint_as_float(c << 16);
    uint32_t b[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float q = x[j] * inv;
      q = fmaf(fmaf(-q, cf, x[j]), inv, q);
      b[j] = __float_as_uint(q + 12582912.f);
    }
    const uint32_t lo = __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(b[3], b[2], 0x04000c0cu);
    return lo | hi;
  }
}

// Four 8-bit values as two packed pairs of bf16, without their scale (exact).
template <int T>
__device__ __forceinline__ u32x2 values4(uint32_t w) {
  u32x2 r;
  if constexpr (T == kKvE4m3) {
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true));
  } else {  // whole numbers up to 127: the upper half of the fp32 is the bf16
    uint32_t f[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = __float_as_uint((float)(int)(int8_t)(w >> (8 * j)));
    r[0] = __builtin_amdgcn_perm(f[1], f[0], 0x07060302u);
    r[1] = __builtin_amdgcn_perm(f[3], f[2], 0x07060302u);
  }
  return r;
}

// 4 x 4 bytes: byte j of w[i] <-> byte i of w[j].
__device__ __forceinline__ void turn_bytes(uint32_t (&w)[4]) {
  // pairs of rows, then pairs of pairs
  const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), b = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u);
  const uint32_t c = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u), d = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
  w[0] = __builtin_amdgcn_perm(c, a, 0x05040100u);
  w[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
  w[2] = __builtin_amdgcn_perm(d, b, 0x05040100u);
  w[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
}
// Lanes 0..31 of b <-> lanes 32..63 of a; and the same between the two rows of 16 lanes in either half.  Their own inverses.
__device__ __forceinline__ void swap32(uint32_t& a, uint32_t& b) {
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  a = r[0];
  b = r[1];
}
__device__ __forceinline__ void swap16(uint32_t& a, uint32_t& b) {
  const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
  a = r[0];
  b = r[1];
}

}  // namespace ds
