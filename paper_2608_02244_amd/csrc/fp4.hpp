// The 4-bit cache: elements e2m1 (+-{0, 0.5, 1, 1.5, 2, 3, 4, 6}) with one scale 2^e for 32
// neighbours of a head, held as the byte e + 127 (255: the block holds what is not finite).
//
// 16 tokens of one head of a page are a group, 17 D bytes in one piece:
//   key codes     [16 tokens][D/2]           byte i of a token: elements 2i (low), 2i + 1
//   value codes   [4][16 pieces][4 tokens][D/32]  a piece is D/16 neighbouring elements
//   key scales    [16 tokens][D/32]
//   value scales  [4][D/32][4 tokens]
// Values lie so that what a lane of the second product's operand needs (the same D/16
// elements of four tokens) is one load; a token still has whole bytes to itself, so tokens
// of one group may be stored by different waves.  16 tokens of a D of 128 are 17 lines of
// 128 bytes.
#pragma once
#include "half.hpp"

namespace fs {

constexpr int GROUP_SHIFT = 4, GROUP = 1 << GROUP_SHIFT;

template <int D>
struct Group4 {
  static constexpr int VALUES = 8 * D, KEY_SCALES = 16 * D, VALUE_SCALES = 16 * D + D / 2,
                       BYTES = 17 * D;
  static constexpr int BLOCKS = D / 32;  // scales of a token
  static constexpr int PIECE = D / 32;   // bytes of a token in a piece of the values
  // byte offsets of token t: its key codes, its part of value piece n, the scales of block b
  __device__ static int key(int t) { return t * (D / 2); }
  __device__ static int value(int t, int n) {
    return VALUES + (((t >> 2) * 16 + n) * 4 + (t & 3)) * PIECE;
  }
  __device__ static int key_scale(int t, int b) { return KEY_SCALES + t * BLOCKS + b; }
  __device__ static int value_scale(int t, int b) {
    return VALUE_SCALES + ((t >> 2) * BLOCKS + b) * 4 + (t & 3);
  }
};

// Exponents of the scales: all values of a block are normal numbers of the element type, or
// f16's smallest ones (0.5 * 2^-23), and none exceeds its largest (6 * 2^13).
template <class T>
constexpr int LEAST_SCALE = __is_same(T, F16) ? 127 - 23 : 127 - 125;
template <class T>
constexpr int MOST_SCALE = __is_same(T, F16) ? 127 + 13 : 127 + 125;

// The scale byte of a block whose largest magnitude has these bits (32-bit float, sign
// cleared): the least 2^e with |x| <= 6 2^e.  6 2^e = 1.5 2^(e + 2), so e + 2 is the
// exponent of |x|, or one more where its mantissa is above 1.5 (the carry).
template <class T>
__device__ __forceinline__ int scale_byte(uint32_t bits) {
  if (bits >= 0x7f800000u) return 255;
  const int e = (int)((bits + 0x3fffffu) >> 23) - 2;
  return min(max(e, LEAST_SCALE<T>), MOST_SCALE<T>);
}

__device__ __forceinline__ float scale_of(uint32_t byte) {
  return __builtin_bit_cast(float, byte << 23);
}

// Eight numbers to eight codes of one scale, each rounded to nearest even.
__device__ __forceinline__ uint32_t codes8(const float* x, float scale) {
  uint32_t r = 0;
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[0], x[1], scale, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2], x[3], scale, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4], x[5], scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6], x[7], scale, 3);
}

// f of the whole numbers 0 .. N - 1 as types, for operands that have to be constants.
template <int I>
struct Const {
  static constexpr int value = I;
};
template <int N, int I = 0, class F>
__device__ __forceinline__ void each(F f) {
  if constexpr (I < N) {
    f(Const<I>{});
    each<N, I + 1>(f);
  }
}

// Byte SEL of a dword of codes to two elements.
template <class T, int SEL>
__device__ __forceinline__ uint32_t values2(uint32_t codes, float scale) {
  if constexpr (__is_same(T, Bf16))
    return __builtin_bit_cast(uint32_t,
                              __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, SEL));
  else
    return __builtin_bit_cast(uint32_t,
                              __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, SEL));
}

template <class T>
__device__ __forceinline__ u32x4 values8(uint32_t codes, float scale) {
  return (u32x4){values2<T, 0>(codes, scale), values2<T, 1>(codes, scale),
                 values2<T, 2>(codes, scale), values2<T, 3>(codes, scale)};
}

// A 64-bit number to 32 bits so that rounding it again to fewer bits gives what rounding the
// number itself gives: towards zero, the last bit set where something was cut off.
__device__ __forceinline__ float to_odd(double x) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint32_t hi = (uint32_t)(b >> 32), lo = (uint32_t)b;
  const uint32_t e = (hi >> 20) & 0x7ff;
  uint32_t r;
  if (e - 897u < 254u) {  // a normal number of 32 bits: exponent and mantissa from the 64
    r = (hi & 0x80000000u) | (((hi & 0x7fffffffu) << 3 | lo >> 29) - (896u << 23));
    r |= (lo & 0x1fffffffu) != 0;
  } else {
    const float f = (float)x;
    r = __builtin_bit_cast(uint32_t, f);
    if (fabs((double)f) > fabs(x)) --r;
    if ((double)__builtin_bit_cast(float, r) != x) r |= 1;
  }
  return __builtin_bit_cast(float, r);
}

}  // namespace fs
