// 16-bit element types of the step's operators: conversions and packs.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fs {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct Bf16 {
  using elem = __bf16;
  using x2 = bf16x2;
  using x8 = bf16x8;
  __device__ static f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
  __device__ static f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};

struct F16 {
  using elem = _Float16;
  using x2 = f16x2;
  using x8 = f16x8;
  __device__ static f32x4 mfma16(f16x8 a, f16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
  __device__ static f32x16 mfma32(f16x8 a, f16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
};

// Two floats to one dword of 16-bit elements, each rounded to nearest even.
template <class T>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  typename T::x2 r;
  r[0] = (typename T::elem)a;
  r[1] = (typename T::elem)b;
  return __builtin_bit_cast(uint32_t, r);
}

}  // namespace fs
