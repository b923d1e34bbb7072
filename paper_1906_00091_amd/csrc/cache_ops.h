// What the kernels over a paged cache share: operands of mfma 16x16, a cap's tanh.
#pragma once

#include <math.h>

#include <type_traits>

#include "heads.h"

namespace dlrm {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kInf = __builtin_inff();
constexpr int kKeys = 32;          // of a tile
constexpr int kTablePages = 1024;  // pages of a chunk, at most

// operand of mfma 16x16: 8 values a lane; lane group g = lane / 16 holds values 8g..8g+7 of 32
template <int DT>
struct Op16;
template <>
struct Op16<DLRM_BF16> {
  u32x4 v;
  __device__ static inline f32x4 mma(const Op16& a, const Op16& b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a.v), __builtin_bit_cast(bf16x8, b.v), c, 0, 0, 0);
  }
};
template <>
struct Op16<DLRM_F16> {
  u32x4 v;
  __device__ static inline f32x4 mma(const Op16& a, const Op16& b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a.v), __builtin_bit_cast(f16x8, b.v), c, 0, 0, 0);
  }
};
template <>
struct Op16<DLRM_F32> {
  float f[8];
  __device__ static inline f32x4 mma(const Op16& a, const Op16& b, f32x4 c) {
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.f[j], b.f[j], c, 0, 0, 0);
    return c;
  }
};
template <int DT>
__device__ inline Op16<DT> op16_load(const char* p) {
  Op16<DT> o;
  if constexpr (DT == DLRM_F32) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 16);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      o.f[j] = a[j];
      o.f[4 + j] = b[j];
    }
  } else {
    o.v = load16(p);
  }
  return o;
}
template <int DT>
__device__ inline Op16<DT> op16_zero() {
  Op16<DT> o;
  if constexpr (DT == DLRM_F32) {
#pragma unroll
    for (int j = 0; j < 8; ++j) o.f[j] = 0.0f;
  } else {
    o.v = u32x4{0, 0, 0, 0};
  }
  return o;
}
template <int DT>
__device__ inline Op16<DT> op16_set(const float* f) {
  Op16<DT> o;
  if constexpr (DT == DLRM_F32) {
#pragma unroll
    for (int j = 0; j < 8; ++j) o.f[j] = f[j];
  } else {
    o.v = narrow<DT>(f);
  }
  return o;
}

// tanh(z).  16-bit rows take an exponential and a reciprocal, each good to 2^-23, where what that adds to a score (less than cap 2^-21) is at most an eighth of
// the rounding of a weight; else the library's, whose error is relative to z.  (256 sequences of up to 8192 items, 16 query heads on 4, bf16, d 128, capped:
// 412 us, 423 with the library's, also where that only stands beside the other.)
template <bool LARGE>
__device__ inline float bent16(float z) {
  if constexpr (LARGE) return tanhf(z);
  return 1.0f - 2.0f * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(z * (2.0f * kLog2e)) + 1.0f);
}

}  // namespace dlrm
