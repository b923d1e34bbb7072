// Rows of heads: what the kernels that read a history in order share (views, storage types, argument checks).
#pragma once

#include "common.h"

namespace dlrm {

constexpr int64_t kLaunchThreads = (int64_t)1 << 31;  // of one launch at most, where a call may need several (the device's limit: 2^32 - 1)

// one dlrm_heads on its way to a kernel, strides in bytes
struct Rows {
  char* p;
  int64_t st, sh;
};

__device__ inline char* row_of(const Rows& r, int64_t t, int h) { return r.p + t * r.st + h * r.sh; }

// (the stride along an axis of one element means nothing, and is not passed on)
__host__ inline Rows rows_of(const dlrm_heads* x, int64_t n, int H, int d, int eb) {
  return Rows{static_cast<char*>(x->data), (n > 1 ? x->stride_t : d) * eb, (H > 1 ? x->stride_h : d) * eb};
}

// Checks a view of H heads of d columns, n items.
__host__ inline int check_heads(const dlrm_heads* x, int64_t n, int H, int d, int eb) {
  if (!x || (!x->data && n > 0)) return DLRM_ERR_NULL;
  if (reinterpret_cast<uintptr_t>(x->data) & 15) return DLRM_ERR_BAD_SHAPE;
  // (as in rows_of; a tile's rows are reached with 32-bit byte offsets)
  const int64_t st = n > 1 ? x->stride_t : d, sh = H > 1 ? x->stride_h : d;
  if (st < d || sh < d || st > (1 << 23) || sh >= (int64_t)1 << 40) return DLRM_ERR_BAD_SHAPE;
  if (((st * eb) & 15) != 0 || ((sh * eb) & 15) != 0) return DLRM_ERR_BAD_SHAPE;
  return DLRM_OK;
}

__host__ inline int check_head_shape(int Hq, int Hk, int d, int dtype) {
  if (!dtype_ok(dtype)) return DLRM_ERR_BAD_DTYPE;
  if (Hq < 1 || Hq > DLRM_MAX_HEADS || Hk < 1 || Hq % Hk != 0) return DLRM_ERR_BAD_SHAPE;
  if (d < 8 || d > DLRM_MAX_HEAD_DIM || (d & 7)) return DLRM_ERR_BAD_SHAPE;
  return DLRM_OK;
}

// 16-byte chunk <- fp32 values, rounded to nearest-even once where the storage type has 16 bits
template <int DT>
__device__ inline u32x4 narrow(const float* f) {
  if constexpr (DT == DLRM_F32) {
    return u32x4{f2u(f[0]), f2u(f[1]), f2u(f[2]), f2u(f[3])};
  } else if constexpr (DT == DLRM_F16) {
    return u32x4{float2_to_half2(f[0], f[1]), float2_to_half2(f[2], f[3]), float2_to_half2(f[4], f[5]), float2_to_half2(f[6], f[7])};
  } else {
    typedef __bf16 b16x8 __attribute__((ext_vector_type(8)));
    b16x8 v;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (__bf16)f[j];
    return __builtin_bit_cast(u32x4, v);
  }
}

// A weight w >= 0 as the sum of two 16-bit numbers, 8 at a time: `high` is w rounded down, `low` what is left.  low is above zero wherever high is (by less than fp32's
// rounding would add), so that both products with an infinite value are that infinity: zero times it, or an infinity less another, would be NaN.
template <int DT>
__device__ inline void two_parts(const float* w, u32x4& high, u32x4& low) {
  constexpr float LEAST = DT == DLRM_F16 ? 0x1p-24f : 0x1p-126f;  // of fp16, subnormal numbers and all, and of the normal ones
  if constexpr (DT == DLRM_F16) {
#pragma unroll
    for (int j = 0; j < 4; ++j) high[j] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(w[2 * j], w[2 * j + 1]));
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) high[j] = __builtin_amdgcn_perm(f2u(w[2 * j + 1]), f2u(w[2 * j]), 0x07060302u);
  }
  float h[8], l[8];
  Tab<DT>::widen(high, h);
#pragma unroll
  for (int j = 0; j < 8; ++j) l[j] = fmaxf(w[j] - h[j], fminf(h[j], LEAST));
  low = narrow<DT>(l);
}

int check_cache(const dlrm_kv_cache* c);  // qk_rope.hip

}  // namespace dlrm
