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

__host__ inline int check_rel_bias(const dlrm_rel_bias* b) {
  if (!b || !b->table) return DLRM_ERR_NULL;
  if (b->n < 1 || b->n > DLRM_MAX_BUCKETS) return DLRM_ERR_BAD_SHAPE;
  return b->n > 1 && !b->bounds ? DLRM_ERR_NULL : DLRM_OK;
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

// 4 columns of a row
template <int DT>
__device__ inline void store4(char* to, f32x4 v) {
  if constexpr (DT == DLRM_F32) {
    *reinterpret_cast<f32x4*>(to) = v;
  } else {
    const float y[8] = {v[0], v[1], v[2], v[3], 0, 0, 0, 0};
    const u32x4 r = narrow<DT>(y);
    *reinterpret_cast<u32x2*>(to) = u32x2{r.x, r.y};
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

// The bucket of a distance: how many of the n - 1 bounds are at most it.  bounds: 2^steps - 1 of them at least, the largest integer past those that there are, which a
// distance may reach: what that adds is taken off.  Found by halves, so bounds that do not ascend give some bucket too, none past the last.
__device__ inline int bucket_of(const int* bounds, int n, int steps, int away) {
  int b = 0;
  for (int step = 1 << steps >> 1; step > 0; step >>= 1) b += bounds[b + step - 1] <= away ? step : 0;
  return min(b, n - 1);
}
// orders a wavefront's own accesses of LDS, which the compiler takes for those of one lane
__device__ inline void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Whether no bound is there twice, for a wavefront.
__device__ inline bool bounds_differ(const int32_t* bounds, int n) {
  uint64_t same = 0;
  int before = 0;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    if (64 * half >= n - 1) break;
    const int i = 64 * half + lane_id(), b = bounds[min(i, n - 2)];
    const int left = __builtin_amdgcn_update_dpp(before, b, 0x138, 0xf, 0xf, false);  // wave_shr:1
    same |= __ballot(b == left && i > 0 && i < n - 1);
    before = __builtin_amdgcn_readlane(b, 63);
  }
  return same == 0;
}
constexpr int kWindowEnd = 0x7fffffff - 64;  // the last distance that a window by marks may start from

// The buckets of 64 neighbouring distances, least + lane, by a wavefront; starts: the lanes, but the first, whose bucket is not the one before's.  By marks, where no bound is
// there twice and least <= kWindowEnd (else a window would meet the largest integer behind the bounds): the bounds up to `least` are counted, and those among the
// distances mark their places in `marks` (64 places in LDS of the wavefront's own), which are counted up to each lane's.  Two round trips through LDS, where halving
// takes one for each step.
template <typename T>
__device__ inline int buckets_from(const int* bounds, int n, int steps, bool by_marks, int least, T* marks, uint64_t& starts) {
  const int lane = lane_id();
  if (__builtin_expect(!by_marks, 0)) {
    const int bucket = bucket_of(bounds, n, steps, (int)((uint32_t)least + lane));
    const int before = __shfl_up(bucket, 1, DLRM_WAVE);
    starts = __ballot(lane > 0 && bucket != before);
    wave_fence();
    return bucket;
  }
  int base = 0;
  wave_fence();
  marks[lane] = T(0);
  wave_fence();
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    if (64 * half >= n - 1) break;
    const int b = 64 * half + lane < n - 1 ? bounds[64 * half + lane] : 0x7fffffff;
    base += __popcll(__ballot(b <= least));
    const uint32_t at = (uint32_t)b - (uint32_t)least;  // (the bound past all others is 2^31 - 1: no difference of integers)
    if (at - 1u < 63u) marks[at] = T(1);
  }
  wave_fence();
  const bool mark = marks[lane] != T(0);
  wave_fence();
  starts = __ballot(mark);
  return base + mark + __builtin_amdgcn_mbcnt_hi((uint32_t)(starts >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)starts, 0));
}
// A bias times `unit`; one that is there to hide its bucket (the lowest number of a type, or any so low that a row of nothing else would leave fp32 no digit of its
// scores) is -inf.
__device__ inline float bias_in(float t, float unit) { return t <= DLRM_BIAS_HIDES ? -__builtin_inff() : t * unit; }
__device__ inline void load_bounds(int* to, const int32_t* bounds, int n, int steps, int threads) {
  for (int i = threadIdx.x; i < 1 << steps; i += threads) to[i] = i < n - 1 ? bounds[i] : 0x7fffffff;
}

int check_cache(const dlrm_kv_cache* c);  // qk_rope.hip

}  // namespace dlrm
