// Attention of one new item per sequence over a paged cache of keys and values.
//
// Bound by memory: the cache is read once.  All query heads of a key head (16 at a time) are the columns of one matrix tile, so a key row
// is loaded once for all of them, straight from its page into the registers that the product takes it in: a lane's 16 bytes are
// 8 consecutive columns of one key.  S^T = K Q^T leaves a lane four keys of one head, and those registers are, with the contracted
// index permuted, what O^T = V^T P^T takes; values pass through a piece of LDS that belongs to the wavefront alone, to be read by
// columns.  So the wavefronts of a workgroup run without a barrier, each with its own running maximum and sum, over
// every fourth tile of 32 keys, and are joined once at the end.  256 sequences of up to 8192 items, 16 query heads on 4, bf16, d 128, capped: 421 us for
// 2.15 GB, 5.1 TB/s; a large copy on the same card moves 4.7.
//
// The length is split over workgroups in chunks; their parts (unnormalised sums, maxima, weights) are joined by a second kernel in
// the order of the chunks.
#include <math.h>

#include <initializer_list>
#include <type_traits>

#include "heads.h"

namespace dlrm {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kInf = __builtin_inff();
constexpr int kKeys = 32, kHeads = 16;
constexpr int kTablePages = 1024;  // pages of a chunk, at most

struct CacheArgs {
  Rows q, out;
  const char* k;
  const char* v;
  const int32_t* table;
  const int32_t* lens;
  const float* slopes;
  int B, Hq, Hk, d, cols, n_pages, page_shift, max_len;  // max_len: the table's items at most
  int chunk, splits, blocks;  // keys of a chunk; chunks of a sequence; groups of 16 heads of a key head
  float scale, cap;
  float* po;  // [B][Hq][splits][d] unnormalised sums
  float* pm;  // [B][Hq][splits][2] maximum (powers of two), sum of weights
};

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

// items of sequence s that are read
__device__ inline int length_of(const CacheArgs& a, int s) { return max(0, min(a.lens[s], a.max_len)); }

template <int DT, int DP, int WAVES, bool LARGE>
__global__ __launch_bounds__(64 * WAVES) void cache_attn_kernel(CacheArgs a) {
  constexpr int EB = Tab<DT>::EB, E = Tab<DT>::ELEMS, STEPS = DP / 32, NB = DP / 16;
  constexpr int CH = DP * EB / 16, NV = kKeys * CH / DLRM_WAVE;  // chunks of a row; of a tile, per lane
  constexpr int STRIDE = DP * EB + 16;
  constexpr int OS = DP + 4;  // row of the joined sums
  // fp16: weights, at most 1, are made 2^15 times as large, sums and all: those of a long cache's many keys are not lost below 2^-24
  constexpr float LIFT = DT == DLRM_F16 ? 15.0f : 0.0f;
  constexpr int VBYTES = WAVES * kKeys * STRIDE, OBYTES = WAVES * kHeads * OS * 4;
  __shared__ __attribute__((aligned(16))) char lds[VBYTES > OBYTES ? VBYTES : OBYTES];
  __shared__ int pages[kTablePages];
  __shared__ float stat[WAVES][2][kHeads];
  const int split = blockIdx.x % a.splits, rest = blockIdx.x / a.splits;
  const int blk = rest % a.blocks, hk = rest / a.blocks % a.Hk, s = rest / a.blocks / a.Hk;
  const int G = a.Hq / a.Hk;
  const int lane = lane_id(), g = lane >> 4, n = lane & 15, wave = wave_id();
  const int head = hk * G + blk * kHeads + n;  // of this lane's column
  const bool head_there = blk * kHeads + n < G;
  // the chunk's page numbers and the queries are loaded beside the length, not after it
  // (Keys are counted from the chunk's start: a cache may hold up to 2^31 - 1 items, and a sum past its end would leave 32 bits.)
  const int start = split * a.chunk, page0 = start >> a.page_shift;
  const int most_pages = min(((start + min(a.chunk, a.max_len - start) - 1) >> a.page_shift) + 1, a.cols) - page0;
  for (int p = threadIdx.x; p < most_pages; p += 64 * WAVES) pages[p] = a.table[(int64_t)s * a.cols + page0 + p];
  Op16<DT> qf[STEPS];
  const char* qrow = row_of(a.q, s, head_there ? head : hk * G);
#pragma unroll
  for (int st = 0; st < STEPS; ++st) {
    qf[st] = op16_zero<DT>();
    if (head_there && 32 * st + 8 * g < a.d) qf[st] = op16_load<DT>(qrow + (32 * st + 8 * g) * EB);
  }
  const float c = a.scale * kLog2e, slope = a.slopes && head_there ? a.slopes[head] * kLog2e : 0.0f;
  const bool bend = a.cap > 0.0f;
  const float zs = bend ? a.scale / a.cap : 0.0f, cl = a.cap * kLog2e;
  const int len = length_of(a, s), n_keys = min(len - start, a.chunk);
  if (n_keys <= 0 && split > 0) return;  // the first chunk of an empty sequence gives zeros
  __syncthreads();

  const int row_bytes = a.d * EB, mask = (1 << a.page_shift) - 1;
  const int64_t head_bytes = (int64_t)row_bytes << a.page_shift, page_bytes = head_bytes * a.Hk;
  // Byte offset of the row of the chunk's key i; a key past the end, or on a page that is not there, gives the first row of the cache and false.
  // No load stands in a branch (the wait for it would come with the branch's end): what came for no reason is masked where it is used.
  auto row_at = [&](int i, bool& there) -> int64_t {
    const int j = start + min(i, n_keys - 1), p = pages[(j >> a.page_shift) - page0];
    there = i < n_keys && p >= 0 && p < a.n_pages;
    return there ? p * page_bytes + hk * head_bytes + (int64_t)((j & mask) * row_bytes) : 0;
  };
  char* vs = lds + wave * kKeys * STRIDE;
  Op16<DT> kf[2][STEPS];
  u32x4 vf[NV];
  bool seen[2];
  uint32_t v_there = 0;  // bit i: chunk i of the values
  // columns past d: another chunk of the same row; the query's zeros there cancel the key's, and the values' are never written out
  int kcol[STEPS];
#pragma unroll
  for (int st = 0; st < STEPS; ++st) kcol[st] = min(32 * st + 8 * g, a.d - 8) * EB;
  auto fetch = [&](int j0) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int64_t at = row_at(j0 + 16 * u + n, seen[u]);
#pragma unroll
      for (int st = 0; st < STEPS; ++st) kf[u][st] = op16_load<DT>(a.k + at + kcol[st]);
    }
    v_there = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int id = lane + i * DLRM_WAVE, r = id / CH, cc = min(id % CH, a.d / E - 1);
      bool there;
      const int64_t at = row_at(j0 + r, there);
      v_there |= there ? 1u << i : 0u;
      vf[i] = load16(a.v + at + cc * 16);
    }
  };

  f32x4 o[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) o[b] = f32x4{0, 0, 0, 0};
  float m = -kInf, l = 0.0f;
  const int to_newest = len - 1 - start;  // from the chunk's first key
  int j0 = wave * kKeys;
  if (j0 < n_keys) fetch(j0);
  for (; j0 < n_keys; j0 += WAVES * kKeys) {
    f32x4 sc[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      sc[u] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int st = 0; st < STEPS; ++st) sc[u] = Op16<DT>::mma(kf[u][st], qf[st], sc[u]);
    }
    // which of the four keys of each register set are there: their lanes know
    const uint64_t have0 = __ballot(seen[0]), have1 = __ballot(seen[1]);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int id = lane + i * DLRM_WAVE;
      *reinterpret_cast<u32x4*>(vs + (id / CH) * STRIDE + (id % CH) * 16) = v_there >> i & 1 ? vf[i] : u32x4{0, 0, 0, 0};
    }
    const int jn = j0 + WAVES * kKeys;
    if (jn < n_keys) fetch(jn);
    float x[8];
    float top = -kInf;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int key = 4 * g + r;
        float y = sc[u][r];
        y = bend ? bent16<LARGE>(y * zs) * cl : y * c;
        y -= slope * (float)(to_newest - (j0 + 16 * u + key));
        x[4 * u + r] = ((u ? have1 : have0) >> key) & 1 ? y : -kInf;
        top = fmaxf(top, x[4 * u + r]);
      }
    top = fmaxf(top, __shfl_xor(top, 16, DLRM_WAVE));
    top = fmaxf(top, __shfl_xor(top, 32, DLRM_WAVE));
    const float m1 = fmaxf(m, top), ms = m1 == -kInf ? 0.0f : m1;
    const float f = __builtin_amdgcn_exp2f(m - ms);
    m = m1;
    l *= f;
#pragma unroll
    for (int b = 0; b < NB; ++b) o[b] *= f;
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      x[r] = __builtin_amdgcn_exp2f(x[r] - (ms - LIFT));
      l += x[r];
    }
    // 16-bit rows: weights in two parts, each in a product of its own.  (The matrix cores wait for memory here: 256 sequences of up to 8192 items
    // 413 -> 419 us, one of 131072 items 48.5 -> 49; the result's error 2.07e-3 -> 1.63e-3 of it in bf16, which is its own rounding.)
    Op16<DT> p, p_low;
    if constexpr (EB == 2)
      two_parts<DT>(x, p.v, p_low.v);
    else
      p = op16_set<DT>(x);
    // the values' columns: rows 4g..4g+3 and 16+4g..16+4g+3 of the tile for lane group g
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      Op16<DT> vt;
      if constexpr (EB == 2) {
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        const char* q = vs + (4 * g + (n >> 2)) * STRIDE + (16 * b + 4 * (n & 3)) * 2;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)q);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(q + 16 * STRIDE));
        const u32x2 l2 = __builtin_bit_cast(u32x2, lo), h2 = __builtin_bit_cast(u32x2, hi);
        vt.v = u32x4{l2.x, l2.y, h2.x, h2.y};
      } else {
        const char* q = vs + 4 * g * STRIDE + (16 * b + n) * 4;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          vt.f[j] = *reinterpret_cast<const float*>(q + j * STRIDE);
          vt.f[4 + j] = *reinterpret_cast<const float*>(q + (16 + j) * STRIDE);
        }
      }
      o[b] = Op16<DT>::mma(vt, p, o[b]);
      if constexpr (EB == 2) o[b] = Op16<DT>::mma(vt, p_low, o[b]);
    }
    __builtin_amdgcn_wave_barrier();
  }
  l += __shfl_xor(l, 16, DLRM_WAVE);
  l += __shfl_xor(l, 32, DLRM_WAVE);
  __syncthreads();  // every wavefront is done with its values
  if (g == 0) {
    stat[wave][0][n] = m;
    stat[wave][1][n] = l;
  }
  float* os = reinterpret_cast<float*>(lds);
#pragma unroll
  for (int b = 0; b < NB; ++b)
    *reinterpret_cast<f32x4*>(os + (wave * kHeads + n) * OS + 16 * b + 4 * g) = o[b];
  __syncthreads();
  // join the wavefronts: a thread takes 4 columns of a head
  const int per_head = a.d / 4, rows = min(kHeads, G - blk * kHeads);
  for (int id = threadIdx.x; id < rows * per_head; id += 64 * WAVES) {
    const int hn = id / per_head, col = id % per_head * 4, hd = hk * G + blk * kHeads + hn;
    float top = -kInf;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) top = fmaxf(top, stat[w][0][hn]);
    const float ms = top == -kInf ? 0.0f : top;
    f32x4 sum = {0, 0, 0, 0};
    float total = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const float f = __builtin_amdgcn_exp2f(stat[w][0][hn] - ms);
      total += f * stat[w][1][hn];
      sum += f * *reinterpret_cast<const f32x4*>(os + (w * kHeads + hn) * OS + col);
    }
    if (a.splits == 1) {
      const float inv = total > 0.0f ? 1.0f / total : 0.0f;
      char* dst = row_of(a.out, s, hd) + col * EB;
      sum *= inv;
      if constexpr (DT == DLRM_F32) {
        *reinterpret_cast<f32x4*>(dst) = sum;
      } else {
        const float y[8] = {sum[0], sum[1], sum[2], sum[3], 0, 0, 0, 0};
        const u32x4 r = narrow<DT>(y);
        *reinterpret_cast<u32x2*>(dst) = u32x2{r.x, r.y};
      }
    } else {
      const int64_t at = ((int64_t)s * a.Hq + hd) * a.splits + split;
      *reinterpret_cast<f32x4*>(a.po + at * a.d + col) = sum;
      if (col == 0) {
        a.pm[at * 2] = top;
        a.pm[at * 2 + 1] = total;
      }
    }
  }
}

// Joins the chunks of one sequence and head: the chunks' factors are made 512 at a time, then half a wavefront takes every 16th chunk,
// 4 columns a lane, four chunks in flight.
constexpr int kJoinThreads = 512;
template <int DT>
__global__ __launch_bounds__(kJoinThreads) void cache_join_kernel(CacheArgs a) {
  constexpr int ROWS = kJoinThreads / 32, AHEAD = 4;
  __shared__ float red[kJoinThreads / DLRM_WAVE];
  __shared__ f32x4 part[ROWS][32];
  __shared__ float factor[kJoinThreads];
  const int64_t row = blockIdx.x;
  const int s = (int)(row / a.Hq), head = (int)(row - (int64_t)s * a.Hq);
  const int len = length_of(a, s), n = len > 0 ? (len - 1) / a.chunk + 1 : 1;
  const float* pm = a.pm + row * a.splits * 2;
  const float* po = a.po + row * a.splits * a.d;
  const int y = threadIdx.x >> 5, col = (threadIdx.x & 31) * 4, wave = wave_id();
  auto over_block = [&](float v, auto f) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = f(v, __shfl_xor(v, o, DLRM_WAVE));
    if (lane_id() == 0) red[wave] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int i = 1; i < kJoinThreads / DLRM_WAVE; ++i) v = f(v, red[i]);
    __syncthreads();
    return v;
  };
  float top = -kInf;
  for (int i = threadIdx.x; i < n; i += kJoinThreads) top = fmaxf(top, pm[2 * i]);
  top = over_block(top, [](float u, float v) { return fmaxf(u, v); });
  const float ms = top == -kInf ? 0.0f : top;
  f32x4 sum = {0, 0, 0, 0};
  float total = 0.0f;
  for (int i0 = 0; i0 < n; i0 += kJoinThreads) {
    const int i = i0 + threadIdx.x;
    float f = 0.0f;
    if (i < n) {
      f = __builtin_amdgcn_exp2f(pm[2 * i] - ms);
      total += f * pm[2 * i + 1];
    }
    factor[threadIdx.x] = f;
    __syncthreads();
    const int m = min(n - i0, kJoinThreads);
    if (col < a.d) {
      for (int r = y; r < m; r += AHEAD * ROWS) {
        f32x4 v[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) v[j] = loadf4(po + (int64_t)(i0 + (r + j * ROWS < m ? r + j * ROWS : r)) * a.d + col);
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
          // (past the end both are zero: zero times the row that was loaded instead would be NaN where that holds an infinity)
          const bool there = r + j * ROWS < m;
          sum += (there ? factor[r + j * ROWS] : 0.0f) * (there ? v[j] : f32x4{0, 0, 0, 0});
        }
      }
    }
    __syncthreads();
  }
  total = over_block(total, [](float u, float v) { return u + v; });
  part[y][threadIdx.x & 31] = sum;
  __syncthreads();
  if (y != 0 || col >= a.d) return;
  sum = f32x4{0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < ROWS; ++i) sum += part[i][threadIdx.x];
  sum *= total > 0.0f ? 1.0f / total : 0.0f;
  char* dst = row_of(a.out, s, head) + col * Tab<DT>::EB;
  if constexpr (DT == DLRM_F32) {
    *reinterpret_cast<f32x4*>(dst) = sum;
  } else {
    const float v[8] = {sum[0], sum[1], sum[2], sum[3], 0, 0, 0, 0};
    const u32x4 r = narrow<DT>(v);
    *reinterpret_cast<u32x2*>(dst) = u32x2{r.x, r.y};
  }
}

// Keys of a chunk: 1024 workgroups, four a CU, and at least two tiles a wavefront.  (The 256 sequences above, weights in one part: 436 us with chunks for 1024
// workgroups, 474 for 2048, 498 for 4096, 537 for 8192, whose joins read more.  One sequence of 131072 items on 4 key heads, four workgroups if it were not
// split: 49 us with its join.)
constexpr int kWanted = 1024, kLeastChunk = 256;
static int64_t groups_of(const dlrm_kv_cache* c, int Hq) { return (int64_t)c->B * c->Hk * ((Hq / c->Hk + kHeads - 1) / kHeads); }
static int64_t most_of_chunk(const dlrm_kv_cache* c) { return (int64_t)(kTablePages - 1) * c->page; }  // (it need not start on a page)
static int chunk_of(const dlrm_kv_cache* c, int Hq, int max_len) {
  int64_t n = (groups_of(c, Hq) * max_len + kWanted - 1) / kWanted;
  if (n < kLeastChunk) n = kLeastChunk;
  n = (n + 127) / 128 * 128;
  if (n > most_of_chunk(c)) n = most_of_chunk(c);
  return (int)(n > max_len ? max_len : n);
}

// the arguments for n sequences from sequence s0 on
static CacheArgs sequences_of(CacheArgs a, int64_t s0, int64_t n) {
  a.q.p += s0 * a.q.st;
  a.out.p += s0 * a.out.st;
  a.table += s0 * a.cols;
  a.lens += s0;
  if (a.po) {
    a.po += s0 * a.Hq * a.splits * a.d;
    a.pm += s0 * a.Hq * a.splits * 2;
  }
  a.B = (int)n;
  return a;
}

static int check_cache_attn(const dlrm_kv_cache* c, int Hq, int max_len) {
  if (int st = check_cache(c)) return st;
  if (int st = check_head_shape(Hq, c->Hk, c->d, c->dtype)) return st;
  if (max_len < 1) return DLRM_ERR_BAD_SHAPE;
  return DLRM_OK;
}

// The most chunks that a bound of up to max_len gives a sequence.  (Chunks are rounded up, so a smaller bound may give more of them than max_len: 8
// sequences, 16 query heads on 4, 33 chunks for 8256 items and 48 for 8000.)  A chunk has the fewest keys there are, as many as a page table's piece holds, or
// enough for kWanted workgroups.
static int64_t most_splits(const dlrm_kv_cache* c, int Hq, int max_len) {
  const int64_t held = (int64_t)c->table_cols * c->page, n = max_len > held ? held : max_len;
  const int64_t short_chunks = (n - 1) / kLeastChunk + 1, table_pieces = (n - 1) / most_of_chunk(c) + 1;
  const int64_t workgroups = (kWanted - 1) / groups_of(c, Hq) + 1, most = workgroups > table_pieces ? workgroups : table_pieces;
  return short_chunks < most ? short_chunks : most;
}

}  // namespace dlrm

using namespace dlrm;

extern "C" size_t dlrm_cache_attn_workspace_bytes(const dlrm_kv_cache* c, int32_t Hq, int32_t max_len) {
  if (check_cache_attn(c, Hq, max_len) != DLRM_OK) return 0;
  const size_t n = (size_t)c->B * Hq * most_splits(c, Hq, max_len) * (c->d + 2) * sizeof(float);
  return (n + 255) / 256 * 256;
}

extern "C" int32_t dlrm_cache_attn(const dlrm_kv_cache* c, const int32_t* lens, int32_t max_len, int32_t Hq, const dlrm_heads* q,
                                   const dlrm_heads* out, const float* slopes, float scale, float cap, void* workspace,
                                   size_t workspace_bytes, void* stream) {
  if (int st = check_cache_attn(c, Hq, max_len)) return st;
  if (!lens) return DLRM_ERR_NULL;
  if (!(scale > 0.0f) || !isfinite(scale) || !(cap >= 0.0f) || !isfinite(cap)) return DLRM_ERR_BAD_SHAPE;
  const int eb = elem_bytes(c->dtype);
  for (const dlrm_heads* x : {q, out})
    if (int st = check_heads(x, c->B, Hq, c->d, eb)) return st;
  CacheArgs a = {};
  a.q = rows_of(q, c->B, Hq, c->d, eb);
  a.out = rows_of(out, c->B, Hq, c->d, eb);
  a.k = static_cast<const char*>(c->k);
  a.v = static_cast<const char*>(c->v);
  a.table = c->table;
  a.lens = lens;
  a.slopes = slopes;
  a.B = c->B;
  a.Hq = Hq;
  a.Hk = c->Hk;
  a.d = c->d;
  a.cols = c->table_cols;
  a.n_pages = c->n_pages;
  a.page_shift = ilog2_ceil(c->page);
  const int64_t held = (int64_t)c->table_cols * c->page;
  a.max_len = max_len > held ? (int)held : max_len;
  a.chunk = chunk_of(c, Hq, a.max_len);
  a.splits = (a.max_len - 1) / a.chunk + 1;
  a.blocks = (Hq / c->Hk + kHeads - 1) / kHeads;
  a.scale = scale;
  a.cap = cap;
  // a launch takes fewer than 2^32 threads: more sequences than that go in several
  const int64_t per_seq = (int64_t)a.splits * a.blocks * a.Hk, join_per_seq = a.splits > 1 ? Hq : 0;
  const int64_t most = 256 * per_seq > kJoinThreads * join_per_seq ? 256 * per_seq : kJoinThreads * join_per_seq;
  const int64_t each = kLaunchThreads / most;
  if (each == 0) return DLRM_ERR_BAD_SHAPE;
  const int64_t grid = per_seq * a.B;
  if (a.splits > 1) {
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < dlrm_cache_attn_workspace_bytes(c, Hq, max_len))
      return DLRM_ERR_WORKSPACE;
    a.po = static_cast<float*>(workspace);
    a.pm = a.po + (int64_t)a.B * Hq * a.splits * a.d;
  }
  // Short sequences, and enough of them: a wavefront each, with nothing to join.  (1356 of 24 items, 8 key heads, fp32, d 32: 22 us, 47 with four
  // wavefronts; 2048 of up to 200, 4 key heads, fp32, d 64: 95 us, 133.  64 of up to 64, 8 key heads, bf16, d 64: 6.6 us, 5.6 with four, and
  // 2048 of up to 512, 4 key heads, bf16, d 64: 114 us, 110.)
  const bool one_wave = a.max_len <= 256 && grid > 8 * (int64_t)a.max_len;
  hipStream_t st = static_cast<hipStream_t>(stream);
  auto by_type = [&](auto dt) {
    auto with_cap = [&](auto dp, auto large) {
      for (int64_t s0 = 0; s0 < a.B; s0 += each) {
        const CacheArgs b = sequences_of(a, s0, a.B - s0 < each ? a.B - s0 : each);
        const unsigned n = (unsigned)(per_seq * b.B);
        if (one_wave)
          hipLaunchKernelGGL((cache_attn_kernel<dt(), dp(), 1, large()>), dim3(n), dim3(64), 0, st, b);
        else
          hipLaunchKernelGGL((cache_attn_kernel<dt(), dp(), 4, large()>), dim3(n), dim3(256), 0, st, b);
        DLRM_CHECK_LAUNCH();
        if (a.splits > 1) {
          hipLaunchKernelGGL(cache_join_kernel<dt()>, dim3((unsigned)(b.B * Hq)), dim3(kJoinThreads), 0, st, b);
          DLRM_CHECK_LAUNCH();
        }
      }
      return (int)DLRM_OK;
    };
    auto go = [&](auto dp) {
      if constexpr (dt() != DLRM_F32) {
        if (a.cap <= (dt() == DLRM_F16 ? 128.0f : 1024.0f)) return with_cap(dp, std::integral_constant<bool, false>{});
      }
      return with_cap(dp, std::integral_constant<bool, true>{});
    };
    if (a.d <= 32) return go(std::integral_constant<int, 32>{});
    if (a.d <= 64) return go(std::integral_constant<int, 64>{});
    if (a.d <= 96) return go(std::integral_constant<int, 96>{});
    return go(std::integral_constant<int, 128>{});
  };
  switch (c->dtype) {
    case DLRM_F32: return by_type(std::integral_constant<int, DLRM_F32>{});
    case DLRM_F16: return by_type(std::integral_constant<int, DLRM_F16>{});
    default: return by_type(std::integral_constant<int, DLRM_BF16>{});
  }
}
