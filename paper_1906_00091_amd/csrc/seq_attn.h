// Attention over the sequences of a CSR batch, forward and backward, on the matrix cores.
//
// Everything is tiled for mfma 32x32: a wavefront owns 32 rows of one sequence and head (queries in the forward and in the
// queries' gradient, keys in the keys' and values' gradients) and walks the other side in tiles that the workgroup's four
// wavefronts stage in LDS together.  The products are arranged so that the wavefront's own rows are the columns of every
// accumulator: S^T = K Q^T, O^T = V^T P^T and so on.  Then a lane holds one row of the softmax (two lanes share it, one half of each
// tile's keys each), maxima, sums and rescaling are plain vector arithmetic, and the weights leave one product in the very registers in
// which the next one takes them: the accumulator's rows 8i + 4h + 0..3 of lane half h, taken as they come, are a permutation of
// the contracted index, and the other operand is read from LDS in the same permutation (ds_read_b64_tr_b16 gives a lane four consecutive
// rows of a column).
// Nothing passes between lanes but one exchange of the two halves' maxima a tile.
//
// fp32 operands run the same code: a fragment of 8 values a lane is 8 products of mfma 32x32x2 in place of one of 32x32x16.
// With 16-bit types the weights and their gradients are rounded to that type before the second product, as the matrix cores
// take it; sums of weights and all accumulators stay fp32.
#pragma once

#include <type_traits>

#include "heads.h"

namespace dlrm {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kInf = __builtin_inff();

// An operand of a product: 8 consecutive values of the contracted index for one row, per lane (lane half h: values 8h..8h+7 of 16).
template <int DT>
struct Op;

template <>
struct Op<DLRM_BF16> {
  bf16x8 v;
  __device__ inline void set(int j, float f) { v[j] = (__bf16)f; }
  __device__ inline float get(int j) const { return (float)v[j]; }
  __device__ static inline f32x16 mma(const Op& a, const Op& b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, b.v, c, 0, 0, 0);
  }
};
template <>
struct Op<DLRM_F16> {
  f16x8 v;
  __device__ inline void set(int j, float f) { v[j] = (_Float16)f; }
  __device__ inline float get(int j) const { return (float)v[j]; }
  __device__ static inline f32x16 mma(const Op& a, const Op& b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a.v, b.v, c, 0, 0, 0);
  }
};
template <>
struct Op<DLRM_F32> {
  f32x4 v[2];
  __device__ inline void set(int j, float f) { v[j >> 2][j & 3] = f; }
  __device__ inline float get(int j) const { return v[j >> 2][j & 3]; }
  __device__ static inline f32x16 mma(const Op& a, const Op& b, f32x16 c) {
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.get(j), b.get(j), c, 0, 0, 0);
    return c;
  }
};

template <int DT>
__device__ inline Op<DT> op_zero() {
  Op<DT> o;
#pragma unroll
  for (int j = 0; j < 8; ++j) o.set(j, 0.0f);
  return o;
}
template <int DT>
__device__ inline Op<DT> op_load(const char* p) {  // 8 consecutive values, 16-byte aligned
  Op<DT> o;
  if constexpr (DT == DLRM_F32) {
    o.v[0] = *reinterpret_cast<const f32x4*>(p);
    o.v[1] = *reinterpret_cast<const f32x4*>(p + 16);
  } else {
    o.v = *reinterpret_cast<const decltype(o.v)*>(p);
  }
  return o;
}

// A tile of rows in LDS.  Rows are padded: row reads of 16 bytes by 16 and more consecutive rows, and column reads of 4 consecutive rows,
// then meet few banks twice (a row stride that is an odd multiple of 16 bytes modulo the 256 bytes of all banks).
template <int DT, int DP>
struct Tile {
  static constexpr int EB = Tab<DT>::EB;
  static constexpr int ROW = DP * EB;
  static constexpr int STRIDE = ROW + (DP == 128 && EB == 2 ? 48 : 16);

  // operand whose row is row r of the tile, values 16 * step + 8 h ...
  __device__ static inline Op<DT> by_row(const char* s, int r, int step, int h) {
    return op_load<DT>(s + r * STRIDE + (16 * step + 8 * h) * EB);
  }
  // operand whose row is column 32 * block + lane % 32 of the tile, and whose contracted values are the tile's rows
  // row0 + 4h + 0..3 and row0 + 8 + 4h + 0..3: the accumulator's order
  __device__ static inline Op<DT> by_column(const char* s, int row0, int block, int lane) {
    Op<DT> o;
    const int h = lane >> 5;
    if constexpr (EB == 2) {
      typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
      const char* p = s + (row0 + 4 * h + ((lane & 15) >> 2)) * STRIDE + (32 * block + (lane & 16) + 4 * (lane & 3)) * 2;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 8 * STRIDE));
      o.v = __builtin_bit_cast(decltype(o.v), __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      const char* p = s + (row0 + 4 * h) * STRIDE + (32 * block + (lane & 31)) * 4;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        o.v[0][j] = *reinterpret_cast<const float*>(p + j * STRIDE);
        o.v[1][j] = *reinterpret_cast<const float*>(p + (8 + j) * STRIDE);
      }
    }
    return o;
  }
};

constexpr int kSeqThreads = 256, kSeqWaves = 4;

// A tile on its way from global memory to LDS, in the registers of the workgroup's threads.
template <int DT, int DP, int ROWS>
struct Staged {
  static constexpr int CH = DP * Tab<DT>::EB / 16;  // chunks of 16 bytes in a row
  static constexpr int N = (ROWS * CH + kSeqThreads - 1) / kSeqThreads;
  u32x4 v[N];
  // rows row0.. of which `n` are there, columns < d; the rest are zeros
  __device__ inline void load(const char* base, int64_t stride, int n, int d) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int id = threadIdx.x + i * kSeqThreads, r = id / CH, c = id % CH;
      v[i] = u32x4{0, 0, 0, 0};
      if (r < n && r < ROWS && c * Tab<DT>::ELEMS < d) v[i] = load16(base + ((uint32_t)r * (uint32_t)stride + c * 16u));
    }
  }
  __device__ inline void store(char* s) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int id = threadIdx.x + i * kSeqThreads, r = id / CH, c = id % CH;
      if (ROWS * CH % kSeqThreads == 0 || r < ROWS) *reinterpret_cast<u32x4*>(s + r * Tile<DT, DP>::STRIDE + c * 16) = v[i];
    }
  }
};

struct SeqArgs {
  Rows q, k, v, out, dout, dq, dk, dv;
  const int64_t* q_off;
  const int64_t* k_off;
  const int32_t* prefix;
  const float* slopes;
  float* lse;    // [Hq, Tq]
  float* delta;  // [Hq, Tq]
  int64_t Tq;
  int B, Hq, Hk, d, causal;
  int slots;       // of 128 rows
  int per_seq;     // slots of a sequence where all have the same number, else 0
  float scale, cap;
};

// Slot -> sequence and first row.  A sequence with n rows needs ceil(n / 128) slots, and how many rows it has stands in device memory.
// Where all sequences fit into few slots each gets as many as the longest may need.  Else sequence s starts at slot off[s] / 128 + s, which leaves it
// enough; slots past its rows end at once.  The sequence is found by all 64 lanes at once: each step asks 64 places.
constexpr int kSlotRows = 128;
__device__ inline bool find_slot(const int64_t* off, int B, int per_seq, int slot, int& seq, int& row0) {
  if (per_seq > 0) {
    seq = slot / per_seq;
    row0 = (slot - seq * per_seq) * kSlotRows;
    return true;
  }
  int lo = 0, hi = B;
  while (hi - lo > 1) {
    const int step = (hi - lo + 63) >> 6, s = lo + lane_id() * step;
    const bool before = s < hi && off[s] / kSlotRows + s <= slot;
    const int n = __popcll(__ballot(before));  // >= 1: the first place always is
    hi = min(lo + n * step, hi);
    lo = lo + (n - 1) * step;
  }
  seq = __builtin_amdgcn_readfirstlane(lo);
  row0 = (slot - (int)(off[seq] / kSlotRows) - seq) * kSlotRows;
  return true;
}

// tanh from one exponential; fp32 operands take the library's, whose error near 0 is relative
template <int DT>
__device__ inline float bent(float z) {
  if constexpr (DT == DLRM_F32) {
    return tanhf(z);
  } else {
    return 1.0f - 2.0f * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(z * (2.0f * kLog2e)) + 1.0f);
  }
}

// the other lane half's value
__device__ inline float other_half(float v) { return __shfl_xor(v, 32, DLRM_WAVE); }

// Rows t of an accumulator set acc^T [DP columns x 32 rows]: row lane % 32, columns 32 b + 8 g + 4 h + 0..3.
template <int DT, int NB>
__device__ inline void store_rows(const f32x16* acc, float f, char* row, int d, int h) {
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int c = 32 * b + 8 * g + 4 * h;
      if (c >= d) continue;
      const float x0 = acc[b][4 * g] * f, x1 = acc[b][4 * g + 1] * f, x2 = acc[b][4 * g + 2] * f, x3 = acc[b][4 * g + 3] * f;
      if constexpr (DT == DLRM_F32) {
        *reinterpret_cast<f32x4*>(row + c * 4) = f32x4{x0, x1, x2, x3};
      } else if constexpr (DT == DLRM_F16) {
        *reinterpret_cast<u32x2*>(row + c * 2) = u32x2{float2_to_half2(x0, x1), float2_to_half2(x2, x3)};
      } else {
        typedef __bf16 b16x4 __attribute__((ext_vector_type(4)));
        *reinterpret_cast<b16x4*>(row + c * 2) = b16x4{(__bf16)x0, (__bf16)x1, (__bf16)x2, (__bf16)x3};
      }
    }
}

// Operands of a row held in registers: values 16 * step + 8 h + 0..7, zeros past d or where the row is not there.
template <int DT, int STEPS>
__device__ inline void own_rows(Op<DT>* f, const char* row, bool there, int d, int h) {
#pragma unroll
  for (int s = 0; s < STEPS; ++s) {
    f[s] = op_zero<DT>();
    if (there && 16 * s + 8 * h < d) f[s] = op_load<DT>(row + (16 * s + 8 * h) * Tab<DT>::EB);
  }
}

// What a sequence's rows may see: keys [0, vis(i)) for query i.
struct Span {
  int nq, nk, shift, prefix, causal;  // shift: a query's place is i + shift
  __device__ inline int vis(int i) const {
    if (!causal) return nk;
    const int v = max(i + shift + 1, prefix);
    return min(max(v, 0), nk);
  }
  __device__ inline int first_query(int j) const { return !causal || j < prefix ? 0 : max(0, j - shift); }  // that sees key j
};
__device__ inline Span span_of(const SeqArgs& a, int s, int64_t& q0, int64_t& k0) {
  q0 = a.q_off[s];
  k0 = a.k_off[s];
  Span x;
  x.nq = (int)(a.q_off[s + 1] - q0);
  x.nk = (int)(a.k_off[s + 1] - k0);
  x.shift = x.nk - x.nq;
  x.causal = a.causal;
  x.prefix = a.prefix ? a.prefix[s] : 0;
  return x;
}

// Key j of accumulator register r of subtile u, lane half h
__device__ inline int acc_row(int r, int h) { return 8 * (r >> 2) + 4 * h + (r & 3); }

template <int DT>
struct Score {  // of one head
  float c, zs, cl, slope;
  bool bend;
  __device__ inline Score(const SeqArgs& a, int head) {
    bend = a.cap > 0.0f;
    c = a.scale * kLog2e;
    zs = bend ? a.scale / a.cap : 0.0f;
    cl = a.cap * kLog2e;
    slope = a.slopes ? a.slopes[head] * kLog2e : 0.0f;
  }
  // product -> score in powers of two, without the factor `c` where there is neither cap nor slope
  __device__ inline bool simple(const SeqArgs& a) const { return !bend && a.slopes == nullptr; }
};

// ---------------------------------------------------------------------------------------------------------------
// Forward: a workgroup takes 128 queries of one head (32 a wavefront), tiles of 64 keys and values go by, two of them in LDS.
template <int DT, int DP>
__global__ __launch_bounds__(kSeqThreads, DT == DLRM_F32 ? 1 : 2) void seq_attn_fwd_kernel(SeqArgs a) {
  constexpr int BK = 64, STEPS = DP / 16, NB = DP / 32;
  typedef Tile<DT, DP> T;
  __shared__ __attribute__((aligned(16))) char sk[2][BK * T::STRIDE];
  __shared__ __attribute__((aligned(16))) char sv[2][BK * T::STRIDE];
  const int hh = blockIdx.x % a.Hq, slot = a.slots - 1 - blockIdx.x / a.Hq;  // late rows see most keys: first
  const int G = a.Hq / a.Hk, hk = hh % a.Hk, head = hk * G + hh / a.Hk;
  int seq, row0;
  find_slot(a.q_off, a.B, a.per_seq, slot, seq, row0);
  int64_t q0, k0;
  const Span sp = span_of(a, seq, q0, k0);
  if (row0 >= sp.nq) return;
  const int lane = lane_id(), h = lane >> 5, w0 = row0 + wave_id() * 32, i = w0 + (lane & 31);
  const bool there = i < sp.nq;
  Op<DT> qf[STEPS];
  own_rows<DT, STEPS>(qf, row_of(a.q, q0 + i, head), there, a.d, h);
  const int vis = there ? sp.vis(i) : 0;
  const int wave_vis = w0 < sp.nq ? sp.vis(min(w0 + 31, sp.nq - 1)) : 0, wave_full = w0 < sp.nq ? sp.vis(w0) : 0;
  const int end = sp.vis(min(row0 + kSlotRows - 1, sp.nq - 1));
  const Score<DT> sc(a, head);
  const bool simple = sc.simple(a);
  const float place = (float)(i + sp.shift);

  f32x16 o[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) o[b] = f32x16{};
  float m = -kInf, l = 0.0f;

  const char* kb = row_of(a.k, k0, hk);
  const char* vb = row_of(a.v, k0, hk);
  const int tiles = (end + BK - 1) / BK;
  Staged<DT, DP, BK> tk, tv;
  if (tiles > 0) {
    tk.load(kb, a.k.st, sp.nk, a.d);
    tv.load(vb, a.v.st, sp.nk, a.d);
    tk.store(sk[0]);
    tv.store(sv[0]);
  }
  __syncthreads();
  for (int t = 0; t < tiles; ++t) {
    const int j0 = t * BK;
    if (t + 1 < tiles) {
      tk.load(kb + (int64_t)(j0 + BK) * a.k.st, a.k.st, sp.nk - j0 - BK, a.d);
      tv.load(vb + (int64_t)(j0 + BK) * a.v.st, a.v.st, sp.nk - j0 - BK, a.d);
    }
    if (j0 < wave_vis) {
      const char* ks = sk[t & 1];
      const char* vs = sv[t & 1];
      f32x16 s[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        s[u] = f32x16{};
#pragma unroll
        for (int st = 0; st < STEPS; ++st) s[u] = Op<DT>::mma(T::by_row(ks, 32 * u + (lane & 31), st, h), qf[st], s[u]);
      }
      float c = sc.c;
      if (!simple) {
        c = 1.0f;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            float x = sc.bend ? bent<DT>(s[u][r] * sc.zs) * sc.cl : s[u][r] * sc.c;
            s[u][r] = x - sc.slope * fabsf(place - (float)(j0 + 32 * u + acc_row(r, h)));
          }
      }
      if (j0 + BK > wave_full) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (j0 + 32 * u + acc_row(r, h) >= vis) s[u][r] = -kInf;
      }
      float top = s[0][0];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, s[u][r]);
      top = fmaxf(top, other_half(top));
      const float m1 = fmaxf(m, top * c);
      const float ms = m1 == -kInf ? 0.0f : m1;  // nothing seen yet: every weight below is exp2(-inf)
      if (__ballot(m1 > m)) {
        const float f = __builtin_amdgcn_exp2f(m - ms);
        l *= f;
#pragma unroll
        for (int b = 0; b < NB; ++b) o[b] *= f;
        m = m1;
      }
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          Op<DT> p;
#pragma unroll
          for (int r = 0; r < 8; ++r) {
            const float e = __builtin_amdgcn_exp2f(fmaf(s[u][8 * g + r], c, -ms));
            l += e;
            p.set(r, e);
          }
#pragma unroll
          for (int b = 0; b < NB; ++b) o[b] = Op<DT>::mma(T::by_column(vs, 32 * u + 16 * g, b, lane), p, o[b]);
        }
    }
    if (t + 1 < tiles) {
      tk.store(sk[(t + 1) & 1]);
      tv.store(sv[(t + 1) & 1]);
    }
    __syncthreads();
  }
  l += other_half(l);
  if (!there) return;
  store_rows<DT, NB>(o, l > 0.0f ? 1.0f / l : 0.0f, row_of(a.out, q0 + i, head), a.d, h);
  if (a.lse && h == 0) a.lse[(int64_t)head * a.Tq + q0 + i] = l > 0.0f ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -kInf;
}

// Weight and score gradient of one product: s -> p = exp2(score - lse), ds = p (dp - delta) d score / d product / scale
template <int DT>
__device__ inline void weight_and_grad(const Score<DT>& sc, float s, float away, float lse2, float dp, float delta, float& p, float& ds) {
  float x, f = 1.0f;
  if (sc.bend) {
    const float t = bent<DT>(s * sc.zs);
    x = t * sc.cl;
    f = 1.0f - t * t;
  } else {
    x = s * sc.c;
  }
  p = __builtin_amdgcn_exp2f(x - sc.slope * away - lse2);
  ds = p * (dp - delta) * f;
}

// a row's lse in powers of two, +inf (all weights 0) for a row that sees nothing or is not there
__device__ inline float lse2_of(const float* lse, int64_t at, bool there) {
  if (!there) return kInf;
  const float x = lse[at];
  return x == -kInf ? kInf : x * kLog2e;
}

// ---------------------------------------------------------------------------------------------------------------
// Queries' gradient, and delta = <dout, out> of every row for the kernel after it.  As the forward, with
// dP^T = V dO^T beside S^T and dQ^T = K^T dS^T.
template <int DT, int DP>
__global__ __launch_bounds__(kSeqThreads, DT == DLRM_F32 ? 1 : 2) void seq_attn_dq_kernel(SeqArgs a) {
  constexpr int BK = 32, STEPS = DP / 16, NB = DP / 32;
  typedef Tile<DT, DP> T;
  __shared__ __attribute__((aligned(16))) char sk[2][BK * T::STRIDE];
  __shared__ __attribute__((aligned(16))) char sv[2][BK * T::STRIDE];
  const int hh = blockIdx.x % a.Hq, slot = a.slots - 1 - blockIdx.x / a.Hq;
  const int G = a.Hq / a.Hk, hk = hh % a.Hk, head = hk * G + hh / a.Hk;
  int seq, row0;
  find_slot(a.q_off, a.B, a.per_seq, slot, seq, row0);
  int64_t q0, k0;
  const Span sp = span_of(a, seq, q0, k0);
  if (row0 >= sp.nq) return;
  const int lane = lane_id(), h = lane >> 5, w0 = row0 + wave_id() * 32, i = w0 + (lane & 31);
  const bool there = i < sp.nq;
  Op<DT> qf[STEPS], df[STEPS];
  own_rows<DT, STEPS>(qf, row_of(a.q, q0 + i, head), there, a.d, h);
  own_rows<DT, STEPS>(df, row_of(a.dout, q0 + i, head), there, a.d, h);
  float delta = 0.0f;
  {
    Op<DT> of[STEPS];
    own_rows<DT, STEPS>(of, row_of(a.out, q0 + i, head), there, a.d, h);
#pragma unroll
    for (int s = 0; s < STEPS; ++s)
#pragma unroll
      for (int j = 0; j < 8; ++j) delta += of[s].get(j) * df[s].get(j);
    delta += other_half(delta);
  }
  const int64_t at = (int64_t)head * a.Tq + q0 + i;
  if (there && h == 0) a.delta[at] = delta;
  const float lse2 = lse2_of(a.lse, at, there);
  const int vis = there ? sp.vis(i) : 0;
  const int wave_vis = w0 < sp.nq ? sp.vis(min(w0 + 31, sp.nq - 1)) : 0, wave_full = w0 < sp.nq ? sp.vis(w0) : 0;
  const int end = sp.vis(min(row0 + kSlotRows - 1, sp.nq - 1));
  const Score<DT> sc(a, head);
  const float place = (float)(i + sp.shift);

  f32x16 g[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) g[b] = f32x16{};
  const char* kb = row_of(a.k, k0, hk);
  const char* vb = row_of(a.v, k0, hk);
  const int tiles = (end + BK - 1) / BK;
  Staged<DT, DP, BK> tk, tv;
  if (tiles > 0) {
    tk.load(kb, a.k.st, sp.nk, a.d);
    tv.load(vb, a.v.st, sp.nk, a.d);
    tk.store(sk[0]);
    tv.store(sv[0]);
  }
  __syncthreads();
  for (int t = 0; t < tiles; ++t) {
    const int j0 = t * BK;
    if (t + 1 < tiles) {
      tk.load(kb + (int64_t)(j0 + BK) * a.k.st, a.k.st, sp.nk - j0 - BK, a.d);
      tv.load(vb + (int64_t)(j0 + BK) * a.v.st, a.v.st, sp.nk - j0 - BK, a.d);
    }
    if (j0 < wave_vis) {
      const char* ks = sk[t & 1];
      const char* vs = sv[t & 1];
      f32x16 s = {}, dp = {};
#pragma unroll
      for (int st = 0; st < STEPS; ++st) {
        s = Op<DT>::mma(T::by_row(ks, lane & 31, st, h), qf[st], s);
        dp = Op<DT>::mma(T::by_row(vs, lane & 31, st, h), df[st], dp);
      }
      const bool masked = j0 + BK > wave_full;
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        Op<DT> ds;
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          const int j = j0 + acc_row(8 * c + r, h);
          float p, x;
          weight_and_grad<DT>(sc, s[8 * c + r], fabsf(place - (float)j), lse2, dp[8 * c + r], delta, p, x);
          if (masked && j >= vis) x = 0.0f;
          ds.set(r, x);
        }
#pragma unroll
        for (int b = 0; b < NB; ++b) g[b] = Op<DT>::mma(T::by_column(ks, 16 * c, b, lane), ds, g[b]);
      }
    }
    if (t + 1 < tiles) {
      tk.store(sk[(t + 1) & 1]);
      tv.store(sv[(t + 1) & 1]);
    }
    __syncthreads();
  }
  if (there) store_rows<DT, NB>(g, a.scale, row_of(a.dq, q0 + i, head), a.d, h);
}

// ---------------------------------------------------------------------------------------------------------------
// Keys' and values' gradients: a workgroup takes 128 keys of one key head (32 a wavefront); the queries and upstream gradients of
// all query heads that share it go by in tiles, so the sum over the heads stays in registers.
// S = Q K^T and dP = dO V^T have the keys as columns; dV^T = dO^T P and dK^T = Q^T dS.
template <int DT, int DP>
__global__ __launch_bounds__(kSeqThreads, 1) void seq_attn_dkv_kernel(SeqArgs a) {
  constexpr int BQ = 32, STEPS = DP / 16, NB = DP / 32;
  typedef Tile<DT, DP> T;
  __shared__ __attribute__((aligned(16))) char sq[2][BQ * T::STRIDE];
  __shared__ __attribute__((aligned(16))) char sd[2][BQ * T::STRIDE];
  __shared__ __attribute__((aligned(16))) float stat[2][2][BQ];  // lse2, delta
  const int hk = blockIdx.x % a.Hk, slot = blockIdx.x / a.Hk;  // early keys are seen by most queries: first
  const int G = a.Hq / a.Hk;
  int seq, row0;
  find_slot(a.k_off, a.B, a.per_seq, slot, seq, row0);
  int64_t q0, k0;
  const Span sp = span_of(a, seq, q0, k0);
  if (row0 >= sp.nk) return;
  const int lane = lane_id(), h = lane >> 5, w0 = row0 + wave_id() * 32, j = w0 + (lane & 31);
  const bool there = j < sp.nk;
  Op<DT> kf[STEPS], vf[STEPS];
  own_rows<DT, STEPS>(kf, row_of(a.k, k0 + j, hk), there, a.d, h);
  own_rows<DT, STEPS>(vf, row_of(a.v, k0 + j, hk), there, a.d, h);
  const int from = there ? sp.first_query(j) : 0x7fffffff;
  const int wave_from = w0 < sp.nk ? sp.first_query(w0) : 0x7fffffff;
  const int wave_full = w0 < sp.nk ? sp.first_query(min(w0 + 31, sp.nk - 1)) : 0x7fffffff;
  const int t0 = sp.first_query(row0) / BQ, tiles = max(0, (sp.nq + BQ - 1) / BQ - t0);

  f32x16 gk[NB], gv[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) gk[b] = gv[b] = f32x16{};
  Staged<DT, DP, BQ> tq, td;
  float st0 = 0.0f;
  auto fetch = [&](int n) {  // tile n of all heads' tiles
    const int head = hk * G + n / tiles, i0 = (t0 + n % tiles) * BQ;
    tq.load(row_of(a.q, q0 + i0, head), a.q.st, sp.nq - i0, a.d);
    td.load(row_of(a.dout, q0 + i0, head), a.dout.st, sp.nq - i0, a.d);
    if (threadIdx.x < 2 * BQ) {
      const int i = threadIdx.x % BQ;
      const int64_t at = (int64_t)head * a.Tq + q0 + i0 + i;
      const bool row = i0 + i < sp.nq;
      st0 = threadIdx.x < BQ ? lse2_of(a.lse, at, row) : row ? a.delta[at] : 0.0f;
    }
  };
  auto put = [&](int n) {
    tq.store(sq[n & 1]);
    td.store(sd[n & 1]);
    if (threadIdx.x < 2 * BQ) stat[n & 1][threadIdx.x / BQ][threadIdx.x % BQ] = st0;
  };
  const int all = tiles * G;
  if (all > 0) {
    fetch(0);
    put(0);
  }
  __syncthreads();
  for (int n = 0; n < all; ++n) {
    if (n + 1 < all) fetch(n + 1);
    const int i0 = (t0 + n % tiles) * BQ;
    if (i0 + BQ > wave_from) {
      const Score<DT> sc(a, hk * G + n / tiles);
      const char* qs = sq[n & 1];
      const char* ds_ = sd[n & 1];
      f32x16 s = {}, dp = {};
#pragma unroll
      for (int st = 0; st < STEPS; ++st) {
        s = Op<DT>::mma(T::by_row(qs, lane & 31, st, h), kf[st], s);
        dp = Op<DT>::mma(T::by_row(ds_, lane & 31, st, h), vf[st], dp);
      }
      const bool masked = i0 < wave_full;
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        Op<DT> p, ds;
#pragma unroll
        for (int r4 = 0; r4 < 2; ++r4) {
          const f32x4 lse2 = *reinterpret_cast<const f32x4*>(&stat[n & 1][0][acc_row(8 * c + 4 * r4, h)]);
          const f32x4 del = *reinterpret_cast<const f32x4*>(&stat[n & 1][1][acc_row(8 * c + 4 * r4, h)]);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int i = i0 + acc_row(8 * c + 4 * r4 + r, h);
            float w, x;
            weight_and_grad<DT>(sc, s[8 * c + 4 * r4 + r], fabsf((float)(i + sp.shift) - (float)j), lse2[r], dp[8 * c + 4 * r4 + r], del[r], w, x);
            if (masked && i < from) w = x = 0.0f;
            p.set(4 * r4 + r, w);
            ds.set(4 * r4 + r, x);
          }
        }
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          gv[b] = Op<DT>::mma(T::by_column(ds_, 16 * c, b, lane), p, gv[b]);
          gk[b] = Op<DT>::mma(T::by_column(qs, 16 * c, b, lane), ds, gk[b]);
        }
      }
    }
    if (n + 1 < all) put(n + 1);
    __syncthreads();
  }
  if (!there) return;
  store_rows<DT, NB>(gk, a.scale, row_of(a.dk, k0 + j, hk), a.d, h);
  store_rows<DT, NB>(gv, 1.0f, row_of(a.dv, k0 + j, hk), a.d, h);
}

// ---------------------------------------------------------------------------------------------------------------
// slots of 128 rows for n rows in B sequences of at most `longest`
__host__ inline bool slots_of(SeqArgs& a, int64_t n, int longest, int heads) {
  const int64_t each = ((int64_t)longest + kSlotRows - 1) / kSlotRows;
  const int64_t even = each * a.B, searched = n / kSlotRows + a.B;
  a.per_seq = even <= searched ? (int)each : 0;
  const int64_t s = even <= searched ? even : searched;
  a.slots = (int)s;
  return s * heads <= 0x7fffffff;
}

template <int DT, typename F>
__host__ inline int for_width(int d, F f) {
  if (d <= 32) return f(std::integral_constant<int, 32>{});
  if (d <= 64) return f(std::integral_constant<int, 64>{});
  if (d <= 96) return f(std::integral_constant<int, 96>{});
  return f(std::integral_constant<int, 128>{});
}

template <int DT>
int launch_seq_fwd(const dlrm_seq_batch* s, SeqArgs a, hipStream_t st) {
  if (!slots_of(a, s->Tq, s->max_q, a.Hq)) return DLRM_ERR_BAD_SHAPE;
  if (a.slots == 0) return DLRM_OK;
  return for_width<DT>(a.d, [&](auto dp) {
    hipLaunchKernelGGL((seq_attn_fwd_kernel<DT, dp()>), dim3((unsigned)(a.slots * a.Hq)), dim3(kSeqThreads), 0, st, a);
    DLRM_CHECK_LAUNCH();
    return (int)DLRM_OK;
  });
}

template <int DT>
int launch_seq_bwd(const dlrm_seq_batch* s, SeqArgs a, hipStream_t st) {
  SeqArgs b = a;
  if (!slots_of(a, s->Tq, s->max_q, a.Hq) || !slots_of(b, s->Tk, s->max_k, a.Hk)) return DLRM_ERR_BAD_SHAPE;
  return for_width<DT>(a.d, [&](auto dp) {
    if (a.slots > 0) {
      hipLaunchKernelGGL((seq_attn_dq_kernel<DT, dp()>), dim3((unsigned)(a.slots * a.Hq)), dim3(kSeqThreads), 0, st, a);
      DLRM_CHECK_LAUNCH();
    }
    if (b.slots > 0) {
      hipLaunchKernelGGL((seq_attn_dkv_kernel<DT, dp()>), dim3((unsigned)(b.slots * b.Hk)), dim3(kSeqThreads), 0, st, b);
      DLRM_CHECK_LAUNCH();
    }
    return (int)DLRM_OK;
  });
}

extern template int launch_seq_fwd<DLRM_F32>(const dlrm_seq_batch*, SeqArgs, hipStream_t);
extern template int launch_seq_fwd<DLRM_F16>(const dlrm_seq_batch*, SeqArgs, hipStream_t);
extern template int launch_seq_fwd<DLRM_BF16>(const dlrm_seq_batch*, SeqArgs, hipStream_t);
extern template int launch_seq_bwd<DLRM_F32>(const dlrm_seq_batch*, SeqArgs, hipStream_t);
extern template int launch_seq_bwd<DLRM_F16>(const dlrm_seq_batch*, SeqArgs, hipStream_t);
extern template int launch_seq_bwd<DLRM_BF16>(const dlrm_seq_batch*, SeqArgs, hipStream_t);

}  // namespace dlrm
