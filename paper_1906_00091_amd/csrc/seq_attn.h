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
// A wavefront that multiplies goes before one that does not (s_setprio): the two of a SIMD then take the matrix core and the vector unit
// by turns (8 histories of up to 4096 items: 2 to 3 % of each kernel).
//
// fp32 operands run the same code: a fragment of 8 values a lane is 8 products of mfma 32x32x2 in place of one of 32x32x16.
// With 16-bit types the weights and their gradients are rounded to that type before the second product, as the matrix cores
// take it; sums of weights and all accumulators stay fp32.  fp16 has few exponents (2^-14 to 2^15 at full precision), so there both are multiplied by
// powers of two that the accumulators are divided by at the end: weights by one that takes the largest possible to 2^15, gradients by one that
// follows the largest met so far (lift_for).  Short walks of up to 64 columns wait for most of their time: they take weights and gradients in two parts, the
// second what the first one's rounding leaves, so that a result's error is its own rounding (2048 histories of up to 200 items, bf16: out 1.9e-3 -> 1.6e-3
// off, dk and dv 2.3e-3 -> 1.7e-3, for 3 % of the time).  Long walks would pay a quarter to a third for it (8 histories of up to 4096 items: 1865 -> 2480 us).
#pragma once

#include <type_traits>

#include "heads.h"

namespace dlrm {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

template <int N>
using Int = std::integral_constant<int, N>;

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

template <int DT>
__device__ inline void op_two_parts(const float* w, Op<DT>& high, Op<DT>& low) {
  u32x4 h, l;
  two_parts<DT>(w, h, l);
  high.v = __builtin_bit_cast(decltype(high.v), h);
  low.v = __builtin_bit_cast(decltype(low.v), l);
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

// Buffer descriptor of `bytes` from base on: loads past them give zeros.  base and bytes are the same for the whole wavefront.
__device__ inline __amdgpu_buffer_rsrc_t span_of_bytes(const char* base, uint32_t bytes) {
  const uint64_t p = reinterpret_cast<uint64_t>(base);
  const uint64_t u = (uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(p >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)p);
  return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(u), 0, __builtin_amdgcn_readfirstlane(bytes), 0x00027000);
}

// A tile on its way from global memory to LDS, in the registers of the workgroup's threads.  Rows past the sequence and columns past d
// are zeros, by the bounds of the buffer descriptor: the loads stand in no branch, so nothing waits for them before the store.
template <int DT, int DP, int ROWS, int THREADS>
struct Staged {
  static constexpr int CH = DP * Tab<DT>::EB / 16;  // chunks of 16 bytes in a row
  static constexpr int N = (ROWS * CH + THREADS - 1) / THREADS;
  u32x4 v[N];
  uint32_t at[N];  // byte offset of each chunk in the tile
  __device__ inline Staged(int64_t stride, int d) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int id = threadIdx.x + i * THREADS, r = id / CH, c = id % CH;
      at[i] = r < ROWS && c * Tab<DT>::ELEMS < d ? (uint32_t)r * (uint32_t)stride + c * 16u : 0xfffffff0u;
    }
  }
  // the n >= 1 rows from base on
  __device__ inline void load(const char* base, int64_t stride, int n, int d) {
    const auto rs = span_of_bytes(base, (uint32_t)(min(n, ROWS) - 1) * (uint32_t)stride + d * Tab<DT>::EB);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = __builtin_amdgcn_raw_buffer_load_b128(rs, at[i], 0, 0);
  }
  __device__ inline void store(char* s) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int id = threadIdx.x + i * THREADS, r = id / CH, c = id % CH;
      if (ROWS * CH % THREADS == 0 || r < ROWS) *reinterpret_cast<u32x4*>(s + r * Tile<DT, DP>::STRIDE + c * 16) = v[i];
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
  float* part;   // [splits][dk, dv][Tk][Hk][d]: sums of the keys' gradients where several workgroups share a block's queries
  int64_t Tq, Tk;
  int B, Hq, Hk, d, causal;
  int splits;    // workgroups that share a block of rows (keys' gradients)
  int by_block;  // the grid is (walk, sequence, block), else walks times slots
  int slots, slot0;  // slots in all, and the first of this launch
  float scale, cap;
};

// Workgroup -> walk (key head + Hk * split), sequence and first row, blocks of ROWS rows, `per` rows for each item of `off`.  A sequence with n rows needs
// ceil(n / ROWS) blocks, and how many rows it has stands in device memory.
// Where all sequences fit into few blocks the grid is (walk, sequence, block), as many blocks as the longest may need: block by block
// through all sequences, so with causal sequences the blocks of most work of every one of them start first.  Else it is walks times
// slots: sequence s starts at slot off[s] * per / ROWS + s, which leaves it enough, and is found by all 64 lanes at once, each step
// asking 64 places; more slots than a launch has threads for go in several.  Workgroups past a sequence's rows end at once.
template <int ROWS>
__device__ inline void find_block(const SeqArgs& a, const int64_t* off, int per, bool last_first, int& walk, int& seq, int& row0) {
  const int walks = a.Hk * a.splits;
  if (a.by_block) {
    walk = blockIdx.x;
    // turned from block to block: workgroups go to the 8 dies in turn, and no die gets all of the same sequences
    seq = blockIdx.y + blockIdx.z;
    if (seq >= a.B) seq %= a.B;
    row0 = (last_first ? gridDim.z - 1 - blockIdx.z : blockIdx.z) * ROWS;
    return;
  }
  const int at = blockIdx.x / walks, slot = last_first ? a.slots - 1 - (a.slot0 + at) : a.slot0 + at;
  walk = blockIdx.x - at * walks;
  int lo = 0, hi = a.B;
  while (hi - lo > 1) {
    const int step = (hi - lo + 63) >> 6, s = lo + lane_id() * step;
    const bool before = s < hi && off[s] * per / ROWS + s <= slot;
    const int n = __popcll(__ballot(before));  // >= 1: the first place always is
    hi = min(lo + n * step, hi);
    lo = lo + (n - 1) * step;
  }
  seq = __builtin_amdgcn_readfirstlane(lo);
  row0 = (slot - (int)(off[seq] * per / ROWS) - seq) * ROWS;
}

// What a score is made of, fixed at compile time: without a cap and slopes an element costs a multiply-add and an exponential.
enum { kPlain = 0, kSlopes = 1, kBend = 2, kLarge = 4 };  // bits; kLarge: a cap that 16-bit rows take as fp32 rows do (with kBend and, slopes or none, kSlopes)

// The score of a product s is, in powers of two, c * y(s) + base - slope * |distance|:
//   without a cap  y = s, c = scale log2 e, base = 0;
//   with a cap     tanh(z) = 1 - 2 r, r = 1 / (exp(2 z) + 1): an exponential and a reciprocal; y = -r, c = 2 cap log2 e,
//                  base = cap log2 e, and the derivative 1 - tanh^2 is 4 r (1 - r) = -4 (y + y^2);
//   fp32 with cap  y = tanh(z) of the library, whose error near 0 is relative; c = cap log2 e, base = 0, derivative 1 - y^2.
// The second form's r is off by up to 2^-23, the score by cap 2^-22 and, with what rounding `base` adds, less than cap 2^-21 whatever its size: an eighth of
// what rounding the weight to 16 bits is at a cap of 128 (fp16) or 1024 (bf16).  Larger caps take the third form, in one cut of each kernel.
// The derivative's constant factor goes into `grad`, which the gradients are multiplied by at the end, as scale does.
template <int DT, int KIND>
struct Score {
  static constexpr bool BEND = (KIND & kBend) != 0, FAST = DT != DLRM_F32 && (KIND & kLarge) == 0;
  float zs, c, base, slope, grad;
  __device__ inline Score(const SeqArgs& a, int head) {
    zs = BEND ? a.scale / a.cap * (FAST ? 2.0f * kLog2e : 1.0f) : 0.0f;
    c = BEND ? a.cap * (FAST ? 2.0f * kLog2e : kLog2e) : a.scale * kLog2e;
    base = BEND && FAST ? a.cap * kLog2e : 0.0f;
    slope = (KIND & kSlopes) && ((KIND & kLarge) == 0 || a.slopes) ? a.slopes[head] * kLog2e : 0.0f;
    grad = BEND && FAST ? -4.0f * a.scale : a.scale;
  }
  __device__ inline float y(float s) const {
    if constexpr (!BEND) return s;
    if constexpr (FAST) return __builtin_amdgcn_rcpf(-1.0f - __builtin_amdgcn_exp2f(s * zs));
    return tanhf(s * zs);
  }
  // exponent of 2 of a weight: the score less `rest`
  __device__ inline float exponent(float y, float away, float rest) const {
    if constexpr ((KIND & kSlopes) != 0) return fmaf(y, c, fmaf(-slope, fabsf(away), -rest));
    return fmaf(y, c, -rest);
  }
  __device__ inline float derivative(float y) const {
    if constexpr (!BEND) return 1.0f;
    return FAST ? fmaf(y, y, y) : fmaf(-y, y, 1.0f);
  }
};

// fp16: log2 of what the weights are multiplied by where they are at most 2^8 (forward, see there) and 1 (gradients)
template <int DT>
constexpr float kWeightLift = DT == DLRM_F16 ? 7.0f : 0.0f;
template <int DT>
constexpr float kGradWeightLift = DT == DLRM_F16 ? 15.0f : 0.0f;

// fp16: the power of two that takes a value of size `top` to 2^8, with room to grow below 2^15 and 22 binades above full precision's end
__device__ inline float lift_for(float top) { return 8.0f - ceilf(__builtin_amdgcn_logf(top)); }
__device__ inline float largest(const f32x16& x) {
  float top = 0.0f;
#pragma unroll
  for (int r = 0; r < 16; ++r) top = fmaxf(top, fabsf(x[r]));
  return top;
}
// whether a gradient of size `top` leaves fp16 (an infinity is not made finite)
__device__ inline bool too_large(float top) { return top > 32768.0f && top < kInf; }

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

// The last step of a product over the columns has none below d where d <= DP - 16.  In fp32 it is left out, where its 8 products of 64 cycles would
// add zeros (13 histories of up to 1999 items, d 72: forward 310 -> 290 us, queries' gradient 430 -> 392, keys' 560 -> 538).
template <int DT, int STEPS>
__device__ inline bool past_d(int st, int d) {
  return DT == DLRM_F32 && st == STEPS - 1 && d <= 16 * st;
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

// ---------------------------------------------------------------------------------------------------------------
// Rows of the forward and of the queries' gradient: the queries of all query heads that share a key head, item by item, are the rows of one
// walk over its keys: row r is item r / G, head r % G of the G.  Short histories and few candidates fill a wavefront's rows this way,
// the keys pass through LDS once for all G, and a causal block ends G times nearer to its diagonal.
// GROUPS x 32 rows a workgroup; PARTS wavefronts share 32 rows, each with its part of a tile's keys, and join at the end: where the rows
// are few, or a product is slow (fp32), the longest rows' walk is what the call waits for.
struct MyRow {
  int64_t t;  // item of q, out, ...
  int i, head;
  bool there;
};
template <int GROUPS, int PARTS>
struct RowWork {
  int seq, row0, group, part, hk, G;
  int64_t q0, k0;
  Span sp;
  MyRow me;
  int vis, wave_vis, wave_full, end;  // keys that my row, the wavefront's last, its first, and the workgroup's last row see
  __device__ inline bool find(const SeqArgs& a) {
    constexpr int ROWS = 32 * GROUPS;
    G = a.Hq / a.Hk;
    find_block<ROWS>(a, a.q_off, G, true, hk, seq, row0);  // late rows see most keys
    sp = span_of(a, seq, q0, k0);
    const int rows = sp.nq * G;
    if (row0 >= rows) return false;
    group = wave_id() % GROUPS;
    part = wave_id() / GROUPS;
    const int w0 = row0 + group * 32, r = w0 + (lane_id() & 31);
    me.there = r < rows;
    auto item = [&](int row) { return G == 1 ? row : row / G; };
    me.i = me.there ? item(r) : 0;
    me.head = hk * G + (me.there ? r - me.i * G : 0);
    me.t = q0 + me.i;
    vis = me.there ? sp.vis(me.i) : 0;
    wave_vis = w0 < rows ? sp.vis(item(min(w0 + 31, rows - 1))) : 0;
    wave_full = w0 < rows ? sp.vis(item(w0)) : 0;
    end = sp.vis(item(min(row0 + ROWS - 1, rows - 1)));
    return true;
  }
};

// x of part 0 becomes x f[0] + (x of part 1) f[1] + ..., through LDS; LDS has to be free.
template <int NB, int GROUPS, int PARTS>
__device__ inline void join_parts(f32x16* x, char* lds, int group, int part, const float* f) {
  constexpr int REGION = GROUPS * NB * 4 * DLRM_WAVE;
  f32x4* at = reinterpret_cast<f32x4*>(lds) + group * NB * 4 * DLRM_WAVE + lane_id();
  if (part > 0) {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        at[(part - 1) * REGION + (b * 4 + q) * DLRM_WAVE] = f32x4{x[b][4 * q], x[b][4 * q + 1], x[b][4 * q + 2], x[b][4 * q + 3]};
  }
  __syncthreads();
  if (part == 0) {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[b][4 * q + e] *= f[0];
#pragma unroll
        for (int p = 1; p < PARTS; ++p) {
          const f32x4 y = at[(p - 1) * REGION + (b * 4 + q) * DLRM_WAVE];
#pragma unroll
          for (int e = 0; e < 4; ++e) x[b][4 * q + e] = fmaf(y[e], f[p], x[b][4 * q + e]);
        }
      }
  }
}

// LDS of a kernel that walks over tiles of BK keys: two tiles of keys and values, one where eight parts take so many keys at a time, or the
// parts' sums.
template <int DT, int DP, int GROUPS, int PARTS, int SUB>
struct Walk {
  static constexpr int BK = 32 * SUB * PARTS, BUFS = PARTS > 2 ? 1 : 2, TILE = BK * Tile<DT, DP>::STRIDE;
  static constexpr int JOIN = (PARTS - 1) * GROUPS * DP / 2 * DLRM_WAVE * 4;
  static constexpr int LDS = 2 * BUFS * TILE > JOIN ? 2 * BUFS * TILE : JOIN;
};

// Wavefronts of a SIMD that the forward's registers are to leave room for: four for short walks of narrow 16-bit rows, one where the rows are
// too few to give a SIMD two.
constexpr int fwd_resident(int dt, int dp, int groups, int parts, int sub) {
  if (groups == 2) return 1;
  return groups == 4 && parts * sub == 1 && dp <= 64 && dt != DLRM_F32 ? 4 : 2;
}

// Forward: tiles of keys and values go by, SUB x 32 keys for each part, two tiles in LDS.
// 8 histories of 2048 to 4096 items, 16 query heads on 4, bf16, d 128, causal, capped: 431 us, 752 TFLOP/s of visible pairs (a large library product
// of bf16 on the same card: 1192), bound by the exponentials and reciprocals beside the products: two wavefronts a SIMD, each of which can
// multiply while the other does not.  2048 histories of up to 200 items, 4 heads, d 64, slopes: 127 us; a workgroup walks over four tiles and
// waits for most of its time (four a CU hide part of it).  fp32, 13 histories of up to 1999 items, d 72: 281 us, 59 TFLOP/s of 154, and 72 with
// the columns that pad 72 to 96.
template <int DT, int DP, int KIND, int GROUPS, int PARTS, int SUB>
__global__ __launch_bounds__(64 * GROUPS * PARTS, fwd_resident(DT, DP, GROUPS, PARTS, SUB)) void seq_attn_fwd_kernel(SeqArgs a) {
  typedef Walk<DT, DP, GROUPS, PARTS, SUB> W;
  constexpr int BK = W::BK, TILE = W::TILE, STEPS = DP / 16, NB = DP / 32, THREADS = 64 * GROUPS * PARTS;
  constexpr bool TWO = DT != DLRM_F32 && DP <= 64 && PARTS * SUB == 1;  // weights in two parts
  typedef Tile<DT, DP> T;
  __shared__ __attribute__((aligned(16))) char lds[W::LDS];
  __shared__ float stat[PARTS > 1 ? PARTS * GROUPS * 2 * 32 : 1];
  RowWork<GROUPS, PARTS> w;
  if (!w.find(a)) return;
  const Span& sp = w.sp;
  const int lane = lane_id(), h = lane >> 5;
  Op<DT> qf[STEPS];
  own_rows<DT, STEPS>(qf, row_of(a.q, w.me.t, w.me.head), w.me.there, a.d, h);
  const Score<DT, KIND> sc(a, w.me.head);
  const int place = w.me.i + sp.shift;  // (distances are taken as integers: fp32 has no odd place past 2^24)

  f32x16 o[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) o[b] = f32x16{};
  float m = -kInf, l = 0.0f;

  const char* kb = row_of(a.k, w.k0, w.hk);
  const char* vb = row_of(a.v, w.k0, w.hk);
  const int tiles = (w.end + BK - 1) / BK;
  Staged<DT, DP, BK, THREADS> tk(a.k.st, a.d), tv(a.v.st, a.d);
  if (tiles > 0) {
    tk.load(kb, a.k.st, sp.nk, a.d);
    tv.load(vb, a.v.st, sp.nk, a.d);
    tk.store(lds);
    tv.store(lds + TILE);
  }
  __syncthreads();
  for (int t = 0; t < tiles; ++t) {
    const int jt = t * BK;
    if (t + 1 < tiles) {
      tk.load(kb + (int64_t)(jt + BK) * a.k.st, a.k.st, sp.nk - jt - BK, a.d);
      tv.load(vb + (int64_t)(jt + BK) * a.v.st, a.v.st, sp.nk - jt - BK, a.d);
    }
    const int j0 = jt + 32 * SUB * w.part;
    if (j0 < w.wave_vis) {
      const char* ks = lds + (t & (W::BUFS - 1)) * 2 * TILE + 32 * SUB * w.part * T::STRIDE;
      const char* vs = ks + TILE;
      f32x16 s[SUB];
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int u = 0; u < SUB; ++u) {
        s[u] = f32x16{};
#pragma unroll
        for (int st = 0; st < STEPS; ++st) {
          if (past_d<DT, STEPS>(st, a.d)) break;
          s[u] = Op<DT>::mma(T::by_row(ks, 32 * u + (lane & 31), st, h), qf[st], s[u]);
        }
      }
      __builtin_amdgcn_s_setprio(0);
      // with slopes the whole score, else what the factor c still goes to, in the multiply-add before the exponential
      const float c = KIND & kSlopes ? 1.0f : sc.c;
      if constexpr (KIND != kPlain) {
        const float away = (float)(place - (j0 + 4 * h));
#pragma unroll
        for (int u = 0; u < SUB; ++u)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            s[u][r] = sc.y(s[u][r]);
            if constexpr ((KIND & kSlopes) != 0) s[u][r] = sc.exponent(s[u][r], away - (float)(32 * u + acc_row(r, 0)), 0.0f);
          }
      }
      if (j0 + 32 * SUB > w.wave_full) {
#pragma unroll
        for (int u = 0; u < SUB; ++u)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (j0 + 32 * u + acc_row(r, h) >= w.vis) s[u][r] = -kInf;
      }
      float top = s[0][0];
#pragma unroll
      for (int u = 0; u < SUB; ++u)
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, s[u][r]);
      top = fmaxf(top, other_half(top));
      // The sums are rescaled only where a maximum grew by more than 2^8: until then weights of up to 2^8 are as good as weights of
      // up to 1 (fp32 sums; 16-bit weights keep their relative precision).  Exact either way: m is whatever the sums were made with.
      if (__ballot(top * c > m + 8.0f)) {
        const float m1 = fmaxf(m, top * c);
        const float f = __builtin_amdgcn_exp2f(m - (m1 == -kInf ? 0.0f : m1));
        l *= f;
#pragma unroll
        for (int b = 0; b < NB; ++b) o[b] *= f;
        m = m1;
      }
      const float ms = m == -kInf ? 0.0f : m - kWeightLift<DT>;  // nothing seen yet: every weight below is exp2(-inf)
#pragma unroll
      for (int u = 0; u < SUB; ++u)
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          Op<DT> p, low;
          float e[8];
#pragma unroll
          for (int r = 0; r < 8; ++r) {
            e[r] = __builtin_amdgcn_exp2f(fmaf(s[u][8 * g + r], c, -ms));
            l += e[r];
            if constexpr (!TWO) p.set(r, e[r]);
          }
          if constexpr (TWO) op_two_parts(e, p, low);
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            const Op<DT> vt = T::by_column(vs, 32 * u + 16 * g, b, lane);
            o[b] = Op<DT>::mma(vt, p, o[b]);
            if constexpr (TWO) o[b] = Op<DT>::mma(vt, low, o[b]);
          }
        }
    }
    if (W::BUFS == 1) __syncthreads();
    if (t + 1 < tiles) {
      tk.store(lds + ((t + 1) & (W::BUFS - 1)) * 2 * TILE);
      tv.store(lds + ((t + 1) & (W::BUFS - 1)) * 2 * TILE + TILE);
    }
    __syncthreads();
  }
  l += other_half(l);
  if constexpr (PARTS > 1) {
    float* st = stat + (w.group * PARTS) * 64 + (lane & 31);
    if (h == 0) {
      st[w.part * 64] = m;
      st[w.part * 64 + 32] = l;
    }
    __syncthreads();
    float top = -kInf, f[PARTS];
#pragma unroll
    for (int p = 0; p < PARTS; ++p) top = fmaxf(top, st[p * 64]);
    const float ts = top == -kInf ? 0.0f : top;
    l = 0.0f;
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
      f[p] = __builtin_amdgcn_exp2f(st[p * 64] - ts);
      l = fmaf(st[p * 64 + 32], f[p], l);
    }
    m = top;
    join_parts<NB, GROUPS, PARTS>(o, lds, w.group, w.part, f);
    if (w.part > 0) return;
  }
  if (!w.me.there) return;
  // (a sum that is NaN is not a row that sees nothing: its lse is NaN too, and the backward's weights with it)
  store_rows<DT, NB>(o, l == 0.0f ? 0.0f : 1.0f / l, row_of(a.out, w.me.t, w.me.head), a.d, h);
  if (a.lse && h == 0)
    a.lse[(int64_t)w.me.head * a.Tq + w.me.t] = l == 0.0f ? -kInf : (m - kWeightLift<DT> + sc.base + __builtin_amdgcn_logf(l)) * kLn2;
}

// a row's lse in powers of two, +inf (all weights 0) for a row that sees nothing or is not there
__device__ inline float lse2_of(float lse, bool there) { return !there || lse == -kInf ? kInf : lse * kLog2e; }

// ---------------------------------------------------------------------------------------------------------------
// Wavefronts of a SIMD that the registers are to leave room for.  fp16 rows of up to 64 columns need one register more than three of them leave, for the
// lift: kept to three (2048 histories of up to 200 items, slopes, forward and backward: 547 us, 586 with two; 535 without a lift), but for slopes and
// a cap together, which would spill eleven.
constexpr int dq_resident(int dt, int dp, int kind, int groups, int parts) {
  if (dt == DLRM_F16 && dp <= 64 && groups == 4 && kind != (kSlopes | kBend)) return 3;
  return groups == 4 || parts == 8 ? 2 : 1;
}

// Queries' gradient, and delta = <dout, out> of every row for the kernel after it.  As the forward, with
// dP^T = V dO^T beside S^T and dQ^T = K^T dS^T.
// The stored output is rounded where rows have 16 bits, and where few keys carry a row's weight that rounding shows in
// ds = p (dp - delta) (a row with one key has dp = delta).  So delta is summed again on the way as sum p dp, in fp32: the kernel after this
// one takes that; a row whose keys all lie in the first 32 has it before its first use here; and for the other rows what the rounding
// of the output leaves is made up for by taking ds in two 16-bit parts, with a second product, where that costs little or is most needed: narrow
// rows (5 %), and slopes, which leave a row few keys of weight (128 columns: 22 %).  dq of the long histories above is 2.4e-3 off (relative, all of it) in one
// part and 1.7e-3 in two, which is its own rounding; of 2048 histories of up to 200 items, slopes, 1.8e-3 in two.
// Bound as the forward is: the sizes above take 576 us (844 TFLOP/s), 197 us and 379 us (66 TFLOP/s).
template <int DT, int DP, int KIND, int GROUPS, int PARTS>
__global__ __launch_bounds__(64 * GROUPS * PARTS, dq_resident(DT, DP, KIND, GROUPS, PARTS)) void seq_attn_dq_kernel(SeqArgs a) {
  typedef Walk<DT, DP, GROUPS, PARTS, 1> W;
  constexpr int BK = W::BK, TILE = W::TILE, STEPS = DP / 16, NB = DP / 32, THREADS = 64 * GROUPS * PARTS;
  constexpr bool TWO = DT != DLRM_F32 && (DP <= 64 || (KIND & kSlopes) != 0);  // ds in two parts
  typedef Tile<DT, DP> T;
  __shared__ __attribute__((aligned(16))) char lds[W::LDS];
  __shared__ float sums[PARTS > 1 ? PARTS * GROUPS * 32 : 1];
  RowWork<GROUPS, PARTS> w;
  if (!w.find(a)) return;
  const Span& sp = w.sp;
  const int lane = lane_id(), h = lane >> 5;
  Op<DT> qf[STEPS], df[STEPS];
  own_rows<DT, STEPS>(qf, row_of(a.q, w.me.t, w.me.head), w.me.there, a.d, h);
  own_rows<DT, STEPS>(df, row_of(a.dout, w.me.t, w.me.head), w.me.there, a.d, h);
  // fp16: ds is made 2^lift times as large.  |dp| <= |dout| |v|, so with 2^lift |dout| near 2^8 values of ordinary size stay far below 2^15, and weights
  // down to 2^-22 above the subnormal numbers; where that does not do, the lift goes down (below).
  constexpr bool LIFT = DT == DLRM_F16;
  float delta = 0.0f, lift = 0.0f;
  {
    Op<DT> of[STEPS];
    own_rows<DT, STEPS>(of, row_of(a.out, w.me.t, w.me.head), w.me.there, a.d, h);
    float square = 0.0f;
#pragma unroll
    for (int s = 0; s < STEPS; ++s)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        delta += of[s].get(j) * df[s].get(j);
        if constexpr (LIFT) square = fmaf(df[s].get(j), df[s].get(j), square);
      }
    delta += other_half(delta);
    if constexpr (LIFT) {
      square += other_half(square);
      if (square > 0.0f && square < kInf) lift = lift_for(sqrtf(square));
    }
  }
  const int64_t at = (int64_t)w.me.head * a.Tq + w.me.t;
  const float lse = w.me.there ? a.lse[at] : 0.0f;
  const Score<DT, KIND> sc(a, w.me.head);
  const int place = w.me.i + sp.shift;
  float rest = lse2_of(lse, w.me.there) - sc.base - lift;  // (so p below is 2^lift times the weight)

  f32x16 g[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) g[b] = f32x16{};
  float sum = 0.0f;  // of p dp
  const char* kb = row_of(a.k, w.k0, w.hk);
  const char* vb = row_of(a.v, w.k0, w.hk);
  const int tiles = (w.end + BK - 1) / BK;
  Staged<DT, DP, BK, THREADS> tk(a.k.st, a.d), tv(a.v.st, a.d);
  if (tiles > 0) {
    tk.load(kb, a.k.st, sp.nk, a.d);
    tv.load(vb, a.v.st, sp.nk, a.d);
    tk.store(lds);
    tv.store(lds + TILE);
  }
  __syncthreads();
  for (int t = 0; t < tiles; ++t) {
    const int jt = t * BK;
    if (t + 1 < tiles) {
      tk.load(kb + (int64_t)(jt + BK) * a.k.st, a.k.st, sp.nk - jt - BK, a.d);
      tv.load(vb + (int64_t)(jt + BK) * a.v.st, a.v.st, sp.nk - jt - BK, a.d);
    }
    const int j0 = jt + 32 * w.part;
    if (j0 < w.wave_vis) {
      const char* ks = lds + (t & (W::BUFS - 1)) * 2 * TILE + 32 * w.part * T::STRIDE;
      const char* vs = ks + TILE;
      f32x16 s = {}, dp = {};
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int st = 0; st < STEPS; ++st) {
        if (past_d<DT, STEPS>(st, a.d)) break;
        s = Op<DT>::mma(T::by_row(ks, lane & 31, st, h), qf[st], s);
        dp = Op<DT>::mma(T::by_row(vs, lane & 31, st, h), df[st], dp);
      }
      __builtin_amdgcn_s_setprio(0);
      const float away = (float)(place - (j0 + 4 * h));
      if (j0 == 0 && w.wave_full <= 32) {  // once a wavefront, and only the first of a sequence
        float all = 0.0f;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float p = __builtin_amdgcn_exp2f(sc.exponent(sc.y(s[r]), away - (float)acc_row(r, 0), rest));
          all += acc_row(r, h) < w.vis ? p * dp[r] : 0.0f;
        }
        all += other_half(all);
        if (w.vis <= 32) delta = all * (LIFT ? __builtin_amdgcn_exp2f(-lift) : 1.0f);
      }
      auto gradient = [&](auto masked) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float y = sc.y(s[r]);
          float p = __builtin_amdgcn_exp2f(sc.exponent(y, away - (float)acc_row(r, 0), rest)), x = dp[r];
          if (masked() && j0 + acc_row(r, h) >= w.vis) p = x = 0.0f;
          sum = fmaf(p, x, sum);
          s[r] = p * (x - delta);
          if constexpr ((KIND & kBend) != 0) s[r] *= sc.derivative(y);
        }
      };
      if (j0 + 32 > w.wave_full)
        gradient(Int<1>{});
      else
        gradient(Int<0>{});
      if constexpr (LIFT) {
        float top = largest(s);
        if (__ballot(too_large(top))) {
          top = fmaxf(top, other_half(top));
          const float down = too_large(top) ? lift_for(top) : 0.0f, f = __builtin_amdgcn_exp2f(down);
          lift += down;
          rest -= down;
          sum *= f;
          s *= f;
#pragma unroll
          for (int b = 0; b < NB; ++b) g[b] *= f;
        }
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        Op<DT> ds, low;
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          ds.set(r, s[8 * c + r]);
          if constexpr (TWO) low.set(r, s[8 * c + r] - ds.get(r));
        }
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          const Op<DT> kt = T::by_column(ks, 16 * c, b, lane);
          g[b] = Op<DT>::mma(kt, ds, g[b]);
          if constexpr (TWO) g[b] = Op<DT>::mma(kt, low, g[b]);
        }
      }
    }
    if (W::BUFS == 1) __syncthreads();
    if (t + 1 < tiles) {
      tk.store(lds + ((t + 1) & (W::BUFS - 1)) * 2 * TILE);
      tv.store(lds + ((t + 1) & (W::BUFS - 1)) * 2 * TILE + TILE);
    }
    __syncthreads();
  }
  if constexpr (LIFT) {
    const float f = __builtin_amdgcn_exp2f(-lift);
    sum *= f;
#pragma unroll
    for (int b = 0; b < NB; ++b) g[b] *= f;
  }
  sum += other_half(sum);
  if constexpr (PARTS > 1) {
    float* st = sums + w.group * 32 + (lane & 31);
    if (h == 0) st[w.part * GROUPS * 32] = sum;
    float ones[PARTS];
#pragma unroll
    for (int p = 0; p < PARTS; ++p) ones[p] = 1.0f;
    join_parts<NB, GROUPS, PARTS>(g, lds, w.group, w.part, ones);
    if (w.part > 0) return;
    sum = 0.0f;
#pragma unroll
    for (int p = 0; p < PARTS; ++p) sum += st[p * GROUPS * 32];
  }
  if (!w.me.there) return;
  if (h == 0) a.delta[at] = sum;
  store_rows<DT, NB>(g, sc.grad, row_of(a.dq, w.me.t, w.me.head), a.d, h);
}

// ---------------------------------------------------------------------------------------------------------------
// Keys' and values' gradients: a workgroup takes KEYS keys of one key head (32 a wavefront); the queries and upstream gradients of
// all query heads that share it go by in tiles, so the sum over the heads stays in registers.
// S = Q K^T and dP = dO V^T have the keys as columns; dV^T = dO^T P and dK^T = Q^T dS.
// Two wavefronts share 32 keys, one for each half of a tile's 64 queries, and add their sums at the end: the keys that all
// queries of a long sequence see are the longest work of all, and go by in half the steps.
// The sizes above: 885 us (733 TFLOP/s: one workgroup of eight wavefronts a CU, which meet at a barrier for each tile), 229 us (latency of short
// walks) and 518 us with 13 for the join (62 TFLOP/s).
template <int DT, int DP, int GROUPS_, int PARTS_>
struct Dkv {
  static constexpr int GROUPS = GROUPS_, PARTS = PARTS_, KEYS = 32 * GROUPS, THREADS = 64 * GROUPS * PARTS, BQ = 32 * PARTS;
  static constexpr int STEPS = DP / 16, NB = DP / 32;
  // Wide 16-bit rows: the values' operands are read from LDS again for every tile, or the accumulators and both operands would
  // not fit the registers of two wavefronts per SIMD.
  static constexpr bool V_LDS = DT != DLRM_F32 && DP > 64;
  typedef Tile<DT, DP> T;
  static constexpr int TILE = BQ * T::STRIDE, V_AT = 4 * TILE, STAT_AT = V_AT + (V_LDS ? KEYS * T::STRIDE : 0);
  static constexpr int BYTES = STAT_AT + 2 * 2 * BQ * 4;
  static constexpr int JOIN = GROUPS * NB * 16 * DLRM_WAVE * 4;  // one of the two sums of half the wavefronts
  static constexpr int LDS = PARTS == 1 || BYTES > JOIN ? BYTES : JOIN;
};

template <int DT, int DP, int KIND, int GROUPS, int PARTS>
__global__ __launch_bounds__(64 * GROUPS * PARTS, DT == DLRM_F32 ? 1 : 2) void seq_attn_dkv_kernel(SeqArgs a) {
  typedef Dkv<DT, DP, GROUPS, PARTS> W;
  typedef typename W::T T;
  constexpr int BQ = W::BQ, STEPS = W::STEPS, NB = W::NB;
  constexpr bool TWO = DT != DLRM_F32 && DP <= 64 && PARTS == 1;  // weights and ds in two parts
  __shared__ __attribute__((aligned(16))) char lds[W::LDS];
  const int G = a.Hq / a.Hk;
  int walk, seq, row0;
  find_block<W::KEYS>(a, a.k_off, 1, false, walk, seq, row0);  // early keys are seen by most queries
  const int split = a.splits == 1 ? 0 : walk / a.Hk, hk = walk - split * a.Hk;
  int64_t q0, k0;
  const Span sp = span_of(a, seq, q0, k0);
  if (row0 >= sp.nk) return;
  const int lane = lane_id(), h = lane >> 5, group = wave_id() % W::GROUPS, part = wave_id() / W::GROUPS;
  const int w0 = row0 + group * 32, j = w0 + (lane & 31);
  const bool there = j < sp.nk;
  Op<DT> kf[STEPS], vf[W::V_LDS ? 1 : STEPS];
  own_rows<DT, STEPS>(kf, row_of(a.k, k0 + j, hk), there, a.d, h);
  if constexpr (W::V_LDS) {
    Staged<DT, DP, W::KEYS, W::THREADS> t(a.v.st, a.d);
    t.load(row_of(a.v, k0 + row0, hk), a.v.st, sp.nk - row0, a.d);
    t.store(lds + W::V_AT);
  } else {
    own_rows<DT, STEPS>(vf, row_of(a.v, k0 + j, hk), there, a.d, h);
  }
  const int from = there ? sp.first_query(j) : 0x7fffffff;
  const int wave_from = w0 < sp.nk ? sp.first_query(w0) : 0x7fffffff;
  const int wave_full = w0 < sp.nk ? sp.first_query(min(w0 + 31, sp.nk - 1)) : 0x7fffffff;
  const int t0 = sp.first_query(row0) / BQ, tiles = max(0, (sp.nq + BQ - 1) / BQ - t0);

  f32x16 gk[NB], gv[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) gk[b] = gv[b] = f32x16{};
  Staged<DT, DP, BQ, W::THREADS> tq(a.q.st, a.d), td(a.dout.st, a.d);
  // lse and delta of the tile's rows: loaded by every thread, row clamped and not yet looked at, so that no branch and no wait comes before
  // the tile is put away
  const int srow = threadIdx.x % BQ;
  const float* const sfrom = (threadIdx.x / BQ & 1 ? a.delta : a.lse) + q0;
  float sraw = 0.0f;
  // this workgroup's share of the tiles of all heads
  const int share = a.splits == 1 ? tiles * G : (tiles * G + a.splits - 1) / a.splits;
  const int first = split * share, all = max(0, min(tiles * G, first + share) - first);
  int head = hk * G, t = t0;  // of the tile that is on its way
  if (first > 0 && tiles > 0) {
    head += first / tiles;
    t += first % tiles;
  }
  const float base = Score<DT, KIND>(a, hk * G).base;
  // fp16: p is 2^15 times the weight, ds made from it, and that times `f` for the product: from nothing met so far (any value is too large) down
  constexpr bool LIFT = DT == DLRM_F16;
  float f = LIFT ? 0x1p60f : 1.0f;
  auto fetch = [&]() {
    const int i0 = t * BQ;
    tq.load(row_of(a.q, q0 + i0, head), a.q.st, sp.nq - i0, a.d);
    td.load(row_of(a.dout, q0 + i0, head), a.dout.st, sp.nq - i0, a.d);
    sraw = sfrom[(int64_t)head * a.Tq + min(i0 + srow, sp.nq - 1)];
  };
  auto put = [&](int n) {
    tq.store(lds + (n & 1) * 2 * W::TILE);
    td.store(lds + ((n & 1) * 2 + 1) * W::TILE);
    if (threadIdx.x < 2 * BQ) {
      const bool row = t * BQ + srow < sp.nq;
      float* stat = reinterpret_cast<float*>(lds + W::STAT_AT) + (n & 1) * 2 * BQ;
      stat[threadIdx.x] = threadIdx.x < BQ ? lse2_of(sraw, row) - base - kGradWeightLift<DT> : row ? sraw : 0.0f;
    }
  };
  if (all > 0) {
    fetch();
    put(0);
  }
  __syncthreads();
  for (int n = 0; n < all; ++n) {
    const int at = head, i0 = t * BQ + 32 * part;
    if (n + 1 < all) {
      if (++t == t0 + tiles) {
        t = t0;
        ++head;
      }
      fetch();
    }
    if (i0 + 32 > wave_from && i0 < sp.nq) {
      const Score<DT, KIND> sc(a, at);
      const char* qs = lds + (n & 1) * 2 * W::TILE + 32 * part * T::STRIDE;
      const char* os = qs + W::TILE;
      const float* stat = reinterpret_cast<const float*>(lds + W::STAT_AT) + (n & 1) * 2 * BQ + 32 * part + 4 * h;
      f32x16 s = {}, dp = {};
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int st = 0; st < STEPS; ++st) {
        if (past_d<DT, STEPS>(st, a.d)) break;
        s = Op<DT>::mma(T::by_row(qs, lane & 31, st, h), kf[st], s);
        dp = Op<DT>::mma(T::by_row(os, lane & 31, st, h), W::V_LDS ? T::by_row(lds + W::V_AT, group * 32 + (lane & 31), st, h) : vf[W::V_LDS ? 0 : st], dp);
      }
      __builtin_amdgcn_s_setprio(0);
      const float away = (float)(i0 + sp.shift + 4 * h - j);
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        const f32x4 rest = *reinterpret_cast<const f32x4*>(stat + 8 * r4);
        const f32x4 del = *reinterpret_cast<const f32x4*>(stat + BQ + 8 * r4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = 4 * r4 + i;
          const float y = sc.y(s[r]);
          const float p = __builtin_amdgcn_exp2f(sc.exponent(y, away + (float)acc_row(r, 0), rest[i]));
          dp[r] = p * (dp[r] - del[i]);
          if constexpr ((KIND & kBend) != 0) dp[r] *= sc.derivative(y);
          s[r] = p;
        }
      }
      if (i0 < wave_full) {
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (i0 + acc_row(r, h) < from) s[r] = dp[r] = 0.0f;
      }
      if constexpr (LIFT) {
        float top = largest(dp);
        if (__ballot(too_large(top * f))) {
          top = fmaxf(top, other_half(top));
          const float f1 = too_large(top * f) ? __builtin_amdgcn_exp2f(lift_for(top)) : f;
#pragma unroll
          for (int b = 0; b < NB; ++b) gk[b] *= f1 / f;
          f = f1;
        }
        dp *= f;
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        Op<DT> p, ds, p_low, ds_low;
        float w[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          if constexpr (!TWO) p.set(r, s[8 * c + r]);
          ds.set(r, dp[8 * c + r]);
          if constexpr (TWO) {
            w[r] = s[8 * c + r];
            ds_low.set(r, dp[8 * c + r] - ds.get(r));
          }
        }
        if constexpr (TWO) op_two_parts(w, p, p_low);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          const Op<DT> ot = T::by_column(os, 16 * c, b, lane);
          gv[b] = Op<DT>::mma(ot, p, gv[b]);
          if constexpr (TWO) gv[b] = Op<DT>::mma(ot, p_low, gv[b]);
          const Op<DT> qt = T::by_column(qs, 16 * c, b, lane);
          gk[b] = Op<DT>::mma(qt, ds, gk[b]);
          if constexpr (TWO) gk[b] = Op<DT>::mma(qt, ds_low, gk[b]);
        }
        __builtin_amdgcn_s_setprio(0);
      }
    }
    if (n + 1 < all) put(n + 1);
    __syncthreads();
  }
  if constexpr (LIFT) {
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      gk[b] *= 1.0f / f * __builtin_amdgcn_exp2f(-kGradWeightLift<DT>);
      gv[b] *= __builtin_amdgcn_exp2f(-kGradWeightLift<DT>);
    }
  }
  if constexpr (PARTS == 2) {  // one of the two gradients after the other
    const float ones[2] = {1.0f, 1.0f};
    join_parts<NB, GROUPS, PARTS>(gk, lds, group, part, ones);
    __syncthreads();
    join_parts<NB, GROUPS, PARTS>(gv, lds, group, part, ones);
  }
  if (part == 1 || !there) return;
  const float grad = Score<DT, KIND>(a, hk * G).grad;
  if (a.splits == 1) {
    store_rows<DT, NB>(gk, grad, row_of(a.dk, k0 + j, hk), a.d, h);
    store_rows<DT, NB>(gv, 1.0f, row_of(a.dv, k0 + j, hk), a.d, h);
  } else {
    const int64_t rows = a.Tk * a.Hk, at = (k0 + j) * a.Hk + hk;
    store_rows<DLRM_F32, NB>(gk, grad, reinterpret_cast<char*>(a.part + (2 * split * rows + at) * a.d), a.d, h);
    store_rows<DLRM_F32, NB>(gv, 1.0f, reinterpret_cast<char*>(a.part + ((2 * split + 1) * rows + at) * a.d), a.d, h);
  }
}

// Sums of the workgroups that shared the keys' blocks, in their order; 8 columns a thread.
template <int DT>
__global__ __launch_bounds__(256) void seq_attn_join_kernel(SeqArgs a) {
  const int chunks = a.d / 8;
  const int64_t rows = a.Tk * a.Hk, id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = id / chunks;
  const int c = (int)(id - row * chunks) * 8, which = blockIdx.y;
  if (row >= rows) return;
  float x[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
  const float* p = a.part + (which * rows + row) * a.d + c;
  for (int s = 0; s < a.splits; ++s, p += 2 * rows * a.d) {
    const f32x4 u = loadf4(p), v = loadf4(p + 4);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[j] += u[j];
      x[4 + j] += v[j];
    }
  }
  const int64_t t = row / a.Hk;
  char* dst = row_of(which ? a.dv : a.dk, t, (int)(row - t * a.Hk)) + c * Tab<DT>::EB;
  store16(dst, narrow<DT>(x));
  if constexpr (DT == DLRM_F32) store16(dst + 16, narrow<DT>(x + 4));
}

// ---------------------------------------------------------------------------------------------------------------
// Launches for n items in B sequences of at most `longest`, `per` rows an item, workgroups of `threads` for `rows` rows (see find_block): calls
// launch(grid), a.slot0 set, as often as it takes.
template <typename F>
__host__ inline int for_blocks(SeqArgs& a, int64_t n, int longest, int per, int rows, int threads, F launch) {
  const int64_t each = ((int64_t)longest * per + rows - 1) / rows, slots = n * per / rows + a.B, walks = (int64_t)a.Hk * a.splits;
  const int64_t most = kLaunchThreads / (threads * walks);  // slots of a launch
  // Block by block while at most two in three are empty: an empty workgroup ends in under two microseconds, while histories one after
  // the other leave the last and longest blocks for the end (8 histories of 2048 to 4096 items: 31 % of the device idle).
  a.by_block = each * a.B <= 3 * slots && a.B <= 65535 && each <= 65535 && each * a.B <= most;
  if (a.by_block) return launch(dim3((unsigned)walks, a.B, (unsigned)each));
  if (slots > 0x7fffffff) return DLRM_ERR_BAD_SHAPE;  // (of 32 rows at least: more than the memory has)
  a.slots = (int)slots;
  for (int64_t at = 0; at < slots; at += most) {
    a.slot0 = (int)at;
    if (int st = launch(dim3((unsigned)((slots - at < most ? slots - at : most) * walks)))) return st;
  }
  return DLRM_OK;
}

// Calls f with the padded width and the kind of score as compile-time constants.
template <int DT, typename F>
__host__ inline int for_kind(const SeqArgs& a, F f) {
  auto by_kind = [&](auto dp) {
    if constexpr (DT != DLRM_F32) {
      if (a.cap > (DT == DLRM_F16 ? 128.0f : 1024.0f)) return f(dp, std::integral_constant<int, kSlopes | kBend | kLarge>{});
    }
    switch ((a.slopes ? kSlopes : 0) | (a.cap > 0.0f ? kBend : 0)) {
      case kPlain: return f(dp, std::integral_constant<int, kPlain>{});
      case kSlopes: return f(dp, std::integral_constant<int, kSlopes>{});
      case kBend: return f(dp, std::integral_constant<int, kBend>{});
      default: return f(dp, std::integral_constant<int, kSlopes | kBend>{});
    }
  };
  if (a.d <= 32) return by_kind(std::integral_constant<int, 32>{});
  if (a.d <= 64) return by_kind(std::integral_constant<int, 64>{});
  if (a.d <= 96) return by_kind(std::integral_constant<int, 96>{});
  return by_kind(std::integral_constant<int, 128>{});
}

// The keys' gradients: workgroups that share a block of keys.  A block walks through all queries of the heads that share its key
// head, and the longest walk bounds the call: it is shared out where it is longer than what every CU has to do on average (little is known
// here: bounds and totals), a piece no shorter than 8 tiles, and the pieces' fp32 sums are joined by a launch of their own.
// (13 histories of up to 1999 items in fp32, two to a block: 620 -> 567 us with the join; 94 of 121 queries and up to 8 keys, eight query heads
// to a key head, fp32, four to a block: 130 -> 67 us forward and backward.)
__host__ inline bool short_walks(const dlrm_seq_batch* s) { return s->max_q <= 256; }
__host__ inline int dkv_splits(const dlrm_seq_batch* s, int Hq, int Hk, int d, int dtype) {
  const bool wide = dtype != DLRM_F32 && (d > 64 || !short_walks(s));
  const int keys = wide ? 128 : 64, tile = short_walks(s) ? 32 : 64, G = Hq / Hk;
  const double resident = short_walks(s) ? 1024 : 256;
  const double walk = (double)((s->max_q + tile - 1) / tile) * G;
  const double blocks = ((double)s->Tk / keys + 0.5 * s->B) * Hk;
  const double mean = blocks * ((double)s->Tq / s->B / tile + 1) * G * (s->causal ? 0.5 : 1.0) / resident;
  int n = (int)(walk / (mean > 8 ? mean : 8) + 0.5);
  n = n < 1 ? 1 : n > 16 ? 16 : n;
  const int64_t bytes = 2 * s->Tk * Hk * d * 4;  // of one workgroup's sums
  while (n > 1 && n * bytes > (int64_t)256 << 20) --n;
  return n;
}

// How the rows' kernels are cut, by what there is of rows and keys (GROUPS x PARTS wavefronts; `sub` tiles of 32 keys to a part and step).
//   k4x1: 16-bit types.  Wavefronts that share 32 rows pay for the join, and gain where the rows are too few to fill the device;
//   k2x1: fp32, whose registers leave a SIMD one wavefront of most kernels: small workgroups begin and end on their own; and two tiles of keys at most;
//   k4x1Short: two tiles at most under many wide rows: four groups read a tile once;
//   k2x2, k4x2: long walks of few rows, which then take half the steps;
//   k1x8: where 32 rows to a workgroup would not give every CU one, if the walk is long and a step's keys fit into LDS.
// Measured, forward / queries' gradient in us:
//   2048 histories of up to 200 items, 4 heads:  fp32, d 64: k4x2 672 / 1004, k2x2 457 / 626, k4x1 379 / 616, k2x1 373 / 501;
//                                                bf16, d 128: k4x1 276 / 394, k2x1 366 / 445
//   128 histories of up to 200 items, 4 heads, bf16, d 128: k2x2 40 / 50, k4x1 23 / 32;  40, fp32, d 64: k2x2 19 / 25, k2x1 27 / 34
//   4 histories of 1000 to 1400 items, 4 heads, bf16, d 128: k2x2 40 / 36, k4x1 43 / 51;  8, 4 heads on 2: k2x2 59 / 61, k4x1 45 / 57
//   64 of 1000 to 1400 items, 4 heads, fp32, d 64: k4x2 630 / 870, k2x1 561 / 763;  13 of up to 2000, 6 heads on 3: k4x2 194 / 266, k2x1 264 / 359
//   2 of 3000 to 4000 items, 8 heads on 2, fp32, d 96: k2x2 552 / 690, k4x2 450 / 629;  4 of 1000 to 1400, 4 heads: k2x2 101 / 125, k4x2 151 / 211
//   16 histories of 2694 items under one or two queries, f16, d 80, all kernels: k2x2 116, k1x8 68;  2 of up to 1762, fp32, d 16: 141 and 89.
// Forward / the whole backward in us, 4 heads (8 in the first group):
//   bf16, d 64: 16 histories of 300 to 700 items (2064 blocks of 32 rows) k2x2 18 / 64, k4x1 17 / 60;  4 of
//   1500 to 2500 (2016) 46 / 124 and 46 / 139;  5 (2520) 49 / 163 and 50 / 166;  8 (4032) 72 / 229 and 57 / 214;  d 96: 16 of 300 to 700 30 / 77 and 23 / 71, 4
//   of 1500 to 2500 60 / 146 and 65 / 164;  d 128: 4 of 300 to 700 21 / 53 and 20 / 58, 8 33 / 71 and 23 / 64, 13 46 / 98 and 26 / 79
//   histories of 1 to 64 items: bf16, d 128, 256 of them k2x1 14 / 37, k4x1Short 13 / 35, 512 26 / 69 and 24 / 67, 2048 95 / 282 and 87 / 280;  d 64,
//   2048 36 / 112 and 40 / 118;  fp16, d 32, 1024 16 / 45 and 18 / 47
//   one query over 600 keys: bf16, d 64, k1x8 10 / 15, k2x2 14 / 21;  16 over 2000 to 4000, d 128: 51 / 163 and 97 / 137;  fp32, d 32: 53 / 93 and 118 / 155
//   4 histories of 40 queries over 600 keys, fp32, d 64: k1x8 20 / 42, k2x2 32 / 56;  2 of 300 over 500 to 600, fp16, d 24: 9 / 18 and 11 / 23
//   one of 1000 items, bf16, d 64: k1x8 11 / 34, k2x2 19 / 43;  8 of 200 queries over 2000 to 4000 keys (216 blocks), d 64: 31 / 71 and 74 / 110;  4 of 500 over
//   500 to 600 (258 blocks: no longer k1x8) 10 / 29 and 13 / 33
enum { k4x1, k4x1Short, k2x1, k2x2, k4x2, k1x8 };
__host__ inline int cut_of(const dlrm_seq_batch* s, const SeqArgs& a, bool f32, bool fits8) {
  const int64_t rows = s->Tq * a.Hq, blocks = rows / 32 + (int64_t)s->B * a.Hk / 2, fill = rows / 128;
  const bool narrow = a.d <= (f32 ? 64 : 96);
  // a tile's rows are reached with 32-bit byte offsets: the 256 keys of k1x8 where the items' strides leave them below 2^32 (the other cuts'
  // tiles have 128 rows at most, of 2^25 bytes at most: check_heads)
  const int64_t st = a.k.st > a.v.st ? a.k.st : a.v.st;
  fits8 = fits8 && 255 * st + 512 < ((int64_t)1 << 32);
  if (s->max_k <= 64) return f32 || a.d <= 64 || fill < 512 ? k2x1 : k4x1Short;
  if (fits8 && blocks <= 256 && s->max_k >= 512) return k1x8;
  if (f32) {
    if (fill >= (s->max_k > 256 ? 1024 : narrow ? 512 : 256)) return k2x1;
    return s->max_k <= 256 || fill < (narrow ? 512 : 384) ? k2x2 : k4x2;
  }
  return s->max_k > 256 && fill < (narrow ? 512 : 256) ? k2x2 : k4x1;
}

template <int DT>
int launch_seq_fwd(const dlrm_seq_batch* s, SeqArgs a, hipStream_t st) {
  return for_kind<DT>(a, [&](auto dp, auto kind) -> int {
    auto go = [&](auto groups, auto parts, auto sub) -> int {
      if (s->Tq == 0) return DLRM_OK;
      constexpr int threads = 64 * groups() * parts();
      return for_blocks(a, s->Tq, s->max_q, a.Hq / a.Hk, 32 * groups(), threads, [&](dim3 grid) -> int {
        hipLaunchKernelGGL((seq_attn_fwd_kernel<DT, dp(), kind(), groups(), parts(), sub()>), grid, dim3(threads), 0, st, a);
        DLRM_CHECK_LAUNCH();
        return DLRM_OK;
      });
    };
    constexpr bool F32 = DT == DLRM_F32, FITS8 = !F32 || dp() <= 64;
    if constexpr ((kind() & kLarge) != 0) {
      return go(Int<2>{}, Int<1>{}, Int<1>{});
    } else {
      const int cut = cut_of(s, a, F32, FITS8);
      if (cut == k2x1) return go(Int<2>{}, Int<1>{}, Int<1>{});
      if (cut == k2x2) return go(Int<2>{}, Int<2>{}, Int<1>{});
      if constexpr (FITS8) {
        if (cut == k1x8) return go(Int<1>{}, Int<8>{}, Int<1>{});
      }
      if constexpr (F32) {
        return go(Int<4>{}, Int<2>{}, Int<1>{});
      } else {
        // Short histories of narrow rows: tiles of 32 keys leave registers for four workgroups a CU.  (2048 histories of up to 200 items, d 64:
        // 127 us, 143 with 64 keys and weights in one part; 500 candidate lists against up to 1000 items, d 40: 48 us, 45.)
        if (cut == k4x1Short || (dp() <= 64 && s->max_k <= 256)) return go(Int<4>{}, Int<1>{}, Int<1>{});
        return go(Int<4>{}, Int<1>{}, Int<2>{});
      }
    }
  });
}

template <int DT>
int launch_seq_bwd(const dlrm_seq_batch* s, SeqArgs a, hipStream_t st) {
  return for_kind<DT>(a, [&](auto dp, auto kind) -> int {
    constexpr bool F32 = DT == DLRM_F32;
    auto dq = [&](auto groups, auto parts) -> int {
      if (s->Tq == 0) return DLRM_OK;
      constexpr int threads = 64 * groups() * parts();
      return for_blocks(a, s->Tq, s->max_q, a.Hq / a.Hk, 32 * groups(), threads, [&](dim3 grid) -> int {
        hipLaunchKernelGGL((seq_attn_dq_kernel<DT, dp(), kind(), groups(), parts()>), grid, dim3(threads), 0, st, a);
        DLRM_CHECK_LAUNCH();
        return DLRM_OK;
      });
    };
    auto dkv = [&](auto groups, auto parts) -> int {
      if (s->Tk == 0) return DLRM_OK;
      constexpr int threads = 64 * groups() * parts();
      const int rc = for_blocks(a, s->Tk, s->max_k, 1, 32 * groups(), threads, [&](dim3 grid) -> int {
        hipLaunchKernelGGL((seq_attn_dkv_kernel<DT, dp(), kind(), groups(), parts()>), grid, dim3(threads), 0, st, a);
        DLRM_CHECK_LAUNCH();
        return DLRM_OK;
      });
      if (rc != DLRM_OK || a.splits == 1) return rc;
      hipLaunchKernelGGL(seq_attn_join_kernel<DT>, dim3(div_up(a.Tk * a.Hk * (a.d / 8), 256), 2), dim3(256), 0, st, a);
      DLRM_CHECK_LAUNCH();
      return DLRM_OK;
    };
    // Four groups of fp32 rows of more than 64 columns need more registers than there are: 13 histories of up to 2000 items, 6 heads on 3, d 96: four
    // of two parts 384 us, two of one 374; d 128: two of two parts 551, of one 484.  (Nor would the keys' gradients with 128 columns fit, below.)
    constexpr bool WIDE = F32 && dp() > 64, WIDEST = F32 && dp() > 96, FITS8 = !F32 || dp() <= 64;
    if constexpr ((kind() & kLarge) != 0) {
      if (int rc = dq(Int<2>{}, Int<1>{})) return rc;
      a.splits = dkv_splits(s, a.Hq, a.Hk, a.d, DT);
      return dkv(Int<2>{}, Int<1>{});
    } else {
      const int cut = cut_of(s, a, F32, FITS8);
      int rc = DLRM_OK;
      if (cut == k2x1 || (WIDE && cut == k4x2))
        rc = dq(Int<2>{}, Int<1>{});
      else if (cut == k2x2)
        rc = dq(Int<2>{}, Int<2>{});
      else if (cut == k1x8) {
        if constexpr (FITS8) rc = dq(Int<1>{}, Int<8>{});
      } else if constexpr (!WIDE) {
        rc = dq(Int<4>{}, Int<F32 ? 2 : 1>{});
      }
      if (rc != DLRM_OK) return rc;
      a.splits = dkv_splits(s, a.Hq, a.Hk, a.d, DT);
      // Short histories: few steps, so nothing is gained by halving them, and small workgroups hide each other's starts.  (2048 histories
      // of up to 200 items, bf16, d 64: two wavefronts of one part 217 us, four 242, eight of two parts 391; 8 of up to 4096, d 128: 1789, 1163, 1038.)
      // (No more than 32 keys: no wavefront without any.  259 histories of one item or none, fp32, d 88: two wavefronts 75 us, one 42.)
      const bool is_short = short_walks(s);
      if constexpr (!WIDEST) {
        if (is_short && s->max_k <= 32) return dkv(Int<1>{}, Int<1>{});
      }
      if constexpr (!F32) {
        return is_short ? dkv(Int<(dp() > 64) ? 4 : 2>{}, Int<1>{}) : dkv(Int<4>{}, Int<2>{});
      } else {
        // 64 histories of 1000 to 1400 items, 4 heads: halved 1203 us with d 64 and 1651 with 96, not halved 1074 and 1485; with 128 columns, which
        // leave no registers for the loads of a whole tile by two wavefronts, 2111 and 2980.
        if constexpr (!WIDEST) {
          if (is_short || s->Tk * a.Hk >= 131072) return dkv(Int<2>{}, Int<1>{});
        }
        return dkv(Int<2>{}, Int<2>{});
      }
    }
  });
}

extern template int launch_seq_fwd<DLRM_F32>(const dlrm_seq_batch*, SeqArgs, hipStream_t);
extern template int launch_seq_fwd<DLRM_F16>(const dlrm_seq_batch*, SeqArgs, hipStream_t);
extern template int launch_seq_fwd<DLRM_BF16>(const dlrm_seq_batch*, SeqArgs, hipStream_t);
extern template int launch_seq_bwd<DLRM_F32>(const dlrm_seq_batch*, SeqArgs, hipStream_t);
extern template int launch_seq_bwd<DLRM_F16>(const dlrm_seq_batch*, SeqArgs, hipStream_t);
extern template int launch_seq_bwd<DLRM_BF16>(const dlrm_seq_batch*, SeqArgs, hipStream_t);

}  // namespace dlrm
