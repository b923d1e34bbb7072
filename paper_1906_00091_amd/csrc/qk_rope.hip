// Norm and rotary position of query and key heads, forward, backward and on the way into a paged cache.
//
// A row of d columns is held by a group of G lanes (a power of two), 16 bytes a lane; the sum of squares and the
// backward's <g w, n> are joined by lane exchanges inside the group.  A group stays with one item and walks its heads, so that the
// item's angles are reduced and their sines and cosines taken once, in registers, for all of its heads: the angle in turns is
// position * frequency / 2 pi in fp64 (1 / 2 pi and two products are rounded: off by 3 2^-53 of the angle at most, 7e-7 radians at 2^31; fp32 would be off
// by 1e-3 radians at position 2^14), its fraction goes to sincospi in fp32.  In the half layout a column's partner lies rot/2 columns away: in another lane at the same
// place of the chunk where rot/2 is a multiple of a chunk's columns (an exchange of the raw chunk), else anywhere (through LDS).
// With p the partner of column j,  y_j = r (c_j w_j x_j + s_j w_p x_p):  the norm's weights go into the coefficients once an item, and
// the exchange of the row as it was loaded does not wait for its norm.
//
// Bound by memory: every row is read and written once.  2048 histories of up to 200 items, 4 + 4 heads of 64 fp32 columns, normed, all rotated: forward
// 151 us for 0.84 GB (5.6 TB/s), backward 249 us for 1.26 GB (5.1 TB/s); a large copy on the same card moves 4.7 TB/s, a read 5.7.
// Few heads of narrow rows are bound by the angles instead (one head each of 16 columns of f16: 2.0 TB/s forward, 1.1 backward).
#include <initializer_list>
#include <type_traits>

#include "heads.h"

namespace dlrm {

struct RopeArgs {
  Rows q, k, v, qo, ko;   // forward
  Rows dqo, dko, dq, dk;  // backward
  int64_t T;
  int Hq, Hk, d, rot;
  int splits, shift_v;  // groups of an item; Hk modulo splits
  const int32_t* pos;
  const float* inv_freq;
  const float* wq;
  const float* wk;
  float eps, mscale;
  float* part;  // [workgroups][2][d] (backward)
  // cache
  char* ck;
  char* cv;
  const int32_t* table;
  const int32_t* seqs;
  int cB, cols, n_pages, page_shift;
};

constexpr int kRopeThreads = 256;
enum { kPairs = 0, kHalfChunks = 1, kHalfAny = 2 };  // where a column's partner is

template <int DT>
struct RopeLane {
  static constexpr int E = Tab<DT>::ELEMS;
  float c[E], s[E];  // of the pair that column j of this lane's chunk is in; (1, 0) where it is not rotated; s signed
};

// sign: +1 forward, -1 backward (the transpose of the rotation)
template <int DT, int MODE>
__device__ inline void lane_angles(const RopeArgs& a, int64_t t, int col0, float sign, RopeLane<DT>& L) {
  constexpr int E = RopeLane<DT>::E;
  const int n = a.rot >> 1;
  const double turn = a.rot > 0 ? (double)a.pos[t] * 0.15915494309189533577 : 0.0;
  constexpr int STEP = MODE == kPairs ? 2 : 1;
#pragma unroll
  for (int j = 0; j < E; j += STEP) {
    const int c = col0 + j;
    float cs = 1.0f, sn = 0.0f;
    if (c < a.rot) {
      const int i = MODE == kPairs ? c >> 1 : c < n ? c : c - n;
      const double x = turn * (double)a.inv_freq[i];
      sincospif((float)(2.0 * (x - rint(x))), &sn, &cs);
      cs *= a.mscale;
      sn *= a.mscale * sign;
    }
    if constexpr (MODE == kPairs) {
      L.c[j] = L.c[j + 1] = cs;
      L.s[j] = -sn;
      L.s[j + 1] = sn;
    } else {
      L.c[j] = cs;
      L.s[j] = c < n ? -sn : sn;
    }
  }
}

// The partner's part of a column's sum: s p, or what leaves the column as it is, bit for bit, where it is not rotated.  (Zero times the partner would not:
// an infinity, or the column itself where it has no partner, would come out as NaN.)
__device__ inline float partner_term(float s, float p, int c, int rot) { return c < rot ? s * p : -0.0f; }

// The partners of this lane's E columns in a row as it was loaded; xs: this wavefront's buffer in LDS (kHalfAny).
template <int DT, int MODE>
__device__ inline void partners(u32x4 raw, const float* x, float* p, int lane, int col0, int rot, float* xs) {
  constexpr int E = Tab<DT>::ELEMS;
  const int n = rot >> 1;
  if constexpr (MODE == kPairs) {
#pragma unroll
    for (int j = 0; j < E; ++j) p[j] = x[j ^ 1];
  } else if constexpr (MODE == kHalfChunks) {
    const int step = n / E;  // lanes to the partner; a lane past the rotated columns takes its own
    const int from = col0 < n ? lane + step : col0 < rot ? lane - step : lane;
    u32x4 q;
#pragma unroll
    for (int j = 0; j < 4; ++j) q[j] = (uint32_t)__shfl((int)raw[j], from, DLRM_WAVE);
    Tab<DT>::widen(q, p);
  } else {
    const float* row = xs + (lane * E - col0);  // of this lane's group
#pragma unroll
    for (int j = 0; j < E; ++j) xs[lane * E + j] = x[j];
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int j = 0; j < E; ++j) {
      const int c = col0 + j;
      p[j] = row[c < n ? c + n : c < rot ? c - n : c];
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// The norm's weights of this lane's columns and of their partners (ones without a norm)
template <int DT, int MODE>
struct Weights {
  static constexpr int E = Tab<DT>::ELEMS;
  float own[E], other[E];
  __device__ inline Weights(const float* w, int col0, int d, int rot) {
#pragma unroll
    for (int j = 0; j < E; ++j) own[j] = other[j] = 1.0f;
    if (w == nullptr) return;
    const int n = rot >> 1, at = min(col0, d - E);
#pragma unroll
    for (int j = 0; j < E; j += 4) load_cols<4>(w + at + j, true, own + j);
    if constexpr (MODE == kPairs) {
#pragma unroll
      for (int j = 0; j < E; ++j) other[j] = own[j ^ 1];
    } else if constexpr (MODE == kHalfChunks) {
      const int from = at >= rot ? at : at < n ? at + n : at - n;
#pragma unroll
      for (int j = 0; j < E; j += 4) load_cols<4>(w + from + j, true, other + j);
    } else {
#pragma unroll
      for (int j = 0; j < E; ++j) other[j] = w[at + j >= rot ? at + j : at + j < n ? at + j + n : at + j - n];
    }
  }
};

// Sum over a group of G lanes, in every lane: exchanges within 16 lanes go through the vector unit.
template <int CTRL>
__device__ inline float dpp(float v) {
  return u2f((uint32_t)__builtin_amdgcn_update_dpp(0, (int)f2u(v), CTRL, 0xf, 0xf, true));
}
template <int G>
__device__ inline float group_sum(float v) {
  if constexpr (G >= 2) v += dpp<0xB1>(v);    // lanes 1 0 3 2 of four
  if constexpr (G >= 4) v += dpp<0x4E>(v);    // lanes 2 3 0 1 of four
  if constexpr (G >= 8) v += dpp<0x141>(v);   // 8 lanes mirrored
  if constexpr (G >= 16) v += dpp<0x140>(v);  // 16 lanes mirrored
  if constexpr (G >= 32) v += __shfl_xor(v, 16, DLRM_WAVE);
  return v;
}

// Forward.  Groups of G lanes; group g of the grid takes item g / splits, and of its queries, keys and values every splits-th head.
// SPLIT: several groups share an item.  Where none do, a head is the same for the whole wavefront, and its address is scalar work.
template <int DT, int MODE, int G, bool SPLIT, bool CACHE>
__global__ __launch_bounds__(kRopeThreads) void qk_rope_fwd_kernel(RopeArgs a) {
  constexpr int E = Tab<DT>::ELEMS;
  __shared__ float xs_all[MODE == kHalfAny ? kRopeThreads * E : 1];
  float* xs = xs_all + (MODE == kHalfAny ? wave_id() * DLRM_WAVE * E : 0);
  const int lane = lane_id(), col0 = (lane & (G - 1)) * E;
  const int64_t group = ((int64_t)blockIdx.x * kRopeThreads + threadIdx.x) / G;
  const int step = SPLIT ? a.splits : 1;
  const int64_t t = SPLIT ? group / step : group;
  // the group's first query, key and value: where every group has one row at most, no two of them meet
  const int fq = SPLIT ? (int)(group - t * step) : 0, fk = SPLIT ? step - 1 - fq : 0;
  const int fv = !SPLIT ? 0 : fk >= a.shift_v ? fk - a.shift_v : fk - a.shift_v + step;
  // lanes of the last group past the row, and groups past the last item, go along with nothing (exchanges need every lane)
  const bool in = t < a.T && col0 < a.d;
  const int64_t tt = t < a.T ? t : a.T - 1;
  const int cb = col0 * Tab<DT>::EB, lb = min(col0, a.d - E) * Tab<DT>::EB;
  // (loads stand in no branch, so that the next row's is in flight while this one is worked on: a lane past the row or a head past the last
  // loads what is there, and it is not used)
  auto load = [&](const Rows& rows, int h, int H) { return load16(row_of(rows, tt, min(h, H - 1)) + lb); };
  u32x4 row_q = load(a.q, fq, a.Hq), row_k = {0, 0, 0, 0};
  if (a.Hk > 0) row_k = load(a.k, fk, a.Hk);
  // the item's page, looked up beside the rows (clamped: whether it is there is asked where it is used)
  int seq = 0, col = 0, page = 0;
  if constexpr (CACHE) {
    seq = a.seqs[tt];
    col = a.pos[tt] >> a.page_shift;
    page = a.table[(int64_t)min(max(seq, 0), a.cB - 1) * a.cols + min(max(col, 0), a.cols - 1)];
  }
  RopeLane<DT> L;
  lane_angles<DT, MODE>(a, tt, col0, 1.0f, L);
  const float inv_d = 1.0f / (float)a.d;

  auto turn = [&](const Rows& rows, int first, int H, u32x4 next, const float* weights, auto to) {
    const Weights<DT, MODE> w(weights, col0, a.d, a.rot);
    float c[E], s[E];
#pragma unroll
    for (int j = 0; j < E; ++j) {
      c[j] = L.c[j] * w.own[j];
      s[j] = L.s[j] * w.other[j];
    }
    for (int h = first; h < H; h += step) {
      u32x4 raw = next;
      next = load(rows, h + step, H);
      if (col0 >= a.d) raw = u32x4{0, 0, 0, 0};
      float x[E], p[E], y[E];
      Tab<DT>::widen(raw, x);
      partners<DT, MODE>(raw, x, p, lane, col0, a.rot, xs);
      float r = 1.0f;
      if (weights != nullptr) {
        float ss = 0.0f;
#pragma unroll
        for (int j = 0; j < E; ++j) ss += x[j] * x[j];
        r = 1.0f / sqrtf(group_sum<G>(ss) * inv_d + a.eps);
      }
#pragma unroll
      for (int j = 0; j < E; ++j) y[j] = r * fmaf(c[j], x[j], partner_term(s[j], p[j], col0 + j, a.rot));
      char* dst = to(h);
      if (in && dst) store16(dst + cb, narrow<DT>(y));
    }
  };
  turn(a.q, fq, a.Hq, row_q, a.wq, [&](int h) { return row_of(a.qo, tt, h); });
  if constexpr (!CACHE) {
    turn(a.k, fk, a.Hk, row_k, a.wk, [&](int h) { return row_of(a.ko, tt, h); });
  } else {
    const int64_t row = (int64_t)a.d * Tab<DT>::EB, head_bytes = row << a.page_shift;
    const bool there = seq >= 0 && seq < a.cB && col >= 0 && col < a.cols && page >= 0 && page < a.n_pages;
    const int64_t at = there ? (int64_t)page * a.Hk * head_bytes + (a.pos[tt] & ((1 << a.page_shift) - 1)) * row : -1;
    turn(a.k, fk, a.Hk, row_k, a.wk, [&](int h) { return at < 0 ? nullptr : a.ck + at + h * head_bytes; });
    for (int h0 = fv; h0 < a.Hk; h0 += 4 * step) {
      u32x4 v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = load(a.v, h0 + i * step, a.Hk);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int h = h0 + i * step;
        if (in && at >= 0 && h < a.Hk) store16(a.cv + at + h * head_bytes + cb, v[i]);
      }
    }
  }
}

// Backward.  Groups share an item as in the forward, and walk from item to item; the weights' gradients of all its rows stay in
// registers, are added over the workgroup's groups once at the end, and one row of sums per workgroup goes to the workspace.
template <int DT, int MODE, int G, bool SPLIT>
__global__ __launch_bounds__(kRopeThreads, 4) void qk_rope_bwd_kernel(RopeArgs a) {
  constexpr int E = Tab<DT>::ELEMS;
  constexpr int NW = kRopeThreads / DLRM_WAVE;
  __shared__ float xs_all[MODE == kHalfAny ? kRopeThreads * E : 1];
  __shared__ float red[NW][2][DLRM_MAX_HEAD_DIM];
  float* xs = xs_all + (MODE == kHalfAny ? wave_id() * DLRM_WAVE * E : 0);
  const int lane = lane_id(), col0 = (lane & (G - 1)) * E;
  const int64_t g0 = ((int64_t)blockIdx.x * kRopeThreads + threadIdx.x) / G;
  const int step = SPLIT ? a.splits : 1;
  const int64_t walkers = (int64_t)gridDim.x * (kRopeThreads / G) / step;  // items in a round
  const int64_t t0 = SPLIT ? g0 / step : g0;
  const int fq = SPLIT ? (int)(g0 - t0 * step) : 0, fk = SPLIT ? step - 1 - fq : 0;  // the group's first query and key head
  const float inv_d = 1.0f / (float)a.d;
  float sq[E], sk[E];
#pragma unroll
  for (int j = 0; j < E; ++j) sq[j] = sk[j] = 0.0f;
  const int cb = col0 * Tab<DT>::EB, lb = min(col0, a.d - E) * Tab<DT>::EB;
  const int64_t rounds = (a.T + walkers - 1) / walkers;  // the same for every lane of the workgroup
  for (int64_t i = 0; i < rounds; ++i) {
    const int64_t t = t0 + i * walkers;
    const bool in = t0 < walkers && t < a.T && col0 < a.d;
    const int64_t tt = t < a.T ? t : a.T - 1;
    auto load = [&](const Rows& rows, int h, int H) { return load16(row_of(rows, tt, min(h, H - 1)) + lb); };
    u32x4 xq = load(a.q, fq, a.Hq), dq = load(a.dqo, fq, a.Hq), xk = {0, 0, 0, 0}, dk = {0, 0, 0, 0};
    if (a.Hk > 0) {
      xk = load(a.k, fk, a.Hk);
      dk = load(a.dko, fk, a.Hk);
    }
    RopeLane<DT> L;
    lane_angles<DT, MODE>(a, tt, col0, -1.0f, L);
    auto turn = [&](const Rows& rows, const Rows& drows, const Rows& to, int first, int H, u32x4 nx, u32x4 nd, const float* wp, float* sum) {
      float w[E];  // (loaded again for every item: the registers are worth more)
#pragma unroll
      for (int j = 0; j < E; ++j) w[j] = 1.0f;
      if (wp != nullptr) {
#pragma unroll
        for (int j = 0; j < E; j += 4) load_cols<4>(wp + min(col0, a.d - E) + j, true, w + j);
      }
      for (int h = first; h < H; h += step) {
        u32x4 rx = nx, rd = nd;
        nx = load(rows, h + step, H);
        nd = load(drows, h + step, H);
        if (col0 >= a.d) rx = rd = u32x4{0, 0, 0, 0};
        float x[E], dy[E], g[E];
        Tab<DT>::widen(rx, x);
        Tab<DT>::widen(rd, dy);
        partners<DT, MODE>(rd, dy, g, lane, col0, a.rot, xs);
#pragma unroll
        for (int j = 0; j < E; ++j) g[j] = fmaf(L.c[j], dy[j], partner_term(L.s[j], g[j], col0 + j, a.rot));
        if (wp != nullptr) {
          float ss = 0.0f, sg = 0.0f, gw[E];
#pragma unroll
          for (int j = 0; j < E; ++j) {
            gw[j] = g[j] * w[j];
            ss += x[j] * x[j];
            sg += gw[j] * x[j];
          }
          ss = group_sum<G>(ss);
          sg = group_sum<G>(sg);
          const float r = 1.0f / sqrtf(ss * inv_d + a.eps);
          const float m = sg * r * r * inv_d;  // mean(g w n) r
#pragma unroll
          for (int j = 0; j < E; ++j) {
            sum[j] += in ? g[j] * (x[j] * r) : 0.0f;
            g[j] = r * (gw[j] - x[j] * m);
          }
        }
        if (in) store16(row_of(to, tt, h) + cb, narrow<DT>(g));
      }
    };
    turn(a.q, a.dqo, a.dq, fq, a.Hq, xq, dq, a.wq, sq);
    turn(a.k, a.dko, a.dk, fk, a.Hk, xk, dk, a.wk, sk);
  }
  if (a.part == nullptr) return;
#pragma unroll
  for (int j = 0; j < E; ++j) {
#pragma unroll
    for (int o = G; o < DLRM_WAVE; o <<= 1) {
      sq[j] += __shfl_xor(sq[j], o, DLRM_WAVE);
      sk[j] += __shfl_xor(sk[j], o, DLRM_WAVE);
    }
    if (lane < G && col0 < a.d) {
      red[wave_id()][0][col0 + j] = sq[j];
      red[wave_id()][1][col0 + j] = sk[j];
    }
  }
  __syncthreads();
  for (int c = threadIdx.x; c < 2 * a.d; c += kRopeThreads) {
    const int w = c >= a.d, col = c - w * a.d;
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < NW; ++i) sum += red[i][w][col];
    a.part[(int64_t)blockIdx.x * 2 * a.d + c] = sum;
  }
}

// dw[c] = sum of the workgroups' rows; 16 columns a workgroup, 64 threads a column, four rows in flight each.  (16 threads a column
// and one row in flight: 50 us for 2048 rows of 256 columns.)
constexpr int kDwThreads = 1024, kDwCols = 16, kDwRows = kDwThreads / kDwCols;
__global__ __launch_bounds__(kDwThreads) void qk_rope_dw_kernel(const float* part, int rows, int d, float* dwq, float* dwk) {
  __shared__ float red[kDwRows][kDwCols + 1];
  const int x = threadIdx.x % kDwCols, y = threadIdx.x / kDwCols, c = blockIdx.x * kDwCols + x;
  float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  if (c < 2 * d) {
    for (int i = y; i < rows; i += 4 * kDwRows) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int r = i + j * kDwRows;
        const float v = part[(int64_t)(r < rows ? r : y) * 2 * d + c];
        sum[j] += r < rows ? v : 0.0f;
      }
    }
  }
  red[y][x] = (sum[0] + sum[1]) + (sum[2] + sum[3]);
  __syncthreads();
  for (int o = kDwRows / 2; o > 0; o >>= 1) {
    if (y < o) red[y][x] += red[y + o][x];
    __syncthreads();
  }
  if (y == 0 && c < 2 * d) {
    float* dst = c < d ? dwq : dwk;
    if (dst) dst[c < d ? c : c - d] = red[0][x];
  }
}

static int check_rope(const dlrm_qk_rope* r) {
  if (!r) return DLRM_ERR_NULL;
  if (int st = check_head_shape(r->Hq, 1, r->d, r->dtype)) return st;
  if (r->Hk < 0 || r->Hk > DLRM_MAX_HEADS) return DLRM_ERR_BAD_SHAPE;
  if (r->T < 0 || r->T > DLRM_MAX_ITEMS) return DLRM_ERR_BAD_SHAPE;
  if (r->rot < 0 || r->rot > r->d || (r->rot & 1)) return DLRM_ERR_BAD_SHAPE;
  if (r->layout != DLRM_ROPE_HALF && r->layout != DLRM_ROPE_INTERLEAVED) return DLRM_ERR_BAD_SHAPE;
  if (r->rot > 0 && (!r->inv_freq || (r->T > 0 && !r->positions))) return DLRM_ERR_NULL;
  if ((r->wq || r->wk) && !(r->eps > 0.0f)) return DLRM_ERR_BAD_SHAPE;
  if ((reinterpret_cast<uintptr_t>(r->wq) & 15) || (reinterpret_cast<uintptr_t>(r->wk) & 15)) return DLRM_ERR_BAD_SHAPE;
  return DLRM_OK;
}

int check_cache(const dlrm_kv_cache* c) {
  if (!c) return DLRM_ERR_NULL;
  if (!c->k || !c->v || !c->table) return DLRM_ERR_NULL;
  if (int st = check_head_shape(c->Hk, 1, c->d, c->dtype)) return st;
  if (c->B < 1 || c->table_cols < 1 || c->n_pages < 1) return DLRM_ERR_BAD_SHAPE;
  if (c->page < 1 || c->page > 1024 || (c->page & (c->page - 1))) return DLRM_ERR_BAD_SHAPE;
  if ((int64_t)c->table_cols * c->page > DLRM_MAX_ITEMS) return DLRM_ERR_BAD_SHAPE;
  if ((reinterpret_cast<uintptr_t>(c->k) & 15) || (reinterpret_cast<uintptr_t>(c->v) & 15)) return DLRM_ERR_BAD_SHAPE;
  return DLRM_OK;
}

static int group_lanes(const dlrm_qk_rope* r) { return pow2_ceil(r->d * elem_bytes(r->dtype) / 16); }

static int partner_mode(const dlrm_qk_rope* r) {
  if (r->layout == DLRM_ROPE_INTERLEAVED) return kPairs;
  return (r->rot / 2) % (16 / elem_bytes(r->dtype)) == 0 ? kHalfChunks : kHalfAny;
}

static RopeArgs rope_args(const dlrm_qk_rope* r) {
  RopeArgs a = {};
  a.T = r->T;
  a.Hq = r->Hq;
  a.Hk = r->Hk;
  a.d = r->d;
  a.rot = r->rot;
  a.splits = 1;
  a.pos = r->positions;
  a.inv_freq = r->inv_freq;
  a.wq = r->wq;
  a.wk = r->Hk > 0 ? r->wk : nullptr;
  a.eps = r->eps;
  a.mscale = r->mscale;
  return a;
}

template <int N>
using Int = std::integral_constant<int, N>;

// Calls f with the storage type, the partner's place, the lanes of a group and whether groups share an item as compile-time constants.
template <typename F>
static int for_row_kind(const dlrm_qk_rope* r, const RopeArgs& a, F f) {
  auto by_split = [&](auto dt, auto md, auto g) { return a.splits > 1 ? f(dt, md, g, Int<1>{}) : f(dt, md, g, Int<0>{}); };
  auto by_lanes = [&](auto dt, auto md) {
    switch (group_lanes(r)) {
      case 2: return by_split(dt, md, Int<2>{});
      case 4: return by_split(dt, md, Int<4>{});
      case 8: return by_split(dt, md, Int<8>{});
      case 16: return by_split(dt, md, Int<16>{});
    }
    return by_split(dt, md, Int<dt() == DLRM_F32 ? 32 : 1>{});  // fp32 rows of more than 64 columns; 16-bit rows of 8
  };
  auto by_mode = [&](auto dt) {
    switch (partner_mode(r)) {
      case kPairs: return by_lanes(dt, Int<kPairs>{});
      case kHalfChunks: return by_lanes(dt, Int<kHalfChunks>{});
      default: return by_lanes(dt, Int<kHalfAny>{});
    }
  };
  switch (r->dtype) {
    case DLRM_F32: return by_mode(Int<DLRM_F32>{});
    case DLRM_F16: return by_mode(Int<DLRM_F16>{});
    default: return by_mode(Int<DLRM_BF16>{});
  }
}

// Groups that share an item's heads: several where the items alone would not fill the device, and, where a row is less than 128 bytes and all
// of an item's rows are more, as many as read 128 bytes side by side if heads lie side by side.  (1.66 million items of 24 rows of 16 bytes, bf16,
// forward and backward: 2.79 ms a group to an item, 0.74 ms with eight.  293 thousand items of two rows of 32 bytes, f16: 73 us, with two groups 96, since
// each works the angles out.)
static int head_splits(const dlrm_qk_rope* r, int heads) {
  const int64_t wanted = 65536 / group_lanes(r);  // 1024 wavefronts
  int64_t s = r->T > 0 ? wanted / r->T : 1;
  if (s < 8 / group_lanes(r) && group_lanes(r) * heads >= 8) s = 8 / group_lanes(r);
  return (int)(s < 1 ? 1 : s > heads ? heads : s);
}

// the forward's arguments for n items from item t0 on
static RopeArgs items_of(RopeArgs a, int64_t t0, int64_t n) {
  for (Rows* x : {&a.q, &a.k, &a.v, &a.qo, &a.ko})
    if (x->p) x->p += t0 * x->st;
  if (a.pos) a.pos += t0;
  if (a.seqs) a.seqs += t0;
  a.T = n;
  return a;
}

template <bool CACHE>
static int launch_fwd(const dlrm_qk_rope* r, RopeArgs a, hipStream_t st) {
  if (r->T == 0) return DLRM_OK;
  a.splits = head_splits(r, r->Hq + r->Hk * (CACHE ? 2 : 1));
  a.shift_v = r->Hk % a.splits;
  const int lanes = a.splits * group_lanes(r);  // of an item
  return for_row_kind(r, a, [&](auto dt, auto md, auto g, auto split) {
    // a launch takes fewer than 2^32 threads: more items than that go in several
    const int64_t each = kLaunchThreads / lanes;
    for (int64_t t0 = 0; t0 < r->T; t0 += each) {
      const RopeArgs b = items_of(a, t0, r->T - t0 < each ? r->T - t0 : each);
      hipLaunchKernelGGL((qk_rope_fwd_kernel<dt(), md(), g(), split(), CACHE>), dim3((unsigned)((b.T * lanes + kRopeThreads - 1) / kRopeThreads)),
                         dim3(kRopeThreads), 0, st, b);
      DLRM_CHECK_LAUNCH();
    }
    return (int)DLRM_OK;
  });
}

static int bwd_blocks(const dlrm_qk_rope* r) {
  const int64_t b = (r->T * head_splits(r, r->Hq + r->Hk) * group_lanes(r) + kRopeThreads - 1) / kRopeThreads;
  return (int)(b > 1024 ? 1024 : b);  // as many as are resident
}

}  // namespace dlrm

using namespace dlrm;

extern "C" int32_t dlrm_qk_rope_fwd(const dlrm_qk_rope* r, const dlrm_heads* q, const dlrm_heads* k, const dlrm_heads* q_out,
                                    const dlrm_heads* k_out, void* stream) {
  if (int st = check_rope(r)) return st;
  const int eb = elem_bytes(r->dtype);
  for (const dlrm_heads* x : {q, q_out})
    if (int st = check_heads(x, r->T, r->Hq, r->d, eb)) return st;
  RopeArgs a = rope_args(r);
  a.q = rows_of(q, r->T, r->Hq, r->d, eb);
  a.qo = rows_of(q_out, r->T, r->Hq, r->d, eb);
  if (r->Hk > 0) {
    for (const dlrm_heads* x : {k, k_out})
      if (int st = check_heads(x, r->T, r->Hk, r->d, eb)) return st;
    a.k = rows_of(k, r->T, r->Hk, r->d, eb);
    a.ko = rows_of(k_out, r->T, r->Hk, r->d, eb);
  }
  return launch_fwd<false>(r, a, static_cast<hipStream_t>(stream));
}

extern "C" int32_t dlrm_qk_rope_append(const dlrm_qk_rope* r, const dlrm_heads* q, const dlrm_heads* k, const dlrm_heads* v,
                                       const dlrm_heads* q_out, const dlrm_kv_cache* c, const int32_t* seqs, void* stream) {
  if (int st = check_rope(r)) return st;
  if (int st = check_cache(c)) return st;
  if (r->Hk != c->Hk || r->d != c->d) return DLRM_ERR_BAD_SHAPE;
  if (r->dtype != c->dtype) return DLRM_ERR_BAD_DTYPE;
  if (r->T > 0 && (!seqs || !r->positions)) return DLRM_ERR_NULL;
  const int eb = elem_bytes(r->dtype);
  for (const dlrm_heads* x : {q, q_out})
    if (int st = check_heads(x, r->T, r->Hq, r->d, eb)) return st;
  for (const dlrm_heads* x : {k, v})
    if (int st = check_heads(x, r->T, r->Hk, r->d, eb)) return st;
  RopeArgs a = rope_args(r);
  a.q = rows_of(q, r->T, r->Hq, r->d, eb);
  a.qo = rows_of(q_out, r->T, r->Hq, r->d, eb);
  a.k = rows_of(k, r->T, r->Hk, r->d, eb);
  a.v = rows_of(v, r->T, r->Hk, r->d, eb);
  a.ck = static_cast<char*>(c->k);
  a.cv = static_cast<char*>(c->v);
  a.table = c->table;
  a.seqs = seqs;
  a.cB = c->B;
  a.cols = c->table_cols;
  a.n_pages = c->n_pages;
  a.page_shift = ilog2_ceil(c->page);
  return launch_fwd<true>(r, a, static_cast<hipStream_t>(stream));
}

extern "C" size_t dlrm_qk_rope_bwd_workspace_bytes(const dlrm_qk_rope* r) {
  if (check_rope(r) != DLRM_OK) return 0;
  const size_t n = (size_t)bwd_blocks(r) * 2 * r->d * sizeof(float);
  return n < 256 ? 256 : (n + 255) / 256 * 256;
}

extern "C" int32_t dlrm_qk_rope_bwd(const dlrm_qk_rope* r, const dlrm_heads* q, const dlrm_heads* k, const dlrm_heads* dq_out,
                                    const dlrm_heads* dk_out, const dlrm_heads* dq, const dlrm_heads* dk, float* dwq, float* dwk,
                                    void* workspace, size_t workspace_bytes, void* stream) {
  if (int st = check_rope(r)) return st;
  const int eb = elem_bytes(r->dtype);
  for (const dlrm_heads* x : {q, dq_out, dq})
    if (int st = check_heads(x, r->T, r->Hq, r->d, eb)) return st;
  RopeArgs a = rope_args(r);
  a.q = rows_of(q, r->T, r->Hq, r->d, eb);
  a.dqo = rows_of(dq_out, r->T, r->Hq, r->d, eb);
  a.dq = rows_of(dq, r->T, r->Hq, r->d, eb);
  if (r->Hk > 0) {
    for (const dlrm_heads* x : {k, dk_out, dk})
      if (int st = check_heads(x, r->T, r->Hk, r->d, eb)) return st;
    a.k = rows_of(k, r->T, r->Hk, r->d, eb);
    a.dko = rows_of(dk_out, r->T, r->Hk, r->d, eb);
    a.dk = rows_of(dk, r->T, r->Hk, r->d, eb);
  }
  const bool norm = a.wq || a.wk;
  if ((a.wq && !dwq) || (a.wk && !dwk)) return DLRM_ERR_NULL;
  if (norm && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < dlrm_qk_rope_bwd_workspace_bytes(r)))
    return DLRM_ERR_WORKSPACE;
  a.part = norm ? static_cast<float*>(workspace) : nullptr;
  a.splits = head_splits(r, r->Hq + r->Hk);
  hipStream_t st = static_cast<hipStream_t>(stream);
  const int blocks = bwd_blocks(r);
  if (blocks > 0) {
    const int rc = for_row_kind(r, a, [&](auto dt, auto md, auto g, auto split) {
      hipLaunchKernelGGL((qk_rope_bwd_kernel<dt(), md(), g(), split()>), dim3(blocks), dim3(kRopeThreads), 0, st, a);
      DLRM_CHECK_LAUNCH();
      return (int)DLRM_OK;
    });
    if (rc != DLRM_OK) return rc;
  }
  if (!norm) return DLRM_OK;
  hipLaunchKernelGGL(qk_rope_dw_kernel, dim3((2 * r->d + kDwCols - 1) / kDwCols), dim3(kDwThreads), 0, st, a.part, blocks, r->d, a.wq ? dwq : nullptr,
                     a.wk ? dwk : nullptr);
  DLRM_CHECK_LAUNCH();
  return DLRM_OK;
}
