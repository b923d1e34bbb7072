// Attention of several new items of every sequence over a paged cache and over one another, and of one new item with a learned bias.
//
// Up to 32 columns ((item, head) pairs of a key head); more: cache_wide.h.
//
// As the attention of one new item: a key row is loaded once, straight from its page into the registers that the product takes it in, S^T = K Q^T leaves a
// lane four keys of one column, and those registers are what O^T = V^T P^T takes; values pass through a piece of LDS of the wavefront's own.  16 columns
// are a tile, and a wavefront has NT of them.  New items are keys behind the cached ones: key j of a sequence is item j of the cache, or row j - len of the new
// ones, and only the address of its row differs.
//
// The length is split over workgroups in chunks; their parts (unnormalised sums, maxima, weights) are joined by a second kernel in the order of the chunks.
//
// Bound by memory where there is enough of it: 256 sequences of up to 8192 items under one item with a bias of 64 buckets, 16 query heads on 4, bf16, d 128, capped:
// 403 us and 5 for the join for 2.15 GB, 5.3 TB/s.  64 sequences of up to 200 items: 11 us, a launch and a chain of loads (length, page, key, value); 64 of up to 200 under trees of 8: 12 us.
#pragma once

#include "cache_ops.h"
#include "tree_args.h"

namespace dlrm {

template <int DT, int DP, int NT, bool LARGE, bool TREE>
__global__ __launch_bounds__(256) void cache_tree_kernel(TreeArgs a) {
  constexpr int WAVES = 4, COLS = 16 * NT;
  constexpr int EB = Tab<DT>::EB, E = Tab<DT>::ELEMS, STEPS = DP / 32, NB = DP / 16;
  constexpr int CH = DP * EB / 16, NV = kKeys * CH / DLRM_WAVE;  // chunks of a row; of a tile, per lane
  constexpr int STRIDE = DP * EB + 16;
  constexpr int OS = DP + 4;  // row of the joined sums
  // fp16: weights are at most 2^8 (below) and made 2^7 times as large, sums and all: those of a long cache's many keys are not lost below 2^-24
  constexpr float LIFT = DT == DLRM_F16 ? 7.0f : 0.0f;
  constexpr int VBYTES = WAVES * kKeys * STRIDE, OBYTES = WAVES * 16 * OS * 4;
  __shared__ __attribute__((aligned(16))) char lds[VBYTES > OBYTES ? VBYTES : OBYTES];
  __shared__ int pages[kTablePages];
  __shared__ float stat[WAVES][2][16];
  __shared__ int bounds[DLRM_MAX_BUCKETS];
  __shared__ int window[WAVES][DLRM_WAVE];  // buckets of a tile's distances
  extern __shared__ float biases[];         // [bias_rows][buckets | 1], in powers of two

  int s, hk, split, blk;
  if (!place_of(a, s, hk, split, blk)) return;
  const int G = a.Hq / a.Hk, c0 = blk * COLS;
  const int lane = lane_id(), g = lane >> 4, n = lane & 15, wave = wave_id();
  const int start = split * a.chunk, page0 = start >> a.page_shift, n_pages = pages_of_chunk(a, start);
  for (int p = threadIdx.x; p < n_pages; p += 256) pages[p] = a.pages[(int64_t)s * a.cols + page0 + p];
  const TreeSeq me(a, s);
  const int n_keys = min(me.total - start, a.chunk), n_cached = min(max(me.len - start, 0), max(n_keys, 0));
  if (c0 >= me.n * G || (n_keys <= 0 && split > 0)) return;  // the first chunk of rows that see nothing gives zeros

  const int row_floats = a.buckets | 1;
  bool by_marks = true;
  if (a.table) {
    load_bounds(bounds, a.bounds, a.buckets, a.bucket_steps, 256);
    load_biases(a, hk, c0, biases, row_floats, WAVES);
    by_marks = bounds_differ(a.bounds, a.buckets);
  }
  // this lane's columns
  Op16<DT> qf[NT][STEPS];
  int item[NT], place[NT];
  float slope[NT];
  const float* bias_row[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int c = c0 + 16 * t + n;
    const bool there = c < me.n * G;
    const int i = there ? c / G : 0, head = hk * G + (there ? c - i * G : 0);
    item[t] = i;
    place[t] = !TREE ? me.len - 1 : a.positions ? a.positions[me.t0 + i] : 0;
    slope[t] = a.slopes ? a.slopes[head] * kLog2e : 0.0f;
    bias_row[t] = biases + (a.bias_rows == G ? head - hk * G : there ? c - c0 : 0) * row_floats;
    const char* row = row_of(a.q, me.t0 + i, head);
#pragma unroll
    for (int st = 0; st < STEPS; ++st) {
      qf[t][st] = op16_zero<DT>();
      if (there && 32 * st + 8 * g < a.d) qf[t][st] = op16_load<DT>(row + (32 * st + 8 * g) * EB);
    }
  }
  const bool bend = a.cap > 0.0f;
  const float zs = bend ? a.scale / a.cap : 0.0f, scale2 = (bend ? a.cap : a.scale) * kLog2e;
  const int last_bound = a.table && a.buckets > 1 ? a.bounds[a.buckets - 2] : -0x7fffffff - 1;
  // places of the wavefront's columns (one of no column counts as the first)
  int low = place[0], high = place[0];
  if constexpr (TREE) {
#pragma unroll
    for (int t = 1; t < NT; ++t) {
      low = min(low, place[t]);
      high = max(high, place[t]);
    }
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) {
      low = min(low, __shfl_xor(low, o, DLRM_WAVE));
      high = max(high, __shfl_xor(high, o, DLRM_WAVE));
    }
  }
  low = __builtin_amdgcn_readfirstlane(low);
  by_marks = by_marks && low <= kWindowEnd;
  const bool close = (uint32_t)__builtin_amdgcn_readfirstlane(high) - (uint32_t)low <= 32;  // one window of 64 distances is enough for a tile
  __syncthreads();

  const int row_bytes = a.d * EB, mask = (1 << a.page_shift) - 1;
  const int64_t head_bytes = (int64_t)row_bytes << a.page_shift, page_bytes = head_bytes * a.Hk;
  // The rows of the chunk's key i; a key past the end, or on a page that is not there, gives the cache's first row and false.  No load stands in a branch (the wait
  // for it would come with the branch's end): what came for no reason is masked where it is used.
  struct Where {
    const char* k;
    const char* v;
    bool there;
  };
  auto row_at = [&](int i) -> Where {
    const int at = min(i, n_cached - 1), j = start + max(at, 0), p = n_cached > 0 ? pages[(j >> a.page_shift) - page0] : -1;
    bool there = i < n_cached && p >= 0 && p < a.n_pages;
    const int64_t off = there ? p * page_bytes + hk * head_bytes + (int64_t)((j & mask) * row_bytes) : 0;
    Where w = {a.k + off, a.v + off, there};
    if constexpr (TREE) {
      const bool fresh = i >= n_cached && i < n_keys;
      const int64_t t = me.t0 + (fresh ? start + i - me.len : 0);
      w.k = fresh ? row_of(a.new_k, t, hk) : w.k;
      w.v = fresh ? row_of(a.new_v, t, hk) : w.v;
      w.there = there || fresh;
    }
    return w;
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
      const Where w = row_at(j0 + 16 * u + n);
      seen[u] = w.there;
#pragma unroll
      for (int st = 0; st < STEPS; ++st) kf[u][st] = op16_load<DT>(w.k + kcol[st]);
    }
    v_there = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int id = lane + i * DLRM_WAVE, r = id / CH, cc = min(id % CH, a.d / E - 1);
      const Where w = row_at(j0 + r);
      v_there |= w.there ? 1u << i : 0u;
      vf[i] = load16(w.v + cc * 16);
    }
  };

  f32x4 o[NT][NB];
  float m[NT], l[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    m[t] = -kInf;
    l[t] = 0.0f;
#pragma unroll
    for (int b = 0; b < NB; ++b) o[t][b] = f32x4{0, 0, 0, 0};
  }
  int j0 = wave * kKeys;
  if (j0 < n_keys) fetch(j0);
  for (; j0 < n_keys; j0 += WAVES * kKeys) {
    f32x4 sc[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        sc[t][u] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int st = 0; st < STEPS; ++st) sc[t][u] = Op16<DT>::mma(kf[u][st], qf[t][st], sc[t][u]);
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
    const int first_key = start + j0 + 4 * g;  // of this lane: first_key + 16 u + r
    const bool any_new = TREE && j0 + kKeys > n_cached;
    const bool far = low - (start + j0 + 31) >= last_bound;
    if (a.table && !any_new && !far && close) {
      uint64_t starts;
      const int b = buckets_from(bounds, a.buckets, a.bucket_steps, by_marks, low - (start + j0 + 31), window[wave], starts);
      wave_fence();
      window[wave][lane] = b;
      wave_fence();
    }
    Op16<DT> p[NT], p_low[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      float x[8];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int r = 0; r < 4; ++r) x[4 * u + r] = (bend ? bent16<LARGE>(sc[t][u][r] * zs) : sc[t][u][r]) * scale2;
      if (any_new) {
        // keys among the new items: places of their own, and a key that is not on the way to this lane's item is hidden
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int key = first_key + 16 * (e >> 2) + (e & 3), u = key - me.len;
          int away = place[t] - key;
          if (u >= 0) {
            const int64_t at = me.t0 + min(u, me.n - 1);
            const int last = a.last ? a.last[at] : me.n - 1;
            if (a.positions) away = place[t] - a.positions[at];
            if (u > item[t] || item[t] > last) x[e] = -kInf;
          }
          if (a.table) x[e] += bias_row[t][bucket_of(bounds, a.buckets, a.bucket_steps, away)];
          x[e] -= slope[t] * fabsf((float)away);
        }
      } else {
        const int away = place[t] - first_key;  // of this lane's first key; its last stands at away - 19
        if (a.table) {
          if (far) {
            const float b = bias_row[t][a.buckets - 1];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] += b;
          } else if (close) {
            const int* at = window[wave] + (place[t] - low) + 31 - 4 * g;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] += bias_row[t][at[-(16 * (e >> 2) + (e & 3))]];
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] += bias_row[t][bucket_of(bounds, a.buckets, a.bucket_steps, away - (16 * (e >> 2) + (e & 3)))];
          }
        }
        if (a.slopes) {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] -= slope[t] * fabsf((float)(away - (16 * (e >> 2) + (e & 3))));
        }
      }
      float top = -kInf;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[e] = ((e >> 2 ? have1 : have0) >> (4 * g + (e & 3))) & 1 ? x[e] : -kInf;
        top = fmaxf(top, x[e]);
      }
      top = fmaxf(top, __shfl_xor(top, 16, DLRM_WAVE));
      top = fmaxf(top, __shfl_xor(top, 32, DLRM_WAVE));
      // The sums are rescaled only where a maximum grew by more than 2^8: until then weights of up to 2^8 are as good as weights of up to 1.
      if (__ballot(top > m[t] + 8.0f)) {
        const float m1 = fmaxf(m[t], top), f = __builtin_amdgcn_exp2f(m[t] - (m1 == -kInf ? 0.0f : m1));
        m[t] = m1;
        l[t] *= f;
#pragma unroll
        for (int b = 0; b < NB; ++b) o[t][b] *= f;
      }
      const float ms = (m[t] == -kInf ? 0.0f : m[t]) - LIFT;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[e] = __builtin_amdgcn_exp2f(x[e] - ms);
        l[t] += x[e];
      }
      // 16-bit rows: weights in two parts, each in a product of its own
      if constexpr (EB == 2)
        two_parts<DT>(x, p[t].v, p_low[t].v);
      else
        p[t] = op16_set<DT>(x);
    }
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
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        o[t][b] = Op16<DT>::mma(vt, p[t], o[t][b]);
        if constexpr (EB == 2) o[t][b] = Op16<DT>::mma(vt, p_low[t], o[t][b]);
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
  // join the wavefronts, 16 columns at a time: a thread takes 4 columns of a row
  float* os = reinterpret_cast<float*>(lds);
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    if (c0 + 16 * t >= me.n * G) break;
    l[t] += __shfl_xor(l[t], 16, DLRM_WAVE);
    l[t] += __shfl_xor(l[t], 32, DLRM_WAVE);
    __syncthreads();  // every wavefront is done with its values, and with the sums before
    if (g == 0) {
      stat[wave][0][n] = m[t];
      stat[wave][1][n] = l[t];
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) *reinterpret_cast<f32x4*>(os + (wave * 16 + n) * OS + 16 * b + 4 * g) = o[t][b];
    __syncthreads();
    const int per_row = a.d / 4, rows = min(16, me.n * G - c0 - 16 * t);
    for (int id = threadIdx.x; id < rows * per_row; id += 256) {
      const int r = id / per_row, col = id % per_row * 4, c = c0 + 16 * t + r, i = c / G, head = hk * G + c - i * G;
      float top = -kInf;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) top = fmaxf(top, stat[w][0][r]);
      const float ms = top == -kInf ? 0.0f : top;
      f32x4 sum = {0, 0, 0, 0};
      float total = 0.0f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        const float f = __builtin_amdgcn_exp2f(stat[w][0][r] - ms);
        total += f * stat[w][1][r];
        sum += f * *reinterpret_cast<const f32x4*>(os + (w * 16 + r) * OS + col);
      }
      if (a.splits == 1) {
        store4<DT>(row_of(a.out, me.t0 + i, head) + col * EB, sum * (total == 0.0f ? 0.0f : 1.0f / total));
      } else {
        const int64_t at = ((me.t0 + i) * a.Hq + head) * a.splits + split;
        *reinterpret_cast<f32x4*>(a.po + at * a.d + col) = sum;
        if (col == 0) {
          a.pm[at * 2] = top;
          a.pm[at * 2 + 1] = total;
        }
      }
    }
  }
}

// Joins the chunks of a row (new item, head): a wavefront a row, half of it every second chunk, 4 columns a lane, four chunks of each half in flight.
template <int DT>
__global__ __launch_bounds__(256) void cache_tree_join_kernel(TreeArgs a) {
  constexpr int AHEAD = 4;
  const int rows = a.max_items * a.Hq, row = blockIdx.x * 4 + wave_id();  // of this sequence
  const int s = a.seq0 + blockIdx.y;
  const TreeSeq me(a, s);
  if (row >= rows || row >= me.n * a.Hq) return;
  const int i = row / a.Hq, head = row - i * a.Hq, n = me.total > 0 ? (me.total - 1) / a.chunk + 1 : 1;
  const int64_t at = ((me.t0 + i) * a.Hq + head) * a.splits;
  const float* pm = a.pm + at * 2;
  const float* po = a.po + at * a.d;
  const int lane = lane_id(), half = lane >> 5, col = (lane & 31) * 4;
  float top = -kInf;
  for (int c = lane; c < n; c += DLRM_WAVE) top = fmaxf(top, pm[2 * c]);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, DLRM_WAVE));
  const float ms = top == -kInf ? 0.0f : top;
  f32x4 sum = {0, 0, 0, 0};
  float total = 0.0f;
  for (int c0 = half; c0 < n; c0 += 2 * AHEAD) {
    f32x4 v[AHEAD];
    float f[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const int c = c0 + 2 * j, there = c < n ? c : c0;
      v[j] = loadf4(po + (int64_t)there * a.d + min(col, a.d - 4));
      f[j] = __builtin_amdgcn_exp2f(pm[2 * there] - ms);
      total += c < n ? f[j] * pm[2 * there + 1] : 0.0f;
    }
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) sum += c0 + 2 * j < n ? f[j] * v[j] : f32x4{0, 0, 0, 0};
  }
  total += __shfl_xor(total, 32, DLRM_WAVE);
#pragma unroll
  for (int e = 0; e < 4; ++e) sum[e] += __shfl_xor(sum[e], 32, DLRM_WAVE);
  if (half != 0 || col >= a.d) return;
  store4<DT>(row_of(a.out, me.t0 + i, head) + col * Tab<DT>::EB, sum * (total == 0.0f ? 0.0f : 1.0f / total));
}

template <int DT>
int launch_cache_tree(const TreeArgs& a, const TreeLaunch& how, hipStream_t st) {
  auto with = [&](auto dp, auto nt, auto large, auto tree) -> int {
    return for_sequences(a, how, [&](const TreeArgs& b) -> int {
      hipLaunchKernelGGL((cache_tree_kernel<DT, dp(), nt(), large(), tree()>), dim3(grid_of(b)), dim3(256), how.lds, st, b);
      DLRM_CHECK_LAUNCH();
      return DLRM_OK;
    });
  };
  auto by_tiles = [&](auto dp, auto large) -> int {
    using T = std::integral_constant<bool, true>;
    if (!a.off) return with(dp, std::integral_constant<int, 1>{}, large, std::integral_constant<bool, false>{});
    if (how.tiles == 1) return with(dp, std::integral_constant<int, 1>{}, large, T{});
    return with(dp, std::integral_constant<int, 2>{}, large, T{});
  };
  auto by_cap = [&](auto dp) -> int {
    if constexpr (DT != DLRM_F32) {
      if (a.cap <= (DT == DLRM_F16 ? 128.0f : 1024.0f)) return by_tiles(dp, std::integral_constant<bool, false>{});
    }
    return by_tiles(dp, std::integral_constant<bool, true>{});
  };
  int rc = DLRM_OK;
  if (how.tiles > 2) rc = launch_cache_wide<DT>(a, how, st);
  else if (a.d <= 32) rc = by_cap(std::integral_constant<int, 32>{});
  else if (a.d <= 64) rc = by_cap(std::integral_constant<int, 64>{});
  else if (a.d <= 96) rc = by_cap(std::integral_constant<int, 96>{});
  else rc = by_cap(std::integral_constant<int, 128>{});
  if (rc != DLRM_OK || a.splits == 1) return rc;
  return for_sequences(a, how, [&](const TreeArgs& b) -> int {
    hipLaunchKernelGGL(cache_tree_join_kernel<DT>, dim3(div_up((int64_t)a.max_items * a.Hq, 4), (unsigned)b.B), dim3(256), 0, st, b);
    DLRM_CHECK_LAUNCH();
    return DLRM_OK;
  });
}

}  // namespace dlrm
