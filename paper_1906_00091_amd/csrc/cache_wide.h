// Attention of several new items of every sequence over a paged cache and over one another, for more than 32 columns ((item, head) pairs of a key head).
//
// The forward of attention over sequences, with a paged cache for keys: wavefronts of 32 columns, tiles of 64 keys and values that the workgroup's WAVES
// wavefronts bring to LDS together, products of 32 x 32 whose accumulators' columns are the wavefront's own.  Where a block's columns are no more than half of what the
// workgroup holds, two wavefronts share 32 of them, each with half of a tile's keys, and join at the end.  New items are keys behind the cached
// ones, as in cache_tree.h.
//
// 16-bit weights enter their product in two parts, as for up to 32 columns: an item's result is off by its own rounding whatever is asked with it.  (One part would take
// 575, 87 and 128 us where two take 683, 103 and 155, the sizes below on one card, and be 1.2 to 1.4 times as far off.)  128 sequences of up to 8192 items with trees of up to 60, 16 query heads
// on 4, bf16, d 128, a bias of 64 buckets, capped: 652 us and 36 for the join, 188 TFLOP/s of visible pairs; with 60 items to 8192 each 1268 and 69, 387 TFLOP/s (vector work 54 % of the
// time, matrix cores 26 %, one after the other for the most part).  The difference is rows of no column in a wavefront's 32 and wavefronts with none in a workgroup.  500
// candidate lists over up to 1000 items, fp16, d 40: 105 us.  One sequence of 131072 items under 64: 157 us and 14, 400 TFLOP/s.
#pragma once

#include "seq_attn.h"
#include "tree_args.h"

namespace dlrm {

constexpr int kWidePages = 1024;  // pages of a chunk, at most

// Registers leave room for four wavefronts a SIMD up to 64 columns, two workgroups of eight a CU: 25 of them are spilled for it (500 candidate lists over up to 1000
// items, fp16, d 40, weights in one part: 89 us, 115 with one workgroup).
template <int DT, int DP, int WAVES, bool BEND>
__global__ __launch_bounds__(64 * WAVES, DT == DLRM_F32 ? 1 : DP <= 64 ? 4 : 2) void cache_wide_kernel(TreeArgs a) {
  typedef Tile<DT, DP> T;
  constexpr bool TWO = DT != DLRM_F32;  // weights in two parts
  constexpr int EB = Tab<DT>::EB, STEPS = DP / 16, NB = DP / 32, THREADS = 64 * WAVES, BK = 64;
  constexpr int CH = DP * EB / 16, N = (BK * CH + THREADS - 1) / THREADS;  // chunks of 16 bytes: of a row; of a tile, per thread
  constexpr int TILE = BK * T::STRIDE, BUFS = 4 * TILE > (DT == DLRM_F32 || WAVES == 8 ? 120 : 70) * 1024 ? 1 : 2;
  constexpr int HALF = WAVES / 2, JOIN = HALF * DP / 2 * DLRM_WAVE * 4, BYTES = 2 * BUFS * TILE > JOIN ? 2 * BUFS * TILE : JOIN;
  __shared__ __attribute__((aligned(16))) char lds[BYTES];
  __shared__ int pages[kWidePages];
  __shared__ float stat[HALF][2][2][32];  // of a group: part, maximum or sum, column
  __shared__ int bounds[kBuckets];
  __shared__ int window[WAVES][DLRM_WAVE];  // buckets of a tile's distances
  __shared__ __attribute__((aligned(16))) int fresh[WAVES][2][32];  // of a tile's keys among the new items: last, place
  extern __shared__ float biases[];             // [bias_rows][buckets | 1], in powers of two

  int s, hk, split, blk;
  if (!place_of(a, s, hk, split, blk)) return;
  const int G = a.Hq / a.Hk, c0 = blk * 32 * WAVES;
  const int lane = lane_id(), h = lane >> 5, wave = __builtin_amdgcn_readfirstlane(wave_id());
  const int start = split * a.chunk, page0 = start >> a.page_shift, n_pages = pages_of_chunk(a, start);
  for (int p = threadIdx.x; p < n_pages; p += THREADS) pages[p] = a.pages[(int64_t)s * a.cols + page0 + p];
  const TreeSeq me(a, s);
  const int n_keys = min(me.total - start, a.chunk), n_cached = min(max(me.len - start, 0), max(n_keys, 0));
  const int columns = me.n * G;
  if (c0 >= columns || (n_keys <= 0 && split > 0)) return;  // the first chunk of rows that see nothing gives zeros

  // (the wavefronts that have work are spread over the four SIMDs: wavefront i is on SIMD i % 4)
  const bool shared = columns - c0 <= 32 * HALF;
  const int sharing = columns - c0 <= 64 ? 2 : HALF;  // groups that share
  const int group = shared ? wave % sharing : wave, part = shared ? wave / sharing : 0;

  bool gone = false;  // a page that the sequence has (each thread looks at those that it loaded)
  for (int p = threadIdx.x; n_cached > 0 && p <= ((start + n_cached - 1) >> a.page_shift) - page0; p += THREADS) gone = gone || pages[p] < 0 || pages[p] >= a.n_pages;
  const int row_floats = a.buckets | 1;
  bool by_marks = true;
  if (a.table) {
    load_bounds(bounds, a.bounds, a.buckets, a.bucket_steps, THREADS);
    load_biases(a, hk, c0, biases, row_floats, WAVES);
    by_marks = bounds_differ(a.bounds, a.buckets);
  }
  // this lane's column
  const int c = c0 + 32 * group + (lane & 31);
  const bool mine = c < columns && part < 2;
  const int item = mine ? c / G : 0, head = hk * G + (mine ? c - item * G : 0);
  const int64_t t = me.t0 + item;
  const int place = a.positions ? a.positions[t] : 0;
  const float slope = a.slopes ? a.slopes[head] * kLog2e : 0.0f;
  const float* bias_row = biases + (a.bias_rows == G ? head - hk * G : mine ? c - c0 : 0) * row_floats;
  Op<DT> qf[STEPS];
  own_rows<DT, STEPS>(qf, row_of(a.q, t, head), mine, a.d, h);
  const float scale2 = (BEND ? a.cap : a.scale) * kLog2e, zs = BEND ? a.scale / a.cap : 0.0f;
  const int last_bound = a.table && a.buckets > 1 ? a.bounds[a.buckets - 2] : -0x7fffffff - 1;
  // places of the wavefront's columns (one of no column counts as the first)
  int low = place, high = place;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    low = min(low, __shfl_xor(low, o, DLRM_WAVE));
    high = max(high, __shfl_xor(high, o, DLRM_WAVE));
  }
  low = __builtin_amdgcn_readfirstlane(low);
  by_marks = by_marks && low <= kWindowEnd;
  high = __builtin_amdgcn_readfirstlane(high);
  const bool close = (uint32_t)high - (uint32_t)low <= 32;  // one window of 64 distances is enough for a tile
  const bool whole = __syncthreads_or(gone) == 0;  // every page of the chunk is there

  const int row_bytes = a.d * EB, mask = (1 << a.page_shift) - 1;
  const int64_t head_bytes = (int64_t)row_bytes << a.page_shift, page_bytes = head_bytes * a.Hk;
  // whether the chunk's key i is there, and its row in the cache
  auto cached_at = [&](int i, int64_t& off) {
    const int j = start + max(min(i, n_cached - 1), 0), p = n_cached > 0 ? pages[(j >> a.page_shift) - page0] : -1;
    const bool there = i < n_cached && p >= 0 && p < a.n_pages;
    off = there ? p * page_bytes + hk * head_bytes + (int64_t)((j & mask) * row_bytes) : 0;
    return there;
  };
  // The tile's rows on their way to LDS; no load stands in a branch, what came for no reason becomes zeros where it is put away.
  u32x4 kv[2][N];
  uint32_t there = 0;
  auto fetch = [&](int j0) {
    there = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int id = threadIdx.x + i * THREADS, r = j0 + id / CH, cc = id % CH;
      int64_t off;
      const bool old = cached_at(r, off), in_row = cc * Tab<DT>::ELEMS < a.d;
      const char* k = a.k + off;
      const char* v = a.v + off;
      bool young = false;
      if (j0 + BK > n_cached) {  // (the same for all threads)
        young = r >= n_cached && r < n_keys;
        const int64_t at = me.t0 + (young ? start + r - me.len : 0);
        k = young ? row_of(a.new_k, at, hk) : k;
        v = young ? row_of(a.new_v, at, hk) : v;
      }
      there |= (old || young) && in_row ? 1u << i : 0u;
      kv[0][i] = load16(k + (in_row ? cc * 16 : 0));
      kv[1][i] = load16(v + (in_row ? cc * 16 : 0));
    }
  };
  auto put = [&](char* to) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int id = threadIdx.x + i * THREADS, r = id / CH, cc = id % CH;
      if (BK * CH % THREADS != 0 && r >= BK) break;
#pragma unroll
      for (int x = 0; x < 2; ++x)
        *reinterpret_cast<u32x4*>(to + x * TILE + r * T::STRIDE + cc * 16) = there >> i & 1 ? kv[x][i] : u32x4{0, 0, 0, 0};
    }
  };

  f32x16 o[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) o[b] = f32x16{};
  float m = -kInf, l = 0.0f;
  const int tiles = n_keys > 0 ? (n_keys + BK - 1) / BK : 0;
  const bool busy = c0 + 32 * group < columns && part < 2;
  if (tiles > 0) {
    fetch(0);
    put(lds);
  }
  __syncthreads();
  for (int tile = 0; tile < tiles; ++tile) {
    if (tile + 1 < tiles) fetch((tile + 1) * BK);
    for (int sub = part; sub < 2; sub += shared ? 2 : 1) {
      const int j0 = tile * BK + 32 * sub;
      if (!busy || j0 >= n_keys) break;
      const char* ks = lds + (tile & (BUFS - 1)) * 2 * TILE + 32 * sub * T::STRIDE;
      const char* vs = ks + TILE;
      f32x16 x = {};
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int st = 0; st < STEPS; ++st) {
        if (past_d<DT, STEPS>(st, a.d)) break;
        x = Op<DT>::mma(T::by_row(ks, lane & 31, st, h), qf[st], x);
      }
      __builtin_amdgcn_s_setprio(0);
      if constexpr (BEND) bend(x, zs);
      // which keys are there (bit i: key i of the tile)
      const int ki = j0 + (lane & 31);
      uint32_t have = j0 + 32 <= n_keys ? 0xffffffffu : (1u << (n_keys - j0)) - 1;
      if (!whole) {
        int64_t off;
        have = (uint32_t)__ballot(cached_at(ki, off) || (ki >= n_cached && ki < n_keys));
      }
      const int key0 = start + j0;  // of the tile's first key
      float cc = scale2;
      if (j0 + 32 > n_cached) {
        // keys among the new items: places of their own, and a key that is not on the way to this lane's item is hidden
        const int u = start + ki - me.len;
        const int64_t at = me.t0 + min(max(u, 0), me.n - 1);
        const int seen_by = u < 0 ? 0x7fffffff : a.last ? a.last[at] : me.n - 1, stands = u < 0 || !a.positions ? start + ki : a.positions[at];
        wave_fence();
        if (lane < 32) {
          fresh[wave][0][lane] = seen_by;
          fresh[wave][1][lane] = stands;
        }
        wave_fence();
        int b[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) b[r] = 0;
        if (a.table)
          for (int step = 1 << a.bucket_steps >> 1; step > 0; step >>= 1)
#pragma unroll
            for (int r = 0; r < 16; ++r) b[r] += bounds[b[r] + step - 1] <= place - fresh[wave][1][acc_row(r, h)] ? step : 0;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int key = key0 + acc_row(r, h) - me.len;
          float y = x[r] * scale2;
          if (a.table) y += bias_row[min(b[r], a.buckets - 1)];
          if (a.slopes) y -= slope * fabsf((float)(place - fresh[wave][1][acc_row(r, h)]));
          x[r] = key >= 0 && (key > item || item > fresh[wave][0][acc_row(r, h)]) ? -kInf : y;
        }
        cc = 1.0f;
      } else if (a.table || a.slopes) {
        cc = 1.0f;
        if (!a.table) {
#pragma unroll
          for (int r = 0; r < 16; ++r) x[r] *= scale2;
        } else if (low - (key0 + 31) >= last_bound) {
          const float y = bias_row[a.buckets - 1];
#pragma unroll
          for (int r = 0; r < 16; ++r) x[r] = fmaf(x[r], scale2, y);
        } else if (close) {
          wave_fence();
          uint64_t starts;
          window[wave][lane] = buckets_from(bounds, a.buckets, a.bucket_steps, by_marks, low - (key0 + 31), window[wave], starts);
          wave_fence();
          const int* at = window[wave] + (place - low) + 31 - 4 * h;
#pragma unroll
          for (int r = 0; r < 16; ++r) x[r] = fmaf(x[r], scale2, bias_row[at[-acc_row(r, 0)]]);
        } else {
          int b[16];
#pragma unroll
          for (int r = 0; r < 16; ++r) b[r] = 0;
          for (int step = 1 << a.bucket_steps >> 1; step > 0; step >>= 1)
#pragma unroll
            for (int r = 0; r < 16; ++r) b[r] += bounds[b[r] + step - 1] <= place - key0 - acc_row(r, h) ? step : 0;
#pragma unroll
          for (int r = 0; r < 16; ++r) x[r] = fmaf(x[r], scale2, bias_row[min(b[r], a.buckets - 1)]);  // (as in bucket_of)
        }
        if (a.slopes) {
          const int away = place - key0 - 4 * h;
#pragma unroll
          for (int r = 0; r < 16; ++r) x[r] = fmaf(-slope, fabsf((float)(away - acc_row(r, 0))), x[r]);
        }
      }
      if (have != 0xffffffffu) {
        const uint32_t bits = have >> (4 * h);
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = bits >> acc_row(r, 0) & 1 ? x[r] : -kInf;
      }
      float top = x[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) top = fmaxf(top, x[r]);
      top = fmaxf(top, other_half(top));
      // (rescaled only where a maximum grew by more than 2^8, as in the forward over sequences)
      if (__ballot(top * cc > m + 8.0f)) {
        const float m1 = fmaxf(m, top * cc), f = __builtin_amdgcn_exp2f(m - (m1 == -kInf ? 0.0f : m1));
        l *= f;
#pragma unroll
        for (int b = 0; b < NB; ++b) o[b] *= f;
        m = m1;
      }
      const float ms = m == -kInf ? 0.0f : m - kWeightLift<DT>;
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        Op<DT> p, low;
        float e[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          e[r] = __builtin_amdgcn_exp2f(fmaf(x[8 * g + r], cc, -ms));
          l += e[r];
          if constexpr (!TWO) p.set(r, e[r]);
        }
        if constexpr (TWO) op_two_parts(e, p, low);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          const Op<DT> vt = T::by_column(vs, 16 * g, b, lane);
          o[b] = Op<DT>::mma(vt, p, o[b]);
          if constexpr (TWO) o[b] = Op<DT>::mma(vt, low, o[b]);
        }
      }
    }
    if (BUFS == 1) __syncthreads();
    if (tile + 1 < tiles) put(lds + ((tile + 1) & (BUFS - 1)) * 2 * TILE);
    __syncthreads();
  }
  l += other_half(l);
  if (shared) {
    if (h == 0 && part < 2) {
      stat[group][part][0][lane] = m;
      stat[group][part][1][lane] = l;
    }
    __syncthreads();
    const float m0 = stat[group][0][0][lane & 31], m1 = stat[group][1][0][lane & 31];
    m = fmaxf(m0, m1);
    const float ms = m == -kInf ? 0.0f : m, f[2] = {__builtin_amdgcn_exp2f(m0 - ms), __builtin_amdgcn_exp2f(m1 - ms)};
    l = stat[group][0][1][lane & 31] * f[0] + stat[group][1][1][lane & 31] * f[1];
    join_parts<NB, HALF, 2>(o, lds, group, part == 1 ? 1 : part == 0 ? 0 : -1, f);
    if (part > 0) return;
  }
  if (!mine) return;
  if (a.splits == 1) {
    store_rows<DT, NB>(o, l == 0.0f ? 0.0f : 1.0f / l, row_of(a.out, t, head), a.d, h);
  } else {
    const int64_t at = (t * a.Hq + head) * a.splits + split;
    store_rows<DLRM_F32, NB>(o, 1.0f, reinterpret_cast<char*>(a.po + at * a.d), a.d, h);
    if (h == 0) {
      a.pm[at * 2] = m;
      a.pm[at * 2 + 1] = l;
    }
  }
}

template <int DT>
int launch_cache_wide(const TreeArgs& a, const TreeLaunch& how, hipStream_t st) {
  auto with = [&](auto dp, auto waves, auto bend) -> int {
    return for_sequences(a, how, [&](const TreeArgs& b) -> int {
      hipLaunchKernelGGL((cache_wide_kernel<DT, dp(), waves(), bend()>), dim3(grid_of(b)), dim3(64 * waves()), how.lds, st, b);
      DLRM_CHECK_LAUNCH();
      return DLRM_OK;
    });
  };
  auto by_cap = [&](auto dp, auto waves) -> int {
    if (a.cap > 0.0f) return with(dp, waves, std::integral_constant<bool, true>{});
    return with(dp, waves, std::integral_constant<bool, false>{});
  };
  auto by_size = [&](auto dp) -> int {
    if constexpr (DT != DLRM_F32) {
      if (how.tiles == 16) return by_cap(dp, Int<8>{});
    }
    return by_cap(dp, Int<4>{});
  };
  if (a.d <= 32) return by_size(Int<32>{});
  if (a.d <= 64) return by_size(Int<64>{});
  if (a.d <= 96) return by_size(Int<96>{});
  return by_size(Int<128>{});
}

}  // namespace dlrm
