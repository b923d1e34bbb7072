// What the kernels of new items over a paged cache are told.
#pragma once

#include "heads.h"

namespace dlrm {

struct TreeArgs {
  Rows q, out, new_k, new_v;
  const char* k;
  const char* v;
  const int32_t* pages;
  const int32_t* lens;
  const int64_t* off;  // [B + 1] of the new items; NULL: one a sequence, at the place of the newest cached item
  const int32_t* last;
  const int32_t* positions;
  const float* slopes;
  const float* table;  // [Hq, buckets] or NULL
  const int32_t* bounds;
  int buckets, bucket_steps, bias_rows;  // bias_rows: heads whose biases a workgroup needs
  int B, Hq, Hk, d, cols, n_pages, page_shift, max_len, max_items;  // max_len: the table's items at most
  int chunk, splits, blocks;  // keys of a chunk; chunks of a sequence; groups of 16 NT columns of a key head
  int seq0;                   // first sequence of this launch
  float scale, cap;
  float* po;  // [T * Hq][splits][d] unnormalised sums
  float* pm;  // [T * Hq][splits][2] maximum (powers of two), sum of weights
};

// A sequence's new items and keys.
struct TreeSeq {
  int64_t t0;      // its first new item
  int n, len, total;  // new items; cached items that are read; keys
  __device__ inline TreeSeq(const TreeArgs& a, int s) {
    len = max(0, min(a.lens[s], a.max_len));
    if (a.off) {
      t0 = a.off[s];
      n = (int)min(a.off[s + 1] - t0, (int64_t)a.max_items);
      total = len + n;
    } else {
      t0 = s;
      n = 1;
      total = len;
    }
  }
};

struct TreeLaunch {
  int tiles;  // of 16 columns to a workgroup
  int64_t each;  // sequences of a launch
  unsigned lds;  // bytes for the biases
};

// Up to 32 columns of a key head (cache_tree.h), and the join of the chunks; more than that (cache_wide.h).
template <int DT>
int launch_cache_tree(const TreeArgs& a, const TreeLaunch& how, hipStream_t st);
template <int DT>
int launch_cache_wide(const TreeArgs& a, const TreeLaunch& how, hipStream_t st);

// Page numbers of the chunk from `start` on, loaded beside the length and not after it: as many as the bound on it may need.
__device__ inline int pages_of_chunk(const TreeArgs& a, int start) {
  return start >= a.max_len ? 0 : ((start + min(a.chunk, a.max_len - start) - 1) >> a.page_shift) + 1 - (start >> a.page_shift);
}
// The biases of the heads that a block's columns (from c0 on) have, in powers of two: row `row` of the block's is that of head `row` of the key head's, or of column
// c0 + row where these are fewer.  A wavefront a row.
__device__ inline void load_biases(const TreeArgs& a, int hk, int c0, float* to, int stride, int waves) {
  const int G = a.Hq / a.Hk;
  for (int row = wave_id(); row < a.bias_rows; row += waves) {
    const float* from = a.table + (int64_t)(hk * G + (a.bias_rows == G ? row : (c0 + row) % G)) * a.buckets;
    for (int b = lane_id(); b < a.buckets; b += DLRM_WAVE) to[row * stride + b] = bias_in(from[b], 1.44269504088896340736f);
  }
}

// kernels take `each` sequences a launch: go(arguments for them)
template <typename F>
__host__ inline int for_sequences(const TreeArgs& a, const TreeLaunch& how, F go) {
  for (int64_t s0 = 0; s0 < a.B; s0 += how.each) {
    TreeArgs b = a;
    b.seq0 = (int)s0;
    b.B = (int)(a.B - s0 < how.each ? a.B - s0 : how.each);
    if (int st = go(b)) return st;
  }
  return DLRM_OK;
}
__host__ inline unsigned grid_of(const TreeArgs& a) { return (unsigned)(((int64_t)a.B * a.Hk * a.splits + 7) / 8 * 8 * a.blocks); }
// Workgroups go to the 8 dies in turn: those of one sequence, key head and chunk, which read the same keys, lie 8 apart.  The chunks of a sequence do not follow one
// another: many sequences have only the first, and these would all go to every second die (500 candidate lists cut in two: 190 us, 117 not cut).
// False past the last.
__device__ inline bool place_of(const TreeArgs& a, int& seq, int& hk, int& split, int& block) {
  const int in_eight = blockIdx.x % (8 * a.blocks), unit = blockIdx.x / (8 * a.blocks) * 8 + in_eight % 8, heads = a.B * a.Hk;
  block = in_eight / 8;
  split = unit / heads;
  const int at = unit - split * heads;
  seq = a.seq0 + at / a.Hk;
  hk = at % a.Hk;
  return split < a.splits;
}

}  // namespace dlrm
