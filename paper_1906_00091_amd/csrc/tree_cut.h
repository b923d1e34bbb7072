// How a call of new items over a paged cache is cut into workgroups: host arithmetic alone.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "dlrm_hot.h"

namespace dlrm {

// Columns of a workgroup in tiles of 16: a wavefront's up to 32 (cache_tree.h), all wavefronts' beyond (cache_wide.h: four wavefronts, or eight); one tile where `max_items` is 0,
// for one item that is in the cache.  (The biases of a block's heads stand in LDS, 33 kB for 64 heads: more than that to a key head keep to the small blocks, which read the cache
// once for each 32 columns.  128 caches of up to 8192 items under up to 60, bf16, d 128, one key head: 64 heads 1.9 ms, 80 heads 6.9.)
constexpr int kWide = 8;  // tiles from which on a workgroup's wavefronts share them
inline int tiles_of(const dlrm_kv_cache* c, int Hq, int max_items) {
  const int G = Hq / c->Hk;
  const int64_t n = (int64_t)max_items * G;
  if (n <= 16) return 1;
  if (n <= 32 || G > 64) return 2;
  return n <= 128 || c->dtype == DLRM_F32 ? kWide : 2 * kWide;
}

constexpr int kPiece = 1024;      // pages of a chunk at most (the kernels' table of them)
constexpr int kLeastChunk = 256;  // keys
inline int64_t blocks_of(const dlrm_kv_cache* c, int Hq, int max_items) {
  const int cols = 16 * tiles_of(c, Hq, max_items);
  return ((int64_t)(max_items < 1 ? 1 : max_items) * (Hq / c->Hk) + cols - 1) / cols;
}
// (2^58 at most; from kMany on none is cut for there being few of them, and this times a length stays far below 2^63)
constexpr int kMany = 2048;
inline int64_t groups_of(const dlrm_kv_cache* c, int Hq, int max_items) {
  const int64_t n = (int64_t)c->B * c->Hk * blocks_of(c, Hq, max_items);
  return n < kMany ? n : kMany;
}
inline int64_t most_of_chunk(const dlrm_kv_cache* c) { return (int64_t)(kPiece - 1) * c->page; }  // (it need not start on a page)
// Keys of a chunk: as many as leave kMany workgroups, so that sequences of mixed lengths fill the device to the end, but no fewer than `fine` for it; else as many as
// leave each CU the workgroups that it holds.  Every chunk leaves a row of sums for each column, which are written and read again.  (Weights in one part: 128 sequences of up to
// 8192 items with trees of up to 60, bf16, d 128: one chunk a sequence 735 us, two 694, four 671;  256 sequences of up to 8192 with one item: 431 and, cut in two,
// 422;  one of 131072 items under 64 with 256 columns, each CU one workgroup 123 us, two 144, four 192, eight 248.)
inline int64_t fill_of(int tiles) { return tiles > kWide ? 256 : tiles == kWide ? 512 : 1024; }
inline int64_t fine_of(int tiles) { return tiles == kWide ? 1024 : 2048; }
inline int chunk_of(const dlrm_kv_cache* c, int tiles, int64_t groups, int64_t total) {
  int64_t n = (groups * total + kMany - 1) / kMany;
  if (n < fine_of(tiles)) {
    n = (groups * total + fill_of(tiles) - 1) / fill_of(tiles);
    if (n > fine_of(tiles) + 128) n = fine_of(tiles) + 128;
  }
  if (n < kLeastChunk) n = kLeastChunk;
  n = (n + 127) / 128 * 128;
  if (n > most_of_chunk(c)) n = most_of_chunk(c);
  return (int)(n > total ? total : n);
}
inline int64_t held_of(const dlrm_kv_cache* c) { return (int64_t)c->table_cols * c->page; }

// The most chunks that bounds of up to max_len cached and `extra` new items give a sequence.  (A smaller bound may give more of them than max_len.)  A chunk has the fewest
// keys there are, as many as a page table's piece holds, enough for `fine` keys, or enough for the workgroups wanted.
inline int64_t most_splits(const dlrm_kv_cache* c, int tiles, int64_t groups, int max_len, int extra) {
  const int64_t held = held_of(c), n = (max_len > held ? held : max_len) + extra;
  if (n < 1) return 1;
  auto pieces = [&](int64_t keys) { return (n - 1) / keys + 1; };
  int64_t most = (fill_of(tiles) - 1) / groups + 1;
  if (pieces(fine_of(tiles)) > most) most = pieces(fine_of(tiles));
  if (pieces(most_of_chunk(c)) > most) most = pieces(most_of_chunk(c));
  return pieces(kLeastChunk) < most ? pieces(kLeastChunk) : most;
}

struct TreeCut {
  int tiles, chunk, splits;  // of 16 columns to a workgroup; keys of a chunk; chunks of a sequence
  int64_t blocks;            // of columns of a key head
};
// max_items new items at most for each sequence, or 0 for one that is in the cache
inline TreeCut tree_cut(const dlrm_kv_cache* c, int Hq, int max_len, int max_items) {
  const int64_t held = held_of(c), total = (max_len > held ? held : max_len) + max_items;
  TreeCut x = {tiles_of(c, Hq, max_items), 1, 1, blocks_of(c, Hq, max_items)};
  if (total > 0) {
    x.chunk = chunk_of(c, x.tiles, groups_of(c, Hq, max_items), total);
    x.splits = (int)((total - 1) / x.chunk) + 1;
  }
  return x;
}
inline size_t parts_bytes(const dlrm_kv_cache* c, int64_t rows, int64_t splits) {
  const size_t n = splits > 1 ? (size_t)rows * splits * (c->d + 2) * sizeof(float) : 0;
  return n < 256 ? 256 : (n + 255) / 256 * 256;
}
// Bytes for `rows` rows under every bound on the length up to max_len
inline size_t tree_workspace(const dlrm_kv_cache* c, int Hq, int64_t rows, int max_len, int max_items) {
  return parts_bytes(c, rows, most_splits(c, tiles_of(c, Hq, max_items), groups_of(c, Hq, max_items), max_len, max_items));
}

}  // namespace dlrm
