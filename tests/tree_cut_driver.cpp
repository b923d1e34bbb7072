// The library's cut of new items over a paged cache (tree_cut.h), for a test on the host.
#include "tree_cut.h"

extern "C" void tree_cut(const dlrm_kv_cache* c, int Hq, int max_len, int max_items, int64_t* to) {
  const dlrm::TreeCut x = dlrm::tree_cut(c, Hq, max_len, max_items);
  to[0] = x.tiles;
  to[1] = x.chunk;
  to[2] = x.splits;
  to[3] = x.blocks;
}
