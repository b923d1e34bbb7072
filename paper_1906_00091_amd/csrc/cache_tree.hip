// Attention of new items over a paged cache: entry points and argument checks (the kernels: cache_tree.h).
#include "tree_args.h"
#include "tree_cut.h"

#include <math.h>

#include <initializer_list>

using namespace dlrm;

static int check_common(const dlrm_kv_cache* c, int Hq) {
  if (int st = check_cache(c)) return st;
  return check_head_shape(Hq, c->Hk, c->d, c->dtype);
}
// Checks the arguments; `items` becomes the bound on a sequence's new items, no looser than their total (1 for none at all).
static int check_tree(const dlrm_kv_cache* c, const dlrm_new_items* x, int Hq, int max_len, int& items) {
  if (int st = check_common(c, Hq)) return st;
  if (!x) return DLRM_ERR_NULL;
  if (max_len < 0 || x->T < 0 || x->T > DLRM_MAX_ITEMS || x->max_items < 1) return DLRM_ERR_BAD_SHAPE;
  items = (int)(x->T < 1 ? 1 : x->max_items > x->T ? x->T : x->max_items);
  // a sequence's keys, and the rows of a key head's queries, are counted in 32 bits, with room for a tile past their end
  const int64_t held = held_of(c), len = max_len > held ? held : max_len, most = 0x7fffffff - 1024;
  if (len + items > most || (int64_t)items * Hq > most) return DLRM_ERR_BAD_SHAPE;
  return DLRM_OK;
}

// One call of either kind: max_items new items, or none.
static int run(const dlrm_kv_cache* c, const int32_t* lens, int max_len, int max_items, int64_t T, int Hq, TreeArgs a, const dlrm_heads* q,
               const dlrm_heads* out, const dlrm_rel_bias* bias, size_t need, void* workspace, size_t workspace_bytes, void* stream) {
  if (!lens) return DLRM_ERR_NULL;
  if (!(a.scale > 0.0f) || !isfinite(a.scale) || !(a.cap >= 0.0f) || !isfinite(a.cap)) return DLRM_ERR_BAD_SHAPE;
  const int eb = elem_bytes(c->dtype);
  for (const dlrm_heads* x : {q, out})
    if (int st = check_heads(x, T, Hq, c->d, eb)) return st;
  if (T == 0) return DLRM_OK;  // nothing to answer
  a.q = rows_of(q, T, Hq, c->d, eb);
  a.out = rows_of(out, T, Hq, c->d, eb);
  a.k = static_cast<const char*>(c->k);
  a.v = static_cast<const char*>(c->v);
  a.pages = c->table;
  a.lens = lens;
  a.B = c->B;
  a.Hq = Hq;
  a.Hk = c->Hk;
  a.d = c->d;
  a.cols = c->table_cols;
  a.n_pages = c->n_pages;
  a.page_shift = ilog2_ceil(c->page);
  const int64_t held = held_of(c);
  a.max_len = max_len > held ? (int)held : max_len;
  a.max_items = max_items < 1 ? 1 : max_items;
  TreeLaunch how = {};
  const TreeCut cut = tree_cut(c, Hq, max_len, max_items);
  how.tiles = cut.tiles;
  a.blocks = (int)cut.blocks;
  a.chunk = cut.chunk;
  a.splits = cut.splits;
  if (bias) {
    a.table = bias->table;
    a.bounds = bias->bounds;
    a.buckets = bias->n;
    a.bucket_steps = ilog2_ceil(bias->n);
    const int G = Hq / c->Hk;
    a.bias_rows = G < 16 * how.tiles ? G : 16 * how.tiles;
    how.lds = (unsigned)(a.bias_rows * (bias->n | 1) * sizeof(float));
  }
  // a launch takes fewer than 2^32 threads, and the joining one 65535 sequences: more than that go in several
  const int64_t per_seq = (int64_t)a.splits * a.Hk * cut.blocks;
  how.each = (kLaunchThreads / 512 - 8 * cut.blocks) / per_seq;
  if (how.each < 1) return DLRM_ERR_BAD_SHAPE;
  if (a.splits > 1) {
    if (how.each > 65535) how.each = 65535;
    const int64_t joins = kLaunchThreads / 256 / (((int64_t)a.max_items * Hq + 3) / 4);
    if (joins < 1) return DLRM_ERR_BAD_SHAPE;
    if (how.each > joins) how.each = joins;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < need) return DLRM_ERR_WORKSPACE;
    a.po = static_cast<float*>(workspace);
    a.pm = a.po + T * Hq * a.splits * a.d;
  }
  hipStream_t st = static_cast<hipStream_t>(stream);
  switch (c->dtype) {
    case DLRM_F32: return launch_cache_tree<DLRM_F32>(a, how, st);
    case DLRM_F16: return launch_cache_tree<DLRM_F16>(a, how, st);
    default: return launch_cache_tree<DLRM_BF16>(a, how, st);
  }
}

extern "C" size_t dlrm_cache_attn_bias_workspace_bytes(const dlrm_kv_cache* c, int32_t Hq, int32_t max_len) {
  if (check_common(c, Hq) != DLRM_OK || max_len < 1) return 0;
  return tree_workspace(c, Hq, (int64_t)c->B * Hq, max_len, 0);
}

extern "C" int32_t dlrm_cache_attn_bias(const dlrm_kv_cache* c, const int32_t* lens, int32_t max_len, const dlrm_rel_bias* bias, int32_t Hq,
                                        const dlrm_heads* q, const dlrm_heads* out, const float* slopes, float scale, float cap, void* workspace,
                                        size_t workspace_bytes, void* stream) {
  if (int st = check_common(c, Hq)) return st;
  if (max_len < 1) return DLRM_ERR_BAD_SHAPE;
  if (int st = check_rel_bias(bias)) return st;
  TreeArgs a = {};
  a.slopes = slopes;
  a.scale = scale;
  a.cap = cap;
  return run(c, lens, max_len, 0, c->B, Hq, a, q, out, bias, dlrm_cache_attn_bias_workspace_bytes(c, Hq, max_len), workspace, workspace_bytes, stream);
}

extern "C" size_t dlrm_cache_tree_attn_workspace_bytes(const dlrm_kv_cache* c, const dlrm_new_items* x, int32_t Hq, int32_t max_len) {
  int items;
  if (check_tree(c, x, Hq, max_len, items) != DLRM_OK) return 0;
  return tree_workspace(c, Hq, x->T * Hq, max_len, items);
}

extern "C" int32_t dlrm_cache_tree_attn(const dlrm_kv_cache* c, const int32_t* lens, int32_t max_len, const dlrm_new_items* x, int32_t Hq,
                                        const dlrm_heads* q, const dlrm_heads* k, const dlrm_heads* v, const dlrm_heads* out,
                                        const dlrm_rel_bias* bias, const float* slopes, float scale, float cap, void* workspace,
                                        size_t workspace_bytes, void* stream) {
  int items;
  if (int st = check_tree(c, x, Hq, max_len, items)) return st;
  if (!x->off || ((bias || slopes) && !x->positions && x->T > 0)) return DLRM_ERR_NULL;
  if (bias) {
    if (int st = check_rel_bias(bias)) return st;
  }
  const int eb = elem_bytes(c->dtype);
  for (const dlrm_heads* y : {k, v})
    if (int st = check_heads(y, x->T, c->Hk, c->d, eb)) return st;
  TreeArgs a = {};
  a.new_k = rows_of(k, x->T, c->Hk, c->d, eb);
  a.new_v = rows_of(v, x->T, c->Hk, c->d, eb);
  a.off = x->off;
  a.last = x->last;
  a.positions = x->positions;
  a.slopes = slopes;
  a.scale = scale;
  a.cap = cap;
  return run(c, lens, max_len, items, x->T, Hq, a, q, out, bias, dlrm_cache_tree_attn_workspace_bytes(c, x, Hq, max_len), workspace,
             workspace_bytes, stream);
}
