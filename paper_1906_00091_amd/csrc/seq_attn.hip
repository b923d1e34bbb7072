// Attention over sequences: entry points and argument checks (the kernels: seq_attn.h).
#include "seq_attn.h"

#include <math.h>

#include <initializer_list>

using namespace dlrm;

// A sequence's items are counted in 32 bits, with room for a tile past its end; a row of the forward is one of an item's heads.
constexpr int64_t kMostRows = 0x7fffffff - 1024;

// Checks the arguments; `seq` becomes the caller's batch with bounds no looser than the totals.
static int check_seq(const dlrm_seq_batch* given, int Hq, int Hk, int d, int dtype, dlrm_seq_batch& seq) {
  if (!given) return DLRM_ERR_NULL;
  seq = *given;
  dlrm_seq_batch* s = &seq;
  if (int st = check_head_shape(Hq, Hk, d, dtype)) return st;
  if (s->B < 1 || s->B == 0x7fffffff || s->Tq < 0 || s->Tk < 0 || s->Tq > DLRM_MAX_ITEMS || s->Tk > DLRM_MAX_ITEMS) return DLRM_ERR_BAD_SHAPE;
  if (s->max_q < 0 || s->max_k < 0 || (s->Tq > 0 && s->max_q == 0) || (s->Tk > 0 && s->max_k == 0)) return DLRM_ERR_BAD_SHAPE;
  if (!s->q_off || !s->k_off) return DLRM_ERR_NULL;
  if ((s->causal != 0 && s->causal != 1) || (s->prefix && !s->causal)) return DLRM_ERR_BAD_SHAPE;
  if (!(s->scale > 0.0f) || !isfinite(s->scale) || !(s->cap >= 0.0f) || !isfinite(s->cap)) return DLRM_ERR_BAD_SHAPE;
  if (s->max_q > s->Tq) s->max_q = (int32_t)s->Tq;
  if (s->max_k > s->Tk) s->max_k = (int32_t)s->Tk;
  if ((int64_t)s->max_q * (Hq / Hk) > kMostRows || s->max_k > kMostRows) return DLRM_ERR_BAD_SHAPE;
  return DLRM_OK;
}

static SeqArgs seq_args(const dlrm_seq_batch* s, int Hq, int Hk, int d) {
  SeqArgs a = {};
  a.q_off = s->q_off;
  a.k_off = s->k_off;
  a.prefix = s->prefix;
  a.slopes = s->slopes;
  a.Tq = s->Tq;
  a.Tk = s->Tk;
  a.splits = 1;
  a.B = s->B;
  a.Hq = Hq;
  a.Hk = Hk;
  a.d = d;
  a.causal = s->causal;
  a.scale = s->scale;
  a.cap = s->cap;
  return a;
}

extern "C" int32_t dlrm_seq_attn_fwd(const dlrm_seq_batch* batch, int32_t Hq, int32_t Hk, int32_t d, int32_t dtype, const dlrm_heads* q,
                                     const dlrm_heads* k, const dlrm_heads* v, const dlrm_heads* out, float* lse, void* stream) {
  dlrm_seq_batch seq;
  if (int st = check_seq(batch, Hq, Hk, d, dtype, seq)) return st;
  const dlrm_seq_batch* s = &seq;
  const int eb = elem_bytes(dtype);
  for (const dlrm_heads* x : {q, out})
    if (int st = check_heads(x, s->Tq, Hq, d, eb)) return st;
  for (const dlrm_heads* x : {k, v})
    if (int st = check_heads(x, s->Tk, Hk, d, eb)) return st;
  SeqArgs a = seq_args(s, Hq, Hk, d);
  a.q = rows_of(q, s->Tq, Hq, d, eb);
  a.k = rows_of(k, s->Tk, Hk, d, eb);
  a.v = rows_of(v, s->Tk, Hk, d, eb);
  a.out = rows_of(out, s->Tq, Hq, d, eb);
  a.lse = lse;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  switch (dtype) {
    case DLRM_F32: return launch_seq_fwd<DLRM_F32>(s, a, hs);
    case DLRM_F16: return launch_seq_fwd<DLRM_F16>(s, a, hs);
    default: return launch_seq_fwd<DLRM_BF16>(s, a, hs);
  }
}

static size_t delta_bytes(const dlrm_seq_batch* s, int Hq) { return ((size_t)Hq * s->Tq * sizeof(float) + 255) / 256 * 256; }

extern "C" size_t dlrm_seq_attn_bwd_workspace_bytes(const dlrm_seq_batch* batch, int32_t Hq, int32_t Hk, int32_t d, int32_t dtype) {
  dlrm_seq_batch seq;
  if (check_seq(batch, Hq, Hk, d, dtype, seq) != DLRM_OK) return 0;
  const dlrm_seq_batch* s = &seq;
  const int splits = dkv_splits(s, Hq, Hk, d, dtype);
  const size_t sums = splits > 1 ? (size_t)splits * 2 * s->Tk * Hk * d * sizeof(float) : 0;
  const size_t n = delta_bytes(s, Hq) + (sums + 255) / 256 * 256;
  return n < 256 ? 256 : n;
}

extern "C" int32_t dlrm_seq_attn_bwd(const dlrm_seq_batch* batch, int32_t Hq, int32_t Hk, int32_t d, int32_t dtype, const dlrm_heads* q,
                                     const dlrm_heads* k, const dlrm_heads* v, const dlrm_heads* out, const float* lse,
                                     const dlrm_heads* dout, const dlrm_heads* dq, const dlrm_heads* dk, const dlrm_heads* dv,
                                     void* workspace, size_t workspace_bytes, void* stream) {
  dlrm_seq_batch seq;
  if (int st = check_seq(batch, Hq, Hk, d, dtype, seq)) return st;
  const dlrm_seq_batch* s = &seq;
  const int eb = elem_bytes(dtype);
  for (const dlrm_heads* x : {q, out, dout, dq})
    if (int st = check_heads(x, s->Tq, Hq, d, eb)) return st;
  for (const dlrm_heads* x : {k, v, dk, dv})
    if (int st = check_heads(x, s->Tk, Hk, d, eb)) return st;
  if (!lse && s->Tq > 0) return DLRM_ERR_NULL;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) ||
      workspace_bytes < dlrm_seq_attn_bwd_workspace_bytes(batch, Hq, Hk, d, dtype))
    return DLRM_ERR_WORKSPACE;
  SeqArgs a = seq_args(s, Hq, Hk, d);
  a.q = rows_of(q, s->Tq, Hq, d, eb);
  a.k = rows_of(k, s->Tk, Hk, d, eb);
  a.v = rows_of(v, s->Tk, Hk, d, eb);
  a.out = rows_of(out, s->Tq, Hq, d, eb);
  a.dout = rows_of(dout, s->Tq, Hq, d, eb);
  a.dq = rows_of(dq, s->Tq, Hq, d, eb);
  a.dk = rows_of(dk, s->Tk, Hk, d, eb);
  a.dv = rows_of(dv, s->Tk, Hk, d, eb);
  a.lse = const_cast<float*>(lse);
  a.delta = static_cast<float*>(workspace);
  a.part = a.delta + delta_bytes(s, Hq) / sizeof(float);
  hipStream_t hs = static_cast<hipStream_t>(stream);
  switch (dtype) {
    case DLRM_F32: return launch_seq_bwd<DLRM_F32>(s, a, hs);
    case DLRM_F16: return launch_seq_bwd<DLRM_F16>(s, a, hs);
    default: return launch_seq_bwd<DLRM_BF16>(s, a, hs);
  }
}
