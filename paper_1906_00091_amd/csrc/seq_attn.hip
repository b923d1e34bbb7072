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

static int check_bias(const dlrm_rel_bias* b, const dlrm_seq_batch* s, int Hq, int Hk) {
  if (int st = check_rel_bias(b)) return st;
  // (wavefronts hold 32 items of one head: the last ones of every head may be empty)
  if ((int64_t)(s->max_q + 31) * (Hq / Hk) > kMostRows) return DLRM_ERR_BAD_SHAPE;
  // (products start from bias / scale, which has to be a number)
  if (s->scale < 0x1p-64f || s->scale > 0x1p64f) return DLRM_ERR_BAD_SHAPE;
  return DLRM_OK;
}

static void set_bias(SeqArgs& a, const dlrm_rel_bias* b) {
  a.table = b->table;
  a.bounds = b->bounds;
  a.buckets = b->n;
  a.bucket_steps = ilog2_ceil(b->n);
}

template <bool BIAS>
static int seq_fwd(const dlrm_seq_batch* batch, const dlrm_rel_bias* bias, int Hq, int Hk, int d, int dtype, const dlrm_heads* q, const dlrm_heads* k,
                   const dlrm_heads* v, const dlrm_heads* out, float* lse, void* stream) {
  dlrm_seq_batch seq;
  if (int st = check_seq(batch, Hq, Hk, d, dtype, seq)) return st;
  const dlrm_seq_batch* s = &seq;
  if constexpr (BIAS) {
    if (int st = check_bias(bias, s, Hq, Hk)) return st;
  }
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
  if constexpr (BIAS) set_bias(a, bias);
  hipStream_t hs = static_cast<hipStream_t>(stream);
  switch (dtype) {
    case DLRM_F32: return launch_seq_fwd<DLRM_F32, BIAS>(s, a, hs);
    case DLRM_F16: return launch_seq_fwd<DLRM_F16, BIAS>(s, a, hs);
    default: return launch_seq_fwd<DLRM_BF16, BIAS>(s, a, hs);
  }
}

extern "C" int32_t dlrm_seq_attn_fwd(const dlrm_seq_batch* batch, int32_t Hq, int32_t Hk, int32_t d, int32_t dtype, const dlrm_heads* q,
                                     const dlrm_heads* k, const dlrm_heads* v, const dlrm_heads* out, float* lse, void* stream) {
  return seq_fwd<false>(batch, nullptr, Hq, Hk, d, dtype, q, k, v, out, lse, stream);
}

extern "C" int32_t dlrm_seq_attn_bias_fwd(const dlrm_seq_batch* batch, const dlrm_rel_bias* bias, int32_t Hq, int32_t Hk, int32_t d, int32_t dtype,
                                          const dlrm_heads* q, const dlrm_heads* k, const dlrm_heads* v, const dlrm_heads* out, float* lse,
                                          void* stream) {
  return seq_fwd<true>(batch, bias, Hq, Hk, d, dtype, q, k, v, out, lse, stream);
}

// What a backward pass keeps in its workspace, in this order.
struct BwdSpace {
  size_t delta, sums, parts, chunks;  // bytes: delta; the keys' gradients of workgroups that share a block; the bias's sums, and those of them joined once
  int64_t n_parts, n_chunks;
  size_t all() const {
    const size_t n = delta + sums + parts + chunks;
    return n < 256 ? 256 : n;
  }
};
static size_t in_lines(size_t n) { return (n + 255) / 256 * 256; }
static BwdSpace bwd_space(const dlrm_seq_batch* s, const dlrm_rel_bias* bias, int Hq, int Hk, int d, int dtype) {
  const int splits = dkv_splits(s, Hq, Hk, d, dtype);
  BwdSpace w = {};
  w.delta = in_lines((size_t)Hq * s->Tq * sizeof(float));
  w.sums = splits > 1 ? in_lines((size_t)splits * 2 * s->Tk * Hk * d * sizeof(float)) : 0;
  if (bias) {
    w.n_parts = bias_parts(s, Hk, d, dtype, splits);
    w.n_chunks = bias_chunks(w.n_parts);
    w.parts = in_lines((size_t)Hq * w.n_parts * bias->n * sizeof(float));
    w.chunks = w.n_chunks > 1 ? in_lines((size_t)Hq * w.n_chunks * bias->n * sizeof(float)) : 0;
  }
  return w;
}

extern "C" size_t dlrm_seq_attn_bwd_workspace_bytes(const dlrm_seq_batch* batch, int32_t Hq, int32_t Hk, int32_t d, int32_t dtype) {
  dlrm_seq_batch seq;
  if (check_seq(batch, Hq, Hk, d, dtype, seq) != DLRM_OK) return 0;
  return bwd_space(&seq, nullptr, Hq, Hk, d, dtype).all();
}

extern "C" size_t dlrm_seq_attn_bias_bwd_workspace_bytes(const dlrm_seq_batch* batch, const dlrm_rel_bias* bias, int32_t Hq, int32_t Hk, int32_t d,
                                                         int32_t dtype) {
  dlrm_seq_batch seq;
  if (check_seq(batch, Hq, Hk, d, dtype, seq) != DLRM_OK || check_bias(bias, &seq, Hq, Hk) != DLRM_OK) return 0;
  return bwd_space(&seq, bias, Hq, Hk, d, dtype).all();
}

// The sums of the bias's score gradients: of `parts` rows of n for each head (blockIdx.y) a workgroup adds up `per`, each strip of threads every STRIPS-th in
// their order, then strip by strip.
__global__ __launch_bounds__(256) void seq_attn_bias_join_kernel(const float* part, int64_t parts, int64_t per, int n, int n_pow2, float* to) {
  __shared__ float sums[256];
  const int strips = 256 / n_pow2, strip = threadIdx.x / n_pow2, b = threadIdx.x % n_pow2;
  const int64_t first = (int64_t)blockIdx.x * per, end = first + per < parts ? first + per : parts;
  const float* at = part + (int64_t)blockIdx.y * parts * n + b;
  float sum = 0.0f;
  if (b < n) {
#pragma unroll 8
    for (int64_t p = first + strip; p < end; p += strips) sum += at[p * n];
  }
  sums[threadIdx.x] = sum;
  __syncthreads();
  if (strip > 0 || b >= n) return;
  for (int i = 1; i < strips; ++i) sum += sums[i * n_pow2 + b];
  to[((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * n + b] = sum;
}

static int join_bias(const BwdSpace& w, const float* parts, float* chunks, int Hq, int n, float* dtable, hipStream_t st) {
  const int p2 = pow2_ceil(n);
  const int64_t per = (w.n_parts + w.n_chunks - 1) / w.n_chunks;
  const bool twice = w.n_chunks > 1;
  hipLaunchKernelGGL(seq_attn_bias_join_kernel, dim3((unsigned)w.n_chunks, Hq), dim3(256), 0, st, parts, w.n_parts, per, n, p2, twice ? chunks : dtable);
  DLRM_CHECK_LAUNCH();
  if (!twice) return DLRM_OK;
  hipLaunchKernelGGL(seq_attn_bias_join_kernel, dim3(1, Hq), dim3(256), 0, st, (const float*)chunks, w.n_chunks, w.n_chunks, n, p2, dtable);
  DLRM_CHECK_LAUNCH();
  return DLRM_OK;
}

template <bool BIAS>
static int seq_bwd(const dlrm_seq_batch* batch, const dlrm_rel_bias* bias, int Hq, int Hk, int d, int dtype, const dlrm_heads* q, const dlrm_heads* k,
                   const dlrm_heads* v, const dlrm_heads* out, const float* lse, const dlrm_heads* dout, const dlrm_heads* dq, const dlrm_heads* dk,
                   const dlrm_heads* dv, float* dtable, void* workspace, size_t workspace_bytes, void* stream) {
  dlrm_seq_batch seq;
  if (int st = check_seq(batch, Hq, Hk, d, dtype, seq)) return st;
  const dlrm_seq_batch* s = &seq;
  if constexpr (BIAS) {
    if (int st = check_bias(bias, s, Hq, Hk)) return st;
    if (!dtable) return DLRM_ERR_NULL;
  }
  const int eb = elem_bytes(dtype);
  for (const dlrm_heads* x : {q, out, dout, dq})
    if (int st = check_heads(x, s->Tq, Hq, d, eb)) return st;
  for (const dlrm_heads* x : {k, v, dk, dv})
    if (int st = check_heads(x, s->Tk, Hk, d, eb)) return st;
  if (!lse && s->Tq > 0) return DLRM_ERR_NULL;
  const BwdSpace w = bwd_space(s, BIAS ? bias : nullptr, Hq, Hk, d, dtype);
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < w.all()) return DLRM_ERR_WORKSPACE;
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
  char* at = static_cast<char*>(workspace);
  a.delta = reinterpret_cast<float*>(at);
  a.part = reinterpret_cast<float*>(at + w.delta);
  a.bias_part = reinterpret_cast<float*>(at + w.delta + w.sums);
  a.bias_parts = w.n_parts;
  if constexpr (BIAS) set_bias(a, bias);
  hipStream_t hs = static_cast<hipStream_t>(stream);
  int rc;
  switch (dtype) {
    case DLRM_F32: rc = launch_seq_bwd<DLRM_F32, BIAS>(s, a, hs); break;
    case DLRM_F16: rc = launch_seq_bwd<DLRM_F16, BIAS>(s, a, hs); break;
    default: rc = launch_seq_bwd<DLRM_BF16, BIAS>(s, a, hs);
  }
  if constexpr (BIAS) {
    if (rc == DLRM_OK) rc = join_bias(w, a.bias_part, reinterpret_cast<float*>(at + w.delta + w.sums + w.parts), Hq, bias->n, dtable, hs);
  }
  return rc;
}

extern "C" int32_t dlrm_seq_attn_bwd(const dlrm_seq_batch* batch, int32_t Hq, int32_t Hk, int32_t d, int32_t dtype, const dlrm_heads* q,
                                     const dlrm_heads* k, const dlrm_heads* v, const dlrm_heads* out, const float* lse,
                                     const dlrm_heads* dout, const dlrm_heads* dq, const dlrm_heads* dk, const dlrm_heads* dv,
                                     void* workspace, size_t workspace_bytes, void* stream) {
  return seq_bwd<false>(batch, nullptr, Hq, Hk, d, dtype, q, k, v, out, lse, dout, dq, dk, dv, nullptr, workspace, workspace_bytes, stream);
}

extern "C" int32_t dlrm_seq_attn_bias_bwd(const dlrm_seq_batch* batch, const dlrm_rel_bias* bias, int32_t Hq, int32_t Hk, int32_t d, int32_t dtype,
                                          const dlrm_heads* q, const dlrm_heads* k, const dlrm_heads* v, const dlrm_heads* out, const float* lse,
                                          const dlrm_heads* dout, const dlrm_heads* dq, const dlrm_heads* dk, const dlrm_heads* dv, float* dtable,
                                          void* workspace, size_t workspace_bytes, void* stream) {
  return seq_bwd<true>(batch, bias, Hq, Hk, d, dtype, q, k, v, out, lse, dout, dq, dk, dv, dtable, workspace, workspace_bytes, stream);
}
