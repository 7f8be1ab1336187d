// C ABI of the operators beside the layers: argument validation and launches. Host code only.
#include <math.h>
#include <string.h>

#include <algorithm>
#include <new>
#include <vector>

#include "entry.h"
#include "kernels.h"

using namespace slapo;

namespace {

inline int64_t element_bytes(int dtype) { return dtype == SLAPO_FP32 ? 4 : 2; }

// ---- cross attention ------------------------------------------------------------------------------------
int check_cross(const slapo_cross_attn_desc* d) {
  if (!d) return SLAPO_ERR_NULL;
  if (!known_dtype(d->dtype)) return SLAPO_ERR_UNSUPPORTED;
  if (d->batch <= 0 || d->q_len <= 0 || d->kv_len <= 0 || d->heads <= 0 || d->kv_heads <= 0) return SLAPO_ERR_SHAPE;
  if (d->heads % d->kv_heads != 0) return SLAPO_ERR_SHAPE;
  if (d->head_dim != 64 && d->head_dim != 128) return SLAPO_ERR_UNSUPPORTED;
  if (!(d->scale >= 0.f) || !(d->scale < INFINITY)) return SLAPO_ERR_SHAPE;
  if (d->batch > 65535 || d->heads > 65535) return SLAPO_ERR_UNSUPPORTED;   // (launch dimensions)
  const int64_t width = (int64_t)d->heads * d->head_dim, kv_width = (int64_t)d->kv_heads * d->head_dim;
  const struct { int64_t stride, width, tokens; } arrays[] = {{d->q_stride, width, d->q_len}, {d->kv_stride, kv_width, d->kv_len}, {d->out_stride, width, d->q_len}};
  for (const auto& a : arrays) {
    if (a.stride != 0 && a.stride < a.width) return SLAPO_ERR_SHAPE;
    if (a.stride % 8 != 0) return SLAPO_ERR_ALIGN;
    // a sample's offsets are 32-bit, also those of the rows of a last tile that reach beyond it
    if ((a.stride > a.width ? a.stride : a.width) * element_bytes(d->dtype) * (a.tokens + 256) >= ((int64_t)1 << 31)) return SLAPO_ERR_UNSUPPORTED;
  }
  // (launch dimensions: blocks of 16 fp32 rows in one; blocks of 64 rows of all heads, and 1024 threads for each head, in one)
  const int64_t rows = (int64_t)d->q_len * (d->heads / d->kv_heads);
  if (rows >= ((int64_t)1 << 26)) return SLAPO_ERR_UNSUPPORTED;
  if ((int64_t)d->batch * d->kv_heads >= ((int64_t)1 << 21)) return SLAPO_ERR_UNSUPPORTED;
  if ((int64_t)d->batch * d->kv_heads * ((std::max(rows, (int64_t)d->kv_len) + 63) / 64) >= ((int64_t)1 << 23)) return SLAPO_ERR_UNSUPPORTED;
  return SLAPO_OK;
}

CrossShape cross_shape(const slapo_cross_attn_desc* d) {
  CrossShape s;
  s.batch = d->batch; s.q_len = d->q_len; s.kv_len = d->kv_len; s.heads = d->heads; s.kv_heads = d->kv_heads;
  s.group = d->heads / d->kv_heads;
  s.scale = d->scale > 0.f ? d->scale : 1.f / sqrtf((float)d->head_dim);
  const int64_t width = (int64_t)d->heads * d->head_dim;
  s.q_stride = d->q_stride ? d->q_stride : width;
  s.out_stride = d->out_stride ? d->out_stride : width;
  s.kv_stride = d->kv_stride ? d->kv_stride : (int64_t)d->kv_heads * d->head_dim;
  // division by an invariant: with 2^(l-1) < group <= 2^l and m = floor(2^32 (2^l - group) / group) + 1, r / group is
  // (floor(r m / 2^32) + r) >> l; the sum stays below 2^32 for r < 2^31
  int l = 0;
  while (((int64_t)1 << l) < s.group) ++l;
  s.div_mul = (uint32_t)(((((uint64_t)1 << l) - s.group) << 32) / s.group + 1);
  s.div_shift = (uint32_t)l;
  return s;
}

// ---- rotary positions of several axes -------------------------------------------------------------------
int check_rope_axes(const slapo_rope_axes_desc* d) {
  if (!d) return SLAPO_ERR_NULL;
  if (!known_dtype(d->dtype)) return SLAPO_ERR_UNSUPPORTED;
  if (d->ladder != SLAPO_ROPE_SHARED && d->ladder != SLAPO_ROPE_PER_AXIS) return SLAPO_ERR_UNSUPPORTED;
  if (d->rows <= 0 || d->heads <= 0 || d->head_dim <= 0 || d->axes <= 0) return SLAPO_ERR_SHAPE;
  if (d->axes > ROPE_MAX_AXES || d->head_dim > 2 * ROPE_MAX_PAIRS || d->heads > (1 << 20)) return SLAPO_ERR_UNSUPPORTED;
  if (d->rows >= ((int64_t)1 << 31)) return SLAPO_ERR_UNSUPPORTED;
  if (d->head_dim % 8 != 0 || d->in_stride % 8 != 0 || d->out_stride % 8 != 0) return SLAPO_ERR_ALIGN;
  int64_t pairs = 0;
  for (int a = 0; a < d->axes; ++a) {
    if (d->pairs[a] < 0) return SLAPO_ERR_SHAPE;
    pairs += d->pairs[a];
  }
  if (pairs > d->head_dim / 2) return SLAPO_ERR_SHAPE;
  if (!(d->base > 1.f) || !(d->base < INFINITY)) return SLAPO_ERR_SHAPE;
  const int64_t width = (int64_t)d->heads * d->head_dim;
  if ((d->in_stride != 0 && d->in_stride < width) || (d->out_stride != 0 && d->out_stride < width)) return SLAPO_ERR_SHAPE;
  if (std::max(d->in_stride, width) >= ((int64_t)1 << 28) || std::max(d->out_stride, width) >= ((int64_t)1 << 28))   // (byte counts below fit 64 bits)
    return SLAPO_ERR_UNSUPPORTED;
  return SLAPO_OK;
}

// ---- gradient norm ----------------------------------------------------------------------------------------
inline int64_t grad_segments(const slapo_grad& g) {
  const int64_t per = GRAD_SEGMENT / element_bytes(g.dtype);
  return (g.count + per - 1) / per;
}
// Checks the arrays and counts their segments.
int check_grads(int32_t n, const slapo_grad* grads, bool pointers, int64_t* segments) {
  if (n < 0) return SLAPO_ERR_SHAPE;
  if (n > 0 && !grads) return SLAPO_ERR_NULL;
  *segments = 0;
  for (int i = 0; i < n; ++i) {
    const slapo_grad& g = grads[i];
    if (!known_dtype(g.dtype)) return SLAPO_ERR_UNSUPPORTED;
    if (g.count < 0) return SLAPO_ERR_SHAPE;
    if (g.count >= ((int64_t)1 << 40)) return SLAPO_ERR_UNSUPPORTED;
    *segments += grad_segments(g);
    if (*segments >= ((int64_t)1 << 31)) return SLAPO_ERR_UNSUPPORTED;
    if (!pointers || g.count == 0) continue;
    if (!g.grad) return SLAPO_ERR_NULL;
    if (misaligned(g.grad) || misaligned(g.out)) return SLAPO_ERR_ALIGN;
  }
  return SLAPO_OK;
}
// Outputs share memory with nothing but the gradient that they scale: everything is written once, and nobody else reads it meanwhile.
int check_shared_memory(int32_t n, const slapo_grad* grads) {
  struct Span { uintptr_t from, to; int of; bool written; };
  std::vector<Span> spans;
  spans.reserve(2 * (size_t)n);
  for (int i = 0; i < n; ++i) {
    const slapo_grad& g = grads[i];
    const uintptr_t b = (uintptr_t)(g.count * element_bytes(g.dtype)), in = (uintptr_t)g.grad, out = (uintptr_t)g.out;
    if (b == 0) continue;
    const bool in_place = !g.out || out == in;
    spans.push_back({in, in + b, i, in_place});
    if (!in_place) spans.push_back({out, out + b, i, true});
  }
  std::sort(spans.begin(), spans.end(), [](const Span& a, const Span& b) { return a.from < b.from; });
  uintptr_t any = 0, written = 0;   // how far the spans so far reach
  for (const Span& s : spans) {
    if (s.from < written || (s.written && s.from < any)) return SLAPO_ERR_SHAPE;
    any = std::max(any, s.to);
    if (s.written) written = std::max(written, s.to);
  }
  return SLAPO_OK;
}
int check_plan(const slapo_grad_plan* p) {
  if (!p || !p->memory) return SLAPO_ERR_NULL;
  if (p->segments < 0 || p->segments >= ((int64_t)1 << 31)) return SLAPO_ERR_SHAPE;
  return SLAPO_OK;
}

}  // namespace

extern "C" {

int slapo_cross_attn_workspace(const slapo_cross_attn_desc* d, size_t* fwd_bytes, size_t* bwd_bytes) {
  if (!fwd_bytes || !bwd_bytes) return SLAPO_ERR_NULL;
  const int rc = check_cross(d);
  if (rc) return rc;
  const CrossShape s = cross_shape(d);
  *fwd_bytes = cross_attn_fwd_ws_bytes(d->dtype, d->head_dim, s);
  *bwd_bytes = cross_attn_bwd_ws_bytes(d->dtype, d->head_dim, s);
  return SLAPO_OK;
}

int slapo_cross_attn_fwd(const slapo_cross_attn_desc* d, const void* q, const void* k, const void* v, const int32_t* kv_lens, void* out,
                         float* lse, void* ws, size_t ws_bytes, void* stream) {
  const int rc = check_cross(d);
  if (rc) return rc;
  if (!q || !k || !v || !out) return SLAPO_ERR_NULL;
  const CrossShape s = cross_shape(d);
  const size_t need = cross_attn_fwd_ws_bytes(d->dtype, d->head_dim, s);
  if (!ws && need) return SLAPO_ERR_NULL;
  if (misaligned(q) || misaligned(k) || misaligned(v) || misaligned(out) || misaligned(ws)) return SLAPO_ERR_ALIGN;
  if (ws_bytes < need) return SLAPO_ERR_WORKSPACE;
  CrossOperands p = {};
  p.q = q; p.k = k; p.v = v; p.lens = kv_lens; p.o = out; p.lse = lse; p.ws = (float*)ws;
  entry_error();
  launch_cross_attn_fwd(d->dtype, d->head_dim, s, p, (hipStream_t)stream);
  return finish();
}

int slapo_cross_attn_bwd(const slapo_cross_attn_desc* d, const void* q, const void* k, const void* v, const int32_t* kv_lens, const void* out,
                         const void* dout, const float* lse, void* dq, void* dk, void* dv, void* ws, size_t ws_bytes, void* stream) {
  const int rc = check_cross(d);
  if (rc) return rc;
  if (!q || !k || !v || !out || !dout || !lse || !dq || !dk || !dv || !ws) return SLAPO_ERR_NULL;
  for (const void* a : {q, k, v, out, dout, (const void*)dq, (const void*)dk, (const void*)dv, (const void*)ws})
    if (misaligned(a)) return SLAPO_ERR_ALIGN;
  const CrossShape s = cross_shape(d);
  if (ws_bytes < cross_attn_bwd_ws_bytes(d->dtype, d->head_dim, s)) return SLAPO_ERR_WORKSPACE;
  CrossOperands p = {};
  p.q = q; p.k = k; p.v = v; p.lens = kv_lens; p.out = out; p.dout = dout; p.lse = const_cast<float*>(lse); p.dq = dq; p.dk = dk; p.dv = dv; p.ws = (float*)ws;
  entry_error();
  launch_cross_attn_bwd(d->dtype, d->head_dim, s, p, (hipStream_t)stream);
  return finish();
}

int slapo_rope_axes(const slapo_rope_axes_desc* d, const int32_t* positions, const void* in, void* out, int inverse, void* stream) {
  const int rc = check_rope_axes(d);
  if (rc) return rc;
  if (!positions || !in || !out) return SLAPO_ERR_NULL;
  if (misaligned(in) || misaligned(out)) return SLAPO_ERR_ALIGN;
  RopeAxes r;
  const int64_t width = (int64_t)d->heads * d->head_dim, eb = element_bytes(d->dtype);
  r.rows = d->rows; r.heads = d->heads; r.head_dim = d->head_dim; r.axes = d->axes;
  r.in_stride = d->in_stride ? d->in_stride : width;
  r.out_stride = d->out_stride ? d->out_stride : width;
  // in place every row is read and written by the same block; anything else that shares memory would be read after it is written
  if ((in != out || r.in_stride != r.out_stride) &&
      overlap(in, (size_t)(((r.rows - 1) * r.in_stride + width) * eb), out, (size_t)(((r.rows - 1) * r.out_stride + width) * eb))) return SLAPO_ERR_SHAPE;
  r.first[0] = 0;
  for (int a = 0; a < ROPE_MAX_AXES; ++a) r.first[a + 1] = r.first[a] + (a < d->axes ? d->pairs[a] : 0);
  r.turned = r.first[d->axes];
  r.own_ladders = d->ladder == SLAPO_ROPE_PER_AXIS;
  r.inverse = inverse ? 1 : 0;
  r.log2_base = log2((double)d->base);
  entry_error();
  launch_rope_axes(d->dtype, r, positions, in, out, (hipStream_t)stream);
  return finish();
}

int slapo_grad_plan_bytes(int32_t n, const slapo_grad* grads, size_t* bytes) {
  if (!bytes) return SLAPO_ERR_NULL;
  int64_t segments;
  const int rc = check_grads(n, grads, false, &segments);
  if (rc) return rc;
  *bytes = grad_plan_layout(segments).total;
  return SLAPO_OK;
}

int slapo_grad_plan_build(int32_t n, const slapo_grad* grads, void* memory, slapo_grad_plan* plan, void* stream) {
  int64_t segments;
  int rc = check_grads(n, grads, true, &segments);
  if (rc) return rc;
  if (!memory || !plan) return SLAPO_ERR_NULL;
  if (misaligned(memory)) return SLAPO_ERR_ALIGN;
  try {
    if ((rc = check_shared_memory(n, grads))) return rc;
    std::vector<GradArray> arrays((size_t)n);
    int64_t first = 0;
    for (int i = 0; i < n; ++i) {
      arrays[i] = {grads[i].grad, grads[i].out ? grads[i].out : const_cast<void*>(grads[i].grad), grads[i].count, first, grads[i].dtype};
      first += grad_segments(grads[i]);
    }
    *plan = {memory, segments};
    entry_error();
    launch_grad_plan(n, arrays.data(), memory, (hipStream_t)stream);
  } catch (const std::bad_alloc&) {   // (host memory for a table of the arrays)
    return SLAPO_ERR_WORKSPACE;
  }
  return finish();
}

int slapo_grad_sumsq(const slapo_grad_plan* plan, int accumulate, double* sumsq, void* stream) {
  const int rc = check_plan(plan);
  if (rc) return rc;
  if (!sumsq) return SLAPO_ERR_NULL;
  if ((reinterpret_cast<uintptr_t>(sumsq) & 7u) != 0) return SLAPO_ERR_ALIGN;
  entry_error();
  launch_grad_sumsq(plan->segments, plan->memory, accumulate ? 1 : 0, sumsq, (hipStream_t)stream);
  return finish();
}

int slapo_grad_clip(const slapo_grad_plan* plan, const double* sumsq, float max_norm, float* norm, void* stream) {
  const int rc = check_plan(plan);
  if (rc) return rc;
  if (!sumsq) return SLAPO_ERR_NULL;
  if (!(max_norm > 0.f)) return SLAPO_ERR_SHAPE;
  if ((reinterpret_cast<uintptr_t>(sumsq) & 7u) != 0 || (reinterpret_cast<uintptr_t>(norm) & 3u) != 0) return SLAPO_ERR_ALIGN;
  entry_error();
  launch_grad_clip(plan->segments, plan->memory, sumsq, max_norm, norm, (hipStream_t)stream);
  return finish();
}

}  // extern "C"
