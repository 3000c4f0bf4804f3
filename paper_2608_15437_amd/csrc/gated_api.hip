// C ABI of the gated operators (norms of queries and keys with rotary
// positions, the gated delta rule): argument validation, workspace layout and
// launches.  No allocation, no host synchronisation, no state between calls.
#include <cmath>

#include "sequence_checks.hpp"

using namespace mmbev;

namespace {

// ------------------------------------------------------------ norms of heads

mmbev_status_t head_norm_ok(const mmbev_head_norm_t* t) {
  if (!t || t->rows < 0 || t->heads < 1 || t->kv_heads < 1 || !known_type(t->dtype)) return MMBEV_ERR_INVALID_ARG;
  if (t->weight_dtype != MMBEV_F32 && t->weight_dtype != t->dtype) return MMBEV_ERR_INVALID_ARG;
  if (t->rotary_dim < 2 || t->rotary_dim % 2 != 0 || t->rotary_dim > t->dim) return MMBEV_ERR_INVALID_ARG;
  if (t->layout != MMBEV_ROTARY_HALF && t->layout != MMBEV_ROTARY_INTERLEAVED) return MMBEV_ERR_INVALID_ARG;
  if (!(t->eps >= 0.0f) || !std::isfinite(t->eps)) return MMBEV_ERR_INVALID_ARG;
  if (t->rows > kMaxRows || t->heads > 1024 || t->kv_heads > 1024 || t->dim > 256) return MMBEV_ERR_UNSUPPORTED;
  return MMBEV_OK;
}

struct Positions {
  const int32_t* at;
  int64_t stride;
  int32_t axes;
  const uint64_t* steps;
  const uint8_t* axis;
};

bool positions_ok(const mmbev_head_norm_t* t, const Positions& p) {
  if (p.axes < 1 || p.axes > 8 || !aligned(p.at, 4) || !aligned(p.steps, 8)) return false;
  if (t->rows > 0 && (!p.at || !p.steps || !p.axis)) return false;
  return p.stride >= 0 && (t->rows <= 1 || p.stride >= p.axes) && p.stride < kMaxStride && reachable(t->rows, p.stride);
}

HeadNormArgs head_norm_args(const mmbev_head_norm_t* t, int32_t arrays, const Positions& p, const void* q_weight, const void* k_weight,
                            const int64_t* row_count, int32_t* fault) {
  HeadNormArgs a{};
  a.weight[0] = q_weight;
  a.weight[1] = k_weight;
  a.positions = p.at;
  a.position_stride = p.stride;
  a.axes = p.axes;
  a.steps = p.steps;
  a.axis = p.axis;
  a.row_count = row_count;
  a.fault = fault;
  a.rows = t->rows;
  a.heads[0] = t->heads;
  a.heads[1] = t->kv_heads;
  a.dim = t->dim;
  a.rotary_dim = t->rotary_dim;
  a.interleaved = t->layout == MMBEV_ROTARY_INTERLEAVED;
  a.weight_f32 = t->weight_dtype == MMBEV_F32;
  a.past = arrays * t->rows * (t->heads + t->kv_heads) * t->dim * size_of(t->dtype) > kPastCaches;
  a.eps = t->eps;
  a.inv_dim = (float)(1.0 / t->dim);
  return a;
}

// An output may be its own input's very rows and heads, and shares no element with the other arrays.
bool outputs_apart(const mmbev_head_norm_t* t, const mmbev_heads_t (&out)[2], std::initializer_list<const mmbev_heads_t*> q,
                   std::initializer_list<const mmbev_heads_t*> k) {
  const int32_t H[2] = {t->heads, t->kv_heads};
  for (int o = 0; o < 2; ++o)
    for (int i = 0; i < 2; ++i)
      for (const mmbev_heads_t* in : i ? k : q)
        if (!(o == i && same(*in, out[o])) && meet(*in, H[i], t->dim, out[o], H[o], t->dim, t->rows, t->dtype)) return false;
  return !meet(out[0], H[0], t->dim, out[1], H[1], t->dim, t->rows, t->dtype);
}

}  // namespace

extern "C" {

mmbev_status_t mmbev_head_norm_rotary(const mmbev_head_norm_t* t, mmbev_heads_t q, mmbev_heads_t k, const void* q_weight,
                                      const void* k_weight, const int32_t* positions, int64_t position_stride, int32_t axes,
                                      const uint64_t* steps, const uint8_t* axis, const int64_t* row_count, mmbev_heads_t q_out,
                                      mmbev_heads_t k_out, int32_t* fault, void* stream) {
  const mmbev_status_t st = head_norm_ok(t);
  if (st != MMBEV_OK) return st;
  const Positions p{positions, position_stride, axes, steps, axis};
  for (const mmbev_heads_t* x : {&q, &q_out})
    if (!heads_ok(*x, t->rows, t->heads, t->dim, t->dtype)) return MMBEV_ERR_INVALID_ARG;
  for (const mmbev_heads_t* x : {&k, &k_out})
    if (!heads_ok(*x, t->rows, t->kv_heads, t->dim, t->dtype)) return MMBEV_ERR_INVALID_ARG;
  if (!positions_ok(t, p) || !aligned(q_weight, size_of(t->weight_dtype)) || !aligned(k_weight, size_of(t->weight_dtype)))
    return MMBEV_ERR_INVALID_ARG;
  const mmbev_heads_t out[2] = {q_out, k_out};
  if (!outputs_apart(t, out, {&q}, {&k})) return MMBEV_ERR_INVALID_ARG;
  HeadNormArgs a = head_norm_args(t, 2, p, q_weight, k_weight, row_count, fault);
  put(q, &a.x[0], &a.x_row[0], &a.x_head[0]);
  put(k, &a.x[1], &a.x_row[1], &a.x_head[1]);
  put(q_out, &a.out[0], &a.out_row[0], &a.out_head[0]);
  put(k_out, &a.out[1], &a.out_row[1], &a.out_head[1]);
  return status_of(launch_head_norm(a, t->dtype, (hipStream_t)stream));
}

size_t mmbev_head_norm_rotary_backward_workspace_bytes(const mmbev_head_norm_t* t) {
  if (head_norm_ok(t) != MMBEV_OK) return 0;
  const HeadNormArgs a = head_norm_args(t, 3, {}, nullptr, nullptr, nullptr, nullptr);
  return align256((size_t)head_norm_backward_grid(a, t->dtype) * 2 * t->dim * 4);
}

mmbev_status_t mmbev_head_norm_rotary_backward(const mmbev_head_norm_t* t, mmbev_heads_t dq_out, mmbev_heads_t dk_out, mmbev_heads_t q,
                                               mmbev_heads_t k, const void* q_weight, const void* k_weight, const int32_t* positions,
                                               int64_t position_stride, int32_t axes, const uint64_t* steps, const uint8_t* axis,
                                               const int64_t* row_count, mmbev_heads_t dq, mmbev_heads_t dk, float* dq_weight,
                                               float* dk_weight, int32_t* fault, void* workspace, size_t workspace_bytes, void* stream) {
  const mmbev_status_t st = head_norm_ok(t);
  if (st != MMBEV_OK) return st;
  const Positions p{positions, position_stride, axes, steps, axis};
  for (const mmbev_heads_t* x : {&dq_out, &q, &dq})
    if (!heads_ok(*x, t->rows, t->heads, t->dim, t->dtype)) return MMBEV_ERR_INVALID_ARG;
  for (const mmbev_heads_t* x : {&dk_out, &k, &dk})
    if (!heads_ok(*x, t->rows, t->kv_heads, t->dim, t->dtype)) return MMBEV_ERR_INVALID_ARG;
  if (!positions_ok(t, p) || !aligned(q_weight, size_of(t->weight_dtype)) || !aligned(k_weight, size_of(t->weight_dtype)) ||
      !aligned(dq_weight, 4) || !aligned(dk_weight, 4))
    return MMBEV_ERR_INVALID_ARG;
  const mmbev_heads_t out[2] = {dq, dk};
  if (!outputs_apart(t, out, {&dq_out, &q}, {&dk_out, &k})) return MMBEV_ERR_INVALID_ARG;
  const bool sums = dq_weight || dk_weight;
  if (sums && !workspace_ok(workspace, workspace_bytes, mmbev_head_norm_rotary_backward_workspace_bytes(t))) return MMBEV_ERR_WORKSPACE;
  HeadNormArgs a = head_norm_args(t, 3, p, q_weight, k_weight, row_count, fault);
  put(q, &a.x[0], &a.x_row[0], &a.x_head[0]);
  put(k, &a.x[1], &a.x_row[1], &a.x_head[1]);
  put(dq_out, &a.dy[0], &a.dy_row[0], &a.dy_head[0]);
  put(dk_out, &a.dy[1], &a.dy_row[1], &a.dy_head[1]);
  put(dq, &a.out[0], &a.out_row[0], &a.out_head[0]);
  put(dk, &a.out[1], &a.out_row[1], &a.out_head[1]);
  a.partial = sums ? (float*)workspace : nullptr;
  a.dweight[0] = dq_weight;
  a.dweight[1] = dk_weight;
  return status_of(launch_head_norm_backward(a, t->dtype, (hipStream_t)stream));
}

}  // extern "C"
