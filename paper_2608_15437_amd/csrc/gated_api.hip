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

HeadNormArgs head_norm_args(const mmbev_head_norm_t* t, const Positions& p, const void* q_weight, const void* k_weight,
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

// ------------------------------------------------------------ gated delta rule

// A sequence and head is a workgroup's work; long sequences are cut so that the workgroups fill the chip's compute units,
// in parts of at least kDeltaLeast rows, and none where none can be longer than kDeltaWhole, among more sequences than a
// workgroup can look through in passing, or where the heads alone come to so many that there are under kDeltaLeastCuts
// shares (then a single sequence has a workgroup a head, of fp32 heads over 64 from 86 on, be that fewer than there are units).
constexpr int64_t kComputeUnits = 256;
constexpr int64_t kDeltaWhole = 512;
constexpr int32_t kDeltaLeast = 128;
constexpr int32_t kDeltaCutSequences = 1024;

struct DeltaPlan {
  int32_t cuts, run;
  // (cut_kind lies first)
  size_t off_from[2], off_state, off_map, off_run[2], off_end[2], off_grad, off_turned, off_before, off_after, off_left, off_due, total;
};

mmbev_status_t delta_ok(const mmbev_attention_t* t, bool step) {
  if (!t || t->rows < 0 || t->reserved != 0 || !known_type(t->dtype)) return MMBEV_ERR_INVALID_ARG;
  if (t->heads < 1 || t->kv_heads < 1 || t->heads % t->kv_heads != 0) return MMBEV_ERR_INVALID_ARG;
  if (t->key_dim < 1 || t->value_dim < 1) return MMBEV_ERR_INVALID_ARG;
  if (!std::isfinite(t->scale) || t->scale == 0.0f) return MMBEV_ERR_INVALID_ARG;
  if (!step && (t->num_sequences < 1 || t->num_sequences > 65535 || t->max_length < 0)) return MMBEV_ERR_INVALID_ARG;
  if (t->rows > kMaxRows || t->heads > 256 || t->key_dim > 128 || t->value_dim > 128) return MMBEV_ERR_UNSUPPORTED;
  // a workgroup each, and the parts of cut sequences
  if ((step ? t->rows : (int64_t)t->num_sequences + 1024) * t->heads > kMostGroups) return MMBEV_ERR_UNSUPPORTED;
  return MMBEV_OK;
}

DeltaPlan delta_plan(const mmbev_attention_t* t, bool backward) {
  DeltaPlan p{};
  // workgroups that the chip takes at once
  const int64_t slots = kComputeUnits * delta_groups(t->dtype == MMBEV_F16, size_of(t->dtype), t->key_dim, t->value_dim);
  const int64_t longest = t->max_length > 0 ? std::min(t->max_length, t->rows) : t->rows;
  if (longest > kDeltaWhole && t->num_sequences <= kDeltaCutSequences) {
    // so many parts that with the sequences that are not cut there are about `units` of them: at least half the units
    const int64_t units = std::max<int64_t>(2, slots / t->heads);
    const int64_t parts = units - std::min<int64_t>(t->num_sequences, units / 2);
    p.cuts = (int32_t)std::max<int64_t>(1, std::min(parts, (t->rows + kDeltaLeast - 1) / kDeltaLeast));
  }
  // steps one after the other: a run's boundaries and the runs
  p.run = 1;
  while (p.run * p.run < p.cuts) ++p.run;
  const size_t cuts = p.cuts >= kDeltaLeastCuts ? p.cuts : 0, runs = (cuts + p.run - 1) / p.run;
  const size_t state = (size_t)t->heads * t->key_dim * t->value_dim * 4, maps = cuts * t->heads * t->key_dim * t->key_dim * 4;
  size_t at = align256(cuts * 4);
  auto take = [&](size_t bytes) {
    const size_t from = at;
    at = align256(at + bytes);
    return from;
  };
  for (int i = 0; i < (backward ? 2 : 1); ++i) {
    p.off_from[i] = take(cuts * 4);
    p.off_run[i] = take(maps);
    p.off_end[i] = take(runs * state);
  }
  p.off_state = take(cuts * state);
  p.off_map = take(maps);
  if (backward) {
    p.off_turned = take(maps);
    const size_t chunks = (size_t)delta_slots(t->rows, t->num_sequences), rows = (size_t)t->rows * t->heads * t->value_dim * 4;
    p.off_grad = take(cuts * state);
    p.off_before = take(chunks * state);
    p.off_after = take(chunks * state);
    p.off_left = take(rows);
    p.off_due = take(rows);
  }
  p.total = std::max<size_t>(at, 256);
  return p;
}

// The gradients' launch over chunks.
bool too_many_chunks(const mmbev_attention_t* t) { return delta_slots(t->rows, t->num_sequences) * t->kv_heads > kMostGroups; }

// Gates: fp32 [rows][heads].
bool gates_ok(const mmbev_rows_t& g, const mmbev_attention_t* t) { return rows_ok(g, t->rows, t->heads, MMBEV_F32, false); }

bool gates_too_wide(std::initializer_list<const mmbev_rows_t*> arrays, int64_t rows) {
  for (const mmbev_rows_t* t : arrays)
    if (rows > 1 && t->row_stride > INT32_MAX) return true;
  return false;
}

// An array of rows of heads of any type, in units of two bytes.
struct Array {
  mmbev_heads_t t;
  int32_t heads, dim;
};
Array array_of(const mmbev_heads_t& t, int32_t heads, int32_t dim, int32_t dtype) {
  const int32_t units = size_of(dtype) / 2;
  return {{t.data, t.row_stride * units, t.head_stride * units}, heads, dim * units};
}
Array array_of(const mmbev_rows_t& t, int32_t width) { return array_of(mmbev_heads_t{t.data, t.row_stride, width}, 1, width, MMBEV_F32); }

bool share(const Array& x, const Array& y, int64_t rows) { return meet(x.t, x.heads, x.dim, y.t, y.heads, y.dim, rows, MMBEV_BF16); }

// `written` against each other and against the arrays behind them.
bool any_meet(std::initializer_list<Array> arrays, int written, int64_t rows) {
  for (int i = 0; i < written; ++i)
    for (int j = i + 1; j < (int)arrays.size(); ++j)
      if (share(arrays.begin()[i], arrays.begin()[j], rows)) return true;
  return false;
}

Span states_of(const float* s, size_t bytes) { return {(uintptr_t)s, (uintptr_t)s + (s ? bytes : 0)}; }

void put_delta(DeltaArgs& a, const mmbev_attention_t* t, const mmbev_heads_t& q, const mmbev_heads_t& k, const mmbev_heads_t& v,
               const mmbev_rows_t& log_decay, const mmbev_rows_t& beta, const int64_t* offsets, const DeltaPlan& p, char* ws) {
  a.offsets = offsets;
  a.rows = t->rows;
  a.B = t->num_sequences;
  a.cuts = p.cuts;
  a.longest_first = t->num_sequences <= kOrderedSequences && (int64_t)t->num_sequences * t->heads > kComputeUnits;
  a.least = kDeltaLeast;
  put(q, &a.q, &a.q_row, &a.q_head);
  put(k, &a.k, &a.k_row, &a.k_head);
  put(v, &a.v, &a.v_row, &a.v_head);
  a.log_decay = (const float*)log_decay.data;
  a.g_row = (int32_t)log_decay.row_stride;
  a.beta = (const float*)beta.data;
  a.b_row = (int32_t)beta.row_stride;
  a.H = t->heads;
  a.group = t->heads / t->kv_heads;
  a.kd = t->key_dim;
  a.vd = t->value_dim;
  a.past = t->rows * (t->heads + t->kv_heads) * (t->key_dim + t->value_dim) * size_of(t->dtype) > kPastCaches;
  a.scale = t->scale;
  a.cut_kind = (int32_t*)ws;
  a.cut_state = (float*)(ws + p.off_state);
  a.cut_map = (float*)(ws + p.off_map);
  a.run = p.run;
  for (int i = 0; i < 2; ++i) {
    a.from_run[i] = (int32_t*)(ws + p.off_from[i]);
    a.run_map[i] = (float*)(ws + p.off_run[i]);
    a.run_end[i] = (float*)(ws + p.off_end[i]);
  }
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
  HeadNormArgs a = head_norm_args(t, p, q_weight, k_weight, row_count, fault);
  put(q, &a.x[0], &a.x_row[0], &a.x_head[0]);
  put(k, &a.x[1], &a.x_row[1], &a.x_head[1]);
  put(q_out, &a.out[0], &a.out_row[0], &a.out_head[0]);
  put(k_out, &a.out[1], &a.out_row[1], &a.out_head[1]);
  return status_of(launch_head_norm(a, t->dtype, (hipStream_t)stream));
}

size_t mmbev_head_norm_rotary_backward_workspace_bytes(const mmbev_head_norm_t* t) {
  if (head_norm_ok(t) != MMBEV_OK) return 0;
  const HeadNormArgs a = head_norm_args(t, {}, nullptr, nullptr, nullptr, nullptr);
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
  HeadNormArgs a = head_norm_args(t, p, q_weight, k_weight, row_count, fault);
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

size_t mmbev_gated_delta_workspace_bytes(const mmbev_attention_t* t, int32_t backward) {
  if (delta_ok(t, false) != MMBEV_OK || (backward && too_many_chunks(t))) return 0;
  return delta_plan(t, backward != 0).total;
}

mmbev_status_t mmbev_gated_delta(const mmbev_attention_t* t, mmbev_heads_t q, mmbev_heads_t k, mmbev_heads_t v, mmbev_rows_t log_decay,
                                 mmbev_rows_t beta, const int64_t* offsets, const float* initial_state, mmbev_heads_t out,
                                 float* final_state, int32_t* fault, void* workspace, size_t workspace_bytes, void* stream) {
  const mmbev_status_t st = delta_ok(t, false);
  if (st != MMBEV_OK) return st;
  const int32_t T = t->dtype, H = t->heads, K = t->kv_heads;
  const int64_t R = t->rows;
  if (!heads_ok(q, R, H, t->key_dim, T) || !heads_ok(k, R, K, t->key_dim, T) || !heads_ok(v, R, K, t->value_dim, T) ||
      !heads_ok(out, R, H, t->value_dim, T) || !gates_ok(log_decay, t) || !gates_ok(beta, t))
    return MMBEV_ERR_INVALID_ARG;
  if (!offsets || !aligned(offsets, 8) || !aligned(initial_state, 4) || !aligned(final_state, 4)) return MMBEV_ERR_INVALID_ARG;
  if (too_wide({&q, &k, &v, &out}, R) || gates_too_wide({&log_decay, &beta}, R)) return MMBEV_ERR_UNSUPPORTED;
  const size_t state = (size_t)t->num_sequences * H * t->key_dim * t->value_dim * 4;
  if (overlap(states_of(initial_state, state), states_of(final_state, state))) return MMBEV_ERR_INVALID_ARG;
  if (any_meet({array_of(out, H, t->value_dim, T), array_of(q, H, t->key_dim, T), array_of(k, K, t->key_dim, T),
                array_of(v, K, t->value_dim, T), array_of(log_decay, H), array_of(beta, H)},
               1, R))
    return MMBEV_ERR_INVALID_ARG;
  const DeltaPlan p = delta_plan(t, false);
  if (!workspace_ok(workspace, workspace_bytes, p.total)) return MMBEV_ERR_WORKSPACE;
  DeltaArgs a{};
  put_delta(a, t, q, k, v, log_decay, beta, offsets, p, (char*)workspace);
  put(out, &a.out, &a.o_row, &a.o_head);
  a.init = initial_state;
  a.final_state = final_state;
  a.fault = fault;
  return status_of(launch_delta(a, T, (hipStream_t)stream));
}

mmbev_status_t mmbev_gated_delta_backward(const mmbev_attention_t* t, mmbev_heads_t dout, mmbev_heads_t q, mmbev_heads_t k, mmbev_heads_t v,
                                          mmbev_rows_t log_decay, mmbev_rows_t beta, const int64_t* offsets, const float* initial_state,
                                          const float* dfinal_state, mmbev_heads_t dq, mmbev_heads_t dk, mmbev_heads_t dv,
                                          mmbev_rows_t dlog_decay, mmbev_rows_t dbeta, float* dinitial_state, int32_t* fault,
                                          void* workspace, size_t workspace_bytes, void* stream) {
  const mmbev_status_t st = delta_ok(t, false);
  if (st != MMBEV_OK) return st;
  const int32_t T = t->dtype, H = t->heads, K = t->kv_heads;
  const int64_t R = t->rows;
  if (!heads_ok(dout, R, H, t->value_dim, T) || !heads_ok(q, R, H, t->key_dim, T) || !heads_ok(k, R, K, t->key_dim, T) ||
      !heads_ok(v, R, K, t->value_dim, T) || !heads_ok(dq, R, H, t->key_dim, T) || !heads_ok(dk, R, K, t->key_dim, T) ||
      !heads_ok(dv, R, K, t->value_dim, T))
    return MMBEV_ERR_INVALID_ARG;
  if (!gates_ok(log_decay, t) || !gates_ok(beta, t) || !gates_ok(dlog_decay, t) || !gates_ok(dbeta, t)) return MMBEV_ERR_INVALID_ARG;
  if (!offsets || !aligned(offsets, 8) || !aligned(initial_state, 4) || !aligned(dfinal_state, 4) || !aligned(dinitial_state, 4))
    return MMBEV_ERR_INVALID_ARG;
  if (too_wide({&dout, &q, &k, &v, &dq, &dk, &dv}, R) || gates_too_wide({&log_decay, &beta, &dlog_decay, &dbeta}, R) || too_many_chunks(t))
    return MMBEV_ERR_UNSUPPORTED;
  const size_t state = (size_t)t->num_sequences * H * t->key_dim * t->value_dim * 4;
  for (const float* in : {initial_state, dfinal_state})
    if (overlap(states_of(dinitial_state, state), states_of(in, state))) return MMBEV_ERR_INVALID_ARG;
  // the gradients against the inputs and against each other
  if (any_meet({array_of(dq, H, t->key_dim, T), array_of(dk, K, t->key_dim, T), array_of(dv, K, t->value_dim, T), array_of(dlog_decay, H),
                array_of(dbeta, H), array_of(dout, H, t->value_dim, T), array_of(q, H, t->key_dim, T), array_of(k, K, t->key_dim, T),
                array_of(v, K, t->value_dim, T), array_of(log_decay, H), array_of(beta, H)},
               5, R))
    return MMBEV_ERR_INVALID_ARG;
  const DeltaPlan p = delta_plan(t, true);
  if (!workspace_ok(workspace, workspace_bytes, p.total)) return MMBEV_ERR_WORKSPACE;
  char* ws = (char*)workspace;
  DeltaGradArgs a{};
  put_delta(a, t, q, k, v, log_decay, beta, offsets, p, ws);
  put(dout, &a.dout, &a.d_row, &a.d_head);
  put(dq, &a.dq, &a.dq_row, &a.dq_head);
  put(dk, &a.dk, &a.dk_row, &a.dk_head);
  put(dv, &a.dv, &a.dv_row, &a.dv_head);
  a.dlog_decay = (float*)dlog_decay.data;
  a.dg_row = (int32_t)dlog_decay.row_stride;
  a.dbeta = (float*)dbeta.data;
  a.db_row = (int32_t)dbeta.row_stride;
  a.init = initial_state;
  a.fault = fault;
  a.cut_grad = (float*)(ws + p.off_grad);
  a.cut_turned = (float*)(ws + p.off_turned);
  a.before = (float*)(ws + p.off_before);
  a.after = (float*)(ws + p.off_after);
  a.left_over = (float*)(ws + p.off_left);
  a.due = (float*)(ws + p.off_due);
  return status_of(launch_delta_backward(a, dfinal_state, dinitial_state, T, (hipStream_t)stream));
}

mmbev_status_t mmbev_gated_delta_step(const mmbev_attention_t* t, mmbev_heads_t q, mmbev_heads_t k, mmbev_heads_t v, mmbev_rows_t log_decay,
                                      mmbev_rows_t beta, const int32_t* slots, int64_t num_slots, float* state, mmbev_heads_t out,
                                      int32_t* fault, void* stream) {
  const mmbev_status_t ok = delta_ok(t, true);
  if (ok != MMBEV_OK) return ok;
  const int32_t T = t->dtype, H = t->heads, K = t->kv_heads;
  const int64_t R = t->rows;
  if (!heads_ok(q, R, H, t->key_dim, T) || !heads_ok(k, R, K, t->key_dim, T) || !heads_ok(v, R, K, t->value_dim, T) ||
      !heads_ok(out, R, H, t->value_dim, T) || !gates_ok(log_decay, t) || !gates_ok(beta, t))
    return MMBEV_ERR_INVALID_ARG;
  if (!aligned(slots, 4) || num_slots < 0) return MMBEV_ERR_INVALID_ARG;
  // a workgroup reads its head's q, k and v before it writes its out: they may be one, unless other heads read them too
  const Array to = array_of(out, H, t->value_dim, T);
  const bool own = H == K;
  if ((!same(q, out) && share(array_of(q, H, t->key_dim, T), to, R)) || (!(own && same(k, out)) && share(array_of(k, K, t->key_dim, T), to, R)) ||
      (!(own && same(v, out)) && share(array_of(v, K, t->value_dim, T), to, R)) || share(array_of(log_decay, H), to, R) ||
      share(array_of(beta, H), to, R))
    return MMBEV_ERR_INVALID_ARG;
  if (num_slots > kMaxRows) return MMBEV_ERR_UNSUPPORTED;
  if (R > 0 && num_slots > 0 && (!state || !aligned(state, 16))) return MMBEV_ERR_INVALID_ARG;
  if (!slots && num_slots < R) return MMBEV_ERR_INVALID_ARG;
  DeltaStepArgs a{};
  put(q, &a.q, &a.q_row, &a.q_head);
  put(k, &a.k, &a.k_row, &a.k_head);
  put(v, &a.v, &a.v_row, &a.v_head);
  put(out, &a.out, &a.o_row, &a.o_head);
  a.log_decay = (const float*)log_decay.data;
  a.g_row = log_decay.row_stride;
  a.beta = (const float*)beta.data;
  a.b_row = beta.row_stride;
  a.slots = slots;
  a.num_slots = num_slots;
  a.state = state;
  a.fault = fault;
  a.rows = R;
  a.H = H;
  a.group = H / K;
  a.kd = t->key_dim;
  a.vd = t->value_dim;
  a.scale = t->scale;
  return status_of(launch_delta_step(a, T, (hipStream_t)stream));
}

}  // extern "C"
