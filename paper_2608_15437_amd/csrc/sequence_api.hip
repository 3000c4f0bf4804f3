// C ABI of the sequence operators: argument validation, workspace layout and
// launches.  No allocation, no host synchronisation, no state between calls.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <initializer_list>

#include "sequence.hpp"

using namespace mmbev;

namespace {

constexpr int64_t kMaxRows = INT32_MAX;

int32_t size_of(int32_t dtype) { return dtype == MMBEV_F32 ? 4 : 2; }

bool known_type(int32_t dtype) { return dtype == MMBEV_F32 || dtype == MMBEV_F16 || dtype == MMBEV_BF16; }

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

bool aligned(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

constexpr int64_t kMaxStride = (int64_t)1 << 40;

// Strides and rows that each are in range: the last row's elements lie inside an address space (2^58 bytes or fewer on).
bool reachable(int64_t rows, int64_t stride) { return rows <= 1 || stride <= ((int64_t)1 << 56) / (rows - 1); }

// Rows of `width` elements: there (or, optional, absent), aligned to the element, rows apart.
bool rows_ok(const mmbev_rows_t& t, int64_t rows, int32_t width, int32_t dtype, bool optional) {
  if (!t.data) return optional || rows == 0;
  return aligned(t.data, size_of(dtype)) && (rows <= 1 || t.row_stride >= width) && t.row_stride >= 0 && t.row_stride < kMaxStride &&
         reachable(rows, t.row_stride);
}

bool heads_ok(const mmbev_heads_t& t, int64_t rows, int32_t heads, int32_t dim, int32_t dtype) {
  if (!t.data) return rows == 0;
  if (!aligned(t.data, size_of(dtype)) || t.row_stride < 0 || t.head_stride < 0) return false;
  if (t.row_stride >= kMaxStride || t.head_stride >= kMaxStride || !reachable(rows, t.row_stride)) return false;
  if (heads > 1 && t.head_stride < dim) return false;
  // heads inside a row, or rows inside a head
  const int64_t row = (int64_t)(heads - 1) * t.head_stride + dim;
  return rows <= 1 || t.row_stride >= row || (t.row_stride >= dim && t.head_stride >= (rows - 1) * t.row_stride + dim);
}

// The attention walks' row strides take 31 bits: a row's address is then one 32 x 32-bit product.
bool too_wide(std::initializer_list<const mmbev_heads_t*> arrays, int64_t rows) {
  for (const mmbev_heads_t* t : arrays)
    if (rows > 1 && t->row_stride > INT32_MAX) return true;
  return false;
}

// First and past-the-last byte of rows of heads.
struct Span {
  uintptr_t lo, hi;
};
Span span_of(const mmbev_heads_t& t, int64_t rows, int32_t heads, int32_t dim, int32_t dtype) {
  if (!t.data || rows == 0) return {0, 0};
  const uintptr_t lo = (uintptr_t)t.data;
  const int64_t last = (rows - 1) * t.row_stride + (int64_t)(heads - 1) * t.head_stride + dim;
  return {lo, lo + (uintptr_t)last * size_of(dtype)};
}
bool overlap(Span a, Span b) { return a.lo < b.hi && b.lo < a.hi; }

int64_t floor_div(int64_t a, int64_t b) { return a / b - (a % b != 0 && a < 0); }

// Runs of `width` elements every `stride`, `count` of them.
struct Runs {
  int64_t stride, count, width;
};

// Whether any run of y, whose first is `shift` elements behind x's first, has an element of a run of x.
bool runs_meet(const Runs& x, const Runs& y, int64_t shift) {
  if (shift >= (x.count - 1) * x.stride + x.width || shift + (y.count - 1) * y.stride + y.width <= 0) return false;
  if (x.stride == y.stride || y.count == 1) {
    // y's run j begins m elements into x's run first + j and may reach into the next
    const int64_t first = floor_div(shift, x.stride), m = shift - first * x.stride;
    auto there = [&](int64_t i) { return i < x.count && i + y.count > 0; };  // one of x's runs i .. i + y.count - 1
    if (m < x.width && there(first)) return true;
    // (a single run of y may reach over several of x's)
    return m + y.width > x.stride && first + 1 < x.count && first + (m + y.width - 1) / x.stride + y.count > 0;
  }
  if (x.count == 1) return runs_meet(y, x, -shift);
  if (x.count + y.count > 4096) return true;  // not told apart
  for (int64_t i = 0, j = 0; i < x.count && j < y.count;) {
    const int64_t a = i * x.stride, b = shift + j * y.stride;
    if (a < b + y.width && b < a + x.width) return true;
    a < b ? ++i : ++j;
  }
  return false;
}

// Whether two arrays of `rows` rows of heads have an element in common.  Exact where both have their heads inside rows of
// one stride, or their rows inside heads of one; else arrays whose first and last elements enclose one another's count as
// having one.
bool meet(const mmbev_heads_t& x, int32_t x_heads, int32_t x_dim, const mmbev_heads_t& y, int32_t y_heads, int32_t y_dim, int64_t rows,
          int32_t dtype) {
  if (!x.data || !y.data || rows == 0) return false;
  if (!overlap(span_of(x, rows, x_heads, x_dim, dtype), span_of(y, rows, y_heads, y_dim, dtype))) return false;
  const int64_t bytes = (int64_t)((uintptr_t)y.data - (uintptr_t)x.data);  // both are aligned to the element
  const int64_t shift = bytes / size_of(dtype);
  const Runs xh{x_heads > 1 ? x.head_stride : x_dim, x_heads, x_dim}, yh{y_heads > 1 ? y.head_stride : y_dim, y_heads, y_dim};
  if (rows == 1) return runs_meet(xh, yh, shift);
  auto extent = [](const Runs& r) { return (r.count - 1) * r.stride + r.width; };
  // `step` elements a time, x's and y's runs inside each
  auto nested = [&](int64_t step, int64_t x_count, int64_t y_count, const Runs& xr, const Runs& yr) {
    const int64_t k = floor_div(shift, step), o = shift - k * step;  // y's item j lies o behind x's item j + k
    auto both = [&](int64_t d) { return d < x_count && d + y_count > 0; };
    return (both(k) && runs_meet(xr, yr, o)) || (both(k + 1) && runs_meet(xr, yr, o - step));
  };
  if (x.row_stride == y.row_stride && x.row_stride >= extent(xh) && x.row_stride >= extent(yh))
    return nested(x.row_stride, rows, rows, xh, yh);
  const Runs xr{x.row_stride, rows, x_dim}, yr{y.row_stride, rows, y_dim};
  if (x_heads > 1 && y_heads > 1 && x.head_stride == y.head_stride && x.head_stride >= extent(xr) && x.head_stride >= extent(yr))
    return nested(x.head_stride, x_heads, y_heads, xr, yr);
  return true;
}

// The same rows, heads and strides.
bool same(const mmbev_heads_t& x, const mmbev_heads_t& y) {
  return x.data == y.data && x.row_stride == y.row_stride && x.head_stride == y.head_stride;
}

// The same for rows without heads: apart, or (own) the very same rows.
bool rows_apart(const mmbev_rows_t& x, const mmbev_rows_t& y, int64_t rows, int32_t width, int32_t dtype, bool own) {
  if (own && x.data == y.data && (rows <= 1 || x.row_stride == y.row_stride)) return true;
  return !meet({x.data, x.row_stride, width}, 1, width, {y.data, y.row_stride, width}, 1, width, rows, dtype);
}

mmbev_status_t norm_ok(const mmbev_norm_t* n) {
  if (!n || n->rows < 0 || n->width < 1 || !known_type(n->dtype)) return MMBEV_ERR_INVALID_ARG;
  if (n->weight_dtype != MMBEV_F32 && n->weight_dtype != n->dtype) return MMBEV_ERR_INVALID_ARG;
  if (!(n->eps >= 0.0f) || !std::isfinite(n->eps)) return MMBEV_ERR_INVALID_ARG;
  if (n->rows > kMaxRows || n->width > 8192) return MMBEV_ERR_UNSUPPORTED;
  return MMBEV_OK;
}

NormArgs norm_args(const mmbev_norm_t* n, int32_t arrays, const int64_t* row_count, int32_t* fault) {
  NormArgs a{};
  a.past = arrays * n->rows * n->width * size_of(n->dtype) > kPastCaches;
  a.rows = n->rows;
  a.width = n->width;
  a.weight_f32 = n->weight_dtype == MMBEV_F32;
  a.eps = n->eps;
  a.inv_width = (float)(1.0 / n->width);
  a.row_count = row_count;
  a.fault = fault;
  return a;
}

mmbev_status_t status_of(hipError_t e) { return e == hipSuccess ? MMBEV_OK : MMBEV_ERR_HIP; }

// ------------------------------------------------------------ attention

// A sequence and head is a workgroup's work, but long ones are cut so that the
// workgroups fill the chip's compute units once.
constexpr int64_t kComputeUnits = 256;
// None is cut where none can be longer than this (it would take two more
// launches than it saves), nor among more sequences than a workgroup can look
// through in passing.
constexpr int64_t kAttnWhole = 512;
constexpr int32_t kAttnCutSequences = 1024;

struct AttnPlan {
  int32_t least;      // rows of a part
  int64_t slots;      // workgroups that the chip takes at once
  int32_t cuts;       // of the forward walks
  int32_t grad_cuts;  // of the backward walk
  int32_t group;      // its heads a workgroup
  size_t off_rows, off_state, off_part, total;
};

mmbev_status_t attention_ok(const mmbev_attention_t* t, bool step) {
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

// Heads that one workgroup of the backward walk takes of those that share keys and values.
int32_t grad_group(const mmbev_attention_t* t) {
  const int32_t shared = t->heads / t->kv_heads;
  int32_t group = kAttnGroupMost(std::max(t->key_dim, t->value_dim));
  while (shared % group != 0) group /= 2;
  return group;
}

// Rows of a part, at least: enough that its state is a small part of what is
// read for them.  Short calls want more parts, the backward pass with its two
// states fewer: a frame's 5,442 rows of 4 x 128 forward in 41 us with 128
// rows and 51 with 256, the gradients of 18,608 in 171 and 165.
int32_t least_rows(const mmbev_attention_t* t, bool backward) {
  return backward && std::max(t->key_dim, t->value_dim) > 64 ? 256 : 128;
}

// No sequence is longer than this, as far as the call says.
bool short_rows(const mmbev_attention_t* t) {
  return (t->max_length > 0 ? std::min(t->max_length, t->rows) : t->rows) <= kAttnWhole;
}

// Parts that rows are shared out over, so that with the sequences that are
// not cut there are about `units` of them and no second round of a few: at
// least half the units. `heads`: workgroups of a part.
int32_t cuts_for(const mmbev_attention_t* t, int64_t heads, int64_t slots, bool backward) {
  if (short_rows(t) || t->num_sequences > kAttnCutSequences) return 0;
  const int64_t least = least_rows(t, backward), units = std::max<int64_t>(2, slots / heads);
  const int64_t parts = units - std::min<int64_t>(t->num_sequences, units / 2);
  return (int32_t)std::max<int64_t>(1, std::min(parts, (t->rows + least - 1) / least));
}

AttnPlan attention_plan(const mmbev_attention_t* t, bool backward) {
  AttnPlan p{};
  const bool half = t->dtype != MMBEV_F32;
  const int32_t wide = std::max(t->key_dim, t->value_dim);
  // (three a unit for the gradients of heads of 32, whatever share one's registers allow: 8 frames of 16 heads over 4,
  // 716 us instead of 883)
  p.slots = kComputeUnits * (!backward ? walk_waves(half, wide) : wide <= 32 ? 3 : grad_waves(half, wide));
  p.least = least_rows(t, backward);
  p.cuts = cuts_for(t, t->heads, p.slots, backward);
  if (backward) {
    p.group = grad_group(t);
    p.grad_cuts = cuts_for(t, t->heads / p.group, p.slots, true);
  }
  // the forward walk's, then the backward one's
  const size_t all = p.cuts + p.grad_cuts;
  size_t at = 0;
  p.off_rows = at;
  at = align256(at + all * 4);
  p.off_state = at;
  at = align256(at + all * t->heads * t->key_dim * t->value_dim * 4);
  p.off_part = at;
  if (backward && t->heads != t->kv_heads * p.group)
    at = align256(at + (size_t)t->rows * (t->heads / p.group) * (t->key_dim + t->value_dim) * 4);
  p.total = std::max<size_t>(at, 256);
  return p;
}

void put_walk(AttnWalk& a, const mmbev_attention_t* t, const float* log_decay, const int64_t* offsets, bool backwards, const AttnPlan& p,
              char* ws) {
  const int32_t cuts = backwards ? p.grad_cuts : p.cuts, before = backwards ? p.cuts : 0;
  const int64_t heads = backwards ? t->heads / p.group : t->heads;
  a.log_decay = log_decay;
  a.offsets = offsets;
  a.rows = t->rows;
  a.B = t->num_sequences;
  a.H = t->heads;
  a.scale = t->scale;
  a.init_scale = a.final_scale = 1.0f;
  a.cuts = cuts;
  a.longest_first = t->num_sequences <= kOrderedSequences && t->num_sequences * heads > p.slots;
  a.past = t->rows * (t->heads + t->kv_heads) * (t->key_dim + t->value_dim) * size_of(t->dtype) > kPastCaches;
  a.least = p.least;
  a.reversed = backwards;
  a.cut_rows = (int32_t*)(ws + p.off_rows) + before;
  a.cut_state = (float*)(ws + p.off_state) + (int64_t)before * t->heads * t->key_dim * t->value_dim;
}

template <typename P, typename R>
void put(const mmbev_heads_t& t, P** data, R* row, int64_t* head) {
  *data = t.data;
  *row = (R)t.row_stride;
  *head = t.head_stride;
}

bool workspace_ok(const void* ws, size_t bytes, size_t need) { return ws && aligned(ws, 256) && bytes >= need; }

}  // namespace

extern "C" {

mmbev_status_t mmbev_layer_norm(const mmbev_norm_t* norm, mmbev_rows_t x, mmbev_rows_t residual, const void* weight,
                                const void* bias, const int64_t* row_count, mmbev_rows_t out, mmbev_rows_t out_sum,
                                float* out_mean, float* out_rstd, int32_t* fault, void* stream) {
  const mmbev_status_t st = norm_ok(norm);
  if (st != MMBEV_OK) return st;
  const int64_t R = norm->rows;
  const int32_t C = norm->width, T = norm->dtype;
  if (!rows_ok(x, R, C, T, false) || !rows_ok(residual, R, C, T, true) || !rows_ok(out, R, C, T, false) ||
      !rows_ok(out_sum, R, C, T, true))
    return MMBEV_ERR_INVALID_ARG;
  if (!aligned(weight, size_of(norm->weight_dtype)) || !aligned(bias, size_of(norm->weight_dtype))) return MMBEV_ERR_INVALID_ARG;
  for (const mmbev_rows_t* in : {&x, &residual})
    for (const mmbev_rows_t* to : {&out, &out_sum})
      if (!rows_apart(*in, *to, R, C, T, true)) return MMBEV_ERR_INVALID_ARG;
  if (!rows_apart(out, out_sum, R, C, T, false)) return MMBEV_ERR_INVALID_ARG;
  NormArgs a = norm_args(norm, 2 + (residual.data != nullptr) + (out_sum.data != nullptr), row_count, fault);
  a.x = x.data;
  a.x_stride = x.row_stride;
  a.skip = residual.data;
  a.skip_stride = residual.row_stride;
  a.weight = weight;
  a.bias = bias;
  a.out = out.data;
  a.out_stride = out.row_stride;
  a.sum = out_sum.data;
  a.sum_stride = out_sum.row_stride;
  a.mean = out_mean;
  a.rstd = out_rstd;
  return status_of(launch_norm(a, T, (hipStream_t)stream));
}

size_t mmbev_layer_norm_backward_workspace_bytes(const mmbev_norm_t* norm) {
  if (norm_ok(norm) != MMBEV_OK) return 0;
  return align256((size_t)norm_backward_grid(norm->rows, norm->width, norm->dtype) * 2 * norm->width * 4);
}

mmbev_status_t mmbev_layer_norm_backward(const mmbev_norm_t* norm, mmbev_rows_t dy, mmbev_rows_t s,
                                         const void* weight, const float* mean, const float* rstd, mmbev_rows_t dskip,
                                         const int64_t* row_count, mmbev_rows_t dx, float* dweight, float* dbias,
                                         int32_t* fault, void* workspace, size_t workspace_bytes, void* stream) {
  const mmbev_status_t st = norm_ok(norm);
  if (st != MMBEV_OK) return st;
  const int64_t R = norm->rows;
  const int32_t C = norm->width, T = norm->dtype;
  if (!rows_ok(dy, R, C, T, false) || !rows_ok(s, R, C, T, false) || !rows_ok(dskip, R, C, T, true) ||
      !rows_ok(dx, R, C, T, false))
    return MMBEV_ERR_INVALID_ARG;
  if (R > 0 && (!mean || !rstd)) return MMBEV_ERR_INVALID_ARG;
  for (const mmbev_rows_t* in : {&dy, &s, &dskip})
    if (!rows_apart(*in, dx, R, C, T, true)) return MMBEV_ERR_INVALID_ARG;
  if (!aligned(weight, size_of(norm->weight_dtype))) return MMBEV_ERR_INVALID_ARG;
  const bool sums = dweight || dbias;
  if (sums && !workspace_ok(workspace, workspace_bytes, mmbev_layer_norm_backward_workspace_bytes(norm)))
    return MMBEV_ERR_WORKSPACE;
  NormArgs a = norm_args(norm, 3 + (dskip.data != nullptr), row_count, fault);
  a.x = s.data;
  a.x_stride = s.row_stride;
  a.dy = dy.data;
  a.dy_stride = dy.row_stride;
  a.skip = dskip.data;
  a.skip_stride = dskip.row_stride;
  a.weight = weight;
  a.mean = const_cast<float*>(mean);
  a.rstd = const_cast<float*>(rstd);
  a.out = dx.data;
  a.out_stride = dx.row_stride;
  a.partial = sums ? (float*)workspace : nullptr;
  a.dweight = dweight;
  a.dbias = dbias;
  return status_of(launch_norm_backward(a, T, (hipStream_t)stream));
}

mmbev_status_t mmbev_make_rotary(const mmbev_rotary_ladder_t* t, uint64_t* out_steps, uint8_t* out_axis) {
  if (!t || !out_steps || !out_axis || t->reserved != 0) return MMBEV_ERR_INVALID_ARG;
  if (t->rotary_dim < 2 || t->rotary_dim > 1024 || t->rotary_dim % 2 != 0) return MMBEV_ERR_INVALID_ARG;
  const int32_t P = t->rotary_dim / 2;
  if (t->axes < 1 || t->axes > 8 || t->axes > P) return MMBEV_ERR_INVALID_ARG;
  if (!(t->base > 1.0) || !std::isfinite(t->base)) return MMBEV_ERR_INVALID_ARG;
  if (t->scaling < MMBEV_ROTARY_PLAIN || t->scaling > MMBEV_ROTARY_PARTS) return MMBEV_ERR_INVALID_ARG;
  if (t->scaling != MMBEV_ROTARY_PLAIN && (!(t->factor >= 1.0) || !std::isfinite(t->factor))) return MMBEV_ERR_INVALID_ARG;
  if (t->scaling == MMBEV_ROTARY_PARTS &&
      (!(t->length > 0.0) || !std::isfinite(t->length) || !(t->slow > 0.0) || !(t->fast > t->slow) || !std::isfinite(t->fast)))
    return MMBEV_ERR_INVALID_ARG;
  const double two_pi = 6.283185307179586476925286766559;
  for (int32_t a = 0; a < t->axes; ++a) {
    const int32_t first = P * a / t->axes, n = P * (a + 1) / t->axes - first;
    for (int32_t j = 0; j < n; ++j) {
      double base = t->base;
      if (t->scaling == MMBEV_ROTARY_BASE && n > 1) base *= std::pow(t->factor, (double)n / (n - 1));
      double turns = std::pow(base, -(double)j / n) / two_pi;
      if (t->scaling == MMBEV_ROTARY_LINEAR) turns /= t->factor;
      if (t->scaling == MMBEV_ROTARY_PARTS) {
        const double share = std::min(1.0, std::max(0.0, (turns * t->length - t->slow) / (t->fast - t->slow)));
        turns = share * turns + (1.0 - share) * turns / t->factor;
      }
      // at most 1 / (2 pi) of a turn, so the product fits; the double's 53 bits are exact in it
      out_steps[first + j] = (uint64_t)std::ldexp(turns, 64);
      out_axis[first + j] = (uint8_t)a;
    }
  }
  return MMBEV_OK;
}

mmbev_status_t mmbev_rotary(const mmbev_rotary_t* t, mmbev_heads_t x, const int32_t* positions, int64_t position_stride,
                            int32_t axes, const uint64_t* steps, const uint8_t* axis, const int64_t* row_count,
                            mmbev_heads_t out, int32_t* fault, void* stream) {
  if (!t || t->rows < 0 || t->heads < 1 || t->dim < 1 || !known_type(t->dtype)) return MMBEV_ERR_INVALID_ARG;
  if (t->rotary_dim < 2 || t->rotary_dim % 2 != 0 || t->rotary_dim > t->dim) return MMBEV_ERR_INVALID_ARG;
  if (t->layout != MMBEV_ROTARY_HALF && t->layout != MMBEV_ROTARY_INTERLEAVED) return MMBEV_ERR_INVALID_ARG;
  if (t->inverse != 0 && t->inverse != 1) return MMBEV_ERR_INVALID_ARG;
  if (axes < 1 || axes > 8) return MMBEV_ERR_INVALID_ARG;
  if (t->rows > kMaxRows || t->heads > 1024 || t->dim > 1024) return MMBEV_ERR_UNSUPPORTED;
  if (!heads_ok(x, t->rows, t->heads, t->dim, t->dtype) || !heads_ok(out, t->rows, t->heads, t->dim, t->dtype))
    return MMBEV_ERR_INVALID_ARG;
  if (t->rows > 0 && (!positions || !aligned(positions, 4) || !steps || !aligned(steps, 8) || !axis)) return MMBEV_ERR_INVALID_ARG;
  if (position_stride < 0 || (t->rows > 1 && position_stride < axes) || position_stride >= kMaxStride ||
      !reachable(t->rows, position_stride))
    return MMBEV_ERR_INVALID_ARG;
  if (!same(x, out) && meet(x, t->heads, t->dim, out, t->heads, t->dim, t->rows, t->dtype)) return MMBEV_ERR_INVALID_ARG;
  RotaryArgs a{};
  a.x = x.data;
  a.out = out.data;
  a.positions = positions;
  a.steps = steps;
  a.axis = axis;
  a.row_count = row_count;
  a.fault = fault;
  a.rows = t->rows;
  a.x_row = x.row_stride;
  a.x_head = x.head_stride;
  a.out_row = out.row_stride;
  a.out_head = out.head_stride;
  a.position_stride = position_stride;
  a.heads = t->heads;
  a.dim = t->dim;
  a.rotary_dim = t->rotary_dim;
  a.axes = axes;
  a.interleaved = t->layout == MMBEV_ROTARY_INTERLEAVED;
  a.inverse = t->inverse;
  a.copy_rest = !same(x, out);
  a.past = 2 * t->rows * t->heads * t->dim * size_of(t->dtype) > kPastCaches;
  return status_of(launch_rotary(a, t->dtype, (hipStream_t)stream));
}

size_t mmbev_linear_attention_workspace_bytes(const mmbev_attention_t* attention, int32_t backward) {
  if (attention_ok(attention, false) != MMBEV_OK) return 0;
  return attention_plan(attention, backward != 0).total;
}

mmbev_status_t mmbev_linear_attention(const mmbev_attention_t* t, mmbev_heads_t q, mmbev_heads_t k, mmbev_heads_t v,
                                      const float* log_decay, const int64_t* offsets, const float* initial_state,
                                      mmbev_heads_t out, float* final_state, int32_t* fault, void* workspace,
                                      size_t workspace_bytes, void* stream) {
  const mmbev_status_t st = attention_ok(t, false);
  if (st != MMBEV_OK) return st;
  if (!heads_ok(q, t->rows, t->heads, t->key_dim, t->dtype) || !heads_ok(k, t->rows, t->kv_heads, t->key_dim, t->dtype) ||
      !heads_ok(v, t->rows, t->kv_heads, t->value_dim, t->dtype) || !heads_ok(out, t->rows, t->heads, t->value_dim, t->dtype))
    return MMBEV_ERR_INVALID_ARG;
  if (!log_decay || !aligned(log_decay, 4) || !offsets || !aligned(offsets, 8) || !aligned(initial_state, 4) ||
      !aligned(final_state, 4))
    return MMBEV_ERR_INVALID_ARG;
  if (too_wide({&q, &k, &v, &out}, t->rows)) return MMBEV_ERR_UNSUPPORTED;
  const size_t state = (size_t)t->num_sequences * t->heads * t->key_dim * t->value_dim * 4;
  if (initial_state && final_state &&
      overlap({(uintptr_t)initial_state, (uintptr_t)initial_state + state}, {(uintptr_t)final_state, (uintptr_t)final_state + state}))
    return MMBEV_ERR_INVALID_ARG;
  if (meet(q, t->heads, t->key_dim, out, t->heads, t->value_dim, t->rows, t->dtype) ||
      meet(k, t->kv_heads, t->key_dim, out, t->heads, t->value_dim, t->rows, t->dtype) ||
      meet(v, t->kv_heads, t->value_dim, out, t->heads, t->value_dim, t->rows, t->dtype))
    return MMBEV_ERR_INVALID_ARG;
  const AttnPlan p = attention_plan(t, false);
  if (!workspace_ok(workspace, workspace_bytes, p.total)) return MMBEV_ERR_WORKSPACE;
  AttnArgs a{};
  put_walk(a, t, log_decay, offsets, false, p, (char*)workspace);
  put(q, &a.a, &a.a_row, &a.a_head);
  put(k, &a.b, &a.b_row, &a.b_head);
  put(v, &a.c, &a.c_row, &a.c_head);
  put(out, &a.out, &a.o_row, &a.o_head);
  a.a_div = 1;
  a.b_div = a.c_div = t->heads / t->kv_heads;
  a.ad = t->key_dim;
  a.cd = t->value_dim;
  a.init = initial_state;
  a.final_state = final_state;
  a.exact_state = final_state != nullptr;
  a.fault = fault;
  return status_of(launch_attention(a, t->dtype, (hipStream_t)stream));
}

mmbev_status_t mmbev_linear_attention_backward(const mmbev_attention_t* t, mmbev_heads_t dout, mmbev_heads_t q,
                                               mmbev_heads_t k, mmbev_heads_t v, const float* log_decay,
                                               const int64_t* offsets, const float* initial_state,
                                               const float* dfinal_state, mmbev_heads_t dq, mmbev_heads_t dk,
                                               mmbev_heads_t dv, float* dinitial_state, int32_t* fault, void* workspace,
                                               size_t workspace_bytes, void* stream) {
  const mmbev_status_t ok = attention_ok(t, false);
  if (ok != MMBEV_OK) return ok;
  const int32_t T = t->dtype, H = t->heads, K = t->kv_heads, group = H / K;
  const int64_t R = t->rows;
  if (!heads_ok(dout, R, H, t->value_dim, T) || !heads_ok(q, R, H, t->key_dim, T) || !heads_ok(k, R, K, t->key_dim, T) ||
      !heads_ok(v, R, K, t->value_dim, T) || !heads_ok(dq, R, H, t->key_dim, T) || !heads_ok(dk, R, K, t->key_dim, T) ||
      !heads_ok(dv, R, K, t->value_dim, T))
    return MMBEV_ERR_INVALID_ARG;
  if (!log_decay || !aligned(log_decay, 4) || !offsets || !aligned(offsets, 8) || !aligned(initial_state, 4) ||
      !aligned(dfinal_state, 4) || !aligned(dinitial_state, 4))
    return MMBEV_ERR_INVALID_ARG;
  if (too_wide({&dout, &q, &k, &v, &dq, &dk, &dv}, R)) return MMBEV_ERR_UNSUPPORTED;
  const size_t state = (size_t)t->num_sequences * H * t->key_dim * t->value_dim * 4;
  const Span di = {(uintptr_t)dinitial_state, (uintptr_t)dinitial_state + (dinitial_state ? state : 0)};
  for (const float* in : {initial_state, dfinal_state})
    if (in && dinitial_state && overlap(di, {(uintptr_t)in, (uintptr_t)in + state})) return MMBEV_ERR_INVALID_ARG;
  struct Array {
    const mmbev_heads_t& t;
    int32_t heads, dim;
  };
  // the gradients against the inputs and against each other
  const Array arrays[] = {{dq, H, t->key_dim},  {dk, K, t->key_dim}, {dv, K, t->value_dim}, {dout, H, t->value_dim},
                          {q, H, t->key_dim}, {k, K, t->key_dim},  {v, K, t->value_dim}};
  for (int i = 0; i < 3; ++i)
    for (int j = i + 1; j < 7; ++j)
      if (meet(arrays[i].t, arrays[i].heads, arrays[i].dim, arrays[j].t, arrays[j].heads, arrays[j].dim, R, T)) return MMBEV_ERR_INVALID_ARG;
  const AttnPlan p = attention_plan(t, true);
  if (!workspace_ok(workspace, workspace_bytes, p.total)) return MMBEV_ERR_WORKSPACE;
  char* ws = (char*)workspace;
  hipStream_t st = (hipStream_t)stream;

  // dq: the forward walk of (dout, v, k), whose state is the transposed one; it
  // shares its launches, hence the chip, with the other
  AttnArgs a{};
  put_walk(a, t, log_decay, offsets, false, p, ws);
  put(dout, &a.a, &a.a_row, &a.a_head);
  put(v, &a.b, &a.b_row, &a.b_head);
  put(k, &a.c, &a.c_row, &a.c_head);
  put(dq, &a.out, &a.o_row, &a.o_head);
  a.a_div = 1;
  a.b_div = a.c_div = group;
  a.ad = t->value_dim;
  a.cd = t->key_dim;
  a.init = initial_state;
  a.init_swapped = 1;
  a.fault = fault;

  // dv and dk: backwards, the carried state that of q and dout, divided by scale
  AttnGradArgs b{};
  put_walk(b, t, log_decay, offsets, true, p, ws);
  put(q, &b.q, &b.q_row, &b.q_head);
  put(dout, &b.dout, &b.d_row, &b.d_head);
  put(k, &b.k, &b.k_row, &b.k_head);
  put(v, &b.v, &b.v_row, &b.v_head);
  put(dk, &b.dk, &b.dk_row, &b.dk_head);
  put(dv, &b.dv, &b.dv_row, &b.dv_head);
  b.ad = t->key_dim;
  b.cd = t->value_dim;
  b.init = dfinal_state;
  b.init_scale = 1.0f / t->scale;
  b.final_state = dinitial_state;
  b.final_scale = t->scale;
  b.exact_state = dinitial_state != nullptr;
  b.kv_div = group;
  b.group = p.group;
  b.parts = group != p.group;
  const int32_t parts = H / p.group;
  b.part_k = (float*)(ws + p.off_part);
  b.part_v = b.part_k + (size_t)R * parts * t->key_dim;
  AttnArgs s{};
  static_cast<AttnWalk&>(s) = b;
  put(q, &s.b, &s.b_row, &s.b_head);
  put(dout, &s.c, &s.c_row, &s.c_head);
  s.b_div = s.c_div = 1;
  if (launch_attention_backward(a, b, s, T, st) != hipSuccess) return MMBEV_ERR_HIP;
  for (int which = 0; b.parts && which < 2; ++which) {
    AttnSumArgs u{};
    u.part = which ? b.part_v : b.part_k;
    put(which ? dv : dk, &u.out, &u.out_row, &u.out_head);
    u.rows = R;
    u.offsets = offsets;
    u.B = t->num_sequences;
    u.parts = parts;
    u.group = group / p.group;
    u.dim = which ? t->value_dim : t->key_dim;
    if (launch_attention_sum(u, T, st) != hipSuccess) return MMBEV_ERR_HIP;
  }
  return MMBEV_OK;
}

mmbev_status_t mmbev_linear_attention_step(const mmbev_attention_t* t, mmbev_heads_t q, mmbev_heads_t k, mmbev_heads_t v,
                                           const float* log_decay, const int32_t* slots, int64_t num_slots, float* state,
                                           mmbev_heads_t out, int32_t* fault, void* stream) {
  const mmbev_status_t ok = attention_ok(t, true);
  if (ok != MMBEV_OK) return ok;
  if (!heads_ok(q, t->rows, t->heads, t->key_dim, t->dtype) || !heads_ok(k, t->rows, t->kv_heads, t->key_dim, t->dtype) ||
      !heads_ok(v, t->rows, t->kv_heads, t->value_dim, t->dtype) || !heads_ok(out, t->rows, t->heads, t->value_dim, t->dtype))
    return MMBEV_ERR_INVALID_ARG;
  if (!log_decay || !aligned(log_decay, 4) || !aligned(slots, 4) || num_slots < 0) return MMBEV_ERR_INVALID_ARG;
  // a workgroup reads its head's q, k and v before it writes its out: they may be one, unless other heads read them too
  const bool own = t->heads == t->kv_heads;
  if ((!same(q, out) && meet(q, t->heads, t->key_dim, out, t->heads, t->value_dim, t->rows, t->dtype)) ||
      (!(own && same(k, out)) && meet(k, t->kv_heads, t->key_dim, out, t->heads, t->value_dim, t->rows, t->dtype)) ||
      (!(own && same(v, out)) && meet(v, t->kv_heads, t->value_dim, out, t->heads, t->value_dim, t->rows, t->dtype)))
    return MMBEV_ERR_INVALID_ARG;
  if (num_slots > kMaxRows) return MMBEV_ERR_UNSUPPORTED;
  if (t->rows > 0 && num_slots > 0 && (!state || !aligned(state, 16))) return MMBEV_ERR_INVALID_ARG;
  if (!slots && num_slots < t->rows) return MMBEV_ERR_INVALID_ARG;
  AttnStepArgs a{};
  put(q, &a.q, &a.q_row, &a.q_head);
  put(k, &a.k, &a.k_row, &a.k_head);
  put(v, &a.v, &a.v_row, &a.v_head);
  a.out = out.data;
  a.o_row = out.row_stride;
  a.o_head = out.head_stride;
  a.log_decay = log_decay;
  a.slots = slots;
  a.num_slots = num_slots;
  a.state = state;
  a.fault = fault;
  a.rows = t->rows;
  a.H = t->heads;
  a.group = t->heads / t->kv_heads;
  a.kd = t->key_dim;
  a.vd = t->value_dim;
  a.scale = t->scale;
  return status_of(launch_attention_step(a, t->dtype, (hipStream_t)stream));
}

}  // extern "C"
