// What the C entry points of the sequence operators check of their arguments.
#pragma once

#include <algorithm>
#include <initializer_list>

#include "sequence.hpp"

namespace mmbev {
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

mmbev_status_t status_of(hipError_t e) { return e == hipSuccess ? MMBEV_OK : MMBEV_ERR_HIP; }

template <typename P, typename R>
void put(const mmbev_heads_t& t, P** data, R* row, int64_t* head) {
  *data = t.data;
  *row = (R)t.row_stride;
  *head = t.head_stride;
}

bool workspace_ok(const void* ws, size_t bytes, size_t need) { return ws && aligned(ws, 256) && bytes >= need; }

}  // namespace
}  // namespace mmbev
