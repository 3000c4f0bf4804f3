// Norms of queries and keys for each head, turned by their positions in the
// same pass, and the gradients:
//   r = 1 / sqrt(mean(x^2) + eps),  h = x r,  y = R(h * w)
//   d = R^-1 dy,  a = d * w,  dx = r (a - h mean(a * h)),  dw = sum of d * h
//
// LANES neighbouring lanes hold a head, two 16-byte packs each: of the part
// that turns, the packs of the pairs' first and second elements or two packs of
// neighbouring pairs; of the rest, two packs that turn by nothing.  A group of
// lanes takes several heads of one row and one array, so that it works the
// sines and cosines out and loads the weights once for all of them (the fewer
// rows, the fewer heads, so that small calls spread out).
// The operator moves bytes; beside them are some 15 operations an element and
// 50 a pair for its angle.
//
// The weights' gradients: a group stays with its heads and walks the rows that
// its workgroup takes (every grid-th block of them) with its columns' sums in
// registers; the workgroup's groups add theirs in LDS, and a second launch adds
// the workgroups' rows, all in a fixed order.
#include <algorithm>

#include "rotary.hpp"

namespace mmbev {

namespace {

constexpr int kHeadThreads = 256;
constexpr int kHeadsAtOnce = 4;  // whose loads are in flight together

struct HeadShape {
  int32_t lanes;             // of a head
  int32_t turned, items;     // of them with pairs, and with elements
  int32_t parts[2], each;    // a row's groups of lanes, of queries and of keys, and the heads of one
  int32_t rows_block;
};

// What a lane has of every head: where its packs are, and its pairs' angles.
template <typename T, bool INTERLEAVED>
struct Place {
  static constexpr int V = kPackOf<T>;
  int at[2], left[2];  // first element of a pack, elements from there on
  bool turned;
  float sn[V], cs[V];

  __device__ __forceinline__ void set(const HeadNormArgs& a, const HeadShape& s, int lane) {
    const int half = a.rotary_dim / 2;
    turned = lane < s.turned;
    if (!turned) {
      const int c = a.rotary_dim + (lane - s.turned) * 2 * V;
      at[0] = c;
      at[1] = c + V;
      left[0] = lane < s.items ? a.dim - c : 0;
      left[1] = left[0] - V;
    } else if (INTERLEAVED) {
      at[0] = lane * 2 * V;
      at[1] = at[0] + V;
      left[0] = a.rotary_dim - at[0];
      left[1] = left[0] - V;
    } else {
      at[0] = lane * V;
      at[1] = half + at[0];
      left[0] = left[1] = half - at[0];
    }
  }
  __device__ __forceinline__ void angles(const HeadNormArgs& a, int64_t row, int lane) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      sn[e] = 0.0f;
      cs[e] = 1.0f;
    }
    if (!turned) return;
    const int half = a.rotary_dim / 2;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      // pairs past the last turn by its angle; they are not stored
      const int j = min(lane * V + e, half - 1), ax = min((int)a.axis[j], a.axes - 1);
      const uint64_t phase = (uint64_t)(int64_t)a.positions[row * a.position_stride + ax] * a.steps[j];
      sincos_of_phase((uint32_t)(phase >> 32), sn[e], cs[e]);
    }
  }
  // pair e: element first(e) of the first pack or, of neighbouring pairs, of either
  __device__ __forceinline__ void turn(float (&x)[2][V], bool back) const {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      float& u = INTERLEAVED ? x[e / (V / 2)][e % (V / 2) * 2] : x[0][e];
      float& v = INTERLEAVED ? x[e / (V / 2)][e % (V / 2) * 2 + 1] : x[1][e];
      const float p = u, q = v, s = back ? -sn[e] : sn[e];
      u = __builtin_fmaf(p, cs[e], -(q * s));
      v = __builtin_fmaf(p, s, q * cs[e]);
    }
  }
};

template <typename T, int V>
struct Two {
  Pack<T, V> p[2];
};

template <typename T, int V>
__device__ __forceinline__ Two<T, V> load_two(const T* x, const int (&at)[2], const int (&left)[2], bool past) {
  Two<T, V> r;
#pragma unroll
  for (int i = 0; i < 2; ++i) r.p[i] = past && left[i] >= V ? load_past<T, V>(x + at[i]) : load_some<T, V>(x + at[i], left[i]);
  return r;
}

template <typename T, int V>
__device__ __forceinline__ void widen(float (&to)[2][V], const Two<T, V>& from) {
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int e = 0; e < V; ++e) to[i][e] = (float)from.p[i].v[e];
}

template <typename T, int V>
__device__ __forceinline__ void store_two(T* x, const float (&f)[2][V], const int (&at)[2], const int (&left)[2], bool past) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    Pack<T, V> r;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      float y = f[i][e];
      // the value as rounded to fp32: a multiply-add fused with its conversion to fp16 in one loop, but not in another,
      // would round the same head in two ways
      if constexpr (__is_same(T, f16)) asm("" : "+v"(y));
      r.v[e] = (T)y;
    }
    store_some<T, V>(x + at[i], r, left[i], past);
  }
}

template <typename T, int V>
__device__ __forceinline__ void load_weights(float (&w)[2][V], const void* p, bool f32, const int (&at)[2], const int (&left)[2]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (!p) {
#pragma unroll
      for (int e = 0; e < V; ++e) w[i][e] = 1.0f;
    } else if (f32) {
      const Pack<float, V> r = load_some<float, V>(static_cast<const float*>(p) + at[i], left[i]);
#pragma unroll
      for (int e = 0; e < V; ++e) w[i][e] = r.v[e];
    } else {
      const Pack<T, V> r = load_some<T, V>(static_cast<const T*>(p) + at[i], left[i]);
#pragma unroll
      for (int e = 0; e < V; ++e) w[i][e] = (float)r.v[e];
    }
  }
}

// Reciprocal root of the mean square (elements past the head are zeros).
template <int LANES, int V>
__device__ __forceinline__ float head_rstd(const float (&x)[2][V], const HeadNormArgs& a) {
  float sq = 0.0f;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int e = 0; e < V; ++e) sq = __builtin_fmaf(x[i][e], x[i][e], sq);
  return 1.0f / __builtin_sqrtf(__builtin_fmaf(group_sum<LANES>(sq), a.inv_dim, a.eps));
}

// The group's array and heads.
struct Share {
  int which, h0, h1;
  __device__ __forceinline__ Share(const HeadNormArgs& a, const HeadShape& s, int part) {
    which = part >= s.parts[0];
    h0 = (part - (which ? s.parts[0] : 0)) * s.each;
    h1 = min(h0 + s.each, which ? a.heads[1] : a.heads[0]);
  }
};

template <typename T, bool INTERLEAVED, int LANES>
__global__ __launch_bounds__(kHeadThreads) void head_norm_kernel(HeadNormArgs a, HeadShape s) {
  constexpr int V = kPackOf<T>;
  const int64_t n = rows_in_use(a.row_count, a.rows, a.fault);
  const int parts = s.parts[0] + s.parts[1], group = threadIdx.x / LANES, lane = threadIdx.x % LANES;
  const int r = group / parts;
  const int64_t row = a.first_row + (int64_t)blockIdx.x * s.rows_block + r;
  if (r >= s.rows_block || row >= n) return;
  const Share share(a, s, group - r * parts);
  const int which = share.which;
  Place<T, INTERLEAVED> place;
  place.set(a, s, lane);
  float w[2][V];
  load_weights<T, V>(w, which ? a.weight[1] : a.weight[0], a.weight_f32, place.at, place.left);
  const int64_t x_head = which ? a.x_head[1] : a.x_head[0], out_head = which ? a.out_head[1] : a.out_head[0];
  const T* x = static_cast<const T*>(which ? a.x[1] : a.x[0]) + row * (which ? a.x_row[1] : a.x_row[0]) + share.h0 * x_head;
  T* out = static_cast<T*>(which ? a.out[1] : a.out[0]) + row * (which ? a.out_row[1] : a.out_row[0]) + share.h0 * out_head;
  place.angles(a, row, lane);
  auto finish = [&](const Two<T, V>& from, T* to) {
    float f[2][V];
    widen<T, V>(f, from);
    const float rstd = head_rstd<LANES, V>(f, a);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) f[i][e] = f[i][e] * rstd * w[i][e];
    place.turn(f, false);
    store_two<T, V>(to, f, place.at, place.left, a.past);
  };
  int h = share.h0;
  for (; h + kHeadsAtOnce <= share.h1; h += kHeadsAtOnce, x += kHeadsAtOnce * x_head, out += kHeadsAtOnce * out_head) {
    Two<T, V> t[kHeadsAtOnce];
#pragma unroll
    for (int i = 0; i < kHeadsAtOnce; ++i) t[i] = load_two<T, V>(x + i * x_head, place.at, place.left, a.past);
#pragma unroll
    for (int i = 0; i < kHeadsAtOnce; ++i) finish(t[i], out + i * out_head);
  }
  for (; h < share.h1; ++h, x += x_head, out += out_head) finish(load_two<T, V>(x, place.at, place.left, a.past), out);
}

template <typename T, bool INTERLEAVED, int LANES>
__global__ __launch_bounds__(kHeadThreads) void head_norm_backward_kernel(HeadNormArgs a, HeadShape s) {
  constexpr int V = kPackOf<T>;
  __shared__ float s_sum[kHeadThreads / LANES][LANES * 2 * V + 1];
  const int64_t n = rows_in_use(a.row_count, a.rows, a.fault);
  const int parts = s.parts[0] + s.parts[1], group = threadIdx.x / LANES, lane = threadIdx.x % LANES;
  const int r = group / parts;
  const Share share(a, s, group - r * parts);
  const int which = share.which;
  Place<T, INTERLEAVED> place;
  place.set(a, s, lane);
  float w[2][V], dw[2][V];
  load_weights<T, V>(w, which ? a.weight[1] : a.weight[0], a.weight_f32, place.at, place.left);
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int e = 0; e < V; ++e) dw[i][e] = 0.0f;
  const int64_t x_head = which ? a.x_head[1] : a.x_head[0], dy_head = which ? a.dy_head[1] : a.dy_head[0],
                out_head = which ? a.out_head[1] : a.out_head[0];
  auto finish = [&](const Two<T, V>& from, const Two<T, V>& grad, T* to) {
    float f[2][V], d[2][V], dot = 0.0f;
    widen<T, V>(f, from);
    widen<T, V>(d, grad);
    const float rstd = head_rstd<LANES, V>(f, a);
    place.turn(d, true);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        f[i][e] *= rstd;
        dw[i][e] = __builtin_fmaf(d[i][e], f[i][e], dw[i][e]);
        d[i][e] *= w[i][e];
        dot = __builtin_fmaf(d[i][e], f[i][e], dot);
      }
    dot = group_sum<LANES>(dot) * a.inv_dim;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) d[i][e] = rstd * __builtin_fmaf(-f[i][e], dot, d[i][e]);
    store_two<T, V>(to, d, place.at, place.left, a.past);
  };
  if (r < s.rows_block)
    for (int64_t row = (int64_t)blockIdx.x * s.rows_block + r; row < n; row += (int64_t)gridDim.x * s.rows_block) {
      const T* x = static_cast<const T*>(which ? a.x[1] : a.x[0]) + row * (which ? a.x_row[1] : a.x_row[0]) + share.h0 * x_head;
      const T* dy = static_cast<const T*>(which ? a.dy[1] : a.dy[0]) + row * (which ? a.dy_row[1] : a.dy_row[0]) + share.h0 * dy_head;
      T* out = static_cast<T*>(which ? a.out[1] : a.out[0]) + row * (which ? a.out_row[1] : a.out_row[0]) + share.h0 * out_head;
      place.angles(a, row, lane);
      int h = share.h0;
      for (; h + 2 <= share.h1; h += 2, x += 2 * x_head, dy += 2 * dy_head, out += 2 * out_head) {
        Two<T, V> t[2], g[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          t[i] = load_two<T, V>(x + i * x_head, place.at, place.left, a.past);
          g[i] = load_two<T, V>(dy + i * dy_head, place.at, place.left, a.past);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) finish(t[i], g[i], out + i * out_head);
      }
      if (h < share.h1) finish(load_two<T, V>(x, place.at, place.left, a.past), load_two<T, V>(dy, place.at, place.left, a.past), out);
    }
  if (!a.partial) return;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (e < place.left[i]) s_sum[group][place.at[i] + e] = dw[i][e];
  __syncthreads();
  for (int c = threadIdx.x; c < 2 * a.dim; c += kHeadThreads) {
    const int k = c >= a.dim, at = c - (k ? a.dim : 0);
    const int first = k ? s.parts[0] : 0, end = k ? parts : s.parts[0];
    float t = 0.0f;
    for (int i = 0; i < s.rows_block; ++i)
      for (int p = first; p < end; ++p) t += s_sum[i * parts + p][at];
    a.partial[(int64_t)blockIdx.x * 2 * a.dim + c] = t;
  }
}

HeadShape head_shape(const HeadNormArgs& a, int32_t vec) {
  HeadShape s;
  const int32_t half = a.rotary_dim / 2;
  s.turned = (half + vec - 1) / vec;  // vec pairs a lane
  s.items = s.turned + (a.dim - a.rotary_dim + 2 * vec - 1) / (2 * vec);
  s.lanes = 4;
  while (s.lanes < s.items) s.lanes *= 2;
  // sixteen heads share an angle unless that leaves the chip under four waves a SIMD, or a row with more groups than
  // a workgroup has
  const int32_t heads = a.heads[0] + a.heads[1], groups = kHeadThreads / s.lanes;
  const int64_t wanted = 256 * 4 * 4 * 64;
  s.each = (int32_t)std::max<int64_t>(1, std::min<int64_t>(16, a.rows * s.lanes * heads / wanted));
  auto count = [&](int i) { return (a.heads[i] + s.each - 1) / s.each; };
  while (count(0) + count(1) > groups) ++s.each;
  s.parts[0] = count(0);
  s.parts[1] = count(1);
  s.rows_block = groups / (s.parts[0] + s.parts[1]);
  return s;
}

template <typename T, bool BACKWARD, int LANES>
void launch_lanes(const HeadNormArgs& a, const HeadShape& s, int64_t groups, hipStream_t st) {
  const dim3 grid((uint32_t)groups), block(kHeadThreads);
  if constexpr (BACKWARD) {
    if (a.interleaved)
      hipLaunchKernelGGL((head_norm_backward_kernel<T, true, LANES>), grid, block, 0, st, a, s);
    else
      hipLaunchKernelGGL((head_norm_backward_kernel<T, false, LANES>), grid, block, 0, st, a, s);
  } else {
    if (a.interleaved)
      hipLaunchKernelGGL((head_norm_kernel<T, true, LANES>), grid, block, 0, st, a, s);
    else
      hipLaunchKernelGGL((head_norm_kernel<T, false, LANES>), grid, block, 0, st, a, s);
  }
}

// dim <= 256, so at most 64 lanes of 2 packs hold a head.
template <typename T, bool BACKWARD>
void launch_groups(const HeadNormArgs& a, const HeadShape& s, int64_t groups, hipStream_t st) {
  switch (s.lanes) {
    case 4: launch_lanes<T, BACKWARD, 4>(a, s, groups, st); break;
    case 8: launch_lanes<T, BACKWARD, 8>(a, s, groups, st); break;
    case 16: launch_lanes<T, BACKWARD, 16>(a, s, groups, st); break;
    case 32: launch_lanes<T, BACKWARD, 32>(a, s, groups, st); break;
    default: launch_lanes<T, BACKWARD, 64>(a, s, groups, st);
  }
}

template <typename T>
hipError_t head_norm_of(const HeadNormArgs& a, hipStream_t st) {
  const HeadShape s = head_shape(a, kPackOf<T>);
  HeadNormArgs part = a;
  for (; part.first_row < a.rows; part.first_row += kMostGroups * s.rows_block) {
    const int64_t groups = std::min((a.rows - part.first_row + s.rows_block - 1) / s.rows_block, kMostGroups);
    launch_groups<T, false>(part, s, groups, st);
  }
  return hipGetLastError();
}

}  // namespace

int32_t head_norm_backward_grid(const HeadNormArgs& a, int32_t dtype) {
  const int64_t per = head_shape(a, dtype == MMBEV_F32 ? 4 : 8).rows_block;
  return (int32_t)std::max<int64_t>(1, std::min<int64_t>((a.rows + per - 1) / per, kNormGrid));
}

hipError_t launch_head_norm(const HeadNormArgs& a, int32_t dtype, hipStream_t st) {
  if (a.rows == 0) return hipSuccess;
  return dtype == MMBEV_F32   ? head_norm_of<float>(a, st)
         : dtype == MMBEV_F16 ? head_norm_of<f16>(a, st)
                              : head_norm_of<bf16>(a, st);
}

hipError_t launch_head_norm_backward(const HeadNormArgs& a, int32_t dtype, hipStream_t st) {
  const int32_t grid = head_norm_backward_grid(a, dtype);
  const HeadShape s = head_shape(a, dtype == MMBEV_F32 ? 4 : 8);
  if (dtype == MMBEV_F32)
    launch_groups<float, true>(a, s, grid, st);
  else if (dtype == MMBEV_F16)
    launch_groups<f16, true>(a, s, grid, st);
  else
    launch_groups<bf16, true>(a, s, grid, st);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.partial) return e;
  return launch_weight_sum(a.partial, grid, a.dim, a.dweight[0], a.dweight[1], st);
}

}  // namespace mmbev
