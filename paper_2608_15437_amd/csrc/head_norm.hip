// Norms of queries and keys for each head, turned by their positions in the
// same pass, and the gradients:
//   r = 1 / sqrt(mean(x^2) + eps),  h = x r,  y = R(h * w)
//   d = R^-1 dy,  a = d * w,  dx = r (a - h mean(a * h)),  dw = sum of d * h
//
// LANES neighbouring lanes hold a head, two 16-byte packs each: of the part
// that turns, the packs of the pairs' first and second elements or two packs of
// neighbouring pairs; of the rest, two packs that turn by nothing.  Where both
// parts have a whole pack (FULL) every access is one: the last pack of a part
// begins so that it ends with the part, lanes with none of their own do the
// last one's work, and what two lanes have counts once in the sums and is
// stored twice, the same.  A group of
// lanes takes several heads of one row and one array, so that it works the
// sines and cosines out and loads the weights once for all of them (the fewer
// rows, the fewer heads, so that small calls spread out).
// The operator moves bytes; beside them are some 15 operations an element and
// 50 a pair for its angle.  (Storing past the caches, as the other sequence
// operators' large calls do, costs here, where a store has 64 bytes a head:
// 921,997 rows of 8 + 4 heads 701 us instead of 566, gradients of 213,879 in
// fp32 676 instead of 554.)  Measured: 921,997 rows of 8 + 4 heads of 64 in
// bf16 571 us, 5.0 TB/s; gradients of 213,879 rows of 8 + 8 heads in fp32 501
// us, 5.2 TB/s, HBM's; of 18,608 rows of 4 + 4 heads of 100 in fp16 31 us, 2.9
// TB/s (200-byte heads, lanes that share elements, three axes' angles, and 1,163
// blocks of rows over 1,024 workgroups, of which 139 go round twice: with the
// sums' launch 33.6 us, of 16,384 rows, once round, 29.4, of 32,768, twice,
// 44.3); a frame's 5,442 rows in 10 us, the chain from position to angle to row.
//
// The weights' gradients: a group stays with its heads and walks the rows that
// its workgroup takes (every grid-th block of them) with its columns' sums in
// registers; the workgroup's groups add theirs in LDS, and a second launch adds
// the workgroups' rows, all in a fixed order.
#include <algorithm>
#include <type_traits>

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
  int32_t full, ragged;      // see FULL; some elements are two lanes'
};

// What a lane has of every head: where its packs are, and its pairs' angles.
template <typename T, bool INTERLEAVED, bool FULL>
struct Place {
  static constexpr int V = kPackOf<T>;
  int at[2];    // first element of a pack
  int left[2];  // elements from there on (not FULL)
  int skip[2];  // elements that are another lane's too (FULL)
  bool turned, ragged;
  float sn[V], cs[V];

  // The i-th of a part's packs, of its `size` elements from `begin` on.
  __device__ __forceinline__ void put(int which, int i, int begin, int size, bool there) {
    const int first = begin + i * V, last = begin + size - V;
    at[which] = FULL ? min(first, last) : first;
    left[which] = there ? begin + size - first : 0;
    skip[which] = there ? min(max(first - last, 0), V) : V;
  }
  __device__ __forceinline__ void set(const HeadNormArgs& a, const HeadShape& s, int lane) {
    const bool there = lane < s.items;
    if (FULL) lane = min(lane, s.items - 1);
    turned = lane < s.turned;
    ragged = s.ragged;
    // neighbouring lanes' first packs lie next to each other, and so do their second ones
    if (!turned) {
      put(0, lane - s.turned, a.rotary_dim, a.dim - a.rotary_dim, there);
      put(1, lane - s.turned + s.items - s.turned, a.rotary_dim, a.dim - a.rotary_dim, there);
    } else if (INTERLEAVED) {
      put(0, lane, 0, a.rotary_dim, there);
      put(1, lane + s.turned, 0, a.rotary_dim, there);
    } else {
      put(0, lane, 0, a.rotary_dim / 2, there);
      put(1, lane, a.rotary_dim / 2, a.rotary_dim / 2, there);
    }
  }
  // an element of the lane's own
  __device__ __forceinline__ bool own(int which, int e) const { return FULL ? e >= skip[which] : e < left[which]; }
  __device__ __forceinline__ int width(int which) const { return FULL ? V : left[which]; }
  __device__ __forceinline__ Pack<T, V> load(const T* x, int which) const {
    if constexpr (FULL)
      return load_pack<T, V>(x + at[which]);
    else
      return load_some<T, V>(x + at[which], left[which]);
  }
  __device__ __forceinline__ void store(T* x, int which, const Pack<T, V>& r) const {
    if constexpr (FULL)
      store_pack<T, V>(x + at[which], r);
    else
      store_some<T, V>(x + at[which], r, left[which]);
  }
  __device__ __forceinline__ void angles(const HeadNormArgs& a, int64_t row) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      sn[e] = 0.0f;
      cs[e] = 1.0f;
    }
    if (!turned) return;
    const int half = a.rotary_dim / 2;
    const int32_t* positions = a.positions + row * a.position_stride;
    // of up to four axes all are loaded together with the table, not after it
    int32_t of_axis[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) of_axis[i] = positions[min(i, a.axes - 1)];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      // pairs past the last turn by its angle; they are not stored
      const int pair = INTERLEAVED ? at[e / (V / 2)] / 2 + e % (V / 2) : at[0] + e;
      const int j = min(pair, half - 1), ax = min((int)a.axis[j], a.axes - 1);
      int32_t p = ax == 0 ? of_axis[0] : ax == 1 ? of_axis[1] : ax == 2 ? of_axis[2] : of_axis[3];
      if (a.axes > 4) p = positions[ax];
      const uint64_t phase = (uint64_t)(int64_t)p * a.steps[j];
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

template <typename P, typename T, int V>
__device__ __forceinline__ Two<T, V> load_two(const P& place, const T* x) {
  return {{place.load(x, 0), place.load(x, 1)}};
}

template <typename T, int V>
__device__ __forceinline__ void widen(float (&to)[2][V], const Two<T, V>& from) {
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int e = 0; e < V; ++e) to[i][e] = (float)from.p[i].v[e];
}

template <typename P, typename T, int V>
__device__ __forceinline__ void store_two(const P& place, T* x, const float (&f)[2][V]) {
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
    place.store(x, i, r);
  }
}

template <typename P, typename T, int V>
__device__ __forceinline__ void load_weights(const P& place, float (&w)[2][V], const void* p, bool f32) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (!p) {
#pragma unroll
      for (int e = 0; e < V; ++e) w[i][e] = 1.0f;
    } else if (f32) {
      const Pack<float, V> r = load_some<float, V>(static_cast<const float*>(p) + place.at[i], place.width(i));
#pragma unroll
      for (int e = 0; e < V; ++e) w[i][e] = r.v[e];
    } else {
      const Pack<T, V> r = load_some<T, V>(static_cast<const T*>(p) + place.at[i], place.width(i));
#pragma unroll
      for (int e = 0; e < V; ++e) w[i][e] = (float)r.v[e];
    }
  }
}

// Sum over the head of x * y, the lane's own elements (past the head both are zeros).
template <int LANES, typename P, int V>
__device__ __forceinline__ float head_sum(const P& place, const float (&x)[2][V], const float (&y)[2][V]) {
  float t = 0.0f;
  if (place.ragged) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) t = __builtin_fmaf(place.own(i, e) ? x[i][e] : 0.0f, y[i][e], t);
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) t = __builtin_fmaf(x[i][e], y[i][e], t);
  }
  return group_sum<LANES>(t);
}

// Reciprocal root of the mean square, off by a step at most.
template <int LANES, typename P, int V>
__device__ __forceinline__ float head_rstd(const P& place, const float (&x)[2][V], const HeadNormArgs& a) {
  return __builtin_amdgcn_rsqf(__builtin_fmaf(head_sum<LANES, P, V>(place, x, x), a.inv_dim, a.eps));
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

template <typename T, bool INTERLEAVED, int LANES, bool FULL>
__global__ __launch_bounds__(kHeadThreads) void head_norm_kernel(HeadNormArgs a, HeadShape s) {
  constexpr int V = kPackOf<T>;
  const int64_t n = rows_in_use(a.row_count, a.rows, a.fault);
  const int parts = s.parts[0] + s.parts[1], group = threadIdx.x / LANES, lane = threadIdx.x % LANES;
  const int r = group / parts;
  const int64_t row = a.first_row + (int64_t)blockIdx.x * s.rows_block + r;
  if (r >= s.rows_block || row >= n) return;
  const Share share(a, s, group - r * parts);
  const int which = share.which;
  using P = Place<T, INTERLEAVED, FULL>;
  P place;
  place.set(a, s, lane);
  float w[2][V];
  load_weights<P, T, V>(place, w, which ? a.weight[1] : a.weight[0], a.weight_f32);
  const int64_t x_head = which ? a.x_head[1] : a.x_head[0], out_head = which ? a.out_head[1] : a.out_head[0];
  const T* x = static_cast<const T*>(which ? a.x[1] : a.x[0]) + row * (which ? a.x_row[1] : a.x_row[0]);
  T* out = static_cast<T*>(which ? a.out[1] : a.out[0]) + row * (which ? a.out_row[1] : a.out_row[0]);
  auto load = [&](Two<T, V> (&t)[kHeadsAtOnce], int h) {
#pragma unroll
    for (int i = 0; i < kHeadsAtOnce; ++i) t[i] = load_two<P, T, V>(place, x + (int64_t)min(h + i, share.h1 - 1) * x_head);
  };
  auto finish = [&](const Two<T, V>& from, T* to) {
    float f[2][V];
    widen<T, V>(f, from);
    const float rstd = head_rstd<LANES, P, V>(place, f, a);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) f[i][e] = f[i][e] * rstd * w[i][e];
    place.turn(f, false);
    store_two<P, T, V>(place, to, f);
  };
  // the first heads' loads before the angles' work, the next ones' before these are stored
  Two<T, V> t[kHeadsAtOnce], next[kHeadsAtOnce];
  load(t, share.h0);
  place.angles(a, row);
  for (int h = share.h0; h < share.h1; h += kHeadsAtOnce) {
    if (h + kHeadsAtOnce < share.h1) load(next, h + kHeadsAtOnce);
#pragma unroll
    for (int i = 0; i < kHeadsAtOnce; ++i) {
      if (h + i < share.h1) finish(t[i], out + (int64_t)(h + i) * out_head);
      t[i] = next[i];
    }
  }
}

template <typename T, bool INTERLEAVED, int LANES, bool FULL>
__global__ __launch_bounds__(kHeadThreads) void head_norm_backward_kernel(HeadNormArgs a, HeadShape s) {
  constexpr int V = kPackOf<T>;
  __shared__ float s_sum[kHeadThreads / LANES][LANES * 2 * V + 1];
  const int64_t n = rows_in_use(a.row_count, a.rows, a.fault);
  const int parts = s.parts[0] + s.parts[1], group = threadIdx.x / LANES, lane = threadIdx.x % LANES;
  const int r = group / parts;
  const Share share(a, s, group - r * parts);
  const int which = share.which;
  using P = Place<T, INTERLEAVED, FULL>;
  P place;
  place.set(a, s, lane);
  float w[2][V], dw[2][V];
  load_weights<P, T, V>(place, w, which ? a.weight[1] : a.weight[0], a.weight_f32);
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int e = 0; e < V; ++e) dw[i][e] = 0.0f;
  const int64_t x_head = which ? a.x_head[1] : a.x_head[0], dy_head = which ? a.dy_head[1] : a.dy_head[0],
                out_head = which ? a.out_head[1] : a.out_head[0];
  auto finish = [&](const Two<T, V>& from, const Two<T, V>& grad, T* to) {
    float f[2][V], d[2][V];
    widen<T, V>(f, from);
    widen<T, V>(d, grad);
    const float rstd = head_rstd<LANES, P, V>(place, f, a);
    place.turn(d, true);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        f[i][e] *= rstd;
        dw[i][e] = __builtin_fmaf(d[i][e], f[i][e], dw[i][e]);
        d[i][e] *= w[i][e];
      }
    const float dot = head_sum<LANES, P, V>(place, d, f) * a.inv_dim;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) d[i][e] = rstd * __builtin_fmaf(-f[i][e], dot, d[i][e]);
    store_two<P, T, V>(place, to, d);
  };
  if (r < s.rows_block)
    for (int64_t row = (int64_t)blockIdx.x * s.rows_block + r; row < n; row += (int64_t)gridDim.x * s.rows_block) {
      const T* x = static_cast<const T*>(which ? a.x[1] : a.x[0]) + row * (which ? a.x_row[1] : a.x_row[0]);
      const T* dy = static_cast<const T*>(which ? a.dy[1] : a.dy[0]) + row * (which ? a.dy_row[1] : a.dy_row[0]);
      T* out = static_cast<T*>(which ? a.out[1] : a.out[0]) + row * (which ? a.out_row[1] : a.out_row[0]);
      for (int h = share.h0; h < share.h1; h += 2) {
        const int other = min(h + 1, share.h1 - 1);
        const Two<T, V> t[2] = {load_two<P, T, V>(place, x + h * x_head), load_two<P, T, V>(place, x + other * x_head)};
        const Two<T, V> g[2] = {load_two<P, T, V>(place, dy + h * dy_head), load_two<P, T, V>(place, dy + other * dy_head)};
        if (h == share.h0) place.angles(a, row);
        finish(t[0], g[0], out + h * out_head);
        if (other != h) finish(t[1], g[1], out + other * out_head);
      }
    }
  if (!a.partial) return;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (place.own(i, e)) s_sum[group][place.at[i] + e] = dw[i][e];
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
  const int32_t rest = a.dim - a.rotary_dim, part = a.interleaved ? a.rotary_dim : half;
  s.full = part >= vec && (rest == 0 || rest >= vec);
  s.lanes = 4;
  while (s.lanes < s.items) s.lanes *= 2;
  s.ragged = s.lanes > s.items || part % (a.interleaved ? 2 * vec : vec) != 0 || rest % (2 * vec) != 0;
  // At most sixteen heads share their angles, and no more than leave the chip two waves a SIMD; a workgroup has room for
  // a row's groups.  Groups wait for those with most heads, and an angle costs about as much as three heads: of 8 + 4 heads
  // in groups of 4, 921,997 rows took 755 us, in groups of 8 864.
  const int32_t heads = a.heads[0] + a.heads[1], groups = kHeadThreads / s.lanes;
  const int64_t wanted = 256 * 4 * 2 * 64;
  const int32_t most = (int32_t)std::max<int64_t>(1, std::min<int64_t>(16, a.rows * s.lanes * heads / wanted));
  auto count = [&](int i, int32_t each) { return (a.heads[i] + each - 1) / each; };
  int64_t best = INT64_MAX;
  for (int32_t each = 1; each <= 1024; ++each) {
    const int64_t parts = count(0, each) + count(1, each);
    if (parts > groups) continue;
    if (each > most && best != INT64_MAX) break;
    if (parts * (each + 3) < best) {
      best = parts * (each + 3);
      s.each = each;
    }
  }
  s.parts[0] = count(0, s.each);
  s.parts[1] = count(1, s.each);
  s.rows_block = groups / (s.parts[0] + s.parts[1]);
  return s;
}

template <typename T, bool BACKWARD, int LANES>
void launch_lanes(const HeadNormArgs& a, const HeadShape& s, int64_t groups, hipStream_t st) {
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((uint32_t)groups), dim3(kHeadThreads), 0, st, a, s); };
  auto full = [&](auto which) {
    constexpr bool FULL = decltype(which)::value;
    if constexpr (BACKWARD)
      a.interleaved ? go(head_norm_backward_kernel<T, true, LANES, FULL>) : go(head_norm_backward_kernel<T, false, LANES, FULL>);
    else
      a.interleaved ? go(head_norm_kernel<T, true, LANES, FULL>) : go(head_norm_kernel<T, false, LANES, FULL>);
  };
  s.full ? full(std::true_type{}) : full(std::false_type{});
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
