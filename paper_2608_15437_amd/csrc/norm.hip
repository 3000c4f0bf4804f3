// Layer norm over rows and its gradients, with the residual sum of the block
// in the forward pass and the skip connection's gradient in the backward one.
//
// Both passes read each row once and keep it in registers: LANES neighbouring
// lanes hold a row, PACKS 16-byte packs each, so that a 64-wide row of 16-bit
// elements takes 8 lanes and a wave has eight rows in flight.  The mean and
// the centred sum of squares are two passes over registers (the variance of
// values far from zero keeps its bits), each a butterfly of register moves.
// They move bytes and nothing else bounds them: about 20 operations an
// element against the chip's 32 per byte.  Rows of 921,997 x 256 bf16: 303 us
// with the residual sum (6.2 TB/s), 347 for the gradients with the skip
// connection's (5.5 TB/s).
//
// The weight's gradient is a sum over all rows of products whose columns lie
// across the lanes.  Each thread keeps its columns' sums in registers over the
// rows that its workgroup takes (every grid-th group of rows), the workgroup's
// threads add theirs in LDS, and a second launch adds the workgroups' rows of
// partial sums in a fixed order: no atomics, the same bits every time.
#include <algorithm>

#include "sequence.hpp"

namespace mmbev {

namespace {

constexpr int kNormThreads = 256;

// Weight or bias of the thread's columns (fp32 or the rows' type).
template <typename T, int VEC>
__device__ __forceinline__ void load_weight(float (&w)[VEC], const void* p, bool f32, int c, int n, float none) {
  if (!p) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) w[e] = none;
    return;
  }
  if (f32) {
    const Pack<float, VEC> r = load_some<float, VEC>(static_cast<const float*>(p) + c, n);
#pragma unroll
    for (int e = 0; e < VEC; ++e) w[e] = r.v[e];
  } else {
    const Pack<T, VEC> r = load_some<T, VEC>(static_cast<const T*>(p) + c, n);
#pragma unroll
    for (int e = 0; e < VEC; ++e) w[e] = (float)r.v[e];
  }
}

// Sum over the lanes of a row: a group of a wave, or all of the workgroup's
// waves through LDS (s_part: one word a wave; its first barrier also keeps
// the words of the sum before).
template <int LANES>
__device__ __forceinline__ float row_sum(float x, float* s_part) {
  if constexpr (LANES <= 64) {
    return group_sum<LANES>(x);
  } else {
    x = group_sum<64>(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s_part[threadIdx.x >> 6] = x;
    __syncthreads();
    float t = 0.0f;
#pragma unroll
    for (int w = 0; w < LANES / 64; ++w) t += s_part[w];
    return t;
  }
}

template <typename T, int LANES, int PACKS>
__global__ __launch_bounds__(kNormThreads) void norm_kernel(NormArgs a) {
  constexpr int VEC = kPackOf<T>, ROWS = kNormThreads / LANES;
  __shared__ float s_part[4];
  const int64_t n = rows_in_use(a.row_count, a.rows, a.fault);
  const int64_t row0 = a.first_row + (int64_t)blockIdx.x * ROWS, row = row0 + threadIdx.x / LANES;
  const int lane = threadIdx.x % LANES;
  if (row0 >= n) return;
  const bool live = row < n;
  float f[PACKS][VEC];
  float sum = 0.0f;
  if (live) {
    const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
    const T* res = a.skip ? static_cast<const T*>(a.skip) + row * a.skip_stride : nullptr;
#pragma unroll
    for (int p = 0; p < PACKS; ++p) {
      const int c = (p * LANES + lane) * VEC;
      const Pack<T, VEC> r = load_some<T, VEC>(x + c, a.width - c);
#pragma unroll
      for (int e = 0; e < VEC; ++e) f[p][e] = (float)r.v[e];
    }
    if (res) {
#pragma unroll
      for (int p = 0; p < PACKS; ++p) {
        const int c = (p * LANES + lane) * VEC;
        Pack<T, VEC> r = load_some<T, VEC>(res + c, a.width - c);
        // the norm is taken of the rounded sum: it is what the backward pass will read
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          r.v[e] = (T)(f[p][e] + (float)r.v[e]);
          f[p][e] = (float)r.v[e];
        }
        if (a.sum) store_some<T, VEC>(static_cast<T*>(a.sum) + row * a.sum_stride + c, r, a.width - c, a.past);
      }
    } else if (a.sum) {
#pragma unroll
      for (int p = 0; p < PACKS; ++p) {
        const int c = (p * LANES + lane) * VEC;
        Pack<T, VEC> r;
#pragma unroll
        for (int e = 0; e < VEC; ++e) r.v[e] = (T)f[p][e];
        store_some<T, VEC>(static_cast<T*>(a.sum) + row * a.sum_stride + c, r, a.width - c, a.past);
      }
    }
#pragma unroll
    for (int p = 0; p < PACKS; ++p)
#pragma unroll
      for (int e = 0; e < VEC; ++e) sum += f[p][e];
  }
  const float mean = row_sum<LANES>(sum, s_part) * a.inv_width;
  float sq = 0.0f;
  if (live) {
#pragma unroll
    for (int p = 0; p < PACKS; ++p) {
      const int left = a.width - (p * LANES + lane) * VEC;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        f[p][e] -= mean;
        if (e < left) sq = __builtin_fmaf(f[p][e], f[p][e], sq);
      }
    }
  }
  const float var = row_sum<LANES>(sq, s_part) * a.inv_width;
  const float rstd = 1.0f / __builtin_sqrtf(var + a.eps);
  if (!live) return;
  if (lane == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
  T* out = static_cast<T*>(a.out) + row * a.out_stride;
#pragma unroll
  for (int p = 0; p < PACKS; ++p) {
    const int c = (p * LANES + lane) * VEC, left = a.width - c;
    float w[VEC], b[VEC];
    load_weight<T, VEC>(w, a.weight, a.weight_f32, c, left, 1.0f);
    load_weight<T, VEC>(b, a.bias, a.weight_f32, c, left, 0.0f);
    Pack<T, VEC> r;
#pragma unroll
    for (int e = 0; e < VEC; ++e) r.v[e] = (T)__builtin_fmaf(f[p][e] * rstd, w[e], b[e]);
    store_some<T, VEC>(out + c, r, left, a.past);
  }
}

template <typename T, int LANES, int PACKS>
__global__ __launch_bounds__(kNormThreads) void norm_backward_kernel(NormArgs a) {
  constexpr int VEC = kPackOf<T>, ROWS = kNormThreads / LANES;
  __shared__ float s_part[4];
  const int64_t n = rows_in_use(a.row_count, a.rows, a.fault);
  const int lane = threadIdx.x % LANES;
  float dw[PACKS][VEC], db[PACKS][VEC], w[PACKS][VEC];
#pragma unroll
  for (int p = 0; p < PACKS; ++p) {
    const int c = (p * LANES + lane) * VEC;
    load_weight<T, VEC>(w[p], a.weight, a.weight_f32, c, a.width - c, 1.0f);
#pragma unroll
    for (int e = 0; e < VEC; ++e) dw[p][e] = db[p][e] = 0.0f;
  }
  for (int64_t row0 = (int64_t)blockIdx.x * ROWS; row0 < n; row0 += (int64_t)gridDim.x * ROWS) {
    const int64_t row = row0 + threadIdx.x / LANES;
    const bool live = row < n;
    float g[PACKS][VEC], h[PACKS][VEC];
    float rstd = 0.0f, s1 = 0.0f, s2 = 0.0f;
    if (live) {
      const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
      const T* dy = static_cast<const T*>(a.dy) + row * a.dy_stride;
      const float mean = a.mean[row];
      rstd = a.rstd[row];
#pragma unroll
      for (int p = 0; p < PACKS; ++p) {
        const int c = (p * LANES + lane) * VEC, left = a.width - c;
        const Pack<T, VEC> rx = load_some<T, VEC>(x + c, left), rd = load_some<T, VEC>(dy + c, left);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float d = (float)rd.v[e];  // zero past the row: its terms vanish
          h[p][e] = e < left ? ((float)rx.v[e] - mean) * rstd : 0.0f;
          dw[p][e] = __builtin_fmaf(d, h[p][e], dw[p][e]);
          db[p][e] += d;
          g[p][e] = d * w[p][e];
          s1 += g[p][e];
          s2 = __builtin_fmaf(g[p][e], h[p][e], s2);
        }
      }
    }
    s1 = row_sum<LANES>(s1, s_part) * a.inv_width;
    s2 = row_sum<LANES>(s2, s_part) * a.inv_width;
    if (!live) continue;
    T* dx = static_cast<T*>(a.out) + row * a.out_stride;
#pragma unroll
    for (int p = 0; p < PACKS; ++p) {
      const int c = (p * LANES + lane) * VEC, left = a.width - c;
      float k[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) k[e] = rstd * (g[p][e] - s1 - h[p][e] * s2);
      if (a.skip) {
        const Pack<T, VEC> rs = load_some<T, VEC>(static_cast<const T*>(a.skip) + row * a.skip_stride + c, left);
#pragma unroll
        for (int e = 0; e < VEC; ++e) k[e] += (float)rs.v[e];
      }
      Pack<T, VEC> r;
#pragma unroll
      for (int e = 0; e < VEC; ++e) r.v[e] = (T)k[e];
      store_some<T, VEC>(dx + c, r, left, a.past);
    }
  }
  if (!a.partial) return;
  // the workgroup's ROWS row slots added in LDS, in slot order
  float* out = a.partial + (int64_t)blockIdx.x * 2 * a.width;
  if constexpr (ROWS == 1) {
#pragma unroll
    for (int p = 0; p < PACKS; ++p) {
      const int c = (p * LANES + lane) * VEC;
      Pack<float, VEC> u, v;
#pragma unroll
      for (int e = 0; e < VEC; ++e) u.v[e] = dw[p][e], v.v[e] = db[p][e];
      store_some<float, VEC>(out + c, u, a.width - c);
      store_some<float, VEC>(out + a.width + c, v, a.width - c);
    }
  } else {
    constexpr int COLS = LANES * VEC;  // one pack of every lane at a time
    __shared__ float s_sum[ROWS][COLS + 1];
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
      for (int p = 0; p < PACKS; ++p) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < VEC; ++e) s_sum[threadIdx.x / LANES][lane * VEC + e] = which ? db[p][e] : dw[p][e];
        __syncthreads();
        for (int c = threadIdx.x; c < COLS; c += kNormThreads) {
          float t = 0.0f;
#pragma unroll 8
          for (int r = 0; r < ROWS; ++r) t += s_sum[r][c];
          if (p * COLS + c < a.width) out[which * a.width + p * COLS + c] = t;
        }
      }
  }
}

// dweight and dbias: the workgroups' partial rows added up, few columns a
// workgroup so that its threads' loads are all in flight together (32 columns
// and eight threads a column, one after the other: 13 us for 1,024 rows).
constexpr int kSumCols = 16, kSumParts = 64;

__global__ __launch_bounds__(kSumCols * kSumParts) void norm_weight_sum_kernel(const float* partial, int32_t parts, int32_t width,
                                                                               float* dweight, float* dbias) {
  __shared__ float s_sum[kSumParts][kSumCols + 1];
  const int col = threadIdx.x % kSumCols, part = threadIdx.x / kSumCols;
  const int c = blockIdx.x * kSumCols + col, at = min(c, 2 * width - 1);
  float x[kNormGrid / kSumParts];
#pragma unroll
  for (int i = 0; i < kNormGrid / kSumParts; ++i) x[i] = partial[(int64_t)min(part + i * kSumParts, parts - 1) * 2 * width + at];
  float t = 0.0f;
#pragma unroll
  for (int i = 0; i < kNormGrid / kSumParts; ++i) t += part + i * kSumParts < parts ? x[i] : 0.0f;
  s_sum[part][col] = t;
  __syncthreads();
  if (part != 0 || c >= 2 * width) return;
  t = 0.0f;
#pragma unroll
  for (int i = 0; i < kSumParts; ++i) t += s_sum[i][col];
  if (c < width) {
    if (dweight) dweight[c] = t;
  } else if (dbias) {
    dbias[c - width] = t;
  }
}

// Lanes that hold a row: the fewest that need one pack each, at most a wave;
// wider rows take up to four packs a lane, then the whole workgroup.
struct NormShape {
  int lanes, packs;
};

NormShape norm_shape(int32_t width, int32_t dtype) {
  const int vec = dtype == MMBEV_F32 ? 4 : 8;
  const int packs = (width + vec - 1) / vec;
  if (packs > 256 * 4) return {256, 8};
  if (packs > 256 * 2) return {256, 4};
  if (packs > 256) return {256, 2};
  if (packs > 128) return {64, 4};
  if (packs > 64) return {64, 2};
  int lanes = 1;
  while (lanes < packs) lanes *= 2;
  return {lanes, 1};
}

template <typename T, typename F>
hipError_t with_shape(NormShape s, F&& f) {
  switch (s.lanes) {
    case 1: f(std::integral_constant<int, 1>{}, std::integral_constant<int, 1>{}); break;
    case 2: f(std::integral_constant<int, 2>{}, std::integral_constant<int, 1>{}); break;
    case 4: f(std::integral_constant<int, 4>{}, std::integral_constant<int, 1>{}); break;
    case 8: f(std::integral_constant<int, 8>{}, std::integral_constant<int, 1>{}); break;
    case 16: f(std::integral_constant<int, 16>{}, std::integral_constant<int, 1>{}); break;
    case 32: f(std::integral_constant<int, 32>{}, std::integral_constant<int, 1>{}); break;
    case 64:
      if (s.packs == 1) f(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{});
      if (s.packs == 2) f(std::integral_constant<int, 64>{}, std::integral_constant<int, 2>{});
      if (s.packs == 4) f(std::integral_constant<int, 64>{}, std::integral_constant<int, 4>{});
      break;
    default:
      if (s.packs == 2) f(std::integral_constant<int, 256>{}, std::integral_constant<int, 2>{});
      if (s.packs == 4) f(std::integral_constant<int, 256>{}, std::integral_constant<int, 4>{});
      if constexpr (sizeof(T) == 4)
        if (s.packs == 8) f(std::integral_constant<int, 256>{}, std::integral_constant<int, 8>{});
  }
  return hipGetLastError();
}

template <typename T>
hipError_t norm_of(const NormArgs& a, NormShape s, hipStream_t st) {
  return with_shape<T>(s, [&](auto lanes, auto packs) {
    constexpr int rows = kNormThreads / lanes.value;
    NormArgs part = a;
    for (; part.first_row < a.rows; part.first_row += kMostGroups * rows) {
      const int64_t groups = std::min((a.rows - part.first_row + rows - 1) / rows, kMostGroups);
      hipLaunchKernelGGL((norm_kernel<T, lanes.value, packs.value>), dim3((uint32_t)groups), dim3(kNormThreads), 0, st, part);
    }
  });
}

template <typename T>
hipError_t norm_backward_of(const NormArgs& a, NormShape s, int32_t grid, hipStream_t st) {
  return with_shape<T>(s, [&](auto lanes, auto packs) {
    hipLaunchKernelGGL((norm_backward_kernel<T, lanes.value, packs.value>), dim3((uint32_t)grid), dim3(kNormThreads), 0, st, a);
  });
}

}  // namespace

int32_t norm_backward_grid(int64_t rows, int32_t width, int32_t dtype) {
  const int per = kNormThreads / norm_shape(width, dtype).lanes;
  return (int32_t)std::max<int64_t>(1, std::min<int64_t>((rows + per - 1) / per, kNormGrid));
}

hipError_t launch_norm(const NormArgs& a, int32_t dtype, hipStream_t st) {
  if (a.rows == 0) return hipSuccess;
  const NormShape s = norm_shape(a.width, dtype);
  return dtype == MMBEV_F32   ? norm_of<float>(a, s, st)
         : dtype == MMBEV_F16 ? norm_of<f16>(a, s, st)
                              : norm_of<bf16>(a, s, st);
}

hipError_t launch_weight_sum(const float* partial, int32_t parts, int32_t width, float* first, float* second, hipStream_t st) {
  hipLaunchKernelGGL(norm_weight_sum_kernel, dim3((uint32_t)((2 * width + kSumCols - 1) / kSumCols)), dim3(kSumCols * kSumParts), 0,
                     st, partial, parts, width, first, second);
  return hipGetLastError();
}

hipError_t launch_norm_backward(const NormArgs& a, int32_t dtype, hipStream_t st) {
  const NormShape s = norm_shape(a.width, dtype);
  const int32_t grid = norm_backward_grid(a.rows, a.width, dtype);
  const hipError_t e = dtype == MMBEV_F32   ? norm_backward_of<float>(a, s, grid, st)
                       : dtype == MMBEV_F16 ? norm_backward_of<f16>(a, s, grid, st)
                                            : norm_backward_of<bf16>(a, s, grid, st);
  if (e != hipSuccess || !a.partial) return e;
  return launch_weight_sum(a.partial, grid, a.width, a.dweight, a.dbias, st);
}

}  // namespace mmbev
