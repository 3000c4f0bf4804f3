// Linear attention: what does not depend on the element type's products (the
// joining of segments, the sum over heads that share keys and values, the
// single-row step) and the dispatch over types.
#include <algorithm>

#include "attention.hpp"
#include "attention_types.hpp"

namespace mmbev {

namespace {

// The states at the segments' ends, carried on: seg_state[s] becomes the
// state after segment s of the sequence that goes on beyond it.  One thread
// an element of the state, segments in order; their loads do not wait for
// each other.
__global__ __launch_bounds__(256) void attention_join_kernel(AttnArgs a) {
  const int64_t each = (int64_t)a.ad * a.cd, all = each * a.H;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= all) return;
  const Order o = order_of(a);
  const int64_t per = segment_rows(o.used, a.segments);
  const int32_t count = (int32_t)((o.used + per - 1) / per);
  const float fade = __builtin_amdgcn_exp2f(decay_exponent(a.log_decay, (int)(i / each)) * (float)per);
  float x = 0.0f;
#pragma unroll 8
  for (int32_t s = 0; s + 1 < count; ++s) {
    float* p = a.seg_state + s * all + i;
    const float own = *p;
    x = a.seg_fresh[s] ? own : __builtin_fmaf(fade, x, own);
    *p = x;
  }
}

// Gradients of shared keys and values: the heads' parts added in order, in
// fp32, and rounded once.
template <typename T>
__global__ __launch_bounds__(256) void attention_sum_kernel(AttnSumArgs a) {
  const int64_t end = a.offsets[a.B], used = end < 0 ? 0 : end > a.rows ? a.rows : end;
  const int kv = a.H / a.group, per_row = kv * a.dim;
  const int64_t step = (int64_t)gridDim.x * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < used * per_row; i += step) {
    const int64_t row = i / per_row;
    const int u = (int)(i - row * per_row), hk = u / a.dim, c = u - hk * a.dim;
    const float* p = a.part + (row * a.H + hk * a.group) * a.dim + c;
    float t = 0.0f;
    for (int j = 0; j < a.group; ++j) t += p[(int64_t)j * a.dim];
    static_cast<T*>(a.out)[row * a.out_row + hk * a.out_head + c] = (T)t;
  }
}

// One row of a stream: its state read, decayed, updated and written once.
// Bound by the state's bytes.  A thread has four neighbouring columns of
// every (256 / lanes)-th state row, lanes enough for a row of the state; the
// rows' parts of the output meet in LDS.
template <typename T, int LANES>
__global__ __launch_bounds__(256) void attention_step_kernel(AttnStepArgs a) {
  constexpr int PARTS = 256 / LANES;
  __shared__ float s_q[128], s_k[128];
  __shared__ float s_out[PARTS][LANES * 4 + 4];
  const int h = blockIdx.x % a.H;
  const int64_t r = blockIdx.x / a.H;
  const int64_t slot = a.slots ? (int64_t)a.slots[r] : r;
  if (slot < 0) return;
  if (slot >= a.num_slots) {
    if (a.fault && threadIdx.x == 0) atomicOr(a.fault, MMBEV_FAULT_SEQUENCES);
    return;
  }
  const int hk = h / a.group;
  for (int i = threadIdx.x; i < a.kd; i += 256) {
    s_q[i] = (float)static_cast<const T*>(a.q)[r * a.q_row + h * a.q_head + i];
    s_k[i] = (float)static_cast<const T*>(a.k)[r * a.k_row + hk * a.k_head + i];
  }
  const int lane = threadIdx.x % LANES, part = threadIdx.x / LANES, c = lane * 4;
  const Pack<T, 4> rv = load_some<T, 4>(static_cast<const T*>(a.v) + r * a.v_row + hk * a.v_head + c, a.vd - c);
  const float lambda = __expf(fmaxf(fminf(a.log_decay[h], 0.0f), -1.0e4f));
  float* state = a.state + (slot * a.H + h) * a.kd * a.vd;
  __syncthreads();
  float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int i = part; i < a.kd; i += PARTS) {
    Pack<float, 4> s = load_some<float, 4>(state + i * a.vd + c, a.vd - c);
    const float ki = s_k[i], qi = s_q[i];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      s.v[e] = __builtin_fmaf(lambda, s.v[e], ki * (float)rv.v[e]);
      acc[e] = __builtin_fmaf(qi, s.v[e], acc[e]);
    }
    store_some<float, 4>(state + i * a.vd + c, s, a.vd - c);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) s_out[part][c + e] = acc[e];
  __syncthreads();
  if (threadIdx.x < a.vd) {
    float t = 0.0f;
#pragma unroll
    for (int p = 0; p < PARTS; ++p) t += s_out[p][threadIdx.x];
    static_cast<T*>(a.out)[r * a.o_row + h * a.o_head + threadIdx.x] = (T)(t * a.scale);
  }
}

template <typename T>
hipError_t step_of(const AttnStepArgs& a, hipStream_t st) {
  const dim3 grid((uint32_t)(a.rows * a.H));
  if (a.vd <= 32)
    hipLaunchKernelGGL((attention_step_kernel<T, 8>), grid, dim3(256), 0, st, a);
  else if (a.vd <= 64)
    hipLaunchKernelGGL((attention_step_kernel<T, 16>), grid, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((attention_step_kernel<T, 32>), grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

// Offsets that break the contract: 0 .. <= rows, non-decreasing.
__global__ __launch_bounds__(256) void attention_check_kernel(const int64_t* offsets, int32_t B, int64_t rows, int32_t* fault) {
  const int32_t b = blockIdx.x * 256 + threadIdx.x;
  if (b >= B) return;
  const int64_t o0 = offsets[b], o1 = offsets[b + 1];
  if ((b == 0 && o0 != 0) || o1 < o0 || o1 > rows) atomicOr(fault, MMBEV_FAULT_SEQUENCES);
}

hipError_t chunks_of(const AttnArgs& a, int32_t dtype, bool state_only, hipStream_t st) {
  return dtype == MMBEV_F32   ? launch_attention_f32(a, state_only, st)
         : dtype == MMBEV_F16 ? launch_attention_f16(a, state_only, st)
                              : launch_attention_bf16(a, state_only, st);
}

}  // namespace

hipError_t launch_attention(const AttnArgs& a, int32_t dtype, hipStream_t st) {
  if (a.fault)
    hipLaunchKernelGGL(attention_check_kernel, dim3((a.B + 255) / 256), dim3(256), 0, st, a.offsets, a.B, a.rows, a.fault);
  if (a.segments) {
    const hipError_t e = chunks_of(a, dtype, true, st);
    if (e != hipSuccess) return e;
    const int64_t all = (int64_t)a.H * a.ad * a.cd;
    hipLaunchKernelGGL(attention_join_kernel, dim3((uint32_t)((all + 255) / 256)), dim3(256), 0, st, a);
  }
  return chunks_of(a, dtype, false, st);
}

hipError_t launch_attention_sum(const AttnSumArgs& a, int32_t dtype, hipStream_t st) {
  const int64_t items = a.rows * (a.H / a.group) * a.dim;
  const dim3 grid((uint32_t)std::max<int64_t>(1, std::min<int64_t>((items + 255) / 256, 16384)));
  if (dtype == MMBEV_F32)
    hipLaunchKernelGGL(attention_sum_kernel<float>, grid, dim3(256), 0, st, a);
  else if (dtype == MMBEV_F16)
    hipLaunchKernelGGL(attention_sum_kernel<f16>, grid, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL(attention_sum_kernel<bf16>, grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_attention_step(const AttnStepArgs& a, int32_t dtype, hipStream_t st) {
  if (a.rows == 0) return hipSuccess;
  return dtype == MMBEV_F32 ? step_of<float>(a, st) : dtype == MMBEV_F16 ? step_of<f16>(a, st) : step_of<bf16>(a, st);
}

}  // namespace mmbev
