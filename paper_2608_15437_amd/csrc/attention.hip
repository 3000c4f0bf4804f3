// Linear attention: what does not depend on the element type's products (the
// joining of cut sequences, the sum over heads that share keys and values, the
// single-row step) and the dispatch over types.
#include <algorithm>

#include "attention.hpp"
#include "attention_types.hpp"

namespace mmbev {

namespace {

// The states at the ends of the parts that go on, carried on through their
// sequences.  A workgroup has 64 elements of the state and its waves take
// neighbouring runs of parts: each carries its own from nothing, the runs'
// ends are carried through LDS, and what comes into a run is added to its
// states with their decay.  So the loads of kJoinWaves * kJoinRun parts are in
// flight together (one wave going through a keyframe's 94 parts, 32 loads at a
// time: 11.8 us).
constexpr int kJoinWaves = 8, kJoinRun = 12;

__global__ __launch_bounds__(kJoinWaves * 64) void attention_join_kernel(AttnPair pair) {
  __shared__ float s_end[kJoinWaves][64];
  __shared__ int32_t s_rows[kJoinWaves];  // of a run that no sequence begins in, else -1
  const AttnArgs& a = pair.walk[blockIdx.z];
  const int64_t each = (int64_t)a.ad * a.cd, all = each * a.H;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int at = blockIdx.x * 64 + lane;
  const bool there = at < each;
  const int64_t i = blockIdx.y * each + min(at, (int)each - 1);
  const Exponent log2 = decay_exponent(a.log_decay, blockIdx.y);
  float carry = 0.0f;
  for (int32_t s0 = 0; s0 < a.cuts; s0 += kJoinWaves * kJoinRun) {
    const int32_t first = s0 + w * kJoinRun;
    float x[kJoinRun];
    int32_t rows[kJoinRun];
#pragma unroll
    for (int j = 0; j < kJoinRun; ++j) {
      const int32_t s = min(first + j, a.cuts - 1);
      x[j] = a.cut_state[s * all + i];
      rows[j] = __builtin_amdgcn_readfirstlane(a.cut_rows[s]);
    }
    int32_t run = rows[0] > 0 ? rows[0] : -1;
#pragma unroll
    for (int j = 1; j < kJoinRun; ++j) {
      if (rows[j] > 0) x[j] = __builtin_fmaf(power(log2, rows[j]), x[j - 1], x[j]);
      run = rows[j] > 0 && run > 0 ? run + rows[j] : -1;
    }
    s_end[w][lane] = x[kJoinRun - 1];
    if (lane == 0) s_rows[w] = run;
    __syncthreads();
    float in = carry;
#pragma unroll
    for (int v = 0; v < kJoinWaves; ++v) {
      if (v == w) in = carry;
      const int32_t r = s_rows[v];
      carry = r > 0 ? __builtin_fmaf(power(log2, r), carry, s_end[v][lane]) : s_end[v][lane];
    }
    __syncthreads();
    bool open = true;  // no sequence has begun since the run's first part
    int32_t upto = 0;
#pragma unroll
    for (int j = 0; j < kJoinRun; ++j) {
      open = open && rows[j] > 0;
      upto += rows[j];
      if (open) x[j] = __builtin_fmaf(power(log2, upto), in, x[j]);
      if (there && first + j < a.cuts && rows[j] > 0) a.cut_state[(first + j) * all + i] = x[j];
    }
  }
}

// Gradients of keys and values that many heads share: the workgroups' parts
// added in order, in fp32, and rounded once.
template <typename T>
__global__ __launch_bounds__(256) void attention_sum_kernel(AttnSumArgs a) {
  const int64_t end = a.offsets[a.B], used = end < 0 ? 0 : end > a.rows ? a.rows : end;
  const int packs = (a.dim + 3) / 4, per_row = a.parts / a.group * packs;
  const int64_t step = (int64_t)gridDim.x * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < used * per_row; i += step) {
    const int64_t row = i / per_row;
    const int u = (int)(i - row * per_row), hk = u / packs, c = (u - hk * packs) * 4;
    const float* p = a.part + (row * a.parts + hk * a.group) * a.dim + c;
    Pack<float, 4> t = load_some<float, 4>(p, a.dim - c);
    for (int j = 1; j < a.group; ++j) {
      const Pack<float, 4> x = load_some<float, 4>(p + (int64_t)j * a.dim, a.dim - c);
#pragma unroll
      for (int e = 0; e < 4; ++e) t.v[e] += x.v[e];
    }
    Pack<T, 4> r;
#pragma unroll
    for (int e = 0; e < 4; ++e) r.v[e] = (T)t.v[e];
    store_some<T, 4>(static_cast<T*>(a.out) + row * a.out_row + hk * a.out_head + c, r, a.dim - c);
  }
}

// One row of a stream: its state read, decayed, updated and written once.
// Bound by the state's bytes, and in small calls by its chain of loads (64
// streams of 8 x 64 x 64, 17 MB: 5.8 us).  A thread has four neighbouring columns of
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
  const float lambda = power(decay_exponent(a.log_decay, h), 1);
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

void check_offsets(const AttnWalk& a, hipStream_t st) {
  if (a.fault)
    hipLaunchKernelGGL(attention_check_kernel, dim3((a.B + 255) / 256), dim3(256), 0, st, a.offsets, a.B, a.rows, a.fault);
}

// The states that go into the parts of cut sequences: made, and carried on.
hipError_t cut_states(const AttnPair& p, int32_t dtype, hipStream_t st) {
  const hipError_t e = dtype == MMBEV_F32   ? launch_attention_states_f32(p, st)
                       : dtype == MMBEV_F16 ? launch_attention_states_f16(p, st)
                                            : launch_attention_states_bf16(p, st);
  if (e != hipSuccess) return e;
  const AttnArgs& a = p.walk[0];
  hipLaunchKernelGGL(attention_join_kernel, dim3((a.ad * a.cd + 63) / 64, a.H, p.items[1] ? 2 : 1), dim3(kJoinWaves * 64), 0, st, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attention(const AttnArgs& a, int32_t dtype, hipStream_t st) {
  check_offsets(a, st);
  if (a.cuts) {
    AttnPair p{};
    p.walk[0] = a;
    p.items[0] = (uint32_t)(a.cuts * a.H);
    const hipError_t e = cut_states(p, dtype, st);
    if (e != hipSuccess) return e;
  }
  return dtype == MMBEV_F32 ? launch_attention_f32(a, st) : dtype == MMBEV_F16 ? launch_attention_f16(a, st) : launch_attention_bf16(a, st);
}

hipError_t launch_attention_backward(const AttnArgs& a, const AttnGradArgs& b, const AttnArgs& states, int32_t dtype, hipStream_t st) {
  check_offsets(a, st);
  if (a.cuts) {  // and then b's are cut too
    AttnPair p{};
    p.walk[0] = a;
    p.walk[1] = states;
    p.items[0] = (uint32_t)(a.cuts * a.H);
    p.items[1] = (uint32_t)(states.cuts * states.H);
    const hipError_t e = cut_states(p, dtype, st);
    if (e != hipSuccess) return e;
  }
  return dtype == MMBEV_F32   ? launch_attention_backward_f32(a, b, st)
         : dtype == MMBEV_F16 ? launch_attention_backward_f16(a, b, st)
                              : launch_attention_backward_bf16(a, b, st);
}

hipError_t launch_attention_sum(const AttnSumArgs& a, int32_t dtype, hipStream_t st) {
  if (a.rows == 0) return hipSuccess;
  const int64_t items = a.rows * (a.parts / a.group) * ((a.dim + 3) / 4);
  const dim3 grid((uint32_t)std::max<int64_t>(1, std::min<int64_t>((items + 255) / 256, 65536)));
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
