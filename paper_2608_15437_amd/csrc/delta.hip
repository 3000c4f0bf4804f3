// The gated delta rule: what does not depend on the rows' element type (the
// joining of cut sequences), the single-row step, and the dispatch over types.
#include <algorithm>

#include "delta.hpp"
#include "delta_types.hpp"

namespace mmbev {

namespace {

// The states at the boundaries between the parts of cut sequences, carried on:
// a part that does not begin its sequence was walked from nothing, and what it
// does to a state was found beside that, so
//   S_e = M_e S_(e-1) + B_e,  backwards  D_e = M_(e+1)^T D_(e+1) + B'_e.
// A workgroup has 16 columns; its waves take 16 rows of a product each and pass
// the state on through LDS.  The next boundary's matrices are loaded before
// this one's product.
constexpr int kJoinTile = 16;

template <int DK, bool BACK>
__device__ __forceinline__ void join(const DeltaArgs& a, bf16 (*s_x)[3 * kJoinTile * (DK + kPlanePad)]) {
  constexpr int STRIDE = DK + kPlanePad, PLANE = kJoinTile * STRIDE, TD = DK >= 64 ? DK / 64 : 1, STEPS = DK / 32;
  const Lane l = lane_of();
  const int h = blockIdx.y, col = blockIdx.x * kJoinTile + l.n;
  const int64_t each = (int64_t)a.kd * a.vd, square = (int64_t)a.kd * a.kd;
  float* state = (BACK ? a.cut_grad : a.cut_state) + h * each;
  const bool own = 16 * TD * l.w < DK;
  const int last = a.cuts - 1;
  struct Next {
    float m[TD][STEPS][8];
    f32x4 b[TD];
    int32_t kind;  // of the boundary, and of the part whose map is there
    bool carries;
  };
  auto fetch = [&](Next& x, int i) {  // the i-th boundary of the walk
    const int e = BACK ? last - i : i, part = BACK ? e + 1 : e;
    x.kind = a.cut_kind[e];
    x.carries = part <= last && a.cut_kind[min(part, last)] == 1;
    const float* m = a.cut_map + ((int64_t)min(part, last) * a.H + h) * square;
    const float* b = state + (int64_t)e * a.H * each;
#pragma unroll
    for (int d = 0; d < TD; ++d) {
      const int row0 = 16 * (l.w * TD + d);
#pragma unroll
      for (int r = 0; r < 4; ++r) x.b[d][r] = b[min(row0 + 4 * l.g + r, a.kd - 1) * a.vd + min(col, a.vd - 1)];
      if (!x.carries) continue;
#pragma unroll
      for (int s = 0; s < STEPS; ++s) {
        if constexpr (BACK) {
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const int row = 32 * s + 8 * l.g + k, c = row0 + l.n;
            const float v = m[min(row, a.kd - 1) * a.kd + min(c, a.kd - 1)];
            x.m[d][s][k] = row < a.kd && c < a.kd ? v : 0.0f;
          }
        } else {
          load_eight(x.m[d][s], m, row0 + l.n, 32 * s + 8 * l.g, a.kd, a.kd);
        }
      }
    }
  };
  Next now, next;
  if (own) fetch(now, 0);
  int turn = 0;
  for (int i = 0; i <= last; ++i, turn ^= 1) {
    if (own && i < last) fetch(next, i + 1);
    if (own) {
      const int e = BACK ? last - i : i;
#pragma unroll
      for (int d = 0; d < TD; ++d) {
        const int row = 16 * (l.w * TD + d) + 4 * l.g;
        f32x4 x;
#pragma unroll
        for (int r = 0; r < 4; ++r) x[r] = row + r < a.kd && col < a.vd && now.kind >= 0 ? now.b[d][r] : 0.0f;
        if (now.kind >= 0 && now.carries && i > 0) {
#pragma unroll
          for (int s = 0; s < STEPS; ++s) x = mma<3>(split<3>(now.m[d][s]), rows_of<3>(s_x[turn ^ 1], PLANE, STRIDE, 0, 32 * s, l), x);
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (row + r < a.kd && col < a.vd) state[(int64_t)e * a.H * each + (row + r) * a.vd + col] = x[r];
        }
        put4<3>(s_x[turn] + l.n * STRIDE + row, PLANE, x);
      }
    }
    __syncthreads();
    now = next;
  }
}

template <int DK>
__global__ __launch_bounds__(kDeltaThreads) void delta_join_kernel(DeltaArgs a) {
  __shared__ __attribute__((aligned(16))) bf16 s_x[2][3 * kJoinTile * (DK + kPlanePad)];
  blockIdx.z == 0 ? join<DK, false>(a, s_x) : join<DK, true>(a, s_x);
}

hipError_t join_states(const DeltaArgs& a, bool backward, hipStream_t st) {
  const dim3 grid((a.vd + kJoinTile - 1) / kJoinTile, a.H, backward ? 2 : 1), block(kDeltaThreads);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, st, a); };
  a.kd <= 32 ? go(delta_join_kernel<32>) : a.kd <= 64 ? go(delta_join_kernel<64>) : go(delta_join_kernel<128>);
  return hipGetLastError();
}

// One row of a stream: its state read once, decayed, corrected and written
// once.  Bound by the state's bytes, and in small calls by its chain: load,
// sum along the key, correct, sum along the query.  A thread has four
// neighbouring columns of every (256 / lanes)-th state row in registers, lanes
// enough for a row of the state; the rows' parts of both sums meet in LDS.
template <typename T, int LANES, int ROWS>
__global__ __launch_bounds__(256) void delta_step_kernel(DeltaStepArgs a) {
  constexpr int PARTS = 256 / LANES;
  __shared__ float s_q[128], s_k[128];
  __shared__ float s_sum[2][PARTS][LANES * 4 + 4];
  const int h = blockIdx.x % a.H;
  const int64_t r = blockIdx.x / a.H;
  const int64_t slot = a.slots ? (int64_t)a.slots[r] : r;
  if (slot < 0) return;
  if (slot >= a.num_slots) {
    if (a.fault && threadIdx.x == 0) atomicOr(a.fault, MMBEV_FAULT_SEQUENCES);
    return;
  }
  const int hk = h / a.group;
  const int lane = threadIdx.x % LANES, part = threadIdx.x / LANES, c = lane * 4;
  float* state = a.state + (slot * a.H + h) * a.kd * a.vd;
  Pack<float, 4> s[ROWS];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const int row = part + i * PARTS;
    s[i] = load_some<float, 4>(state + min(row, a.kd - 1) * a.vd + c, a.vd - c);
  }
  for (int i = threadIdx.x; i < 128; i += 256) {
    const bool there = i < a.kd;
    s_q[i] = there ? (float)static_cast<const T*>(a.q)[r * a.q_row + h * a.q_head + i] : 0.0f;
    s_k[i] = there ? (float)static_cast<const T*>(a.k)[r * a.k_row + hk * a.k_head + i] : 0.0f;
  }
  const Pack<T, 4> rv = load_some<T, 4>(static_cast<const T*>(a.v) + r * a.v_row + hk * a.v_head + c, a.vd - c);
  float step, rest;
  base2_of(a.log_decay[r * a.g_row + h], step, rest);
  const float decay = exp2_of(step, rest), beta = a.beta[r * a.b_row + h];
  __syncthreads();
  float held[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const float k = part + i * PARTS < 128 ? s_k[part + i * PARTS] : 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      s[i].v[e] *= decay;
      held[e] = __builtin_fmaf(k, s[i].v[e], held[e]);
    }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) s_sum[0][part][c + e] = held[e];
  __syncthreads();
  float u[4], acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float t = 0.0f;
#pragma unroll
    for (int p = 0; p < PARTS; ++p) t += s_sum[0][p][c + e];
    u[e] = beta * ((float)rv.v[e] - t);
  }
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const int row = part + i * PARTS;
    if (row >= a.kd) continue;
    const float k = s_k[row], q = s_q[row];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      s[i].v[e] = __builtin_fmaf(k, u[e], s[i].v[e]);
      acc[e] = __builtin_fmaf(q, s[i].v[e], acc[e]);
    }
    store_some<float, 4>(state + row * a.vd + c, s[i], a.vd - c);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) s_sum[1][part][c + e] = acc[e];
  __syncthreads();
  if (threadIdx.x < a.vd) {
    float t = 0.0f;
#pragma unroll
    for (int p = 0; p < PARTS; ++p) t += s_sum[1][p][threadIdx.x];
    static_cast<T*>(a.out)[r * a.o_row + h * a.o_head + threadIdx.x] = (T)(t * a.scale);
  }
}

template <typename T>
hipError_t step_of(const DeltaStepArgs& a, hipStream_t st) {
  const dim3 grid((uint32_t)(a.rows * a.H)), block(256);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, st, a); };
  // lanes of a state row, rows of a thread
  if (a.vd <= 32)
    a.kd <= 64 ? go(delta_step_kernel<T, 8, 2>) : go(delta_step_kernel<T, 8, 4>);
  else if (a.vd <= 64)
    a.kd <= 64 ? go(delta_step_kernel<T, 16, 4>) : go(delta_step_kernel<T, 16, 8>);
  else
    a.kd <= 64 ? go(delta_step_kernel<T, 32, 8>) : go(delta_step_kernel<T, 32, 16>);
  return hipGetLastError();
}

// Offsets that break the contract: 0 .. <= rows, non-decreasing.
__global__ __launch_bounds__(256) void delta_check_kernel(const int64_t* offsets, int32_t B, int64_t rows, int32_t* fault) {
  const int32_t b = blockIdx.x * 256 + threadIdx.x;
  if (b >= B) return;
  const int64_t o0 = offsets[b], o1 = offsets[b + 1];
  if ((b == 0 && o0 != 0) || o1 < o0 || o1 > rows) atomicOr(fault, MMBEV_FAULT_SEQUENCES);
}

void check_offsets(const DeltaArgs& a, hipStream_t st) {
  if (a.fault)
    hipLaunchKernelGGL(delta_check_kernel, dim3((a.B + 255) / 256), dim3(256), 0, st, a.offsets, a.B, a.rows, a.fault);
}

hipError_t walk(const DeltaArgs& a, DeltaMode mode, int32_t dtype, hipStream_t st) {
  return dtype == MMBEV_F32   ? launch_delta_walk_f32(a, mode, st)
         : dtype == MMBEV_F16 ? launch_delta_walk_f16(a, mode, st)
                              : launch_delta_walk_bf16(a, mode, st);
}

}  // namespace

hipError_t launch_delta(const DeltaArgs& a, int32_t dtype, hipStream_t st) {
  check_offsets(a, st);
  if (a.cuts) {
    hipError_t e = walk(a, kDeltaStates, dtype, st);
    if (e == hipSuccess) e = join_states(a, false, st);
    if (e != hipSuccess) return e;
  }
  return walk(a, kDeltaOut, dtype, st);
}

hipError_t launch_delta_backward(const DeltaGradArgs& a, const float* dfinal, float* dinitial, int32_t dtype, hipStream_t st) {
  check_offsets(a, st);
  DeltaArgs back = a;
  back.init = dfinal;
  back.final_state = dinitial;
  hipError_t e = hipSuccess;
  if (a.cuts) {
    e = walk(a, kDeltaStates, dtype, st);
    if (e == hipSuccess) e = walk(back, kDeltaBackStates, dtype, st);
    if (e == hipSuccess) e = join_states(a, true, st);
  }
  if (e == hipSuccess) e = walk(a, kDeltaSave, dtype, st);
  if (e == hipSuccess) e = walk(back, kDeltaBack, dtype, st);
  if (e != hipSuccess) return e;
  return dtype == MMBEV_F32 ? launch_delta_grad_f32(a, st) : dtype == MMBEV_F16 ? launch_delta_grad_f16(a, st) : launch_delta_grad_bf16(a, st);
}

hipError_t launch_delta_step(const DeltaStepArgs& a, int32_t dtype, hipStream_t st) {
  if (a.rows == 0) return hipSuccess;
  return dtype == MMBEV_F32 ? step_of<float>(a, st) : dtype == MMBEV_F16 ? step_of<f16>(a, st) : step_of<bf16>(a, st);
}

}  // namespace mmbev
