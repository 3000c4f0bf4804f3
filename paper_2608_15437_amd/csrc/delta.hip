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
// One boundary after the other, each a product behind its matrix's load, would
// take longer than the walks (a keyframe's 95: 97 us; 126 of heads of 128,
// backwards: 1,530).  So the boundaries are taken in runs, all at once, each
// from nothing together with what the run up to there does to a state (the
// same recurrence from the unit matrix); then the runs' ends are carried on;
// and the walk that begins at a boundary adds the product with the end of the
// run before (add_mapped).
// A workgroup has 16 columns of B or of the map; its waves take 16 rows of a
// product each and pass the result on through LDS.  The next boundary's
// matrices are loaded before this one's product.  Bound by that chain, 2 to 4
// us a boundary: a keyframe's 127 boundaries of 8 heads of 64 24 us, the ends
// 16; 127 of 4 heads of 128, both ways, 123 and 34.  (Four boundaries' loads
// ahead took longer: 40 us instead of 33, 182 instead of 133; so did 32 columns
// of heads of 128, 155.)
constexpr int kJoinTile = 16, kJoinThreads = 256;

__host__ __device__ inline int tiles_of(int columns) { return (columns + kJoinTile - 1) / kJoinTile; }

// The workgroups that read the same maps lie next to each other on the same die (the dies take eight workgroups in turn),
// whose L2 then has them once: a keyframe's joining 33 -> 24 us, 8 frames' both ways 59 -> 43.
struct Chain {
  int chain, tile;
};
__device__ __forceinline__ Chain chain_of(int tiles) {
  const int turn = blockIdx.x / 8;
  return {turn / tiles * 8 + (int)(blockIdx.x % 8), turn % tiles};
}

// A boundary's part of the recurrence: X = map X + add, or X = add.
struct Link {
  const float *map, *add;
  float* to;
  bool there, carries;
};

// X goes from link to link, from what `first` says: nothing (0), the unit matrix (1).  link(i) is the i-th.
template <int DK, typename F>
__device__ __forceinline__ void carry_on(bf16 (*s_x)[3 * kJoinTile * (DK + kPlanePad)], int count, int col, int kd, int columns, bool unit, F&& link) {
  constexpr int STRIDE = DK + kPlanePad, PLANE = kJoinTile * STRIDE, TD = DK >= 64 ? DK / 64 : 1, STEPS = DK / 32;
  const Lane l = lane_of();
  const bool own = 16 * TD * l.w < DK;
  struct Next {
    float m[TD][STEPS][8];
    f32x4 b[TD];
    Link link;
  };
  auto fetch = [&](Next& x, int i) {
    x.link = link(i);
#pragma unroll
    for (int d = 0; d < TD; ++d) {
      const int row0 = 16 * (l.w * TD + d);
      x.b[d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      if (x.link.there && x.link.add) {
#pragma unroll
        for (int r = 0; r < 4; ++r) x.b[d][r] = x.link.add[min(row0 + 4 * l.g + r, kd - 1) * columns + min(col + l.n, columns - 1)];
      }
      if (!x.link.carries) continue;
#pragma unroll
      for (int s = 0; s < STEPS; ++s) load_eight(x.m[d][s], x.link.map, row0 + l.n, 32 * s + 8 * l.g, kd, kd);
    }
  };
  Next now, next;
  if (own) {
    // the start
#pragma unroll
    for (int d = 0; d < TD; ++d) {
      const int row = 16 * (l.w * TD + d) + 4 * l.g;
      f32x4 x;
#pragma unroll
      for (int r = 0; r < 4; ++r) x[r] = unit && row + r == col + l.n ? 1.0f : 0.0f;
      put4<3>(s_x[1] + l.n * STRIDE + row, PLANE, x);
    }
    fetch(now, 0);
  }
  __syncthreads();
  for (int i = 0; i < count; ++i) {
    const int turn = i & 1;
    if (own) {
      if (i + 1 < count) fetch(next, i + 1);
#pragma unroll
      for (int d = 0; d < TD; ++d) {
        const int row = 16 * (l.w * TD + d) + 4 * l.g;
        f32x4 x;
#pragma unroll
        for (int r = 0; r < 4; ++r) x[r] = row + r < kd && col + l.n < columns ? now.b[d][r] : 0.0f;
        if (now.link.carries) {
#pragma unroll
          for (int s = 0; s < STEPS; ++s) x = mma<3>(split<3>(now.m[d][s]), rows_of<3>(s_x[turn ^ 1], PLANE, STRIDE, 0, 32 * s, l), x);
        }
        if (now.link.there && now.link.to) {
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (row + r < kd && col + l.n < columns) now.link.to[(row + r) * columns + col + l.n] = x[r];
        }
        put4<3>(s_x[turn] + l.n * STRIDE + row, PLANE, x);
      }
      now = next;
    }
    __syncthreads();
  }
}

// Up to 64 links' flags, lane i of a wave the i-th's, known to all of them.
struct Flags {
  uint64_t there, carries;
  __device__ __forceinline__ bool is_there(int i) const { return there >> i & 1; }
  __device__ __forceinline__ bool do_carry(int i) const { return carries >> i & 1; }
};

template <int DK, bool BACK>
__device__ __forceinline__ void join_run(const DeltaArgs& a, bf16 (*s_x)[3 * kJoinTile * (DK + kPlanePad)], int run, int tile, int h) {
  const int64_t each = (int64_t)a.kd * a.vd, square = (int64_t)a.kd * a.kd;
  const int tiles = tiles_of(a.vd), first = run * a.run, count = min(a.run, a.cuts - first);
  const bool map = tile >= tiles;
  float* state = BACK ? a.cut_grad : a.cut_state;
  const float* maps = BACK ? a.cut_turned : a.cut_map;
  auto boundary = [&](int i) { return BACK ? first + count - 1 - i : first + i; };
  auto coming_in = [&](int e) { return BACK ? min(e + 1, a.cuts - 1) : e; };  // the part whose map comes in
  const int i = min((int)threadIdx.x & 63, count - 1), e = boundary(i);
  const bool there = a.cut_kind[e] >= 0, carries = there && a.cut_kind[coming_in(e)] == 1 && !(BACK && e + 1 == a.cuts);
  const Flags f = {__ballot(there), __ballot(carries)};
  // boundaries up to the first that does not carry come from the run before
  const int open = min(f.carries == ~0ull ? 64 : __builtin_ctzll(~f.carries), count);
  if (h == 0 && tile == 0 && (int)threadIdx.x < count) a.from_run[BACK][e] = i < open;
  if (map && open == 0) return;
  carry_on<DK>(s_x, map ? open : count, (map ? tile - tiles : tile) * kJoinTile, a.kd, map ? a.kd : a.vd, map, [&](int i) {
    const int64_t at = (int64_t)boundary(i) * a.H + h;
    float* place = map ? a.run_map[BACK] + at * square : state + at * each;
    return Link{maps + ((int64_t)coming_in(boundary(i)) * a.H + h) * square, map ? nullptr : place, place, f.is_there(i), f.do_carry(i) && (map || i > 0)};
  });
}

template <int DK>
__global__ __launch_bounds__(kJoinThreads) void delta_join_kernel(DeltaArgs a) {
  __shared__ __attribute__((aligned(16))) bf16 s_x[2][3 * kJoinTile * (DK + kPlanePad)];
  const int runs = (a.cuts + a.run - 1) / a.run;
  const Chain c = chain_of(tiles_of(a.vd) + tiles_of(a.kd));
  const int run = c.chain / a.H, h = c.chain - run * a.H;
  if (run < runs)
    join_run<DK, false>(a, s_x, run, c.tile, h);
  else if (a.cut_grad && run < 2 * runs)
    join_run<DK, true>(a, s_x, run - runs, c.tile, h);
}

// The runs' ends.
template <int DK, bool BACK>
__device__ __forceinline__ void join_ends(const DeltaArgs& a, bf16 (*s_x)[3 * kJoinTile * (DK + kPlanePad)], int tile, int h) {
  const int runs = (a.cuts + a.run - 1) / a.run;
  const int64_t each = (int64_t)a.kd * a.vd, square = (int64_t)a.kd * a.kd;
  auto run_of = [&](int i) { return BACK ? runs - 1 - i : i; };
  auto boundary = [&](int i) { return BACK ? run_of(i) * a.run : min((run_of(i) + 1) * a.run, a.cuts) - 1; };
  const int e = boundary(min((int)threadIdx.x & 63, runs - 1));
  const bool there = a.cut_kind[e] >= 0;
  const Flags f = {__ballot(there), __ballot(there && a.from_run[BACK][e])};
  carry_on<DK>(s_x, runs, tile * kJoinTile, a.kd, a.vd, false, [&](int i) {
    const int64_t at = (int64_t)boundary(i) * a.H + h;
    return Link{a.run_map[BACK] + at * square, (BACK ? a.cut_grad : a.cut_state) + at * each, a.run_end[BACK] + ((int64_t)run_of(i) * a.H + h) * each,
                f.is_there(i), f.do_carry(i) && i > 0};
  });
}

template <int DK>
__global__ __launch_bounds__(kJoinThreads) void delta_ends_kernel(DeltaArgs a) {
  __shared__ __attribute__((aligned(16))) bf16 s_x[2][3 * kJoinTile * (DK + kPlanePad)];
  const Chain c = chain_of(tiles_of(a.vd));
  if (c.chain < a.H)
    join_ends<DK, false>(a, s_x, c.tile, c.chain);
  else if (a.cut_grad && c.chain < 2 * a.H)
    join_ends<DK, true>(a, s_x, c.tile, c.chain - a.H);
}

hipError_t join_states(const DeltaArgs& a, bool backward, hipStream_t st) {
  const int runs = (a.cuts + a.run - 1) / a.run, chains = backward ? 2 * a.H : a.H;
  auto go = [&](auto join, auto ends) {
    hipLaunchKernelGGL(join, dim3((runs * chains + 7) / 8 * 8 * (tiles_of(a.vd) + tiles_of(a.kd))), dim3(kJoinThreads), 0, st, a);
    hipLaunchKernelGGL(ends, dim3((chains + 7) / 8 * 8 * tiles_of(a.vd)), dim3(kJoinThreads), 0, st, a);
  };
  a.kd <= 32   ? go(delta_join_kernel<32>, delta_ends_kernel<32>)
  : a.kd <= 64 ? go(delta_join_kernel<64>, delta_ends_kernel<64>)
               : go(delta_join_kernel<128>, delta_ends_kernel<128>);
  return hipGetLastError();
}

// One row of a stream: its state read once, decayed, corrected and written
// once.  Bound by the state's bytes, and in small calls by its chain: load,
// sum along the key, correct, sum along the query.  A thread has four
// neighbouring columns of every (256 / lanes)-th state row in registers, lanes
// enough for a row of the state; the rows' parts of both sums meet in LDS.
// 1,024 streams of 8 heads of 128 x 128: 211 us, 5.1 TB/s; 64 of 8 heads of
// 64 x 64: 6.1 us.
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
  if (a.cuts >= kDeltaLeastCuts) {
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
  if (a.cuts >= kDeltaLeastCuts) {
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
