// The sequence operators of a learned voxel encoder (layer norm, rotary
// positions, linear attention with decay): what their kernels share, and
// their host-side launchers.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "delta_rows.hpp"
#include "mmbev.h"

namespace mmbev {

// ------------------------------------------------------------- arguments

// Workgroups of a launch: with 256 threads each they stay under the 2^32
// threads that one may have.  More rows take more launches.
constexpr int64_t kMostGroups = (int64_t)1 << 23;

// Calls that read and write more than this store past the caches: what they
// write would be evicted before another call reads it, and takes the place of
// what they read twice.  (Norm of 921,997 x 256 rows 315 -> 309 us, rotary of
// 213,879 x 16 x 64 169 -> 152, a keyframe's attention 177 -> 169.)  Half of
// the memory-side cache.
constexpr int64_t kPastCaches = (int64_t)128 << 20;

struct NormArgs {
  const void* x;         // forward: x; backward: s
  const void* skip;      // forward: residual; backward: dskip (null: none)
  const void* dy;        // backward
  const void* weight;    // null: ones
  const void* bias;      // null: zeros
  void* out;             // forward: out; backward: dx
  void* sum;             // forward: out_sum (null: not written)
  float* mean;           // backward: read
  float* rstd;
  float* partial;        // backward: [grid][2][width] sums of dy*h and dy, or null
  float* dweight;
  float* dbias;
  const int64_t* row_count;
  int32_t* fault;
  int64_t rows, x_stride, skip_stride, dy_stride, out_stride, sum_stride;
  int64_t first_row;     // of the launch
  int32_t width;
  int32_t weight_f32;    // weight and bias are fp32 (else of the rows' type)
  int32_t past;          // store past the caches
  float eps, inv_width;
};

hipError_t launch_norm(const NormArgs& a, int32_t dtype, hipStream_t st);
hipError_t launch_norm_backward(const NormArgs& a, int32_t dtype, hipStream_t st);
int32_t norm_backward_grid(int64_t rows, int32_t width, int32_t dtype);  // workgroups, hence partial rows

constexpr int kNormGrid = 1024;  // most workgroups of a norm's backward pass: four a CU, a partial row each
// first and second [width]: partial's `parts` <= kNormGrid rows of 2 * width added up (either may be null)
hipError_t launch_weight_sum(const float* partial, int32_t parts, int32_t width, float* first, float* second, hipStream_t st);

struct RotaryArgs {
  const void* x;
  void* out;
  const int32_t* positions;
  const uint64_t* steps;
  const uint8_t* axis;
  const int64_t* row_count;
  int32_t* fault;
  int64_t rows, x_row, x_head, out_row, out_head, position_stride;
  int64_t first_row;     // of the launch
  int32_t heads, dim, rotary_dim, axes;
  int32_t interleaved, inverse, copy_rest;  // copy_rest: out is not x
  int32_t past;          // store past the caches
};

hipError_t launch_rotary(const RotaryArgs& a, int32_t dtype, hipStream_t st);

// Norm and rotation of every head of two arrays of rows: [0] queries, [1] keys.
struct HeadNormArgs {
  const void* x[2];
  const void* dy[2];     // backward
  void* out[2];          // backward: dx
  const void* weight[2]; // null: ones
  float* partial;        // backward: [grid][2][dim] sums of dweight, or null
  float* dweight[2];
  const int32_t* positions;
  const uint64_t* steps;
  const uint8_t* axis;
  const int64_t* row_count;
  int32_t* fault;
  int64_t rows, x_row[2], x_head[2], dy_row[2], dy_head[2], out_row[2], out_head[2], position_stride;
  int64_t first_row;     // of the launch
  int32_t heads[2];
  int32_t dim, rotary_dim, axes;
  int32_t interleaved;
  int32_t weight_f32;    // weights are fp32 (else of the rows' type)
  float eps, inv_dim;
};

hipError_t launch_head_norm(const HeadNormArgs& a, int32_t dtype, hipStream_t st);
hipError_t launch_head_norm_backward(const HeadNormArgs& a, int32_t dtype, hipStream_t st);
int32_t head_norm_backward_grid(const HeadNormArgs& a, int32_t dtype);  // workgroups, hence partial rows

// Waves a SIMD of the walks' kernels, as their registers allow, hence the
// workgroups of four waves that a compute unit takes; `wide`: 32, 64 or 128.
constexpr int walk_waves(bool half, int wide) { return (wide > 64 ? 2 : wide > 32 ? 3 : 4) - (half ? 0 : 1); }
constexpr int grad_waves(bool half, int wide) { return wide > 64 && !half ? 1 : 2; }

constexpr int kOrderedSequences = 256;

// Ragged sequences and how the walks over them are cut.  Positions may run
// backwards.
struct Ranges {
  const int64_t* offsets;
  int64_t rows;
  int32_t B;
  int32_t reversed;
  // sequences are cut at shares of (rows in use) / cuts, at least `least` rows; 0: none is
  int32_t cuts;
  int32_t longest_first;  // the sequences that are not cut, up to kOrderedSequences of them
  int32_t least;          // whole chunks
};

// What the walks of linear attention share; `ad` and `cd` are the state's rows
// and columns.
struct AttnWalk : Ranges {
  const float* log_decay;
  const float* init;      // [B][H][ad][cd], or [B][H][cd][ad] where init_swapped; null: zeros
  float* final_state;     // [B][H][ad][cd]; null: not written
  int32_t* fault;
  int32_t H;
  int32_t ad, cd;
  int32_t init_swapped;
  int32_t exact_state;    // the state is an output: as exact as fp32
  int32_t past;           // store past the caches
  float scale;
  float init_scale, final_scale;  // the state is carried divided by these
  float* cut_state;       // [cuts][H][ad][cd]: the state at the end of every part that goes on
  int32_t* cut_rows;      // [cuts] its rows, 0 where it begins its sequence, -1: there is no such part
};

// out_i = scale * sum_{j <= i} lambda^(i-j) (a_i . b_j) c_j + scale * lambda^(i+1) a_i . init over each sequence: the
// forward pass is (q, k, v), dq is (dout, v, k).  The state alone (of b and c) is also made backwards.
struct AttnArgs : AttnWalk {
  const void *a, *b, *c;
  void* out;
  int64_t a_head, b_head, c_head, o_head;
  int32_t a_row, b_row, c_row, o_row;
  int32_t a_div, b_div, c_div;  // head h of the operator is head h / div of the operand
};

struct AttnGradArgs : AttnWalk {  // dv and dk, backwards; the state's rows are q's, its columns dout's
  const void *q, *dout, *k, *v;
  void *dk, *dv;
  int64_t q_head, d_head, k_head, v_head, dk_head, dv_head;
  int32_t q_row, d_row, k_row, v_row, dk_row, dv_row;
  int32_t kv_div;         // heads that share keys and values
  int32_t group;          // of them a workgroup's: 1, 2 or 4
  int32_t parts;          // not all of them: the sums go to part_k and part_v, fp32 [rows][H / group][dim]
  float *part_k, *part_v;
};

constexpr int32_t kAttnGroupMost(int32_t wide) { return wide <= 32 ? 4 : wide <= 64 ? 2 : 1; }

// One or two walks whose cut sequences' states one launch makes, and their workgroups.
struct AttnPair {
  AttnArgs walk[2];
  uint32_t items[2];
};

hipError_t launch_attention(const AttnArgs& a, int32_t dtype, hipStream_t st);
// states: the arguments of the walk that makes the states of b's cut sequences, (., q, dout) reversed
hipError_t launch_attention_backward(const AttnArgs& a, const AttnGradArgs& b, const AttnArgs& states, int32_t dtype, hipStream_t st);

struct AttnSumArgs {   // out[r][g] = sum over the group's parts of part[r][g * group + i], fp32 [rows][parts][dim]
  const float* part;
  void* out;
  int64_t out_head, rows;
  const int64_t* offsets;
  int32_t out_row;
  int32_t B, parts, group, dim;
};
hipError_t launch_attention_sum(const AttnSumArgs& a, int32_t dtype, hipStream_t st);

struct AttnStepArgs {
  const void *q, *k, *v;
  void* out;
  int64_t q_row, q_head, k_row, k_head, v_row, v_head, o_row, o_head;
  const float* log_decay;
  const int32_t* slots;
  float* state;
  int32_t* fault;
  int64_t rows, num_slots;
  int32_t H, group, kd, vd;
  float scale;
};
hipError_t launch_attention_step(const AttnStepArgs& a, int32_t dtype, hipStream_t st);

// ---- the gated delta rule

// One walk over chunks: forwards over (q, k, v) or, for the gradients,
// backwards over (q, k, dout).
struct DeltaArgs : Ranges {
  const void *q, *k, *v, *dout;
  void* out;
  int64_t q_head, k_head, v_head, d_head, o_head;
  int32_t q_row, k_row, v_row, d_row, o_row;
  int32_t g_row, b_row;   // of log_decay and beta, fp32 [rows][H]
  const float *log_decay, *beta;
  const float* init;      // [B][H][kd][vd]: the state before a sequence; backwards, the gradient of the one after it
  float* final_state;     // the other end's
  int32_t* fault;
  int32_t H, group;       // group: heads that share keys and values
  int32_t kd, vd;
  int32_t past;           // store past the caches
  float scale;
  // boundaries between parts of a cut sequence: kind -1: there is none, 0: the part before it begins its sequence, 1: it does not
  int32_t* cut_kind;      // [cuts]
  float* cut_state;       // [cuts][H][kd][vd]: the state at the boundary
  float* cut_grad;        // its gradient; null: forwards alone
  float* cut_map;         // [cuts][H][kd][kd]: what the part before it does to the state before that part, where kind is 1
  float* cut_turned;      // its transpose (with cut_grad)
  // Boundaries are joined in runs of `run`: [0] forwards, [1] backwards.  Where from_run is set, what lies at a boundary
  // has run_map times the state at the end of the run before it yet to come.
  int32_t run;
  int32_t* from_run[2];   // [cuts]
  float* run_map[2];      // [cuts][H][kd][kd]
  float* run_end[2];      // [runs][H][kd][vd]: the state at a run's last boundary, backwards the gradient at its first
  // the gradients' chunks
  float* before;          // [slots][H][kd][vd]: the state before a chunk
  float* after;           // the gradient of the state after it
  float* left_over;       // [rows][H][vd]: values less what the state holds for their keys
  float* due;             // its gradient
};

// Of one or two shares of the rows none is less than half of a sequence, so none is cut: nothing is launched for parts, and
// they have no room.
constexpr int32_t kDeltaLeastCuts = 3;

// Chunks of a sequence lie next to each other from rows / 32 + sequence on, so no two chunks share a place.
inline int64_t delta_slots(int64_t rows, int64_t B) { return rows / kDeltaRows + B; }

struct DeltaGradArgs : DeltaArgs {
  void *dq, *dk, *dv;
  int64_t dq_head, dk_head, dv_head;
  int32_t dq_row, dk_row, dv_row;
  int32_t dg_row, db_row;
  float *dlog_decay, *dbeta;  // fp32 [rows][H]
};

// Waves a SIMD that the walks' kernels are compiled for, the workgroups that a compute unit takes of them, as LDS and
// those waves allow, and the waves that the gradients' kernel is compiled for; keys and values padded to `key` and `value`.
// (fp16 heads over 32 have three workgroups: with a plan for four, whose last ones begin when the others end, a keyframe
// of 8 heads of 64 took 631 us instead of 575, gradients of 8 crowded frames 3,500 instead of 3,180.)
constexpr int delta_waves(int size, int key, int value) { return size == 4 && (key > 64 || value > 64) ? 1 : 2; }
constexpr int delta_groups(bool f16, int size, int key, int value) {
  const bool wide = key > 64 || value > 64;
  return size == 4 ? (wide ? 1 : 2) : wide ? 2 : f16 && key > 32 ? 3 : 4;
}
constexpr int delta_grad_waves(bool f16, int size, int key, int value) {
  return size == 4 || key > 64 || value > 64 ? 1 : f16 && key > 32 ? 2 : 3;
}

hipError_t launch_delta(const DeltaArgs& a, int32_t dtype, hipStream_t st);
hipError_t launch_delta_backward(const DeltaGradArgs& a, const float* dfinal, float* dinitial, int32_t dtype, hipStream_t st);

struct DeltaStepArgs {
  const void *q, *k, *v;
  void* out;
  int64_t q_row, q_head, k_row, k_head, v_row, v_head, o_row, o_head, g_row, b_row;
  const float *log_decay, *beta;
  const int32_t* slots;
  float* state;
  int32_t* fault;
  int64_t rows, num_slots;
  int32_t H, group, kd, vd;
  float scale;
};
hipError_t launch_delta_step(const DeltaStepArgs& a, int32_t dtype, hipStream_t st);

// ------------------------------------------------------------ device code

using f16 = _Float16;
using bf16 = __bf16;

// N elements as they lie in memory, at any alignment of the element: the
// loads and stores are still as wide as the elements together (gfx950's
// global accesses take any byte address; an aligned row is faster).
template <typename T, int N>
struct Pack {
  T v[N];
};

template <typename T, int N>
__device__ __forceinline__ Pack<T, N> load_pack(const T* p) {
  Pack<T, N> r;
  __builtin_memcpy(&r, p, sizeof(r));
  return r;
}

template <typename T, int N>
__device__ __forceinline__ void store_pack(T* p, const Pack<T, N>& r) {
  __builtin_memcpy(p, &r, sizeof(r));
}

typedef uint32_t words_anywhere __attribute__((ext_vector_type(4), aligned(2)));

// 16 bytes that this call does not read again: past the caches, which keep what
// is read twice.
template <typename T, int N>
__device__ __forceinline__ void store_past(T* p, const Pack<T, N>& r) {
  static_assert(sizeof(r) == 16, "one 16-byte store");
  words_anywhere x;
  __builtin_memcpy(&x, &r, 16);
  // between the two, or the compiler merges this store with the plain one of the branch beside it
  asm volatile("");
  __builtin_nontemporal_store(x, reinterpret_cast<words_anywhere*>(p));
  asm volatile("");
}

// The first `n` of N elements (n may be outside 0..N), zeros after them.
template <typename T, int N>
__device__ __forceinline__ Pack<T, N> load_some(const T* p, int n) {
  if (n >= N) return load_pack<T, N>(p);
  Pack<T, N> r;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    r.v[e] = (T)0.0f;
    if (e < n) r.v[e] = p[e];
  }
  return r;
}

// 16 bytes that no call of this size reads again from a cache.
template <typename T, int N>
__device__ __forceinline__ Pack<T, N> load_past(const T* p) {
  static_assert(sizeof(Pack<T, N>) == 16, "one 16-byte load");
  asm volatile("");  // see store_past
  const words_anywhere x = __builtin_nontemporal_load(reinterpret_cast<const words_anywhere*>(p));
  asm volatile("");
  Pack<T, N> r;
  __builtin_memcpy(&r, &x, 16);
  return r;
}

template <typename T, int N>
__device__ __forceinline__ void store_some(T* p, const Pack<T, N>& r, int n, bool past = false) {
  if (n >= N) {
    if constexpr (sizeof(r) == 16) {
      if (past) {
        store_past<T, N>(p, r);
        return;
      }
    }
    store_pack<T, N>(p, r);
    return;
  }
#pragma unroll
  for (int e = 0; e < N; ++e)
    if (e < n) p[e] = r.v[e];
}

template <typename T>
constexpr int kPackOf = 16 / (int)sizeof(T);  // elements of a 16-byte access

__device__ __forceinline__ float dpp_xor_step(float x, int which) {
  // partner values of a butterfly inside 16 lanes; which is a literal
  const int i = __builtin_bit_cast(int, x);
  switch (which) {
    case 1: return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, i, 0xB1, 0xf, 0xf, true));   // lane ^ 1
    case 2: return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, i, 0x4E, 0xf, 0xf, true));   // lane ^ 2
    case 4: return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, i, 0x141, 0xf, 0xf, true));  // mirror of 8
    default: return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, i, 0x140, 0xf, 0xf, true)); // mirror of 16
  }
}

// Sum over groups of LANES neighbouring lanes (a power of two up to 64),
// known to all of them, in register moves only: quads, mirrored halves of
// 8 and 16 (all lanes of a mirrored part hold the same sum), swapped rows.
template <int LANES>
__device__ __forceinline__ float group_sum(float x) {
  if constexpr (LANES >= 2) x += dpp_xor_step(x, 1);
  if constexpr (LANES >= 4) x += dpp_xor_step(x, 2);
  if constexpr (LANES >= 8) x += dpp_xor_step(x, 4);
  if constexpr (LANES >= 16) x += dpp_xor_step(x, 8);
  if constexpr (LANES >= 32) {
    const unsigned i = __builtin_bit_cast(unsigned, x);
    const auto p = __builtin_amdgcn_permlane16_swap(i, i, false, false);
    x = __builtin_bit_cast(float, (unsigned)p[0]) + __builtin_bit_cast(float, (unsigned)p[1]);
  }
  if constexpr (LANES >= 64) {
    const unsigned i = __builtin_bit_cast(unsigned, x);
    const auto p = __builtin_amdgcn_permlane32_swap(i, i, false, false);
    x = __builtin_bit_cast(float, (unsigned)p[0]) + __builtin_bit_cast(float, (unsigned)p[1]);
  }
  return x;
}

// Largest value of the four lanes of the same number in the wave's rows of 16, known to all of them.
__device__ __forceinline__ float column_max(float x) {
  unsigned i = __builtin_bit_cast(unsigned, x);
  const auto p = __builtin_amdgcn_permlane16_swap(i, i, false, false);
  x = fmaxf(__builtin_bit_cast(float, (unsigned)p[0]), __builtin_bit_cast(float, (unsigned)p[1]));
  i = __builtin_bit_cast(unsigned, x);
  const auto q = __builtin_amdgcn_permlane32_swap(i, i, false, false);
  return fmaxf(__builtin_bit_cast(float, (unsigned)q[0]), __builtin_bit_cast(float, (unsigned)q[1]));
}

// Largest value of a wave, known to all lanes.
__device__ __forceinline__ float group_max(float x) {
  x = fmaxf(x, dpp_xor_step(x, 1));
  x = fmaxf(x, dpp_xor_step(x, 2));
  x = fmaxf(x, dpp_xor_step(x, 4));
  return column_max(fmaxf(x, dpp_xor_step(x, 8)));
}

// Rows in use: the device's count, clamped to the array.
__device__ __forceinline__ int64_t rows_in_use(const int64_t* row_count, int64_t rows, int32_t* fault) {
  if (!row_count) return rows;
  const int64_t n = *row_count;
  const int64_t use = n < 0 ? 0 : n > rows ? rows : n;
  if (use != n && fault && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) atomicOr(fault, MMBEV_FAULT_SEQUENCES);
  return use;
}

}  // namespace mmbev
