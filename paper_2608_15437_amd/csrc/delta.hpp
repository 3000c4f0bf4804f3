// The gated delta rule: the chunked kernels (one translation unit a type
// includes this).
//
// A row first decays the state, then writes what its key does not hold yet:
//   S' = a S,  e = v - k S',  S = S' + k^T (beta e),  out = scale q S.
// In a chunk of 32 rows with G the inclusive sum of log a and
//   X_ij = e^(G_i - G_j) k_i . k_j for j < i,  P_ij = scale e^(G_i - G_j) q_i . k_j for j <= i,
// the rows' e solve (1 + X beta) E = R, R = V - e^G K S; with U = beta E
//   out = scale e^G Q S + P U,  S_after = e^(G_end) S + K^T (e^(G_end - G) U).
// The system is solved in two blocks of 16 rows, whose own inverses 1 + N beta
// (N strictly lower: N = -X - N beta X, column by column) are found once a
// chunk:
//   E_0 = R_0 + N_00 beta R_0,  R_1' = R_1 - X_10 beta E_0,  E_1 = R_1' + N_11 beta R_1'.
// Backwards, with D the gradient of the state after the chunk:
//   W = e^(G_end - G) K D + P^T dout,  Z = (1 + X^T beta)^-1 W (the same blocks, transposed),  dV = beta Z,
//   D_before = e^(G_end) D + (scale e^G Q)^T dout - (e^G K)^T beta Z.
//
// All that a row of the state's columns needs of another is in K, Q, N and P,
// so a wave walks 32 columns (two tiles of 16) alone: its state stays in
// registers from chunk to chunk, and every product's result is the next one's
// operand where it lies.  What the rows do to each other (N and P) is worked out
// once a chunk by the workgroup's waves, two to eight of them, through LDS.
//
// Precision: the state and the gradients of the gates are fp32 and go through
// thousands of chunks, so every product is as exact as fp32's: an operand is
// up to three parts of bf16, whose products of 2^-16 and more are summed (a
// bf16 row is one part, an fp16 row two, an fp32 value three; bf16 has fp32's
// exponents, so nothing is scaled).  An fp32 product this way is six products
// of bf16, 2.7 times as fast as the fp32 ones of the matrix cores.  What only
// enters a 16-bit result has three parts too: with two, 0.4% of the results
// were not the nearest value to their sum instead of 0.03%, and a state that
// was no output lost bits in every chunk.  (128 frames' results took 1,260 us
// that way instead of 1,700, a frame's 68 instead of 77, a keyframe's 420
// instead of 432.)
//
// What bounds the walks: issue of vector instructions (heads of 64 in bf16: 64
// to 73% of the time forwards, 51 to 65% in the gradients' walks: splitting
// results into parts, masks, addresses) and the chain through a chunk, with two
// waves a SIMD, which the registers of a state allow; the matrix cores are busy
// for 15 to 30%, LDS for 18 to 34%.  128 frames of 921,997 rows, 8 heads of 64
// in bf16: 1,680 us, 2.3 TB/s.  Rows fetched two chunks ahead instead of one
// took registers and 6% longer.  A single sequence is walked in parts, its keys
// and values read twice: 120,000 rows 432 us.  Of 16-bit keys over 64 the two
// walks that leave what the gradients need have a state too large for their 256
// registers and spill about 100 of them (344 to 500 bytes of scratch a lane; not
// the one backwards of fp16 values up to 64, which has one wave a SIMD): vector
// instructions are 20% of the time, 18,608 rows of 4 heads of 128 in fp16 take
// 173 and 206 us.
#pragma once

#include <type_traits>

#include "common.hpp"
#include "sequence_parts.hpp"

namespace mmbev {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef bf16 b16x8 __attribute__((ext_vector_type(8)));
typedef bf16 b16x4 __attribute__((ext_vector_type(4)));

// Parts of bf16 that a row's element is, and those of an fp32 value.
template <typename T>
constexpr int kPlanes = sizeof(T) == 4 ? 3 : __is_same(T, f16) ? 2 : 1;
constexpr int kParts = 3;

struct Lane {
  int w, g, n;  // wave; lane / 16; lane % 16
};
__device__ __forceinline__ Lane lane_of() {
  return {__builtin_amdgcn_readfirstlane(threadIdx.x >> 6), (int)(threadIdx.x & 63) >> 4, (int)threadIdx.x & 15};
}

// ------------------------------------------------------ products

// Eight elements a lane of a 32-deep product's operand, in N parts.  Lane l
// holds row (or column) l % 16; with g = l / 16 its elements are 8g .. 8g+7 of
// the depth or, `split`, 4g .. 4g+3 and 16+4g .. 16+4g+3: two results of 16 x 16
// (lane l of a result has column l % 16, rows 4g .. 4g+3) are such an operand.
template <int N>
struct Parts {
  b16x8 p[N];
};

// The sum of the products of two operands' parts, down to those of 2^-8(LEVEL-1).
template <int LEVEL, int NA, int NB>
__device__ __forceinline__ f32x4 mma(const Parts<NA>& a, const Parts<NB>& b, f32x4 c) {
#pragma unroll
  for (int s = LEVEL - 1; s >= 0; --s)
#pragma unroll
    for (int i = 0; i < NA; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j)
        if (i + j == s) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.p[i], b.p[j], c, 0, 0, 0);
  return c;
}

// Two neighbours' next part, taken off them (conversions in pairs: five operations instead of seven).
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef bf16 b16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t take_part(float& x, float& y, bool more) {
  const uint32_t p = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x, y}, b16x2));
  if (more) {
    x -= __builtin_bit_cast(float, p << 16);
    y -= __builtin_bit_cast(float, p & 0xffff0000u);
  }
  return p;
}

template <int N>
__device__ __forceinline__ Parts<N> split(const float (&x)[8]) {
  typedef uint32_t words __attribute__((ext_vector_type(4)));
  words w[N];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float u = x[2 * e], v = x[2 * e + 1];
#pragma unroll
    for (int i = 0; i < N; ++i) w[i][e] = take_part(u, v, i + 1 < N);
  }
  Parts<N> r;
#pragma unroll
  for (int i = 0; i < N; ++i) r.p[i] = __builtin_bit_cast(b16x8, w[i]);
  return r;
}

template <int N>
struct Quarter {
  b16x4 p[N];
};
template <int N>
__device__ __forceinline__ Quarter<N> split(f32x4 x) {
  typedef uint32_t words __attribute__((ext_vector_type(2)));
  words w[N];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    float u = x[2 * e], v = x[2 * e + 1];
#pragma unroll
    for (int i = 0; i < N; ++i) w[i][e] = take_part(u, v, i + 1 < N);
  }
  Quarter<N> r;
#pragma unroll
  for (int i = 0; i < N; ++i) r.p[i] = __builtin_bit_cast(b16x4, w[i]);
  return r;
}

template <int N>
__device__ __forceinline__ Parts<N> split(f32x4 x, f32x4 y) {
  const float z[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
  return split<N>(z);
}

// The first N parts of two results as an operand.
template <int N, int M>
__device__ __forceinline__ Parts<N> both(const Quarter<M>& x, const Quarter<M>& y) {
  Parts<N> r;
#pragma unroll
  for (int i = 0; i < N; ++i) r.p[i] = __builtin_shufflevector(x.p[i], y.p[i], 0, 1, 2, 3, 4, 5, 6, 7);
  return r;
}

// Four values of an operand, in N parts N arrays of LDS apart.
template <int N>
__device__ __forceinline__ void put4(bf16* s, int plane, f32x4 x) {
  const Quarter<N> q = split<N>(x);
#pragma unroll
  for (int i = 0; i < N; ++i) __builtin_memcpy(__builtin_assume_aligned(s + i * plane, 8), &q.p[i], 8);
}

// Operands out of LDS, rows of `stride` elements, parts `plane` apart.
// A row of memory: row row0 + n, elements c0 + 8g ..
template <int N>
__device__ __forceinline__ Parts<N> rows_of(const bf16* s, int plane, int stride, int row0, int c0, const Lane& l) {
  Parts<N> r;
#pragma unroll
  for (int i = 0; i < N; ++i)
    __builtin_memcpy(&r.p[i], __builtin_assume_aligned(s + i * plane + (row0 + l.n) * stride + c0 + 8 * l.g, 16), 16);
  return r;
}

// The same split: elements 4g .. and 16 + 4g ..
template <int N>
__device__ __forceinline__ Parts<N> rows_split(const bf16* s, int plane, int stride, int row0, const Lane& l) {
  Parts<N> r;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const bf16* p = s + i * plane + (row0 + l.n) * stride + 4 * l.g;
    b16x4 x, y;
    __builtin_memcpy(&x, __builtin_assume_aligned(p, 8), 8);
    __builtin_memcpy(&y, __builtin_assume_aligned(p + 16, 8), 8);
    r.p[i] = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
  }
  return r;
}

// A transposed read: lane n of 16 names 4 neighbouring elements of row n / 4 and gets, of the four rows, element n % 4 of
// those that lane n / 4 of each row names.
__device__ __forceinline__ b16x4 read_columns(const bf16* p) {
  using P = __attribute__((address_space(3))) s16x4*;
  return __builtin_bit_cast(b16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(p)));
}

// Down columns, split, the 32 rows of a chunk: lane n has column c0 + n or, of a pair of 16-column tiles whose columns
// are dealt out in fours (STEP 8; the second one's c0 is 4 more), column c0 + 8 (n / 4) + n % 4.
template <int N, int STEP = 4>
__device__ __forceinline__ Parts<N> columns_of(const bf16* s, int plane, int stride, int c0, const Lane& l) {
  Parts<N> r;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const bf16* p = s + i * plane + (4 * l.g + (l.n >> 2)) * stride + c0 + (l.n & 3) * STEP;
    r.p[i] = __builtin_shufflevector(read_columns(p), read_columns(p + 16 * stride), 0, 1, 2, 3, 4, 5, 6, 7);
  }
  return r;
}

// ---- blocks of 16 x 16: 16 deep, so a product's 32 take two of the parts' products at once

constexpr int kBlockStride = 20;  // rows of eight-byte steps over all banks
constexpr int kBlock = 16 * kBlockStride;

struct Block {
  b16x8 high, ends;  // first and second part; first and third
};

template <bool TRANSPOSED>
__device__ __forceinline__ Block block_of(const bf16* s, const Lane& l) {
  b16x4 p[kParts];
#pragma unroll
  for (int i = 0; i < kParts; ++i) {
    if constexpr (TRANSPOSED)
      p[i] = read_columns(s + i * kBlock + (4 * l.g + (l.n >> 2)) * kBlockStride + (l.n & 3) * 4);
    else
      __builtin_memcpy(&p[i], __builtin_assume_aligned(s + i * kBlock + l.n * kBlockStride + 4 * l.g, 8), 8);
  }
  return {__builtin_shufflevector(p[0], p[1], 0, 1, 2, 3, 4, 5, 6, 7), __builtin_shufflevector(p[0], p[2], 0, 1, 2, 3, 4, 5, 6, 7)};
}

// c + block * x
__device__ __forceinline__ f32x4 mma_block(const Block& a, const Quarter<kParts>& q, f32x4 c) {
  c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.ends, __builtin_shufflevector(q.p[2], q.p[0], 0, 1, 2, 3, 4, 5, 6, 7), c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.high, __builtin_shufflevector(q.p[1], q.p[1], 0, 1, 2, 3, 4, 5, 6, 7), c, 0, 0, 0);
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.high, __builtin_shufflevector(q.p[0], q.p[0], 0, 1, 2, 3, 4, 5, 6, 7), c, 0, 0, 0);
}

// ------------------------------------------------------ gates

// 2^(hi + lo), |lo| under 1: the sum's last bits stay in the power.
__device__ __forceinline__ float exp2_of(float hi, float lo) {
  const float x = hi + lo, rest = lo - (x - hi), p = __builtin_amdgcn_exp2f(x);
  return __builtin_fmaf(p, rest * 0.693147181f, p);
}

// A chunk's gates in LDS.  The sums of the log decays, to base 2, are held in
// two parts, multiples of 2^-10 (whose sums and differences are exact) and what
// is left over, so that the decay between two rows has its last bits behind a
// decay of any size too.
struct alignas(16) Gates {
  float hi[kDeltaRows], lo[kDeltaRows];      // inclusive sums
  float beta[kDeltaRows];
  float fade[kDeltaRows], left[kDeltaRows];  // the decay from before the chunk to a row, and from a row to the chunk's end
  float whole;
};

// Inclusive sums over the lanes of each half wave.
__device__ __forceinline__ float half_wave_sums(float x) {
  auto moved = [](float v, auto ctrl) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), ctrl.value, 0xf, 0xf, false));
  };
  x += moved(x, std::integral_constant<int, 0x111>{});  // row_shr:1, 2, 4, 8
  x += moved(x, std::integral_constant<int, 0x112>{});
  x += moved(x, std::integral_constant<int, 0x114>{});
  x += moved(x, std::integral_constant<int, 0x118>{});
  // row_bcast:15 into the second and fourth sixteen lanes
  return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x142, 0xa, 0xf, false));
}

__device__ __forceinline__ float last_of_half(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), kDeltaRows - 1));
}

// A decay of more than e^-104 leaves nothing in fp32; a log decay over 0 counts as 0, NaN stays.
__device__ __forceinline__ float clamp_gate(float g) { return g > 0.0f ? 0.0f : g < -104.0f ? -104.0f : g; }

// A log decay to base 2 in its two parts: log2(e) as fp32 and what that leaves of it.
__device__ __forceinline__ void base2_of(float g, float& step, float& rest) {
  g = clamp_gate(g);
  const float x = g * 1.44269504088896341f;
  step = __builtin_rintf(x * 1024.0f) * (1.0f / 1024.0f);
  rest = (x - step) + __builtin_fmaf(g, 1.44269504088896341f, -x) + g * 1.92596299e-8f;
}

// By one wave: lane r < 32 has row r's gates (0 past the rows).  `left` is multiplied by `times`.
__device__ __forceinline__ void put_gates(Gates& s, float g, float beta, float times) {
  const int r = threadIdx.x & 63;
  float step, rest;
  base2_of(g, step, rest);
  const float hi = half_wave_sums(step), lo = half_wave_sums(rest);
  const float end_hi = last_of_half(hi), end_lo = last_of_half(lo);
  const float fade = exp2_of(hi, lo);
  if (r < kDeltaRows) {
    s.hi[r] = hi;
    s.lo[r] = lo;
    s.beta[r] = beta;
    s.fade[r] = fade;
    s.left[r] = exp2_of(end_hi - hi, end_lo - lo) * times;
    if (r == kDeltaRows - 1) s.whole = fade;
  }
}

__device__ __forceinline__ f32x4 four(const float* s) {
  f32x4 r;
  __builtin_memcpy(&r, __builtin_assume_aligned(s, 16), 16);
  return r;
}

// ------------------------------------------------------ chunks

template <typename T>
constexpr int kRowPad = 16 / (int)sizeof(T);
constexpr int kPlanePad = 8;

// Eight elements of each of a chunk's 32 rows, W to a row, shared out among the threads of NW waves.
template <int W, int NW>
constexpr int kPacks = (kDeltaRows * W / 8 + 64 * NW - 1) / (64 * NW);
template <int W, int NW>
constexpr int kRowsApart = 64 * NW / (W / 8);  // of a thread's packs

// An operand's rows as a thread reads them.  Every load is of an element that
// is there, unconditional where the dim is a multiple of eight (WHOLE: a load
// under a condition is waited for where the paths meet); what is past the rows
// or the row's end is zeroed on the way into LDS.
template <typename T, int W, int NW, bool WHOLE>
struct Source {
  const T* p;  // row 0, the thread's columns
  int64_t stride;
  int dim;

  __device__ __forceinline__ Source(const void* data, int64_t head, int32_t row_stride, int columns) : stride(row_stride), dim(columns) {
    const int c = threadIdx.x % (W / 8) * 8;
    p = static_cast<const T*>(data) + head + (c < dim ? c : 0);
  }
  __device__ __forceinline__ void fetch(Pack<T, 8> (&r)[kPacks<W, NW>], int32_t s0, int32_t hi) const {
    const T* chunk = p + s0 * stride;
#pragma unroll
    for (int i = 0; i < kPacks<W, NW>; ++i) {
      // (rows past the last one are its copies)
      const uint32_t row = min((int)threadIdx.x / (W / 8) + i * kRowsApart<W, NW>, hi - s0 - 1);
      const T* from = chunk + (uint64_t)row * (uint32_t)stride;
      if constexpr (WHOLE)
        r[i] = load_pack<T, 8>(from);
      else
        r[i] = load_some<T, 8>(from, dim - (int)(threadIdx.x % (W / 8)) * 8);
    }
  }
};

// f(row, column, pack), zeros where there is nothing.
template <typename T, int W, int NW, typename F>
__device__ __forceinline__ void each_pack(const Pack<T, 8> (&r)[kPacks<W, NW>], int dim, int n, F&& f) {
  const int row = threadIdx.x / (W / 8), c = threadIdx.x % (W / 8) * 8;
#pragma unroll
  for (int i = 0; i < kPacks<W, NW>; ++i) {
    if (kPacks<W, NW> * kRowsApart<W, NW> > kDeltaRows && row + i * kRowsApart<W, NW> >= kDeltaRows) continue;
    typedef uint32_t words __attribute__((ext_vector_type(sizeof(T) * 2)));
    words x = __builtin_bit_cast(words, r[i]);
    if (n < kDeltaRows || dim < W) {
      const bool there = row + i * kRowsApart<W, NW> < n && c < dim;
#pragma unroll
      for (int e = 0; e < (int)sizeof(T) * 2; ++e) x[e] = there ? x[e] : 0u;
      asm volatile("");  // a branch over the selections: most chunks are whole
    }
    f(row + i * kRowsApart<W, NW>, c, __builtin_bit_cast(Pack<T, 8>, x));
  }
}

template <int N, typename T>
__device__ __forceinline__ void put_planes(bf16* s, int plane, const Pack<T, 8>& x) {
  if constexpr (__is_same(T, bf16)) {
    __builtin_memcpy(__builtin_assume_aligned(s, 16), &x, 16);
  } else {
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = (float)x.v[e];
    const Parts<N> p = split<N>(f);
#pragma unroll
    for (int i = 0; i < N; ++i) __builtin_memcpy(__builtin_assume_aligned(s + i * plane, 16), &p.p[i], 16);
  }
}

// A chunk's rows in LDS as operands: parts of W (and a step of 16 bytes) columns.
template <typename T, int W>
struct Planes {
  static constexpr int stride = W + kPlanePad, plane = kDeltaRows * stride;
  __attribute__((aligned(16))) bf16 v[kPlanes<T> * plane];

  template <int NW>
  __device__ __forceinline__ void put(const Pack<T, 8> (&r)[kPacks<W, NW>], int dim, int n) {
    each_pack<T, W, NW>(r, dim, n, [&](int row, int c, const Pack<T, 8>& x) { put_planes<kPlanes<T>, T>(v + row * stride + c, plane, x); });
  }
  __device__ __forceinline__ Parts<kPlanes<T>> rows(int row0, int c0, const Lane& l) const {
    return rows_of<kPlanes<T>>(v, plane, stride, row0, c0, l);
  }
  template <int STEP = 4>
  __device__ __forceinline__ Parts<kPlanes<T>> columns(int c0, const Lane& l) const {
    return columns_of<kPlanes<T>, STEP>(v, plane, stride, c0, l);
  }
  // elements c .. c+3 of a row
  __device__ __forceinline__ f32x4 at(int row, int c) const {
    f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < kPlanes<T>; ++i) {
      b16x4 p;
      __builtin_memcpy(&p, __builtin_assume_aligned(v + i * plane + row * stride + c, 8), 8);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] += (float)p[e];
    }
    return x;
  }
};

// Values as they are.
template <typename T, int W>
struct Values {
  static constexpr int stride = W + kRowPad<T>;
  __attribute__((aligned(16))) T v[kDeltaRows * stride];

  template <int NW>
  __device__ __forceinline__ void put(const Pack<T, 8> (&r)[kPacks<W, NW>], int dim, int n) {
    each_pack<T, W, NW>(r, dim, n, [&](int row, int c, const Pack<T, 8>& x) { __builtin_memcpy(__builtin_assume_aligned(v + row * stride + c, 16), &x, sizeof(x)); });
  }
  // column c0 + n of rows row0 + 4g ..
  __device__ __forceinline__ f32x4 down(int row0, int c0, const Lane& l) const {
    f32x4 x;
    if constexpr (sizeof(T) == 2) {
      typedef T t4 __attribute__((ext_vector_type(4)));
      const bf16* p = reinterpret_cast<const bf16*>(v) + (row0 + 4 * l.g + (l.n >> 2)) * stride + c0 + (l.n & 3) * 4;
      const t4 t = __builtin_bit_cast(t4, read_columns(p));
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = (float)t[e];
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = v[(row0 + 4 * l.g + e) * stride + c0 + l.n];
    }
    return x;
  }
};

// LDS order between lanes of one wave.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// What the rows of a chunk do to each other (P: where WITH_P), with the rows' beta multiplied in: forwards that of
// the row that is read (N beta, -X beta, P beta), backwards that of the row that reads (beta N, -beta X, P as it is).
constexpr int kPairStride = kDeltaRows + 4, kPairPlane = kDeltaRows * kPairStride;

template <bool WITH_P>
struct Pairs {
  __attribute__((aligned(16))) bf16 n[3][kParts * kBlock];  // N of the first and last 16 rows, -X of the last with the first
  __attribute__((aligned(16))) bf16 p[WITH_P ? kParts * kPairPlane : 8];
  __attribute__((aligned(16))) float x[2][kBlock];      // X of the first and last 16 rows
};

// e^(G_i - G_j), lane n row i0 + n, elements j0 + 4g ..: without exp2_of's last bits, off by |G_i - G_j| 2^-25 of itself.
// (Where j > i it may be infinite.)
__device__ __forceinline__ f32x4 decays(const Gates& s, int i0, int j0, const Lane& l) {
  const float hi = s.hi[i0 + l.n], lo = s.lo[i0 + l.n];
  const f32x4 jh = four(s.hi + j0 + 4 * l.g), jl = four(s.lo + j0 + 4 * l.g);
  f32x4 d;
#pragma unroll
  for (int r = 0; r < 4; ++r) d[r] = __builtin_amdgcn_exp2f((hi - jh[r]) + (lo - jl[r]));
  return d;
}

// x times them where j < i (j <= i with the diagonal), else 0.  Of two blocks of 16 rows, the diagonal ones have j > i.
template <bool SAME>
__device__ __forceinline__ f32x4 decayed(f32x4 x, f32x4 d, bool diagonal, const Lane& l) {
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int above = l.n - 4 * l.g - r;  // i - j
    const float y = x[r] * d[r];
    x[r] = !SAME || above > 0 || (diagonal && above == 0) ? y : 0.0f;
  }
  return x;
}

// a_i . b_j over DK columns: lane n row i0 + n, elements j0 + 4g ..
template <int LEVEL, typename T, int DK>
__device__ __forceinline__ f32x4 dots(const Planes<T, DK>& a, int i0, const Planes<T, DK>& b, int j0, const Lane& l) {
  f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int s = 0; s < DK / 32; ++s) x = mma<LEVEL>(b.rows(j0, 32 * s, l), a.rows(i0, 32 * s, l), x);
  return x;
}

// N = -X - N beta X of both blocks of 16 rows, by one wave: lane i of each half has row i of a block (twice), and takes
// its columns from the last one on, X's rows read out of LDS.  A row needs no other's, so there is no exchange between
// lanes: 120 multiply-adds behind each other's loads, not their results.
template <bool WITH_P, bool BACK>
__device__ __forceinline__ void put_inverses(Pairs<WITH_P>& to, const Gates& s) {
  const int lane = threadIdx.x & 63, block = lane >> 5, i = lane & 15, columns = lane >> 4 & 1;
  const float* x = to.x[block];
  float n[16], beta[16];
#pragma unroll
  for (int c = 0; c < 16; c += 4) {
    const f32x4 mine = four(x + i * kBlockStride + c), b = four(s.beta + 16 * block + c);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      n[c + e] = -mine[e];
      beta[c + e] = b[e];
    }
  }
  f32x4 row[3][4];  // of X: this column's and the next two
  auto load = [&](int j) {
#pragma unroll
    for (int c = 0; c < j; c += 4) row[j % 3][c / 4] = four(x + j * kBlockStride + c);
  };
  load(15);
  load(14);
#pragma unroll
  for (int j = 15; j > 0; --j) {
    if (j > 2) load(j - 2);
    const float m = n[j] * beta[j];
#pragma unroll
    for (int c = 0; c < j; ++c) n[c] = __builtin_fmaf(-m, row[j % 3][c / 4][c % 4], n[c]);
    // done before further rows are loaded: else all of them are at once, and the registers of the whole kernel are gone
#pragma unroll
    for (int c = 0; c < j; ++c) asm volatile("" : "+v"(n[c])::"memory");
  }
  // half of the row a lane
  const float own = s.beta[16 * block + i];
  f32x4 y[2];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float u = n[e] * (BACK ? own : beta[e]), v = n[8 + e] * (BACK ? own : beta[8 + e]);
    y[e / 4][e % 4] = columns ? v : u;
  }
  bf16* p = to.n[block] + i * kBlockStride + 8 * columns;
  put4<kParts>(p, kBlock, y[0]);
  put4<kParts>(p + 4, kBlock, y[1]);
}

// The waves' shares of a chunk's preparation: the inverses, the last rows with the first, the rest (none where there is no
// P), and the gates, a wave each; of two waves the first has the inverses, the second the others.
template <int NW>
__device__ __forceinline__ bool has_share(int share, const Lane& l) {
  return NW >= 4 ? l.w == share : NW == 3 ? l.w == (share == 3 ? 2 : share) : l.w == (share ? 1 : 0);
}

template <typename T, int DK, int NW, bool WITH_P, bool BACK>
__device__ __forceinline__ void put_pairs(Pairs<WITH_P>& to, const Planes<T, DK>& k, const Planes<T, DK>* q, const Gates& s, float scale,
                                          const Lane& l) {
  const f32x4 one = {1.0f, 1.0f, 1.0f, 1.0f};
  if (has_share<NW>(0, l)) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const f32x4 x = decayed<true>(dots<kParts>(k, 16 * b, k, 16 * b, l), decays(s, 16 * b, 16 * b, l), false, l);
      __builtin_memcpy(__builtin_assume_aligned(to.x[b] + l.n * kBlockStride + 4 * l.g, 16), &x, 16);
    }
    wave_fence();
    put_inverses<WITH_P, BACK>(to, s);
  }
  if (has_share<NW>(1, l)) {
    const f32x4 d = decays(s, 16, 0, l), beta = BACK ? one : four(s.beta + 4 * l.g);
    const f32x4 x = d * (BACK ? one * -s.beta[16 + l.n] : -beta);
    put4<kParts>(to.n[2] + l.n * kBlockStride + 4 * l.g, kBlock, decayed<false>(dots<kParts>(k, 16, k, 0, l), x, false, l));
    if constexpr (WITH_P)
      put4<kParts>(to.p + (16 + l.n) * kPairStride + 4 * l.g, kPairPlane, decayed<false>(dots<kParts>(*q, 16, k, 0, l), d * scale * beta, false, l));
  }
  if constexpr (WITH_P) {
    if (has_share<NW>(2, l)) {
#pragma unroll
      for (int i0 = 0; i0 < kDeltaRows; i0 += 16) {
        const f32x4 d = decays(s, i0, i0, l) * scale;
        put4<kParts>(to.p + (i0 + l.n) * kPairStride + i0 + 4 * l.g, kPairPlane,
                    decayed<true>(dots<kParts>(*q, i0, k, i0, l), BACK ? d : d * four(s.beta + i0 + 4 * l.g), true, l));
      }
    }
  }
}

// ------------------------------------------------------ the state of a wave
//
// Columns col0 + 16 tv + n; of a pair of 16-row tiles 2s and 2s + 1 a lane has rows 32 s + 8g .. 8g+7, so a row of K in
// LDS, read 16 bytes a lane, is the matching operand.

template <int DK, int TV>
using State = f32x4[DK / 16][TV];

__device__ __forceinline__ int state_row(int tile, int r, const Lane& l) { return 32 * (tile / 2) + 8 * l.g + 4 * (tile % 2) + r; }

template <int DK, int TV>
__device__ __forceinline__ void load_state(State<DK, TV>& st, const float* from, int kd, int vd, int col0, const Lane& l) {
#pragma unroll
  for (int t = 0; t < DK / 16; ++t)
#pragma unroll
    for (int v = 0; v < TV; ++v) st[t][v] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  if (!from) return;
  // unconditional loads of an element that is there: they do not wait for each other
#pragma unroll
  for (int t = 0; t < DK / 16; ++t)
#pragma unroll
    for (int v = 0; v < TV; ++v)
#pragma unroll
      for (int r = 0; r < 4; ++r) st[t][v][r] = from[min(state_row(t, r, l), kd - 1) * vd + min(col0 + 16 * v + l.n, vd - 1)];
#pragma unroll
  for (int t = 0; t < DK / 16; ++t)
#pragma unroll
    for (int v = 0; v < TV; ++v)
#pragma unroll
      for (int r = 0; r < 4; ++r) st[t][v][r] = state_row(t, r, l) < kd && col0 + 16 * v + l.n < vd ? st[t][v][r] : 0.0f;
}

template <int DK, int TV>
__device__ __forceinline__ void store_state(float* to, const State<DK, TV>& st, int kd, int vd, int col0, const Lane& l) {
#pragma unroll
  for (int t = 0; t < DK / 16; ++t)
#pragma unroll
    for (int v = 0; v < TV; ++v)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = state_row(t, r, l), col = col0 + 16 * v + l.n;
        if (row < kd && col < vd) to[row * vd + col] = st[t][v][r];
      }
}

// Rows of fp32 in global memory as an operand: row `row`, elements c .. c+7; zeros past the matrix.
__device__ __forceinline__ void load_eight(float (&x)[8], const float* p, int row, int c, int rows, int columns) {
  const bool there = row < rows;
  const float* from = p + (int64_t)(there ? row : 0) * columns;
  if (columns % 8 == 0) {
    const Pack<float, 8> t = load_pack<float, 8>(from + (c < columns ? c : 0));
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = there && c < columns ? t.v[e] : 0.0f;
  } else {
    const Pack<float, 8> t = load_some<float, 8>(from + c, columns - c);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = there ? t.v[e] : 0.0f;
  }
}

// st += map * from, both in global memory: map [kd][kd], from [kd][vd].
template <int DK, int TV>
__device__ __forceinline__ void add_mapped(State<DK, TV>& st, const float* map, const float* from, int kd, int vd, int col0, const Lane& l) {
#pragma unroll
  for (int s = 0; s < DK / 32; ++s) {
    Parts<3> x[TV];
#pragma unroll
    for (int v = 0; v < TV; ++v) {
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int row = 32 * s + 8 * l.g + e, col = col0 + 16 * v + l.n;
        y[e] = from[min(row, kd - 1) * vd + min(col, vd - 1)];
        y[e] = row < kd && col < vd ? y[e] : 0.0f;
      }
      x[v] = split<3>(y);
    }
#pragma unroll
    for (int t = 0; t < DK / 16; ++t) {
      float m[8];
      // lane n has the row that comes out in its place of the state
      load_eight(m, map, 32 * (t / 2) + 8 * (l.n >> 2) + 4 * (t % 2) + (l.n & 3), 32 * s + 8 * l.g, kd, kd);
      const Parts<3> p = split<3>(m);
#pragma unroll
      for (int v = 0; v < TV; ++v) st[t][v] = mma<3>(p, x[v], st[t][v]);
    }
  }
}

// ------------------------------------------------------ the walks

// Where a chunk's states are kept: a sequence's chunks from its first row / 32 + its number on.
__device__ __forceinline__ int64_t place_of(int32_t first, int32_t b, int32_t s0) {
  return (int64_t)(first / kDeltaRows) + (s0 - first) / kDeltaRows + b;
}

enum DeltaMode {
  kDeltaStates,      // the states at the ends of the parts that go on, and what those parts do to a state
  kDeltaOut,         // results
  kDeltaSave,        // what the gradients need: the state before each chunk, the rows' e
  kDeltaBackStates,  // the gradients of the states at the parts' starts
  kDeltaBack         // what the gradients need: that of the state after each chunk, Z
};

struct Nothing {};

// A wave has two tiles of 16 columns: what it reads of the rows' operands serves both, and one's products run in the
// other's shadow.  Value columns are padded to W; beside the states of the parts, further waves of the same workgroup walk
// the columns of what the part does to a state.
constexpr int kWalkTiles = 2;
template <int DK, int W, int MODE>
constexpr int kWalkWaves = (MODE == kDeltaStates ? W + DK : W) / (16 * kWalkTiles);

template <typename T, int DK, int W, int MODE>
struct DeltaShared {
  static constexpr bool BACK = MODE >= kDeltaBackStates, QUERIES = MODE == kDeltaOut || BACK;
  template <bool THERE, typename X>
  using If = std::conditional_t<THERE, X, Nothing>;
  Planes<T, DK> k;
  If<QUERIES, Planes<T, DK>> q;
  If<!BACK, Values<T, W>> v;
  If<BACK, Planes<T, W>> d;
  If<MODE == kDeltaOut, Values<T, W>> out;
  Gates gates[2];
  Pairs<QUERIES> pairs;
};

template <typename T, int DK, int W, int MODE, bool WHOLE>
__global__ __launch_bounds__((64 * kWalkWaves<DK, W, MODE>), delta_waves(sizeof(T), DK, W)) void delta_walk_kernel(DeltaArgs a) {
  using Shared = DeltaShared<T, DK, W, MODE>;
  constexpr int NW = kWalkWaves<DK, W, MODE>, TV = kWalkTiles, THREADS = 64 * NW;
  constexpr int NP = kPlanes<T>;
  constexpr bool BACK = Shared::BACK, QUERIES = Shared::QUERIES, STATES = MODE == kDeltaStates || MODE == kDeltaBackStates;
  __shared__ Shared sh;
  const Lane l = lane_of();
  int unit = blockIdx.x / a.H;
  const int h = blockIdx.x - unit * a.H;
  // columns of the state, or of what a part does to it
  const bool map = MODE == kDeltaStates && l.w >= W / (16 * TV);
  const int col0 = 16 * TV * l.w - (map ? W : 0), columns = map ? a.kd : a.vd;
  const Order o = order_of(a);
  Part q;
  const bool found = find_part(q, o, a, unit, STATES);
  if (MODE == kDeltaStates && h == 0 && threadIdx.x == 0) a.cut_kind[unit] = !found ? -1 : q.began ? 1 : 0;
  if (!found) return;
  int32_t lo = q.lo, hi = q.hi;
  bool began = q.began, goes_on = q.goes_on && q.before < a.cuts;
  int32_t boundary = q.before;  // behind the part
  if constexpr (MODE == kDeltaBackStates) {
    // the part behind the boundary
    lo = q.hi;
    hi = q.next;
    began = true;
    goes_on = q.next < q.end && unit + 1 < a.cuts;
    boundary = unit + 1;
  }
  const int64_t each = (int64_t)a.kd * a.vd;
  const int hk = h / a.group;
  const Source<T, DK, NW, WHOLE> from_k(a.k, hk * a.k_head, a.k_row, a.kd), from_q(QUERIES ? a.q : a.k, QUERIES ? h * a.q_head : 0, a.q_row, a.kd);
  const Source<T, W, NW, WHOLE> from_v(BACK ? a.dout : a.v, BACK ? h * a.d_head : hk * a.v_head, BACK ? a.d_row : a.v_row, a.vd);
  const bool own = col0 < columns && !(map && !began);

  if constexpr (QUERIES) {
    // the first rows have nothing of the last ones
    for (int i = threadIdx.x; i < kParts * 16 * 16; i += THREADS)
      sh.pairs.p[i / 256 * kPairPlane + i % 256 / 16 * kPairStride + 16 + i % 16] = (bf16)0.0f;
  }

  Pack<T, 8> rk[kPacks<DK, NW>], rq[kPacks<DK, NW>], rv[kPacks<W, NW>];
  float rg = 0.0f, rb = 0.0f;
  auto fetch = [&](int32_t s0) {
    from_k.fetch(rk, s0, hi);
    if constexpr (QUERIES) from_q.fetch(rq, s0, hi);
    from_v.fetch(rv, s0, hi);
  };
  // a chunk's gates are loaded two chunks ahead of it, and made one ahead
  auto fetch_gates = [&](int32_t s0) {
    const int64_t row = delta_row(s0, threadIdx.x & 31, hi);
    rg = a.log_decay[row * a.g_row + h];
    rb = a.beta[row * a.b_row + h];
  };
  auto make_gates = [&](int32_t s0, int buffer) {
    const bool there = delta_row_there(s0, threadIdx.x & 31, hi);
    put_gates(sh.gates[buffer], there ? rg : 0.0f, there ? rb : 0.0f, BACK ? 1.0f : there ? rb : 0.0f);
  };
  auto put = [&](int32_t s0) {
    const int n = hi - s0;
    sh.k.template put<NW>(rk, a.kd, n);
    if constexpr (QUERIES) sh.q.template put<NW>(rq, a.kd, n);
    if constexpr (BACK)
      sh.d.template put<NW>(rv, a.vd, n);
    else
      sh.v.template put<NW>(rv, a.vd, n);
  };
  auto store_out = [&](int32_t s0) {
    if constexpr (MODE == kDeltaOut) {
      T* po = static_cast<T*>(a.out) + h * a.o_head;
#pragma unroll
      for (int i = 0; i < kPacks<W, NW>; ++i) {
        const int idx = threadIdx.x + i * THREADS, row = idx / (W / 8), c = idx % (W / 8) * 8;
        if (!delta_row_there(s0, row, hi) || c >= a.vd || row >= kDeltaRows) continue;
        Pack<T, 8> x;
        __builtin_memcpy(&x, __builtin_assume_aligned(sh.out.v + row * sh.out.stride + c, 16), sizeof(x));
        store_some<T, 8>(po + (int64_t)(s0 + row) * a.o_row + c, x, a.vd - c, a.past);
      }
    }
  };

  const int chunks = delta_chunks(lo, hi);
  // (past the last chunk the last one again: loads under a condition would be waited for together with the results' stores)
  auto begin = [&](int c) {
    c = min(c, chunks - 1);
    return delta_chunk(lo, BACK ? chunks - 1 - c : c);
  };
  if (chunks > 0) {
    fetch(begin(0));
    if (has_share<NW>(3, l)) fetch_gates(begin(0));
  }

  State<DK, TV> st;
  {
    const float* from = nullptr;
    if constexpr (MODE == kDeltaStates)
      from = !began && a.init ? a.init + ((int64_t)q.b * a.H + h) * each : nullptr;
    else if constexpr (MODE == kDeltaBackStates)
      from = !goes_on && a.init ? a.init + ((int64_t)q.b * a.H + h) * each : nullptr;
    else if constexpr (MODE == kDeltaBack)
      from = goes_on ? a.cut_grad + ((int64_t)boundary * a.H + h) * each : a.init ? a.init + ((int64_t)q.b * a.H + h) * each : nullptr;
    else
      from = began ? a.cut_state + ((int64_t)(boundary - 1) * a.H + h) * each : a.init ? a.init + ((int64_t)q.b * a.H + h) * each : nullptr;
    load_state<DK, TV>(st, map ? nullptr : from, a.kd, columns, col0, l);
    if constexpr (!STATES) {
      // the end of the run of boundaries before
      const int e = BACK ? boundary : boundary - 1, run = BACK ? e / a.run + 1 : e / a.run - 1;
      if ((BACK ? goes_on : began) && own && a.from_run[BACK][e] && run >= 0 && run * a.run < a.cuts)
        add_mapped<DK, TV>(st, a.run_map[BACK] + ((int64_t)e * a.H + h) * a.kd * a.kd, a.run_end[BACK] + ((int64_t)run * a.H + h) * each, a.kd,
                           a.vd, col0, l);
    }
    if (map) {
#pragma unroll
      for (int t = 0; t < DK / 16; ++t)
#pragma unroll
        for (int v = 0; v < TV; ++v)
#pragma unroll
          for (int r = 0; r < 4; ++r) st[t][v][r] = state_row(t, r, l) == col0 + 16 * v + l.n ? 1.0f : 0.0f;
    }
  }

  // arrived: else its first use in the loop would wait, in every round, for all loads that are on their way by then
#pragma unroll
  for (int t = 0; t < DK / 16; ++t)
#pragma unroll
    for (int v = 0; v < TV; ++v) asm volatile("" : "+v"(st[t][v]));

  if (chunks > 0) {
    if (has_share<NW>(3, l)) {
      make_gates(begin(0), 0);
      fetch_gates(begin(1));
    }
    put(begin(0));
    __syncthreads();
  }
  for (int c = 0; c < chunks; ++c) {
    const int32_t s0 = begin(c), next = begin(c + 1);
    const Gates& gates = sh.gates[c & 1];
    fetch(next);
    if (has_share<NW>(3, l)) {
      make_gates(next, (c + 1) & 1);
      fetch_gates(begin(c + 2));
    }
    put_pairs<T, DK, NW, QUERIES, BACK>(sh.pairs, sh.k, reinterpret_cast<const Planes<T, DK>*>(&sh.q), gates, a.scale, l);

    // the products with the state: K S, lane n column n of it; and (Q S) transposed, lane n row n
    f32x4 ks[2][TV], qs[2][TV];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int v = 0; v < TV; ++v) ks[t][v] = qs[t][v] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (own) {
#pragma unroll
      for (int s = 0; s < DK / 32; ++s) {
        Parts<kParts> x[TV];
#pragma unroll
        for (int v = 0; v < TV; ++v) x[v] = split<kParts>(st[2 * s][v], st[2 * s + 1][v]);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const Parts<NP> k = sh.k.rows(16 * t, 32 * s, l);
#pragma unroll
          for (int v = 0; v < TV; ++v) ks[t][v] = mma<kParts>(k, x[v], ks[t][v]);
          if constexpr (MODE == kDeltaOut) {
            const Parts<NP> qr = sh.q.rows(16 * t, 32 * s, l);
#pragma unroll
            for (int v = 0; v < TV; ++v) qs[t][v] = mma<kParts>(x[v], qr, qs[t][v]);
          }
        }
      }
      if constexpr (MODE == kDeltaSave || MODE == kDeltaBack) {
        const int64_t place = place_of(o.bound(q.b), q.b, s0);
        store_state<DK, TV>((BACK ? a.after : a.before) + (place * a.H + h) * each, st, a.kd, a.vd, col0, l);
      }
    }
    __syncthreads();  // the pairs are there
    if (own) {
      const float whole = gates.whole;
      f32x4 fade[2], left[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        fade[t] = four(gates.fade + 16 * t + 4 * l.g);
        left[t] = four(gates.left + 16 * t + 4 * l.g);
      }
      f32x4 e[2][TV];
      Quarter<kParts> ep[2][TV];  // forwards e's parts
      Parts<NP> dout[TV];
      {
        // forwards the first 16 rows first, backwards the last
        constexpr int F = BACK ? 1 : 0, L = 1 - F;
        if constexpr (BACK) {
          // W = what the state's gradient and the results' owe the rows
          const Parts<3> pt[2] = {columns_of<3>(sh.pairs.p, kPairPlane, kPairStride, 0, l),
                                  columns_of<3>(sh.pairs.p, kPairPlane, kPairStride, 16, l)};
#pragma unroll
          for (int v = 0; v < TV; ++v) {
            dout[v] = sh.d.columns(col0 + 16 * v, l);
#pragma unroll
            for (int t = 0; t < 2; ++t) e[t][v] = mma<3>(pt[t], dout[v], ks[t][v] * left[t]);
          }
        } else {
#pragma unroll
          for (int v = 0; v < TV; ++v)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
              if (!map) x = sh.v.down(16 * t, col0 + 16 * v, l);
#pragma unroll
              for (int r = 0; r < 4; ++r) e[t][v][r] = __builtin_fmaf(-fade[t][r], ks[t][v][r], x[r]);
            }
        }
        const Block first = block_of<BACK>(sh.pairs.n[F], l), cross = block_of<BACK>(sh.pairs.n[2], l), last = block_of<BACK>(sh.pairs.n[L], l);
#pragma unroll
        for (int v = 0; v < TV; ++v) {
          e[F][v] = mma_block(first, split<kParts>(e[F][v]), e[F][v]);
          ep[F][v] = split<kParts>(e[F][v]);
          e[L][v] = mma_block(cross, ep[F][v], e[L][v]);
          e[L][v] = mma_block(last, split<kParts>(e[L][v]), e[L][v]);
          if constexpr (MODE == kDeltaOut) ep[L][v] = split<kParts>(e[L][v]);
        }
      }
      if constexpr (MODE == kDeltaSave || MODE == kDeltaBack) {
        float* to = (BACK ? a.due : a.left_over) + (int64_t)h * a.vd;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int32_t row = s0 + 16 * t + 4 * l.g + r;  // (a call with gradients has fewer than 2^29 rows)
#pragma unroll
            for (int v = 0; v < TV; ++v) {
              const int col = col0 + 16 * v + l.n;
              if (row < hi && col < a.vd) to[(int64_t)row * a.H * a.vd + col] = e[t][v][r];
            }
          }
      }
      if constexpr (MODE == kDeltaOut) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const Parts<kParts> p = rows_split<kParts>(sh.pairs.p, kPairPlane, kPairStride, 16 * t, l);
          const float f = gates.fade[16 * t + l.n] * a.scale;
#pragma unroll
          for (int v = 0; v < TV; ++v) {
            const f32x4 x = mma<kParts>(both<kParts>(ep[0][v], ep[1][v]), p, qs[t][v] * f);
            Pack<T, 4> y;
#pragma unroll
            for (int r = 0; r < 4; ++r) y.v[r] = (T)x[r];
            __builtin_memcpy(__builtin_assume_aligned(sh.out.v + (16 * t + l.n) * sh.out.stride + col0 + 16 * v + 4 * l.g, 4 * sizeof(T)), &y, sizeof(y));
          }
        }
      }
      // the state after the chunk (backwards: its gradient before it)
      Parts<kParts> x[TV], y[TV];
      const f32x4 beta[2] = {four(gates.beta + 4 * l.g), four(gates.beta + 16 + 4 * l.g)};
#pragma unroll
      for (int v = 0; v < TV; ++v) {
        if constexpr (BACK) {
          float f[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            f[i] = 0.0f;
#pragma unroll
            for (int p = 0; p < NP; ++p) f[i] += (float)dout[v].p[p][i];
            f[i] *= fade[i / 4][i % 4] * a.scale;
          }
          y[v] = split<kParts>(f);
          x[v] = split<kParts>(-(fade[0] * beta[0] * e[0][v]), -(fade[1] * beta[1] * e[1][v]));
        } else {
          x[v] = split<kParts>(left[0] * e[0][v], left[1] * e[1][v]);  // (beta is in there)
        }
      }
#pragma unroll
      for (int t = 0; t < DK / 16; ++t) {
        const int c0 = 32 * (t / 2) + 4 * (t % 2);
        const Parts<NP> k = sh.k.template columns<8>(c0, l);
#pragma unroll
        for (int v = 0; v < TV; ++v) st[t][v] = mma<kParts>(k, x[v], st[t][v] * whole);
        if constexpr (BACK) {
          const Parts<NP> qc = sh.q.template columns<8>(c0, l);
#pragma unroll
          for (int v = 0; v < TV; ++v) st[t][v] = mma<kParts>(qc, y[v], st[t][v]);
        }
      }
    }
    __syncthreads();  // the results are there, the chunk has been read
    store_out(s0);
    put(next);
    __syncthreads();
  }
  if (!own) return;
  if constexpr (STATES) {
    if (map) {
      const int64_t at = ((int64_t)unit * a.H + h) * a.kd * a.kd;
      store_state<DK, TV>(a.cut_map + at, st, a.kd, a.kd, col0, l);
      if (a.cut_grad) {
#pragma unroll
        for (int t = 0; t < DK / 16; ++t)
#pragma unroll
          for (int v = 0; v < TV; ++v)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int row = state_row(t, r, l), col = col0 + 16 * v + l.n;
              if (row < a.kd && col < a.kd) a.cut_turned[at + col * a.kd + row] = st[t][v][r];
            }
      }
    } else
      store_state<DK, TV>((BACK ? a.cut_grad : a.cut_state) + ((int64_t)unit * a.H + h) * each, st, a.kd, a.vd, col0, l);
  } else {
    if ((BACK ? !began : !goes_on) && a.final_state)
      store_state<DK, TV>(a.final_state + ((int64_t)q.b * a.H + h) * each, st, a.kd, a.vd, col0, l);
  }
}

// ------------------------------------------------------ the gradients of a chunk
//
// With the state S before it, the gradient D of the one after it, and the
// rows' E and Z (U = beta E, Y = beta Z):
//   dQ = scale e^G dout S^T + A K,                   A_ij = scale e^(G_i - G_j) dout_i . u_j, j <= i
//   dK = [-e^G Y S^T - F K] + [e^(G_end - G) U D^T - F^T K + A^T Q],  F_ij = e^(G_i - G_j) y_i . u_j, j < i
//   dV = Y,  dbeta = Z . E.
// A row's G scales what it reads (q and, in the first bracket, k) and divides
// what it writes (the second bracket), so
//   dG_i = q_i . dQ_i + k_i . (first - second)_i,  and G_end has <D, S_after>;
// the gradient of a row's log decay is the sum of dG from it on.  With the term
// in D kept apart, kd_j = k_j . (e^(G_end - G_j) u_j D^T), that is
//   sum_{i >= t} (dG_i without it) + e^(G_end) <D, S> + sum_{j < t} kd_j.
//
// A workgroup has a chunk and the heads that share its key; the walks left S,
// D, E and Z in memory.  Reading them is what bounds it (213,879 rows, 8 heads
// of 64 over 4 in bf16: 3.5 GB in 852 us, 4.1 TB/s): states between chunks of
// 32 rows are four times a chunk's keys and values.

constexpr int kGradWaves = 4;

template <typename T, int DK, int TV>
struct DeltaGradShared {
  Planes<T, DK> k, q;
  Planes<T, 64 * TV> d;
  Planes<float, 64 * TV> y;
  union {  // A and F take U's place when it has been read
    Planes<float, 64 * TV> u;
    struct {
      __attribute__((aligned(16))) bf16 a[3 * kPairPlane], f[3 * kPairPlane];
    };
  };
  __device__ DeltaGradShared() {}
  Gates gates;
  float own[4][kDeltaRows], end[4][kDeltaRows];  // a wave's part of dG and of kd
  float both[4];                                 // of <D, S>
};

// Sum over the four lane groups of the same lane % 16, known to all.
__device__ __forceinline__ float groups_sum(float x) {
  unsigned i = __builtin_bit_cast(unsigned, x);
  const auto p = __builtin_amdgcn_permlane16_swap(i, i, false, false);
  x = __builtin_bit_cast(float, (unsigned)p[0]) + __builtin_bit_cast(float, (unsigned)p[1]);
  i = __builtin_bit_cast(unsigned, x);
  const auto q = __builtin_amdgcn_permlane32_swap(i, i, false, false);
  return __builtin_bit_cast(float, (unsigned)q[0]) + __builtin_bit_cast(float, (unsigned)q[1]);
}

// The sequence whose chunks lie from `place` back, and whether it has one there: first row / 32 + sequence grows with the
// sequence, so 64 are looked at at a time.
__device__ __forceinline__ bool chunk_at(int64_t place, const Order& o, int32_t& b, int32_t& s0, int32_t& hi) {
  const int lane = threadIdx.x & 63;
  int32_t first = 0, count = o.B;  // candidates
  while (count > 1) {
    const int32_t step = (count + 63) / 64, k = first + lane * step;
    const bool upto = k < first + count && (int64_t)(o.bound(min(k, o.B - 1)) / kDeltaRows) + k <= place;
    const uint64_t m = __ballot(upto);
    const int32_t at = m ? 63 - __builtin_clzll(m) : 0;
    count = min(step, count - at * step);
    first += at * step;
  }
  b = __builtin_amdgcn_readfirstlane(first);
  const int32_t lo = o.bound(b);
  hi = o.bound(b + 1);
  const int64_t begin = lo + (place - lo / kDeltaRows - b) * kDeltaRows;
  s0 = (int32_t)begin;
  return begin >= lo && begin < hi;
}

template <typename T, int DK, int TV, bool WHOLE>
__global__ __launch_bounds__(64 * kGradWaves, delta_grad_waves(__is_same(T, f16), sizeof(T), DK, 64 * TV)) void delta_grad_kernel(DeltaGradArgs a) {
  constexpr int NP = kPlanes<T>, W = 64 * TV, TD = DK >= 64 ? DK / 64 : 1, PER = W / 8;
  // where a compute unit has one or two workgroups the states are on their way while the rows are worked on (fp16 heads of
  // 128 214 -> 186 us; the whole call of 8 crowded frames in fp32 4,090 -> 4,050, in fp16 3,195 -> 3,140); where it has
  // three, the registers run out (bf16 890 -> 1,114)
  constexpr bool EARLY = delta_grad_waves(__is_same(T, f16), sizeof(T), DK, W) < 3;
  __shared__ DeltaGradShared<T, DK, TV> sh;
  const Lane l = lane_of();
  const int KV = a.H / a.group, hk = blockIdx.x % KV;
  const int64_t place = blockIdx.x / KV;
  const Order o = order_of(a);
  int32_t b, s0, hi;
  if (!chunk_at(place, o, b, s0, hi)) return;
  const int n = min(hi - s0, kDeltaRows);
  const int64_t each = (int64_t)a.kd * a.vd;
  const bool own = 16 * TD * l.w < DK;
  Pack<T, 8> rk[kPacks<DK, kGradWaves>];
  Source<T, DK, kGradWaves, WHOLE>(a.k, hk * a.k_head, a.k_row, a.kd).fetch(rk, s0, hi);
  float dv[kPacks<W, kGradWaves>][8];
  f32x4 dk[2][TD];
#pragma unroll
  for (int i = 0; i < kPacks<W, kGradWaves>; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) dv[i][e] = 0.0f;
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int d = 0; d < TD; ++d) dk[t][d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  for (int j = 0; j < a.group; ++j) {
    const int h = hk * a.group + j;
    Pack<float, 8> before[W / 32][TD], after[W / 32][TD];
    const float *pb = a.before + (place * a.H + h) * each, *pa = a.after + (place * a.H + h) * each;
    {
      Pack<T, 8> rq[kPacks<DK, kGradWaves>], rd[kPacks<W, kGradWaves>];
      Pack<float, 8> re[kPacks<W, kGradWaves>], rz[kPacks<W, kGradWaves>];
      Source<T, DK, kGradWaves, WHOLE>(a.q, h * a.q_head, a.q_row, a.kd).fetch(rq, s0, hi);
      Source<T, W, kGradWaves, WHOLE>(a.dout, h * a.d_head, a.d_row, a.vd).fetch(rd, s0, hi);
      Source<float, W, kGradWaves, WHOLE>(a.left_over, h * a.vd, a.H * a.vd, a.vd).fetch(re, s0, hi);
      Source<float, W, kGradWaves, WHOLE>(a.due, h * a.vd, a.H * a.vd, a.vd).fetch(rz, s0, hi);
      float g = 0.0f, beta = 0.0f;
      if (l.w == 3 && (int)(threadIdx.x & 31) < n) {
        const int64_t row = s0 + (int)(threadIdx.x & 31);
        g = a.log_decay[row * a.g_row + h];
        beta = a.beta[row * a.b_row + h];
      }
      float rb[kPacks<W, kGradWaves>];
#pragma unroll
      for (int i = 0; i < kPacks<W, kGradWaves>; ++i)
        rb[i] = a.beta[(int64_t)min(s0 + (int)(threadIdx.x + i * 64 * kGradWaves) / PER, hi - 1) * a.b_row + h];
      if constexpr (EARLY) {
#pragma unroll
        for (int s = 0; s < W / 32; ++s)
#pragma unroll
          for (int d = 0; d < TD; ++d) {
            // (rows past the last one are its copies)
            const int row = min(16 * (l.w * TD + d) + l.n, a.kd - 1) * a.vd, c = 32 * s + 8 * l.g;
            if constexpr (WHOLE) {
              before[s][d] = load_pack<float, 8>(pb + row + min(c, a.vd - 8));
              after[s][d] = load_pack<float, 8>(pa + row + min(c, a.vd - 8));
            } else {
              before[s][d] = load_some<float, 8>(pb + row + c, a.vd - c);
              after[s][d] = load_some<float, 8>(pa + row + c, a.vd - c);
            }
          }
      }
      if (j) __syncthreads();  // the head before has been read
      if (j == 0) sh.k.template put<kGradWaves>(rk, a.kd, n);
      sh.q.template put<kGradWaves>(rq, a.kd, n);
      sh.d.template put<kGradWaves>(rd, a.vd, n);
      if (l.w == 3) put_gates(sh.gates, g, beta, 1.0f);
      int i = 0;
      each_pack<float, W, kGradWaves>(re, a.vd, n, [&](int row, int c, Pack<float, 8> x) {
        float dot = 0.0f;
        Pack<float, 8> y;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float z = row < n && c < a.vd ? rz[i].v[e] : 0.0f;
          dot = __builtin_fmaf(z, x.v[e], dot);
          y.v[e] = rb[i] * z;
          x.v[e] = rb[i] * x.v[e];
          dv[i][e] += y.v[e];
        }
        put_planes<3, float>(sh.u.v + row * sh.u.stride + c, sh.u.plane, x);
        put_planes<3, float>(sh.y.v + row * sh.y.stride + c, sh.y.plane, y);
        dot = group_sum<PER>(dot);
        if (c == 0 && row < n) a.dbeta[(int64_t)(s0 + row) * a.db_row + h] = dot;
        ++i;
      });
    }
    __syncthreads();
    const Gates& gates = sh.gates;
    // A (results) and F: lane n row i, elements j0 + 4g ..
    auto pairs = [&](int i0, int j0, bool results) {
      f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int s = 0; s < W / 32; ++s) {
        const Parts<3> u = sh.u.rows(j0, 32 * s, l);
        x = results ? mma<3>(u, sh.d.rows(i0, 32 * s, l), x) : mma<3>(u, sh.y.rows(i0, 32 * s, l), x);
      }
      f32x4 d = decays(gates, i0, j0, l);
      if (results) d = d * a.scale;
      return i0 == j0 ? decayed<true>(x, d, results, l) : decayed<false>(x, d, results, l);
    };
    f32x4 one_pair, other_pair = {0.0f, 0.0f, 0.0f, 0.0f};
    if (l.w < 2) {
      one_pair = pairs(16 * l.w, 16 * l.w, true);
      other_pair = pairs(16 * l.w, 16 * l.w, false);
    } else {
      one_pair = pairs(16, 0, l.w == 2);
    }
    // what comes through the states: lane n row n, elements of dk 4g ..
    f32x4 read_q[2][TD], read_k[2][TD], written[2][TD];
    float both = 0.0f;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int d = 0; d < TD; ++d) read_q[t][d] = read_k[t][d] = written[t][d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (own) {
#pragma unroll
      for (int s = 0; s < W / 32; ++s) {
#pragma unroll
        for (int d = 0; d < TD; ++d) {
          const int row = 16 * (l.w * TD + d) + l.n;
          float x[8], z[8];
          if constexpr (EARLY) {
            const bool there = row < a.kd && 32 * s + 8 * l.g < a.vd;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              x[e] = there ? before[s][d].v[e] : 0.0f;
              z[e] = there ? after[s][d].v[e] : 0.0f;
            }
          } else {
            load_eight(x, pb, row, 32 * s + 8 * l.g, a.kd, a.vd);
            load_eight(z, pa, row, 32 * s + 8 * l.g, a.kd, a.vd);
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) both = __builtin_fmaf(x[e], z[e], both);
          const Parts<3> sp = split<3>(x), gp = split<3>(z);
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            read_q[t][d] = mma<3>(sp, sh.d.rows(16 * t, 32 * s, l), read_q[t][d]);
            read_k[t][d] = mma<3>(sp, sh.y.rows(16 * t, 32 * s, l), read_k[t][d]);
            written[t][d] = mma<3>(gp, sh.u.rows(16 * t, 32 * s, l), written[t][d]);
          }
        }
      }
    }
    both = group_sum<64>(both);
    __syncthreads();  // U has been read
    {
      const int i0 = l.w < 2 ? 16 * l.w : 16, j0 = l.w < 2 ? i0 : 0;
      const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
      put4<3>((l.w == 3 ? sh.f : sh.a) + (i0 + l.n) * kPairStride + j0 + 4 * l.g, kPairPlane, one_pair);
      if (l.w < 2)
        put4<3>(sh.f + (i0 + l.n) * kPairStride + j0 + 4 * l.g, kPairPlane, other_pair);
      else  // the first rows have nothing of the last ones
        put4<3>((l.w == 3 ? sh.f : sh.a) + l.n * kPairStride + 16 + 4 * l.g, kPairPlane, zero);
    }
    __syncthreads();  // A and F are there
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      float own_sum = 0.0f, end_sum = 0.0f;
      if (own) {
        const float fade = gates.fade[16 * t + l.n], left = gates.left[16 * t + l.n];
        const Parts<3> ar = rows_split<3>(sh.a, kPairPlane, kPairStride, 16 * t, l), fr = rows_split<3>(sh.f, kPairPlane, kPairStride, 16 * t, l);
        const Parts<3> ac = columns_of<3>(sh.a, kPairPlane, kPairStride, 16 * t, l), fc = columns_of<3>(sh.f, kPairPlane, kPairStride, 16 * t, l);
#pragma unroll
        for (int d = 0; d < TD; ++d) {
          const int c0 = 16 * (l.w * TD + d), row = 16 * t + l.n, c = c0 + 4 * l.g;
          const Parts<NP> kc = sh.k.columns(c0, l), qc = sh.q.columns(c0, l);
          const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
          const f32x4 dq = mma<3>(kc, ar, read_q[t][d] * (fade * a.scale));
          const f32x4 reads = -mma<3>(kc, fr, read_k[t][d] * fade);
          const f32x4 writes = mma<3>(qc, ac, -mma<3>(kc, fc, zero)), end = written[t][d] * left;
          const f32x4 qv = sh.q.at(row, c), kv = sh.k.at(row, c);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            own_sum += __builtin_fmaf(qv[r], dq[r], kv[r] * (reads[r] - writes[r]));
            end_sum = __builtin_fmaf(kv[r], end[r], end_sum);
          }
          dk[t][d] += reads + writes + end;
          if (row < n) {
            Pack<T, 4> x;
#pragma unroll
            for (int r = 0; r < 4; ++r) x.v[r] = (T)dq[r];
            store_some<T, 4>(static_cast<T*>(a.dq) + (int64_t)(s0 + row) * a.dq_row + h * a.dq_head + c, x, a.kd - c);
          }
        }
      }
      own_sum = groups_sum(own_sum);
      end_sum = groups_sum(end_sum);
      if (l.g == 0) {
        sh.own[l.w][16 * t + l.n] = own_sum;
        sh.end[l.w][16 * t + l.n] = end_sum;
      }
    }
    if ((threadIdx.x & 63) == 0) sh.both[l.w] = both;
    __syncthreads();
    if (l.w == 0) {
      const int r = threadIdx.x & 31, back = kDeltaRows - 1 - r;
      float from = 0.0f, upto = 0.0f;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        from += sh.own[w][back];
        upto += sh.end[w][r];
      }
      const float whole = gates.whole * ((sh.both[0] + sh.both[1]) + (sh.both[2] + sh.both[3]));
      const float after_row = __shfl(half_wave_sums(from), back), before_row = half_wave_sums(upto) - upto;
      if ((threadIdx.x & 63) < n) {
        const int64_t row = s0 + r;
        const float g = a.log_decay[row * a.g_row + h];
        a.dlog_decay[row * a.dg_row + h] = g > 0.0f ? 0.0f : after_row + whole + before_row;
      }
    }
  }
  if (own) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int d = 0; d < TD; ++d) {
        const int row = 16 * t + l.n, c = 16 * (l.w * TD + d) + 4 * l.g;
        if (row >= n) continue;
        Pack<T, 4> x;
#pragma unroll
        for (int r = 0; r < 4; ++r) x.v[r] = (T)dk[t][d][r];
        store_some<T, 4>(static_cast<T*>(a.dk) + (int64_t)(s0 + row) * a.dk_row + hk * a.dk_head + c, x, a.kd - c);
      }
  }
#pragma unroll
  for (int i = 0; i < kPacks<W, kGradWaves>; ++i) {
    const int idx = threadIdx.x + i * 64 * kGradWaves, row = idx / PER, c = idx % PER * 8;
    if (row >= n || c >= a.vd) continue;
    Pack<T, 8> x;
#pragma unroll
    for (int e = 0; e < 8; ++e) x.v[e] = (T)dv[i][e];
    store_some<T, 8>(static_cast<T*>(a.dv) + (int64_t)(s0 + row) * a.dv_row + hk * a.dv_head + c, x, a.vd - c, a.past);
  }
}

// ------------------------------------------------------ launches

// Instances by the key dim padded to 32, 64 or 128 and the value dim to 64 or 128.
template <typename F>
void with_dims(int kd, int vd, F&& f) {
  auto values = [&](auto key) {
    vd <= 64 ? f(key, std::integral_constant<int, 64>{}) : f(key, std::integral_constant<int, 128>{});
  };
  kd <= 32 ? values(std::integral_constant<int, 32>{}) : kd <= 64 ? values(std::integral_constant<int, 64>{}) : values(std::integral_constant<int, 128>{});
}

bool whole_packs(const DeltaArgs& a) { return a.kd % 8 == 0 && a.vd % 8 == 0; }

template <typename T, int MODE>
hipError_t walk_of(const DeltaArgs& a, hipStream_t st) {
  with_dims(a.kd, a.vd, [&](auto key, auto value) {
    constexpr int DK = decltype(key)::value, W = decltype(value)::value;
    constexpr bool states = MODE == kDeltaStates || MODE == kDeltaBackStates;
    static_assert(delta_groups(__is_same(T, f16), sizeof(T), DK, W) * sizeof(DeltaShared<T, DK, W, MODE>) <= 160 * 1024, "the plan's workgroups fit");
    const dim3 grid((uint32_t)((states ? a.cuts : a.cuts + a.B) * (int64_t)a.H));
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(64 * kWalkWaves<DK, W, MODE>), 0, st, a); };
    whole_packs(a) ? go(delta_walk_kernel<T, DK, W, MODE, true>) : go(delta_walk_kernel<T, DK, W, MODE, false>);
  });
  return hipGetLastError();
}

template <typename T>
hipError_t grad_of(const DeltaGradArgs& a, hipStream_t st) {
  with_dims(a.kd, a.vd, [&](auto key, auto value) {
    constexpr int DK = decltype(key)::value, TV = decltype(value)::value / 64;
    const dim3 grid((uint32_t)(delta_slots(a.rows, a.B) * (a.H / a.group)));
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(64 * kGradWaves), 0, st, a); };
    whole_packs(a) ? go(delta_grad_kernel<T, DK, TV, true>) : go(delta_grad_kernel<T, DK, TV, false>);
  });
  return hipGetLastError();
}

template <typename T>
hipError_t delta_walk(const DeltaArgs& a, int mode, hipStream_t st) {
  switch (mode) {
    case kDeltaStates: return walk_of<T, kDeltaStates>(a, st);
    case kDeltaOut: return walk_of<T, kDeltaOut>(a, st);
    case kDeltaSave: return walk_of<T, kDeltaSave>(a, st);
    case kDeltaBackStates: return walk_of<T, kDeltaBackStates>(a, st);
    default: return walk_of<T, kDeltaBack>(a, st);
  }
}

}  // namespace
}  // namespace mmbev
