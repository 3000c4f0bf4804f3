// Linear attention with a decay per head: the chunked kernels (one
// translation unit a type includes this).
//
// With lambda = exp(log_decay) and rows numbered from the sequence's start,
//   out_i = scale * sum_{j <= i} lambda^(i-j) (a_i . b_j) c_j  +  scale * lambda^(i+1) a_i S,
//   S' = lambda^n S + sum_j lambda^(n-1-j) b_j^T c_j
// holds for any run of n rows with the state S before it, so a workgroup walks
// a sequence in chunks of 64 rows and carries S in registers, in fp32.  A
// chunk is three products of 64 rows for the matrix cores and one that updates
// the state; a row's arithmetic, some 8 D + 2 * 64 multiply-adds an element,
// stays several times under what the cores do while the row's bytes arrive,
// so the layout saves bytes and waits, not products:
//
// - everything is computed transposed (out^T = c^T P^T, P^T = b a^T): a
//   product's result then lies across the lanes as the next product wants its
//   operand, so P goes from accumulators to operand in registers, and a lane
//   ends with four neighbouring elements of one output row;
// - a wave owns 16 rows of the chunk and needs only b's rows up to them; a goes
//   from memory straight into the operand, b and c through LDS, where the
//   transposed reads of gfx950 take columns of 16-bit elements;
// - the state's columns are shared out among the waves; each chunk its
//   rounded copy is put into LDS for the product with a;
// - the next chunk's loads are issued before this one's products.
//
// Heads of 8 x 64 in bf16, forward: 128 frames (921,997 rows) 986 us, 3.8 TB/s,
// bound by the chain of a chunk; a sequence of 120,000 rows 172 us, where keys
// and values are read twice, once for the parts' states.  Gradients over 213,879
// rows in 8 sequences 607 us: all of them cut, 2.6 GB moved at 4.3 TB/s.
//
// The gradients are the same recurrence: dq forwards as (dout, v, k); dv and dk
// backwards in time as (k, q, dout) and (v, dout, q), whose states are one
// another's transposes, so one walk makes both (walk_back).
// Backwards the state is carried one decay later, S' = lambda^n S + sum_j
// lambda^(n-j) b_j^T c_j with lambda^i in place of lambda^(i+1), so that a
// gradient of the final state enters undecayed and the last S is the initial
// state's.
//
// 16-bit types: the rows that enter the state are c times its decay in two
// parts, the rounded value and what the rounding left: 16 or 22 bits instead of
// the type's 8 or 11; in bf16 a third part makes them 24 where the state is
// asked for.  P and the state's copy take part in two parts as well, so that a
// result is off by its own rounding and no more (rounded once they add an error
// of that size, 1.4 times it together; the four more products cost 128 frames
// 979 us instead of 918, the gradients of 8 crowded frames 607 instead of 514,
// those of one robot frame's heads of 128, where the parts take turns in LDS,
// 152 instead of 109).
//
// fp16 has too few exponents for what its own values make: a product of two
// rows passes 65,504, a small gradient's decayed rows fall under 2^-24.  So
// whatever becomes fp16 inside is divided by a power of two first and the
// product multiplied by it in fp32: the state's copy (one power), the pairs'
// factors (one a row of the result and 32 rows of the chunk), the decayed rows
// (one a column of the state).  The robot frame's gradients 166 us, 152 without.
#pragma once

#include "common.hpp"
#include "sequence.hpp"

namespace mmbev {
namespace {

constexpr int kAttnThreads = 256, kAttnWaves = 4;
constexpr int kChunk = 64;  // rows of a chunk: 16 a wave

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

// ------------------------------------------------------ operands

// Eight elements a lane, of a 32-deep product.  Lane l holds row (or column)
// l % 16; with g = l / 16 its elements are 8g..8g+7 along a row of memory
// (load_rows) or, down a column, 4g..4g+3 and 16+4g..16+4g+3 (load_cols, and
// two results of 16 x 16: lane l of a result has column l % 16, rows
// 4g..4g+3).  Both operands of a product use the same of the two orders.
template <typename T>
struct Frag {
  T v[8];
};

template <typename T>
__device__ __forceinline__ Frag<T> load_rows(const T* s, int stride, int row0, int col0) {
  const int l = threadIdx.x & 63;
  const T* p = s + (row0 + (l & 15)) * stride + col0 + (l >> 4) * 8;
  Frag<T> f;
  __builtin_memcpy(&f, __builtin_assume_aligned(p, 16), sizeof(f));
  return f;
}

// Along a row in load_cols' order.
template <typename T>
__device__ __forceinline__ Frag<T> load_rows_split(const T* s, int stride, int row0, int col0) {
  const int l = threadIdx.x & 63;
  const T* p = s + (row0 + (l & 15)) * stride + col0 + (l >> 4) * 4;
  Frag<T> f;
  __builtin_memcpy(&f.v[0], __builtin_assume_aligned(p, 4 * sizeof(T)), 4 * sizeof(T));
  __builtin_memcpy(&f.v[4], __builtin_assume_aligned(p + 16, 4 * sizeof(T)), 4 * sizeof(T));
  return f;
}

template <typename T>
__device__ __forceinline__ Frag<T> load_cols(const T* s, int stride, int row0, int col0) {
  const int l = threadIdx.x & 63, g = l >> 4, n = l & 15;
  Frag<T> f;
  if constexpr (sizeof(T) == 2) {
    // a transposed read: lane n of a group of 16 names 4 elements of row n / 4 and gets column n of the four rows
    const T* p = s + (row0 + 4 * g + (n >> 2)) * stride + col0 + (n & 3) * 4;
    using P = __attribute__((address_space(3))) s16x4*;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(p));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(p + 16 * stride));
    __builtin_memcpy(&f.v[0], &lo, 8);
    __builtin_memcpy(&f.v[4], &hi, 8);
  } else {
    const T* p = s + (row0 + 4 * g) * stride + col0 + n;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      f.v[e] = p[e * stride];
      f.v[4 + e] = p[(16 + e) * stride];
    }
  }
  return f;
}

__device__ __forceinline__ f32x4 mma(const Frag<bf16>& a, const Frag<bf16>& b, f32x4 c) {
  typedef bf16 v8 __attribute__((ext_vector_type(8)));
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(const Frag<f16>& a, const Frag<f16>& b, f32x4 c) {
  typedef f16 v8 __attribute__((ext_vector_type(8)));
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(const Frag<float>& a, const Frag<float>& b, f32x4 c) {
#pragma unroll
  for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[e], b.v[e], c, 0, 0, 0);
  return c;
}

// ------------------------------------------------------ sequences

// Positions run over the rows in use, from the last row backwards where the
// call is reversed; sequence k in that order begins at bound(k).
struct Order {
  const int64_t* offsets;
  int64_t ahead[2];  // offsets of this lane's sequence, if it is one of the first 64
  int32_t used, B, reversed;
  __device__ __forceinline__ int32_t clamped(int64_t o) const {
    const int32_t c = o < 0 ? 0 : o > used ? used : (int32_t)o;
    return reversed ? used - c : c;
  }
  __device__ __forceinline__ int32_t bound(int32_t k) const { return clamped(offsets[reversed ? B - k : k]); }
  __device__ __forceinline__ int32_t row(int32_t p) const { return reversed ? used - 1 - p : p; }
  __device__ __forceinline__ int32_t sequence(int32_t k) const { return reversed ? B - 1 - k : k; }
};

__device__ __forceinline__ Order order_of(const AttnWalk& a) {
  Order o;
  o.offsets = a.offsets;
  o.B = a.B;
  o.reversed = a.reversed;
  // all of these loads before the first is waited for
  const int k = min((int)(threadIdx.x & 63), a.B - 1);
  o.ahead[0] = a.offsets[a.reversed ? a.B - k : k];
  o.ahead[1] = a.offsets[a.reversed ? a.B - k - 1 : k + 1];
  const int64_t end = a.offsets[a.B];
  o.used = end < 0 ? 0 : end > a.rows ? (int32_t)a.rows : (int32_t)end;
  return o;
}

// A run of rows that one workgroup walks: a sequence, or a part of one.
struct Part {
  int32_t lo, hi;  // positions
  int32_t b;       // sequence
  int32_t before;  // parts that go on (into another of their sequence) before this one
  bool began;      // a part of the sequence comes before it
  bool goes_on;    // and after it
};

// The r-th longest of up to 256 sequences that are not longer than `most`
// (ties: the first ones first), found bit by bit: the largest length that more
// than r of them reach.  False: there are no more than r.

__device__ __forceinline__ bool find_longest(Part& q, const Order& o, int32_t most, int32_t r) {
  constexpr int N = kOrderedSequences / 64;
  const int lane = threadIdx.x & 63;
  int32_t n[N], s0[N];
  int32_t there = 0;
#pragma unroll
  for (int u = 0; u < N; ++u) {
    n[u] = -1;
    s0[u] = 0;
    if (64 * u < o.B) {
      const int32_t k = 64 * u + lane;
      s0[u] = o.bound(min(k, o.B - 1));
      const int32_t len = max(o.bound(min(k, o.B - 1) + 1) - s0[u], 0);
      n[u] = k < o.B && len <= most ? len : -1;
    }
    there += __popcll(__ballot(n[u] >= 0));
  }
  if (r >= there) return false;
  auto reach = [&](int32_t len) {
    int32_t c = 0;
#pragma unroll
    for (int u = 0; u < N; ++u) c += __popcll(__ballot(n[u] >= len));
    return c;
  };
  int32_t len = 0;
  for (int32_t bit = most > 0 ? 1 << (31 - __builtin_clz(most)) : 0; bit; bit >>= 1)
    if (reach(len | bit) > r) len |= bit;
  int32_t tie = r - reach(len + 1);
#pragma unroll
  for (int u = 0; u < N; ++u) {
    const uint64_t same = __ballot(n[u] == len);
    const int c = __popcll(same);
    if (tie >= 0 && tie < c) {
      const int at = __builtin_ctzll(__ballot(n[u] == len && (int32_t)count_below(same) == tie));
      q.lo = __builtin_amdgcn_readlane(s0[u], at);
      q.hi = q.lo + len;
      q.b = o.sequence(64 * u + at);
    }
    tie -= c;
  }
  return true;
}

// A workgroup's share is the rows in use over a.cuts.  Sequences longer than
// two shares are cut into equal parts of at most one, in whole chunks; the
// others are walked whole.  There are at most a.cuts + B parts, of which at
// most a.cuts go on.  Finds part `index`: the cut sequences' parts come first,
// then the whole ones, the longest first where there are more than the chip
// takes at once (so that the last ones to begin are short).  Or, `going_on`,
// the part of that number among those that go on.  False if there are fewer.
// Every wave looks for itself, 64 sequences at a time: loads, a sum over the
// lanes and ballots, about a microsecond.
__device__ __forceinline__ bool find_part(Part& q, const Order& o, const AttnWalk& a, int32_t index, bool going_on) {
  q.before = 0;
  q.began = q.goes_on = false;
  if (!a.cuts) {
    q.lo = o.bound(index);
    q.hi = max(o.bound(index + 1), q.lo);
    q.b = o.sequence(index);
    return true;
  }
  const int32_t each = (int32_t)(((int64_t)o.used + a.cuts - 1) / a.cuts);
  const int32_t share = max((int32_t)(((int64_t)each + kChunk - 1) / kChunk * kChunk), a.least);
  const int32_t most = (int32_t)min((int64_t)share * 2, (int64_t)INT32_MAX);
  const int lane = threadIdx.x & 63;
  int32_t seen = 0, cut = 0;
  for (int32_t k0 = 0; k0 < o.B; k0 += 64) {
    const int32_t k = min(k0 + lane, o.B - 1);
    const int32_t s0 = k0 == 0 ? o.clamped(o.ahead[0]) : o.bound(k);
    const int32_t n = max((k0 == 0 ? o.clamped(o.ahead[1]) : o.bound(k + 1)) - s0, 0);
    const uint32_t parts = k0 + lane < o.B && n > most ? (uint32_t)(((int64_t)n + share - 1) / share) : 0u;
    const uint64_t cuts = __ballot(parts != 0);
    if (cuts == 0) continue;
    const uint32_t count = parts - (going_on && parts ? 1u : 0u), upto = wave_inclusive_sum(count);
    const uint32_t all = (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
    if ((uint32_t)(index - seen) < all) {
      const int at = __builtin_ctzll(__ballot(upto > (uint32_t)(index - seen)));
      const int32_t n0 = __builtin_amdgcn_readlane(s0, at), len = __builtin_amdgcn_readlane(n, at);
      const int32_t c = __builtin_amdgcn_readlane((int)parts, at);
      const int32_t j = index - seen - (int32_t)__builtin_amdgcn_readlane((int)(upto - count), at);
      const int32_t step = (int32_t)((((int64_t)len + c - 1) / c + kChunk - 1) / kChunk * kChunk);  // <= share
      q.lo = n0 + j * step;
      q.hi = j + 1 < c ? q.lo + step : n0 + len;
      q.b = o.sequence(k0 + at);
      q.before = going_on ? index : index - cut - __popcll(cuts & ((1ull << at) - 1));
      q.began = j > 0 && q.before <= a.cuts;  // more parts than that go on only where the offsets break their contract
      q.goes_on = j + 1 < c;
      return true;
    }
    seen += (int32_t)all;
    cut += __popcll(cuts);
  }
  if (going_on) return false;
  if (a.longest_first) return find_longest(q, o, most, index - seen);
  int32_t r = index - seen;
  for (int32_t k0 = 0; k0 < o.B; k0 += 64) {
    const int32_t k = min(k0 + lane, o.B - 1);
    const int32_t s0 = o.bound(k), n = max(o.bound(k + 1) - s0, 0);
    const uint64_t whole = __ballot(k0 + lane < o.B && n <= most);
    const int c = __popcll(whole);
    if (r < c) {
      const int at = __builtin_ctzll(__ballot((whole >> lane & 1) && (int32_t)count_below(whole) == r));
      q.lo = __builtin_amdgcn_readlane(s0, at);
      q.hi = q.lo + __builtin_amdgcn_readlane(n, at);
      q.b = o.sequence(k0 + at);
      return true;
    }
    r -= c;
  }
  return false;
}

// log2 of a decay, in two parts: its product with many rows is to keep the power's last bits, not the
// exponent's (e^-60 taken of the product rounded once is off by up to 5e-6 of itself).
struct Exponent {
  float hi, lo;
};

__device__ __forceinline__ Exponent decay_exponent(const float* log_decay, int h) {
  // at most 0; -1e4 stands for -inf, whose product with no rows would be NaN; NaN stays what it is
  const float d = log_decay[h], x = d > 0.0f ? 0.0f : d < -1.0e4f ? -1.0e4f : d;
  const float hi = x * 1.44269504088896341f;
  return {hi, __builtin_fmaf(x, 1.44269504088896341f, -hi) + x * 1.92596299e-8f};  // 1 / ln 2 and what fp32 leaves of it
}

// The decay of n rows.
__device__ __forceinline__ float power(const Exponent& e, int n) {
  const float t = e.hi * (float)n, p = __builtin_amdgcn_exp2f(t);
  const float rest = __builtin_fmaf(e.hi, (float)n, -t) + e.lo * (float)n;
  return __builtin_fmaf(p, rest * 0.693147181f, p);
}

// ------------------------------------------------------ parts of a step

template <typename T>
constexpr int kRowPad = 16 / (int)sizeof(T);  // one 16-byte step: rows of a column fall into different banks
template <int D>
constexpr int kTiles = D / 16;
template <int D>
constexpr int kSteps = D / 32;  // 32-deep products along a dim
template <int D>
constexpr int kOwnTiles = D >= 64 ? D / 64 : 1;  // column tiles of the state that a wave owns
template <int D>
constexpr int kPacks = kChunk * D / 8 / kAttnThreads;  // 8-element packs of a thread and tile

// A value that every lane holds, in a scalar register.
__device__ __forceinline__ float uniform(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, x)));
}

// The same value, of which the compiler knows nothing: what is computed from
// it stays where it is used, instead of being kept in registers all through a
// loop that is around it.
__device__ __forceinline__ int opaque(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

struct Lane {
  int w, g, n;  // wave; lane / 16; lane % 16
};

// Powers of the decay that do not change from chunk to chunk.
struct Powers {
  Exponent log2;
  float diag[4], off[4], gap[3];  // scale * lambda^(i-j): of the wave's own tile, and as off * gap of those before it
  float left[4];                  // lambda^(rows after j) of the chunk's last 16 rows; the tiles before them 16 rows more each
  float fade16, fade32, fade48, fade_chunk;

  __device__ __forceinline__ float of(int x) const { return power(log2, x); }
  __device__ __forceinline__ void set(const Exponent& exponent, const Lane& l, float scale, int late) {
    log2 = {uniform(exponent.hi), uniform(exponent.lo)};
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      diag[r] = l.n >= 4 * l.g + r ? of(l.n - 4 * l.g - r) * scale : 0.0f;
      off[r] = of(l.n - 4 * l.g - r + 15) * scale;
      left[r] = of(15 - 4 * l.g - r + late);
    }
#pragma unroll
    for (int d = 0; d < 3; ++d) gap[d] = uniform(of(16 * d + 1));
    fade16 = uniform(of(16));
    fade32 = uniform(of(32));
    fade48 = uniform(of(48));
    fade_chunk = uniform(of(kChunk));
  }
};

// Eight elements into LDS at a multiple of 16 bytes; zeros if they are not to be seen.
template <typename T>
__device__ __forceinline__ void put_pack(T* s, const Pack<T, 8>& r, bool seen) {
  typedef uint32_t words __attribute__((ext_vector_type(sizeof(T) * 2)));
  words x = __builtin_bit_cast(words, r);
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) * 2; ++i) x[i] = seen ? x[i] : 0u;
  __builtin_memcpy(__builtin_assume_aligned(s, 16), &x, sizeof(x));
}

// WHOLE: both dims are multiples of eight, so a pack of eight elements lies in
// a row or past it.  Its loads are unconditional, at an address that is always
// a row's (what lies before the sequence or past the row is zeroed on the way
// into LDS): a load under a condition is waited for where the paths meet.
template <typename T, int N, bool WHOLE>
__device__ __forceinline__ Pack<T, N> load_part(const T* row, int c, int dim) {
  if constexpr (WHOLE)
    return load_pack<T, N>(row + (c < dim ? c : 0));
  else
    return load_some<T, N>(row + c, dim - c);
}

// A chunk's 64 rows of an operand, shared out among the threads.
template <typename T, int D, bool WHOLE>
__device__ __forceinline__ void fetch_tile(Pack<T, 8> (&r)[kPacks<D>], const T* p, int32_t stride, int dim, const Order& o, int32_t c0,
                                           int32_t lo) {
#pragma unroll
  for (int i = 0; i < kPacks<D>; ++i) {
    const int idx = threadIdx.x + i * kAttnThreads;
    const int64_t row = o.row(max(c0 + idx / (D / 8), lo));
    r[i] = load_part<T, 8, WHOLE>(p + row * stride, idx % (D / 8) * 8, dim);
  }
}

template <typename T, int D, bool WHOLE>
__device__ __forceinline__ void put_tile(T* s, const Pack<T, 8> (&r)[kPacks<D>], int dim, int skip) {
#pragma unroll
  for (int i = 0; i < kPacks<D>; ++i) {
    const int idx = threadIdx.x + i * kAttnThreads, row = idx / (D / 8), c = idx % (D / 8) * 8;
    put_pack(s + row * (D + kRowPad<T>) + c, r[i], row >= skip && (!WHOLE || c < dim));
  }
}

// The wave's 16 rows as operands, lane n its row n: in load_rows' order, or in load_cols'.
template <typename T, int D, bool WHOLE, bool SPLIT>
__device__ __forceinline__ void fetch_rows(Frag<T> (&q)[kSteps<D>], const T* p, int32_t stride, int dim, const Order& o, int32_t at,
                                           int32_t lo, const Lane& l) {
  // a row before the first makes a column of the result that is not stored
  const T* row = p + (int64_t)o.row(max(at + l.n, lo)) * stride;
#pragma unroll
  for (int s = 0; s < kSteps<D>; ++s) {
    if constexpr (SPLIT) {
      const Pack<T, 4> x = load_part<T, 4, WHOLE>(row, 32 * s + 4 * l.g, dim), y = load_part<T, 4, WHOLE>(row, 32 * s + 16 + 4 * l.g, dim);
      __builtin_memcpy(&q[s].v[0], &x, sizeof(x));
      __builtin_memcpy(&q[s].v[4], &y, sizeof(y));
    } else {
      const Pack<T, 8> x = load_part<T, 8, WHOLE>(row, 32 * s + 8 * l.g, dim);
      __builtin_memcpy(&q[s], &x, sizeof(x));
    }
  }
}

// What lies past the row's end is zeroed before it is used.
template <typename T, int D, bool WHOLE, bool SPLIT>
__device__ __forceinline__ void take_rows(Frag<T> (&to)[kSteps<D>], const Frag<T> (&from)[kSteps<D>], int dim, const Lane& l) {
#pragma unroll
  for (int s = 0; s < kSteps<D>; ++s) {
    to[s] = from[s];
    if constexpr (WHOLE) {
      if constexpr (SPLIT) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (32 * s + 4 * l.g >= dim) to[s].v[e] = (T)0.0f;
          if (32 * s + 16 + 4 * l.g >= dim) to[s].v[4 + e] = (T)0.0f;
        }
      } else {
        if (32 * s + 8 * l.g >= dim) to[s] = Frag<T>{};
      }
    }
  }
}

// ---- the state: wave w has columns 16 * own * w .., all rows; lane n of a tile column n, rows 4g .. 4g+3

template <int D>
using State = f32x4[kTiles<D>][kOwnTiles<D>];

template <int D>
__device__ __forceinline__ bool owns_state(const Lane& l) {
  return l.w * kOwnTiles<D> < kTiles<D>;
}

template <int D>
__device__ __forceinline__ void load_state(State<D>& st, const float* from, int ad, int cd, bool swapped, float times, const Lane& l) {
#pragma unroll
  for (int kt = 0; kt < kTiles<D>; ++kt)
#pragma unroll
    for (int vt = 0; vt < kOwnTiles<D>; ++vt) st[kt][vt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  if (!from) return;
  // unconditional loads of an element that is there: they do not wait for each other
  const int row0 = opaque(4 * l.g), col0 = opaque(16 * l.w * kOwnTiles<D> + l.n);
  const int step_r = swapped ? 1 : cd, step_c = swapped ? ad : 1;
#pragma unroll
  for (int kt = 0; kt < kTiles<D>; ++kt)
#pragma unroll
    for (int vt = 0; vt < kOwnTiles<D>; ++vt)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        st[kt][vt][r] = from[min(row0 + 16 * kt + r, ad - 1) * step_r + min(col0 + 16 * vt, cd - 1) * step_c];
#pragma unroll
  for (int kt = 0; kt < kTiles<D>; ++kt)
#pragma unroll
    for (int vt = 0; vt < kOwnTiles<D>; ++vt)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        st[kt][vt][r] = row0 + 16 * kt + r < ad && col0 + 16 * vt < cd ? st[kt][vt][r] * times : 0.0f;
}

template <int D>
__device__ __forceinline__ void store_state(float* to, const State<D>& st, int ad, int cd, float times, const Lane& l) {
  const int row0 = opaque(4 * l.g), col0 = opaque(16 * l.w * kOwnTiles<D> + l.n);
#pragma unroll
  for (int kt = 0; kt < kTiles<D>; ++kt)
#pragma unroll
    for (int vt = 0; vt < kOwnTiles<D>; ++vt)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = row0 + 16 * kt + r, col = col0 + 16 * vt;
        if (row < ad && col < cd) to[row * cd + col] = st[kt][vt][r] * times;
      }
}

// fp16: the wave's largest magnitude, for the copy's scale (s_max: a word a wave).
template <int D>
__device__ __forceinline__ void put_max(float* s_max, const State<D>& st, const Lane& l) {
  float m = 0.0f;
#pragma unroll
  for (int kt = 0; kt < kTiles<D>; ++kt)
#pragma unroll
    for (int vt = 0; vt < kOwnTiles<D>; ++vt)
#pragma unroll
      for (int r = 0; r < 4; ++r) m = fmaxf(m, __builtin_fabsf(st[kt][vt][r]));
  m = group_max(m);
  s_max[l.w] = owns_state<D>(l) ? m : 0.0f;
}

// The exponent of the power of two that values are divided by before they become fp16, the largest of them being m: it
// then lies in 2^14 .. 2^15, and a value's second part keeps its bits down to 2^-25 of m.
__device__ __forceinline__ int exponent_under(float m) {
  return m > 0.0f && m < 3.0e38f ? max(-126, __builtin_amdgcn_frexp_expf(m) - 15) : 0;
}

// That of the state's copy.
__device__ __forceinline__ int copy_exponent(const float* s_max) {
  return __builtin_amdgcn_readfirstlane(exponent_under(fmaxf(fmaxf(s_max[0], s_max[1]), fmaxf(s_max[2], s_max[3]))));
}

// The state's copy in LDS, [column][row]; in 16-bit types what its rounding leaves as another, `low`.
template <typename T, int D>
__device__ __forceinline__ void put_state(T* s, T* low, const State<D>& st, float times, const Lane& l) {
#pragma unroll
  for (int vt = 0; vt < kOwnTiles<D>; ++vt)
#pragma unroll
    for (int kt = 0; kt < kTiles<D>; ++kt) {
      const int at = (16 * (l.w * kOwnTiles<D> + vt) + l.n) * (D + kRowPad<T>) + 16 * kt + 4 * l.g;
      Pack<T, 4> q, rest;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float x = __is_same(T, f16) ? st[kt][vt][r] * times : st[kt][vt][r];
        q.v[r] = (T)x;
        if constexpr (sizeof(T) == 2) rest.v[r] = (T)(x - (float)q.v[r]);
      }
      __builtin_memcpy(__builtin_assume_aligned(s + at, 4 * sizeof(T)), &q, sizeof(q));
      if constexpr (sizeof(T) == 2) __builtin_memcpy(__builtin_assume_aligned(low + at, 4 * sizeof(T)), &rest, sizeof(rest));
    }
}

// S += times * sum_j lambda^(rows after j in the chunk) b_j^T c_j.
template <typename T, int D>
__device__ __forceinline__ void add_to_state(State<D>& st, const T* s_b, const T* s_c, const Powers& p, float times, bool third,
                                             const Lane& l) {
  constexpr int SD = D + kRowPad<T>, VT = kOwnTiles<D>;
  constexpr bool HALF = sizeof(T) == 2, THIRD = __is_same(T, bf16), SCALED = __is_same(T, f16);
  // 32 rows at a time; in fp16 all 64, as a column's largest value is looked for among them
  constexpr int STEPS = SCALED ? 2 : 1;
#pragma unroll
  for (int s0 = 0; s0 < 2; s0 += STEPS) {
    Frag<T> hi_part[STEPS][VT], lo_part[STEPS][VT], end_part[STEPS][VT];
    float up[VT];  // fp16: the power of two that the lane's column is divided by
#pragma unroll
    for (int vt = 0; vt < VT; ++vt) {
      float x[STEPS][8], m = 0.0f;
#pragma unroll
      for (int u = 0; u < STEPS; ++u) {
        const Frag<T> c = load_cols(s_c, SD, 32 * (s0 + u), 16 * (l.w * VT + vt));
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float f = (s0 + u == 0 ? (e < 4 ? p.fade48 : p.fade32) : e < 4 ? p.fade16 : 1.0f) * times;
          x[u][e] = (float)c.v[e] * (p.left[e & 3] * f);
          if constexpr (SCALED) m = fmaxf(m, __builtin_fabsf(x[u][e]));
        }
      }
      const int ex = SCALED ? exponent_under(column_max(m)) : 0;
      if constexpr (SCALED) up[vt] = __builtin_ldexpf(1.0f, ex);
#pragma unroll
      for (int u = 0; u < STEPS; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float y = SCALED ? __builtin_ldexpf(x[u][e], -ex) : x[u][e];
          // the value as rounded to fp32: a multiply fused with one of its two conversions to fp16, but not with the
          // other, would leave the parts a step of fp16 apart where it lies next to a tie
          if constexpr (SCALED) asm("" : "+v"(y));
          hi_part[u][vt].v[e] = (T)y;
          if constexpr (HALF) {
            const float rest = y - (float)hi_part[u][vt].v[e];
            lo_part[u][vt].v[e] = (T)rest;
            if constexpr (THIRD) end_part[u][vt].v[e] = (T)(rest - (float)lo_part[u][vt].v[e]);
          }
        }
    }
#pragma unroll
    for (int kt = 0; kt < kTiles<D>; ++kt) {
      f32x4 sum[VT];
#pragma unroll
      for (int vt = 0; vt < VT; ++vt) sum[vt] = SCALED ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : st[kt][vt];
#pragma unroll
      for (int u = 0; u < STEPS; ++u) {
        const Frag<T> bk = load_cols(s_b, SD, 32 * (s0 + u), 16 * kt);
#pragma unroll
        for (int vt = 0; vt < VT; ++vt) {
          sum[vt] = mma(bk, hi_part[u][vt], sum[vt]);
          if constexpr (HALF) sum[vt] = mma(bk, lo_part[u][vt], sum[vt]);
        }
      }
#pragma unroll
      for (int vt = 0; vt < VT; ++vt)
#pragma unroll
        for (int r = 0; r < 4; ++r) st[kt][vt][r] = SCALED ? __builtin_fmaf(sum[vt][r], up[vt], st[kt][vt][r]) : sum[vt][r];
    }
    if constexpr (THIRD)
      if (third) {
#pragma unroll
        for (int kt = 0; kt < kTiles<D>; ++kt) {
          const Frag<T> bk = load_cols(s_b, SD, 32 * s0, 16 * kt);
#pragma unroll
          for (int vt = 0; vt < VT; ++vt) st[kt][vt] = mma(bk, end_part[0][vt], st[kt][vt]);
        }
      }
  }
}

// The state after the chunk.
template <typename T, int D>
__device__ __forceinline__ void update_state(State<D>& st, const T* s_b, const T* s_c, const Powers& p, float fade, bool third,
                                             const Lane& l) {
#pragma unroll
  for (int kt = 0; kt < kTiles<D>; ++kt)
#pragma unroll
    for (int vt = 0; vt < kOwnTiles<D>; ++vt)
#pragma unroll
      for (int r = 0; r < 4; ++r) st[kt][vt][r] *= fade;
  add_to_state<T, D>(st, s_b, s_c, p, 1.0f, third, l);
}

// ---- products for the wave's 16 rows, transposed: lane n its row n, elements 16t + 4g .. of it

template <int D>
using Rows = f32x4[kTiles<D>];

template <int D>
__device__ __forceinline__ void clear(Rows<D>& acc) {
#pragma unroll
  for (int t = 0; t < kTiles<D>; ++t) acc[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
}

// acc += times * (the rows' a) S, S in its parts.  SPLIT: S transposed, a in load_cols' order.
template <typename T, int D, bool SPLIT>
__device__ __forceinline__ void add_state_product(Rows<D>& acc, const T* s_s, const T* s_low, const Frag<T> (&q)[kSteps<D>],
                                                  float times) {
  constexpr int SD = D + kRowPad<T>;
#pragma unroll
  for (int t = 0; t < kTiles<D>; ++t) {
    f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int s = 0; s < kSteps<D>; ++s) {
      x = mma(SPLIT ? load_cols(s_s, SD, 32 * s, 16 * t) : load_rows(s_s, SD, 16 * t, 32 * s), q[s], x);
      if constexpr (sizeof(T) == 2)
        x = mma(SPLIT ? load_cols(s_low, SD, 32 * s, 16 * t) : load_rows(s_low, SD, 16 * t, 32 * s), q[s], x);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) acc[t][r] = __builtin_fmaf(x[r], times, acc[t][r]);
  }
}

// acc += sum over the rows j of the chunk up to the wave's own, scale * lambda^(i-j) (a_i . b_j) c_j.  In 16-bit types
// the pairs' factors take part as the rounded value and what the rounding left; fp16 has too few exponents for products
// of its own values, so there a row's factors are first divided by a power of two.
template <typename T, int D, bool SPLIT>
__device__ __forceinline__ void add_pairs(Rows<D>& acc, const T* s_b, const T* s_c, const Frag<T> (&q)[kSteps<D>], const Powers& pw,
                                          const Lane& l) {
  constexpr int SD = D + kRowPad<T>;
#pragma unroll
  for (int s2 = 0; s2 < 2; ++s2) {
    if (2 * s2 > l.w) continue;
    f32x4 p[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      p[u] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      const int j = 2 * s2 + u;
      if (j > l.w) continue;
#pragma unroll
      for (int s = 0; s < kSteps<D>; ++s)
        p[u] = mma(SPLIT ? load_rows_split(s_b, SD, 16 * j, 32 * s) : load_rows(s_b, SD, 16 * j, 32 * s), q[s], p[u]);
      if (j == l.w) {
#pragma unroll
        for (int r = 0; r < 4; ++r) p[u][r] = l.n >= 4 * l.g + r ? p[u][r] * pw.diag[r] : 0.0f;
      } else {
        const float f = l.w - j == 1 ? pw.gap[0] : l.w - j == 2 ? pw.gap[1] : pw.gap[2];
#pragma unroll
        for (int r = 0; r < 4; ++r) p[u][r] *= pw.off[r] * f;
      }
    }
    int ex = 0;  // of the lane's row of the result
    if constexpr (__is_same(T, f16)) {
      float m = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) m = fmaxf(m, __builtin_fabsf(p[e >> 2][e & 3]));
      ex = exponent_under(column_max(m));
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e >> 2][e & 3] = __builtin_ldexpf(p[e >> 2][e & 3], -ex);
    }
    Frag<T> pf, rest;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if constexpr (__is_same(T, f16)) asm("" : "+v"(p[e >> 2][e & 3]));  // see add_to_state
      pf.v[e] = (T)p[e >> 2][e & 3];
      if constexpr (sizeof(T) == 2) rest.v[e] = (T)(p[e >> 2][e & 3] - (float)pf.v[e]);
    }
#pragma unroll
    for (int t = 0; t < kTiles<D>; ++t) {
      const Frag<T> c = load_cols(s_c, SD, 32 * s2, 16 * t);
      if constexpr (__is_same(T, f16)) {
        const f32x4 x = mma(c, rest, mma(c, pf, f32x4{0.0f, 0.0f, 0.0f, 0.0f}));
        const float up = __builtin_ldexpf(1.0f, ex);
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[t][r] = __builtin_fmaf(x[r], up, acc[t][r]);
      } else {
        acc[t] = mma(c, pf, acc[t]);
        if constexpr (sizeof(T) == 2) acc[t] = mma(c, rest, acc[t]);
      }
    }
  }
}

// The wave's 16 rows from position `at` on, those before `lo` left out.
//
// 16-bit results: a lane's four elements of a tile are eight bytes, and stores
// of 32 bytes a row cost more than the loads of all operands (128 frames: 450
// of 1,190 us).  So two tiles' elements are exchanged among the four lanes of
// a row, in registers, until a lane has 16 bytes and the row's lanes 64 in a
// line; and then two such lines of a row with the row eight further, until a
// store covers eight rows of 128 bytes, a cache line each.
template <bool WHOLE, int D, typename T>
__device__ __forceinline__ void store_rows(T* base, int32_t stride, const Order& o, int32_t at, int32_t lo, const Rows<D>& acc, int dim,
                                           bool past) {
  const int g = (threadIdx.x & 63) >> 4, n = threadIdx.x & 15;
  if constexpr (sizeof(T) == 2) {
    uint32_t line[kTiles<D> / 2][4];
#pragma unroll
    for (int t = 0; t < kTiles<D>; t += 2) {
      uint32_t x[2], y[2];
      Pack<T, 4> u, v;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        u.v[r] = (T)acc[t][r];
        v.v[r] = (T)acc[t + 1][r];
      }
      __builtin_memcpy(x, &u, 8);
      __builtin_memcpy(y, &v, 8);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        // lanes of g 0, 1 take tile t's elements of g and g + 2, those of g 2, 3 tile t + 1's of g - 2 and g
        const auto a = __builtin_amdgcn_permlane32_swap(x[i], y[i], false, false);
        // and then neighbours: g has eighths 2g and 2g + 1 of the 32 elements
        const auto b = __builtin_amdgcn_permlane16_swap(a[0], a[1], false, false);
        line[t / 2][i] = b[0];
        line[t / 2][2 + i] = b[1];
      }
    }
    auto put = [&](const uint32_t (&q)[4], int32_t p, int c) {
      if (p < lo) return;
      T* to = base + (int64_t)o.row(p) * stride + c;
      Pack<T, 8> r;
      __builtin_memcpy(&r, q, 16);
      if constexpr (WHOLE) {
        if (c < dim) store_some<T, 8>(to, r, 8, past);
      } else {
        store_some<T, 8>(to, r, dim - c, past);
      }
    };
    if constexpr (D == 32) {
      put(line[0], at + n, 8 * g);
    } else {
#pragma unroll
      for (int t = 0; t < kTiles<D> / 2; t += 2) {
        uint32_t low[4], high[4];  // of rows n % 8 and n % 8 + 8
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t x = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)line[t][i], 0x128, 0xf, 0xf, true);  // lane n ^ 8's
          const uint32_t y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)line[t + 1][i], 0x128, 0xf, 0xf, true);
          low[i] = n < 8 ? line[t][i] : y;
          high[i] = n < 8 ? x : line[t + 1][i];
        }
        const int c = 32 * t + (n < 8 ? 0 : 32) + 8 * g;
        put(low, at + (n & 7), c);
        put(high, at + (n & 7) + 8, c);
      }
    }
  } else {
    if (at + n < lo) return;
    T* to = base + (int64_t)o.row(at + n) * stride;
#pragma unroll
    for (int t = 0; t < kTiles<D>; ++t) {
      Pack<T, 4> q;
#pragma unroll
      for (int r = 0; r < 4; ++r) q.v[r] = (T)acc[t][r];
      const int c = 16 * t + 4 * g;
      if constexpr (WHOLE) {
        if (c < dim) store_some<T, 4>(to + c, q, 4, past);
      } else {
        store_some<T, 4>(to + c, q, dim - c, past);
      }
    }
  }
}

__device__ __forceinline__ Lane lane_of() {
  Lane l;
  l.w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  l.g = (threadIdx.x & 63) >> 4;
  l.n = threadIdx.x & 15;
  return l;
}

template <typename T, int D>
constexpr int kWavesSimd = walk_waves(sizeof(T) == 2, D);

// ------------------------------------------------------ the kernels

// The state at the end of every part that goes on, from nothing (or the
// initial state, where the part begins the sequence); attention_join_kernel
// then carries them on.
template <typename T, int D, bool WHOLE>
__global__ __launch_bounds__(kAttnThreads, (kWavesSimd<T, D>)) void attention_state_kernel(AttnPair pair) {
  constexpr int SD = D + kRowPad<T>;
  __shared__ __attribute__((aligned(16))) T s_b[kChunk * SD];
  __shared__ __attribute__((aligned(16))) T s_c[kChunk * SD];
  const Lane l = lane_of();
  const bool second = blockIdx.x >= pair.items[0];
  const AttnArgs& a = pair.walk[second];
  const int item = blockIdx.x - (second ? pair.items[0] : 0);
  const int h = item % a.H, unit = item / a.H;
  const Order o = order_of(a);
  Part q;
  const bool found = find_part(q, o, a, unit, true);
  if (h == 0 && threadIdx.x == 0) a.cut_rows[unit] = !found ? -1 : q.began ? q.hi - q.lo : 0;
  if (!found) return;
  const int32_t lo = q.lo, hi = q.hi;
  const T* pb = static_cast<const T*>(a.b) + (int64_t)(h / a.b_div) * a.b_head;
  const T* pc = static_cast<const T*>(a.c) + (int64_t)(h / a.c_div) * a.c_head;

  // from the end back: the walk that follows begins with the rows read last here
  Pack<T, 8> rb[kPacks<D>], rc[kPacks<D>];
  fetch_tile<T, D, WHOLE>(rb, pb, a.b_row, a.ad, o, hi - kChunk, lo);
  fetch_tile<T, D, WHOLE>(rc, pc, a.c_row, a.cd, o, hi - kChunk, lo);
  State<D> st;
  const bool own = owns_state<D>(l);
  Powers pw;
  pw.set(decay_exponent(a.log_decay, h), l, a.scale, a.reversed);
  load_state<D>(st, !q.began && a.init && own ? a.init + ((int64_t)q.b * a.H + h) * a.ad * a.cd : nullptr, a.ad, a.cd, a.init_swapped,
                a.init_scale * pw.of(hi - lo), l);
  for (int32_t c0 = hi - kChunk; c0 + kChunk > lo; c0 -= kChunk) {
    const int skip = max(lo - c0, 0);
    __syncthreads();  // the chunk before has been read
    put_tile<T, D, WHOLE>(s_b, rb, a.ad, skip);
    put_tile<T, D, WHOLE>(s_c, rc, a.cd, skip);
    __syncthreads();
    if (c0 > lo) {
      fetch_tile<T, D, WHOLE>(rb, pb, a.b_row, a.ad, o, c0 - kChunk, lo);
      fetch_tile<T, D, WHOLE>(rc, pc, a.c_row, a.cd, o, c0 - kChunk, lo);
    }
    if (own) add_to_state<T, D>(st, s_b, s_c, pw, uniform(pw.of(hi - c0 - kChunk)), a.exact_state, l);
  }
  if (own) store_state<D>(a.cut_state + ((int64_t)unit * a.H + h) * a.ad * a.cd, st, a.ad, a.cd, 1.0f, l);
}

// The second part of the state's copy lies beside the first where two workgroups of it still fit a compute unit.  Else
// (16-bit heads over 64) it takes the chunks' place: the products with the state come first, then the chunks.  (Taking
// the first part's place when that has been read: 160 us for the robot frame's gradients instead of 152.)
template <typename T, int D>
constexpr bool kStateFirst = sizeof(T) == 2 && D > 64;

// LDS of a walk: two operands' chunks, the state's copy, fp16's largest values.
template <typename T, int D>
struct WalkShared {
  __attribute__((aligned(16))) T chunk[2][kChunk * (D + kRowPad<T>)];
  __attribute__((aligned(16))) T s[D * (D + kRowPad<T>)];
  __attribute__((aligned(16))) T low[sizeof(T) == 2 && !kStateFirst<T, D> ? D * (D + kRowPad<T>) : 8];
  static_assert(!kStateFirst<T, D> || D <= 2 * kChunk, "both chunks hold it");
  float most[4][kAttnWaves];  // of each head that the workgroup takes
};

// out: the walk of (a, b, c).
template <typename T, int D, bool WHOLE>
__device__ __forceinline__ void walk(const AttnArgs& a, int item, WalkShared<T, D>& shared) {
  constexpr bool SCALED = __is_same(T, f16), STATE_FIRST = kStateFirst<T, D>;
  T *s_b = shared.chunk[0], *s_c = shared.chunk[1], *s_s = shared.s, *s_low = STATE_FIRST ? shared.chunk[0] : shared.low;
  float* s_max = shared.most[0];
  const Lane l = lane_of();
  const int h = item % a.H, unit = item / a.H;
  const Order o = order_of(a);
  Part q;
  if (!find_part(q, o, a, unit, false)) return;
  const T* pa = static_cast<const T*>(a.a) + (int64_t)(h / a.a_div) * a.a_head;
  const T* pb = static_cast<const T*>(a.b) + (int64_t)(h / a.b_div) * a.b_head;
  const T* pc = static_cast<const T*>(a.c) + (int64_t)(h / a.c_div) * a.c_head;
  T* po = static_cast<T*>(a.out) + (int64_t)h * a.o_head;
  const bool own = owns_state<D>(l);
  const int64_t state = (int64_t)a.ad * a.cd;

  // whole chunks up to the end, so the first one may begin `skip` rows before the first row: those are zeros in LDS
  const int32_t first = q.hi - (q.hi - q.lo + kChunk - 1) / kChunk * kChunk;
  Pack<T, 8> rb[kPacks<D>], rc[kPacks<D>];
  Frag<T> qa[kSteps<D>], qn[kSteps<D>];
  auto fetch = [&](int32_t c0) {
    fetch_tile<T, D, WHOLE>(rb, pb, a.b_row, a.ad, o, c0, q.lo);
    fetch_tile<T, D, WHOLE>(rc, pc, a.c_row, a.cd, o, c0, q.lo);
    fetch_rows<T, D, WHOLE, false>(qn, pa, a.a_row, a.ad, o, c0 + 16 * l.w, q.lo, l);
  };
  if (q.lo < q.hi) fetch(first);
  const float* from = q.began ? a.cut_state + ((int64_t)(q.before - 1) * a.H + h) * state
                      : a.init ? a.init + ((int64_t)q.b * a.H + h) * state
                               : nullptr;
  bool have_state = from != nullptr;
  State<D> st;
  load_state<D>(st, own ? from : nullptr, a.ad, a.cd, !q.began && a.init_swapped, q.began ? 1.0f : a.init_scale, l);
  if (SCALED && have_state) put_max<D>(s_max, st, l);
  Powers pw;
  pw.set(decay_exponent(a.log_decay, h), l, a.scale, 0);

  for (int32_t c0 = first; c0 < q.hi; c0 += kChunk) {
    const int skip = max(q.lo - c0, 0);
    const bool some = 16 * l.w + 15 >= skip;  // of the wave's rows
    auto put_chunk = [&] {
      put_tile<T, D, WHOLE>(s_b, rb, a.ad, skip);
      put_tile<T, D, WHOLE>(s_c, rc, a.cd, skip);
    };
    __syncthreads();  // the chunk before has been read
    if (!STATE_FIRST) put_chunk();
    take_rows<T, D, WHOLE, false>(qa, qn, a.ad, l);
    const int ex = SCALED && have_state ? copy_exponent(s_max) : 0;
    if (have_state && own) put_state<T, D>(s_s, s_low, st, __builtin_ldexpf(1.0f, -ex), l);
    if (!STATE_FIRST || have_state) __syncthreads();
    if (!STATE_FIRST && c0 + kChunk < q.hi) fetch(c0 + kChunk);
    Rows<D> acc;
    clear<D>(acc);
    if (have_state && some)
      add_state_product<T, D, false>(acc, s_s, s_low, qa, __builtin_ldexpf(pw.of(max(16 * l.w + l.n - skip, 0) + 1) * a.scale, ex));
    if (STATE_FIRST) {
      if (have_state) __syncthreads();
      put_chunk();
      __syncthreads();
      if (c0 + kChunk < q.hi) fetch(c0 + kChunk);
    }
    if (some) {
      add_pairs<T, D, false>(acc, s_b, s_c, qa, pw, l);
      store_rows<WHOLE, D>(po, a.o_row, o, c0 + 16 * l.w, q.lo, acc, a.cd, a.past);
    }
    // the state after the chunk, where something reads it
    if (c0 + kChunk < q.hi || (!q.goes_on && a.final_state)) {
      if (own) update_state<T, D>(st, s_b, s_c, pw, skip ? pw.of(kChunk - skip) : pw.fade_chunk, a.exact_state, l);
      if constexpr (SCALED) put_max<D>(s_max, st, l);
    }
    have_state = true;
  }
  if (!q.goes_on && a.final_state && own)
    store_state<D>(a.final_state + ((int64_t)q.b * a.H + h) * state, st, a.ad, a.cd, 1.0f, l);
}

template <typename T, int D, bool WHOLE>
__global__ __launch_bounds__(kAttnThreads, (kWavesSimd<T, D>)) void attention_kernel(AttnArgs a) {
  __shared__ WalkShared<T, D> shared;
  walk<T, D, WHOLE>(a, blockIdx.x, shared);
}

// dv and dk: one walk backwards, whose state is that of (q, dout) divided by
// scale.  A workgroup takes GROUP of the heads that share its keys and values:
// each chunk it goes through them with a state each, and their sums stay in
// registers.  Where GROUP is not all of them, the sums are fp32 parts that
// attention_sum_kernel adds.
template <typename T, int D, int GROUP, bool WHOLE>
__device__ __forceinline__ void walk_back(const AttnGradArgs& a, int item, WalkShared<T, D>& shared) {
  constexpr bool SCALED = __is_same(T, f16), STATE_FIRST = kStateFirst<T, D>;
  T *s_q = shared.chunk[0], *s_d = shared.chunk[1], *s_s = shared.s, *s_low = STATE_FIRST ? shared.chunk[0] : shared.low;
  float(&s_max)[4][kAttnWaves] = shared.most;
  const Lane l = lane_of();
  const int groups = a.H / GROUP, u = item % groups, unit = item / groups;
  const int h0 = u * GROUP, hk = h0 / a.kv_div;
  const Order o = order_of(a);
  Part q;
  if (!find_part(q, o, a, unit, false)) return;
  const T* pq = static_cast<const T*>(a.q) + (int64_t)h0 * a.q_head;
  const T* pd = static_cast<const T*>(a.dout) + (int64_t)h0 * a.d_head;
  const T* pk = static_cast<const T*>(a.k) + (int64_t)hk * a.k_head;
  const T* pv = static_cast<const T*>(a.v) + (int64_t)hk * a.v_head;
  const bool own = owns_state<D>(l);
  const int64_t state = (int64_t)a.ad * a.cd;

  const int32_t first = q.hi - (q.hi - q.lo + kChunk - 1) / kChunk * kChunk;
  Pack<T, 8> rq[kPacks<D>], rd[kPacks<D>];
  // the next chunk's rows of k and v are loaded with its tiles where the registers allow, else when this chunk's are
  // done with
  constexpr bool AHEAD = D < 128;
  Frag<T> fk[kSteps<D>], fv[kSteps<D>], nk[kSteps<D>], nv[kSteps<D>];
  auto fetch = [&](int32_t c0, int j) {
    fetch_tile<T, D, WHOLE>(rq, pq + j * a.q_head, a.q_row, a.ad, o, c0, q.lo);
    fetch_tile<T, D, WHOLE>(rd, pd + j * a.d_head, a.d_row, a.cd, o, c0, q.lo);
  };
  auto fetch_own = [&](int32_t c0) {
    fetch_rows<T, D, WHOLE, false>(nk, pk, a.k_row, a.ad, o, c0 + 16 * l.w, q.lo, l);
    fetch_rows<T, D, WHOLE, true>(nv, pv, a.v_row, a.cd, o, c0 + 16 * l.w, q.lo, l);
  };
  if (q.lo < q.hi) {
    fetch(first, 0);
    fetch_own(first);
  }
  const float* from = q.began ? a.cut_state + ((int64_t)(q.before - 1) * a.H + h0) * state
                      : a.init ? a.init + ((int64_t)q.b * a.H + h0) * state
                               : nullptr;
  bool have_state = from != nullptr;
  State<D> st[GROUP];
  Powers pw[GROUP];
#pragma unroll
  for (int j = 0; j < GROUP; ++j) {
    load_state<D>(st[j], own && from ? from + j * state : nullptr, a.ad, a.cd, false, q.began ? 1.0f : a.init_scale, l);
    if (SCALED && have_state) put_max<D>(s_max[j], st[j], l);
    pw[j].set(decay_exponent(a.log_decay, h0 + j), l, a.scale, 1);
  }

  for (int32_t c0 = first; c0 < q.hi; c0 += kChunk) {
    const int skip = max(q.lo - c0, 0);
    const bool needed = c0 + kChunk < q.hi || (!q.goes_on && a.final_state);
    const int32_t at = c0 + 16 * l.w;
    const bool some = 16 * l.w + 15 >= skip;  // of the wave's rows
    Rows<D> acc_v, acc_k;  // of one head and not STATE_FIRST: live one after the other
#pragma unroll
    for (int j = 0; j < GROUP; ++j) {
      auto put_chunk = [&] {
        put_tile<T, D, WHOLE>(s_q, rq, a.ad, skip);
        put_tile<T, D, WHOLE>(s_d, rd, a.cd, skip);
      };
      auto fetch_next = [&] {
        if (j + 1 < GROUP) {
          fetch(c0, j + 1);
        } else if (c0 + kChunk < q.hi) {
          fetch(c0 + kChunk, 0);
          if (AHEAD) fetch_own(c0 + kChunk);
        }
      };
      __syncthreads();  // what was in LDS has been read
      if (!STATE_FIRST) put_chunk();
      if (j == 0) {
        take_rows<T, D, WHOLE, false>(fk, nk, a.ad, l);
        take_rows<T, D, WHOLE, true>(fv, nv, a.cd, l);
      }
      const int ex = SCALED && have_state ? copy_exponent(s_max[j]) : 0;
      if (have_state && own) put_state<T, D>(s_s, s_low, st[j], __builtin_ldexpf(1.0f, -ex), l);
      if (!STATE_FIRST || have_state) __syncthreads();
      if (!STATE_FIRST) fetch_next();
      const float fade_in = have_state ? __builtin_ldexpf(pw[j].of(max(16 * l.w + l.n - skip, 0)) * a.scale, ex) : 0.0f;
      auto state_v = [&] {
        if (j == 0) clear<D>(acc_v);
        if (have_state && some) add_state_product<T, D, false>(acc_v, s_s, s_low, fk, fade_in);
      };
      auto state_k = [&] {
        if (j == 0) clear<D>(acc_k);
        if (have_state && some) add_state_product<T, D, true>(acc_k, s_s, s_low, fv, fade_in);
      };
      if (STATE_FIRST) {
        state_v();
        state_k();
        if (have_state) __syncthreads();
        put_chunk();
        __syncthreads();
        fetch_next();
      }
      if (some) {
        if (!STATE_FIRST) state_v();
        add_pairs<T, D, false>(acc_v, s_q, s_d, fk, pw[j], l);
        if (j == GROUP - 1) {
          if (a.parts)
            store_rows<WHOLE, D>(a.part_v + (int64_t)u * a.cd, groups * a.cd, o, at, q.lo, acc_v, a.cd, a.past);
          else
            store_rows<WHOLE, D>(static_cast<T*>(a.dv) + (int64_t)hk * a.dv_head, a.dv_row, o, at, q.lo, acc_v, a.cd, a.past);
        }
        if (!STATE_FIRST) state_k();
        add_pairs<T, D, true>(acc_k, s_d, s_q, fv, pw[j], l);
        if (j == GROUP - 1) {
          if (a.parts)
            store_rows<WHOLE, D>(a.part_k + (int64_t)u * a.ad, groups * a.ad, o, at, q.lo, acc_k, a.ad, a.past);
          else
            store_rows<WHOLE, D>(static_cast<T*>(a.dk) + (int64_t)hk * a.dk_head, a.dk_row, o, at, q.lo, acc_k, a.ad, a.past);
        }
      }
      if (!AHEAD && j == GROUP - 1 && c0 + kChunk < q.hi) fetch_own(c0 + kChunk);
      if (needed) {
        if (own) update_state<T, D>(st[j], s_q, s_d, pw[j], skip ? pw[j].of(kChunk - skip) : pw[j].fade_chunk, a.exact_state, l);
        if constexpr (SCALED) put_max<D>(s_max[j], st[j], l);
      }
    }
    have_state = true;
  }
  if (!q.goes_on && a.final_state && own) {
#pragma unroll
    for (int j = 0; j < GROUP; ++j)
      store_state<D>(a.final_state + ((int64_t)q.b * a.H + h0 + j) * state, st[j], a.ad, a.cd, a.final_scale, l);
  }
}

// The backward pass: both walks in one launch, the longer one's workgroups
// first (one after the other their last workgroups, and twice two more
// launches for the cut sequences' states, left the chip idle: 167 us for one
// robot frame instead of 113, both with factors rounded once).
template <typename T, int D, int GROUP, bool WHOLE>
__global__ __launch_bounds__(kAttnThreads, (grad_waves(sizeof(T) == 2, D))) void attention_backward_kernel(AttnArgs a, AttnGradArgs b,
                                                                                                       uint32_t back_items) {
  __shared__ WalkShared<T, D> shared;
  if (blockIdx.x < back_items)
    walk_back<T, D, GROUP, WHOLE>(b, blockIdx.x, shared);
  else
    walk<T, D, WHOLE>(a, blockIdx.x - back_items, shared);
}

// Instances by the wider of the two dims: 32, 64 or 128, the rest zeros.
template <typename T, bool WHOLE>
void launch_states(const AttnPair& p, hipStream_t st) {
  const int wide = p.walk[0].ad > p.walk[0].cd ? p.walk[0].ad : p.walk[0].cd;
  const dim3 grid(p.items[0] + p.items[1]), block(kAttnThreads);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, st, p); };
  wide <= 32 ? go(attention_state_kernel<T, 32, WHOLE>) : wide <= 64 ? go(attention_state_kernel<T, 64, WHOLE>)
                                                                     : go(attention_state_kernel<T, 128, WHOLE>);
}

template <typename T, bool WHOLE>
void launch_walk(const AttnArgs& a, hipStream_t st) {
  const int wide = a.ad > a.cd ? a.ad : a.cd;
  const dim3 grid((uint32_t)((a.cuts + a.B) * (int64_t)a.H)), block(kAttnThreads);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, st, a); };
  wide <= 32 ? go(attention_kernel<T, 32, WHOLE>) : wide <= 64 ? go(attention_kernel<T, 64, WHOLE>) : go(attention_kernel<T, 128, WHOLE>);
}

template <typename T, bool WHOLE>
void launch_backward(const AttnArgs& a, const AttnGradArgs& b, hipStream_t st) {
  const int wide = b.ad > b.cd ? b.ad : b.cd;
  const uint32_t back = (uint32_t)((b.cuts + b.B) * (int64_t)(b.H / b.group));
  const dim3 grid(back + (uint32_t)((a.cuts + a.B) * (int64_t)a.H)), block(kAttnThreads);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, st, a, b, back); };
  if (wide <= 32)
    b.group == 4 ? go(attention_backward_kernel<T, 32, 4, WHOLE>) : b.group == 2 ? go(attention_backward_kernel<T, 32, 2, WHOLE>)
                                                                                 : go(attention_backward_kernel<T, 32, 1, WHOLE>);
  else if (wide <= 64)
    b.group == 2 ? go(attention_backward_kernel<T, 64, 2, WHOLE>) : go(attention_backward_kernel<T, 64, 1, WHOLE>);
  else
    go(attention_backward_kernel<T, 128, 1, WHOLE>);
}

// WHOLE: see load_part; both walks' dims are the same two.
bool whole_packs(const AttnWalk& a) { return a.ad % 8 == 0 && a.cd % 8 == 0; }

template <typename T>
hipError_t states_of(const AttnPair& p, hipStream_t st) {
  whole_packs(p.walk[0]) ? launch_states<T, true>(p, st) : launch_states<T, false>(p, st);
  return hipGetLastError();
}
template <typename T>
hipError_t walk_of(const AttnArgs& a, hipStream_t st) {
  whole_packs(a) ? launch_walk<T, true>(a, st) : launch_walk<T, false>(a, st);
  return hipGetLastError();
}
template <typename T>
hipError_t backward_of(const AttnArgs& a, const AttnGradArgs& b, hipStream_t st) {
  whole_packs(b) ? launch_backward<T, true>(a, b, st) : launch_backward<T, false>(a, b, st);
  return hipGetLastError();
}

}  // namespace
}  // namespace mmbev
