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
// The gradients are the same recurrence (dout, v, k), and backwards in time
// (k, q, dout) and (v, dout, q); backwards the state is carried one decay
// later, S' = lambda^n S + sum_j lambda^(n-j) b_j^T c_j with lambda^i in the
// first sum's place of lambda^(i+1), so that a gradient of the final state
// enters undecayed and the last S is the initial state's.
//
// 16-bit types: P and the state's copy are rounded to the type for their
// products.  The rows that enter the state are c times its decay in two parts
// (the rounded product and what the rounding left), so the state has 16 or 22
// bits and not the type's 8 or 11; in bf16 a third part makes them 24 where
// the state is asked for.  fp16 has too few exponents for a state that sums
// many rows: its copy is scaled by a power of two per column.
#pragma once

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
  int64_t used;
  int32_t B, reversed;
  __device__ __forceinline__ int64_t bound(int32_t k) const {
    const int64_t o = offsets[reversed ? B - k : k];
    const int64_t c = o < 0 ? 0 : o > used ? used : o;
    return reversed ? used - c : c;
  }
  __device__ __forceinline__ int64_t row(int64_t p) const { return reversed ? used - 1 - p : p; }
  __device__ __forceinline__ int32_t sequence(int32_t k) const { return reversed ? B - 1 - k : k; }
};

__device__ __forceinline__ Order order_of(const AttnArgs& a) {
  Order o;
  o.offsets = a.offsets;
  o.B = a.B;
  o.reversed = a.reversed;
  const int64_t end = a.offsets[a.B];
  o.used = end < 0 ? 0 : end > a.rows ? a.rows : end;
  return o;
}

// Rows of a segment: the rows in use shared out evenly, in whole chunks.
__device__ __forceinline__ int64_t segment_rows(int64_t used, int32_t segments) {
  const int64_t each = (used + segments - 1) / segments;
  return max((each + kChunk - 1) / kChunk * kChunk, (int64_t)kChunk);
}

// First sequence that ends after position p (B if none): the bounds do not
// decrease where the offsets keep their contract, and any k is in bounds.
__device__ __forceinline__ int32_t first_ending_after(const Order& o, int64_t p) {
  int32_t lo = 0, hi = o.B;
  while (lo < hi) {
    const int32_t mid = (lo + hi) >> 1;
    if (o.bound(mid + 1) > p)
      hi = mid;
    else
      lo = mid + 1;
  }
  return lo;
}

__device__ __forceinline__ float decay_exponent(const float* log_decay, int h) {
  // at most 0; -1e4 stands for -inf, whose products with 0 rows would be NaN
  return fmaxf(fminf(log_decay[h], 0.0f), -1.0e4f) * 1.44269504088896341f;
}

template <typename T>
constexpr int kRowPad = 16 / (int)sizeof(T);  // one 16-byte step: rows of a column fall into different banks

// ------------------------------------------------------ the walk

// STATE_ONLY: the state at the end of every segment that a sequence goes on
// beyond, from nothing (or the initial state, where the sequence begins
// inside); attention_join_kernel then carries them on.
template <typename T, int D, bool STATE_ONLY>
__global__ __launch_bounds__(kAttnThreads) void attention_kernel(AttnArgs a) {
  constexpr int SD = D + kRowPad<T>;
  constexpr int KT = D / 16;                     // tiles of 16 along a dim
  constexpr int VT = D >= 64 ? D / 64 : 1;       // state column tiles of a wave
  constexpr int KS = D / 32;                     // 32-deep steps along a dim
  constexpr int PACKS = kChunk * D / 8 / kAttnThreads;  // 8-element packs of a thread, per operand
  constexpr bool HALF = sizeof(T) == 2;
  constexpr bool SCALED = __is_same(T, f16);
  constexpr bool THIRD = __is_same(T, bf16);
  __shared__ __attribute__((aligned(16))) T s_b[kChunk * SD];
  __shared__ __attribute__((aligned(16))) T s_c[kChunk * SD];
  __shared__ __attribute__((aligned(16))) T s_s[STATE_ONLY ? 8 : D * SD];  // state copy, [column][row]
  __shared__ __attribute__((aligned(16))) float s_scale[SCALED && !STATE_ONLY ? D : 4];

  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l = threadIdx.x & 63, g = l >> 4, n = l & 15;
  const int h = blockIdx.x % a.H, unit = blockIdx.x / a.H;
  const Order o = order_of(a);

  int64_t p_lo, p_hi;
  int32_t k = unit, k_end = unit + 1;
  if (a.segments) {
    const int64_t per = segment_rows(o.used, a.segments);
    p_lo = unit * per;
    p_hi = min(p_lo + per, o.used);
    if (unit > 0 && p_lo >= o.used) return;
    k = unit == 0 ? 0 : first_ending_after(o, p_lo);
    k_end = a.B;
  } else {
    p_lo = 0;
    p_hi = o.used;
  }
  if (STATE_ONLY) {
    // only the sequence that goes on beyond the segment counts
    k = first_ending_after(o, p_hi);
    k_end = k + 1;
    const bool goes_on = k < a.B && o.bound(k) < p_hi;
    if (h == 0 && threadIdx.x == 0) a.seg_fresh[unit] = !goes_on || o.bound(k) >= p_lo;
    if (!goes_on) return;
  }

  const T* pa = static_cast<const T*>(a.a) + (int64_t)(h / a.a_div) * a.a_head;
  const T* pb = static_cast<const T*>(a.b) + (int64_t)(h / a.b_div) * a.b_head;
  const T* pc = static_cast<const T*>(a.c) + (int64_t)(h / a.c_div) * a.c_head;
  const int late = a.reversed;

  // powers of the decay that do not change from chunk to chunk
  const float g2 = decay_exponent(a.log_decay, h);
  auto power = [&](int x) { return __builtin_amdgcn_exp2f(g2 * (float)x); };
  const float fade_in = power(16 * w + n + 1 - late) * a.scale;  // of the state, for this lane's row
  float diag[4], off[4], gap[3];  // lambda^(i-j) of the wave's own tile, and as off * gap of those before it
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    diag[r] = n >= 4 * g + r ? power(n - 4 * g - r) * a.scale : 0.0f;
    off[r] = power(n - 4 * g - r + 15) * a.scale;
  }
#pragma unroll
  for (int d = 0; d < 3; ++d) gap[d] = power(16 * d + 1);
  float left[2][8];  // lambda^(rows after j), of a whole chunk
#pragma unroll
  for (int s = 0; s < 2; ++s)
#pragma unroll
    for (int e = 0; e < 8; ++e) left[s][e] = power(kChunk - 1 + late - (32 * s + (e < 4 ? 0 : 12) + 4 * g + e));
  const float fade_chunk = power(kChunk);

  const bool owns_state = w * VT < KT;
  f32x4 st[KT][VT];

  for (; k < k_end; ++k) {
    const int64_t s0 = o.bound(k), s1 = max(o.bound(k + 1), s0);
    if (a.segments && s1 > p_hi && s0 >= p_hi) break;
    const int64_t lo = max(s0, p_lo), hi = min(s1, p_hi);
    const int32_t b = o.sequence(k);
    const bool goes_on = s1 > p_hi;

    // the state before `lo`
    const float* from = nullptr;
    int64_t step_r = a.cd, step_c = 1;
    float times = a.init_scale;
    if (s0 < p_lo) {
      if (!STATE_ONLY) {
        from = a.seg_state + ((int64_t)(unit - 1) * a.H + h) * a.ad * a.cd;
        times = 1.0f;
      }
    } else if (a.init) {
      from = a.init + ((int64_t)b * a.H + h) * a.ad * a.cd;
      if (a.init_swapped) {
        step_r = 1;
        step_c = a.ad;
      }
    }
    bool have_state = from != nullptr;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int vt = 0; vt < VT; ++vt) {
        const int col = 16 * (w * VT + vt) + n;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = 16 * kt + 4 * g + r;
          st[kt][vt][r] = from && row < a.ad && col < a.cd ? from[row * step_r + col * step_c] * times : 0.0f;
        }
      }

    Pack<T, 8> rb[PACKS], rc[PACKS];
    Frag<T> qa[KS], qn[KS];
    auto fetch = [&](int64_t c0) {
#pragma unroll
      for (int i = 0; i < PACKS; ++i) {
        const int idx = threadIdx.x + i * kAttnThreads, r = idx / (D / 8), c = idx % (D / 8) * 8;
        const bool in = c0 + r < hi;
        const int64_t row = o.row(c0 + r);
        rb[i] = load_some<T, 8>(pb + row * a.b_row + c, in ? a.ad - c : 0);
        rc[i] = load_some<T, 8>(pc + row * a.c_row + c, in ? a.cd - c : 0);
      }
      if constexpr (!STATE_ONLY) {
        const int64_t p = c0 + 16 * w + n;
        const int64_t row = o.row(p);
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          const int c = 32 * s + 8 * g;
          const Pack<T, 8> q = load_some<T, 8>(pa + row * a.a_row + c, p < hi ? a.ad - c : 0);
          __builtin_memcpy(&qn[s], &q, sizeof(q));
        }
      }
    };
    if (lo < hi) fetch(lo);

    for (int64_t c0 = lo; c0 < hi; c0 += kChunk) {
      const int len = (int)min((int64_t)kChunk, hi - c0);
      __syncthreads();  // the chunk before has been read
#pragma unroll
      for (int i = 0; i < PACKS; ++i) {
        const int idx = threadIdx.x + i * kAttnThreads, r = idx / (D / 8), c = idx % (D / 8) * 8;
        __builtin_memcpy(__builtin_assume_aligned(s_b + r * SD + c, 16), &rb[i], sizeof(rb[i]));
        __builtin_memcpy(__builtin_assume_aligned(s_c + r * SD + c, 16), &rc[i], sizeof(rc[i]));
      }
      if constexpr (!STATE_ONLY) {
#pragma unroll
        for (int s = 0; s < KS; ++s) qa[s] = qn[s];
        if (have_state && owns_state) {
#pragma unroll
          for (int vt = 0; vt < VT; ++vt) {
            const int col = 16 * (w * VT + vt) + n;
            float shrink = 1.0f;
            if constexpr (SCALED) {
              float m = 0.0f;
#pragma unroll
              for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int r = 0; r < 4; ++r) m = fmaxf(m, __builtin_fabsf(st[kt][vt][r]));
              m = fmaxf(m, __shfl_xor(m, 16));
              m = fmaxf(m, __shfl_xor(m, 32));
              const int ex = m > 0.0f && m < 3.0e38f ? max(-100, min(100, __builtin_amdgcn_frexp_expf(m))) : 0;
              shrink = __builtin_ldexpf(1.0f, -ex);
              if (g == 0) s_scale[col] = __builtin_ldexpf(1.0f, ex);
            }
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) {
              Pack<T, 4> q;
#pragma unroll
              for (int r = 0; r < 4; ++r) q.v[r] = (T)(SCALED ? st[kt][vt][r] * shrink : st[kt][vt][r]);
              __builtin_memcpy(__builtin_assume_aligned(s_s + col * SD + 16 * kt + 4 * g, 4 * sizeof(T)), &q, sizeof(q));
            }
          }
        }
      }
      __syncthreads();
      if (c0 + kChunk < hi) fetch(c0 + kChunk);

      if (!STATE_ONLY && 16 * w < len) {
        f32x4 acc[KT];
#pragma unroll
        for (int t = 0; t < KT; ++t) acc[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        if (have_state) {
#pragma unroll
          for (int t = 0; t < KT; ++t) {
#pragma unroll
            for (int s = 0; s < KS; ++s) acc[t] = mma(load_rows(s_s, SD, 16 * t, 32 * s), qa[s], acc[t]);
            if constexpr (SCALED) {
              f32x4 sc;
              __builtin_memcpy(&sc, __builtin_assume_aligned(s_scale + 16 * t + 4 * g, 16), 16);
#pragma unroll
              for (int r = 0; r < 4; ++r) acc[t][r] *= sc[r];
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[t][r] *= fade_in;
          }
        }
#pragma unroll
        for (int s2 = 0; s2 < 2; ++s2) {
          if (2 * s2 > w) continue;
          f32x4 p[2];
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            p[u] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            const int j = 2 * s2 + u;
            if (j > w) continue;
#pragma unroll
            for (int s = 0; s < KS; ++s) p[u] = mma(load_rows(s_b, SD, 16 * j, 32 * s), qa[s], p[u]);
            if (j == w) {
#pragma unroll
              for (int r = 0; r < 4; ++r) p[u][r] = n >= 4 * g + r ? p[u][r] * diag[r] : 0.0f;
            } else {
              const float f = w - j == 1 ? gap[0] : w - j == 2 ? gap[1] : gap[2];
#pragma unroll
              for (int r = 0; r < 4; ++r) p[u][r] *= off[r] * f;
            }
          }
          Frag<T> pf;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            pf.v[r] = (T)p[0][r];
            pf.v[4 + r] = (T)p[1][r];
          }
#pragma unroll
          for (int t = 0; t < KT; ++t) acc[t] = mma(load_cols(s_c, SD, 32 * s2, 16 * t), pf, acc[t]);
        }
        if (16 * w + n < len) {
          const int64_t row = o.row(c0 + 16 * w + n);
          if (a.out_f32) {
            float* out = static_cast<float*>(a.out) + row * a.o_row + h * a.o_head;
#pragma unroll
            for (int t = 0; t < KT; ++t) {
              Pack<float, 4> q;
#pragma unroll
              for (int r = 0; r < 4; ++r) q.v[r] = acc[t][r];
              store_some<float, 4>(out + 16 * t + 4 * g, q, a.cd - 16 * t - 4 * g);
            }
          } else {
            T* out = static_cast<T*>(a.out) + row * a.o_row + h * a.o_head;
#pragma unroll
            for (int t = 0; t < KT; ++t) {
              Pack<T, 4> q;
#pragma unroll
              for (int r = 0; r < 4; ++r) q.v[r] = (T)acc[t][r];
              store_some<T, 4>(out + 16 * t + 4 * g, q, a.cd - 16 * t - 4 * g);
            }
          }
        }
      }

      // the state after the chunk, where something reads it
      if (owns_state && (c0 + kChunk < hi || (STATE_ONLY ? goes_on : (!goes_on && a.final_state)))) {
        float fade = fade_chunk;
        if (len < kChunk) fade = power(len);
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
          for (int vt = 0; vt < VT; ++vt)
#pragma unroll
            for (int r = 0; r < 4; ++r) st[kt][vt][r] *= fade;
#pragma unroll
        for (int s2 = 0; s2 < 2; ++s2) {
          if (32 * s2 >= len) continue;
          Frag<T> hi_part[VT], lo_part[VT], end_part[VT];
#pragma unroll
          for (int vt = 0; vt < VT; ++vt) {
            const Frag<T> c = load_cols(s_c, SD, 32 * s2, 16 * (w * VT + vt));
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              float f = left[s2][e];
              if (len < kChunk) f = power(max(len - 1 - (32 * s2 + (e < 4 ? 0 : 12) + 4 * g + e), 0) + late);
              float x = (float)c.v[e] * f;
              // the product as rounded to fp32: a multiply fused with one of its two conversions to fp16, but not with
              // the other, would leave the parts a step of fp16 apart where x lies next to a tie
              if constexpr (SCALED) asm("" : "+v"(x));
              hi_part[vt].v[e] = (T)x;
              if constexpr (HALF) {
                const float rest = x - (float)hi_part[vt].v[e];
                lo_part[vt].v[e] = (T)rest;
                if constexpr (THIRD) end_part[vt].v[e] = (T)(rest - (float)lo_part[vt].v[e]);
              }
            }
          }
#pragma unroll
          for (int kt = 0; kt < KT; ++kt) {
            const Frag<T> bk = load_cols(s_b, SD, 32 * s2, 16 * kt);
#pragma unroll
            for (int vt = 0; vt < VT; ++vt) {
              st[kt][vt] = mma(bk, hi_part[vt], st[kt][vt]);
              if constexpr (HALF) st[kt][vt] = mma(bk, lo_part[vt], st[kt][vt]);
              if (THIRD && a.final_state) st[kt][vt] = mma(bk, end_part[vt], st[kt][vt]);
            }
          }
        }
      }
      have_state = true;
    }

    float* to = nullptr;
    float scaled = 1.0f;
    if (STATE_ONLY) {
      to = a.seg_state + ((int64_t)unit * a.H + h) * a.ad * a.cd;
    } else if (!goes_on && a.final_state) {
      to = a.final_state + ((int64_t)b * a.H + h) * a.ad * a.cd;
      scaled = a.final_scale;
    }
    if (to && owns_state) {
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int vt = 0; vt < VT; ++vt) {
          const int col = 16 * (w * VT + vt) + n;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int row = 16 * kt + 4 * g + r;
            if (row < a.ad && col < a.cd) to[(int64_t)row * a.cd + col] = st[kt][vt][r] * scaled;
          }
        }
    }
    if (goes_on) break;
  }
}

// Instances by the wider of the two dims: 32, 64 or 128, the rest zeros.
template <typename T>
hipError_t attention_of(const AttnArgs& a, bool state_only, hipStream_t st) {
  const int wide = a.ad > a.cd ? a.ad : a.cd;
  const dim3 grid((uint32_t)((a.segments ? a.segments : a.B) * (int64_t)a.H));
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kAttnThreads), 0, st, a); };
  if (wide <= 32)
    state_only ? go(attention_kernel<T, 32, true>) : go(attention_kernel<T, 32, false>);
  else if (wide <= 64)
    state_only ? go(attention_kernel<T, 64, true>) : go(attention_kernel<T, 64, false>);
  else
    state_only ? go(attention_kernel<T, 128, true>) : go(attention_kernel<T, 128, false>);
  return hipGetLastError();
}

}  // namespace
}  // namespace mmbev
