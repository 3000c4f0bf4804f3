// Rotary positions: pairs of every head turned by position times step.
//
// The phase of a pair is a wrapping 64-bit product, exact at any position; its
// top 32 bits are a signed fraction of a turn.  The nearest quarter turn is
// taken off as an integer, which leaves at most an eighth of a turn (pi/4
// radians) to the Taylor polynomials of sine and cosine: terms to x^11 and
// x^10, whose next terms are below 2^-29.
//
// A thread owns as many neighbouring pairs as two 16-byte accesses hold, works
// their sines and cosines out once, and turns those pairs of several heads
// (the fewer rows, the fewer heads a thread, so that small calls spread out).
// The operator moves bytes: 7 operations a pair and head beside the loads, and
// some 50 a pair for its angle.
#include <algorithm>

#include "sequence.hpp"

namespace mmbev {

namespace {

constexpr int kRotThreads = 256;

// Heads of one thread, by how many threads the call has: an angle is shared
// by at most eight heads.
struct RotShape {
  int32_t turned, items;  // threads of a row that turn pairs, with those that copy the head's rest
  int32_t head_parts, heads_each;
  int32_t rows_block;
};

__device__ __forceinline__ void sincos_of_phase(uint32_t phase, float& s, float& c) {
  const uint32_t quarter = (phase + 0x20000000u) >> 30;                  // nearest quarter turn
  const float x = (float)(int32_t)(phase - (quarter << 30)) * 1.46291807926715968e-9f;  // 2 pi / 2^32
  const float y = x * x;
  float sp = __builtin_fmaf(y, -2.50521083854417188e-8f, 2.75573192239858907e-6f);  // -1/11!, 1/9!
  sp = __builtin_fmaf(y, sp, -1.98412698412698413e-4f);
  sp = __builtin_fmaf(y, sp, 8.33333333333333333e-3f);
  sp = __builtin_fmaf(y, sp, -1.66666666666666667e-1f);
  sp = __builtin_fmaf(x * y, sp, x);
  float cp = __builtin_fmaf(y, -2.75573192239858907e-7f, 2.48015873015873016e-5f);  // -1/10!, 1/8!
  cp = __builtin_fmaf(y, cp, -1.38888888888888889e-3f);
  cp = __builtin_fmaf(y, cp, 4.16666666666666667e-2f);
  cp = __builtin_fmaf(y, cp, -0.5f);
  cp = __builtin_fmaf(y, cp, 1.0f);
  const float a = (quarter & 1) ? cp : sp, b = (quarter & 1) ? sp : cp;
  s = (quarter & 2) ? -a : a;
  c = ((quarter + 1) & 2) ? -b : b;
}

template <typename T, bool INTERLEAVED>
__global__ __launch_bounds__(kRotThreads) void rotary_kernel(RotaryArgs a, RotShape s) {
  constexpr int V = kPackOf<T>;  // pairs of a thread
  const int64_t n = rows_in_use(a.row_count, a.rows, a.fault);
  const int per_row = s.items * s.head_parts;
  const int64_t row0 = (int64_t)blockIdx.x * s.rows_block;
  if (row0 >= n) return;
  const int half = a.rotary_dim / 2;
  for (int t = threadIdx.x; t < s.rows_block * per_row; t += kRotThreads) {
    const int r = t / per_row, u = t - r * per_row;
    const int part = u / s.items, item = u - part * s.items;
    const int64_t row = row0 + r;
    if (row >= n) return;
    const int h0 = part * s.heads_each, h1 = min(h0 + s.heads_each, a.heads);
    const T* x = static_cast<const T*>(a.x) + row * a.x_row + h0 * a.x_head;
    T* out = static_cast<T*>(a.out) + row * a.out_row + h0 * a.out_head;
    if (item >= s.turned) {  // the head's rest, copied
      const int c = a.rotary_dim + (item - s.turned) * V;
      for (int h = h0; h < h1; ++h, x += a.x_head, out += a.out_head)
        store_some<T, V>(out + c, load_some<T, V>(x + c, a.dim - c), a.dim - c);
      continue;
    }
    const int j0 = item * V, pairs = half - j0;
    float sn[V], cs[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      sn[e] = 0.0f;
      cs[e] = 1.0f;
      if (e < pairs) {
        const int ax = min((int)a.axis[j0 + e], a.axes - 1);
        const uint64_t phase = (uint64_t)(int64_t)a.positions[row * a.position_stride + ax] * a.steps[j0 + e];
        sincos_of_phase((uint32_t)(phase >> 32), sn[e], cs[e]);
        if (a.inverse) sn[e] = -sn[e];
      }
    }
    for (int h = h0; h < h1; ++h, x += a.x_head, out += a.out_head) {
      if constexpr (INTERLEAVED) {
        const int c = 2 * j0;
        Pack<T, V> p = load_some<T, V>(x + c, 2 * pairs), q = load_some<T, V>(x + c + V, 2 * pairs - V);
#pragma unroll
        for (int e = 0; e < V / 2; ++e) {
          const float p0 = (float)p.v[2 * e], p1 = (float)p.v[2 * e + 1];
          const float q0 = (float)q.v[2 * e], q1 = (float)q.v[2 * e + 1];
          p.v[2 * e] = (T)__builtin_fmaf(p0, cs[e], -(p1 * sn[e]));
          p.v[2 * e + 1] = (T)__builtin_fmaf(p0, sn[e], p1 * cs[e]);
          q.v[2 * e] = (T)__builtin_fmaf(q0, cs[e + V / 2], -(q1 * sn[e + V / 2]));
          q.v[2 * e + 1] = (T)__builtin_fmaf(q0, sn[e + V / 2], q1 * cs[e + V / 2]);
        }
        store_some<T, V>(out + c, p, 2 * pairs);
        store_some<T, V>(out + c + V, q, 2 * pairs - V);
      } else {
        Pack<T, V> p = load_some<T, V>(x + j0, pairs), q = load_some<T, V>(x + half + j0, pairs);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float u0 = (float)p.v[e], u1 = (float)q.v[e];
          p.v[e] = (T)__builtin_fmaf(u0, cs[e], -(u1 * sn[e]));
          q.v[e] = (T)__builtin_fmaf(u0, sn[e], u1 * cs[e]);
        }
        store_some<T, V>(out + j0, p, pairs);
        store_some<T, V>(out + half + j0, q, pairs);
      }
    }
  }
}

template <typename T>
hipError_t rotary_of(const RotaryArgs& a, hipStream_t st) {
  RotShape s;
  s.turned = (a.rotary_dim / 2 + kPackOf<T> - 1) / kPackOf<T>;
  const int rest = a.dim - a.rotary_dim;
  s.items = s.turned + (a.copy_rest ? (rest + kPackOf<T> - 1) / kPackOf<T> : 0);
  // eight heads share an angle unless that leaves the chip under four waves a SIMD
  const int64_t wanted = 256 * 4 * 4 * 64;
  s.heads_each = (int32_t)std::max<int64_t>(1, std::min<int64_t>(8, a.rows * s.items * a.heads / wanted));
  s.head_parts = (a.heads + s.heads_each - 1) / s.heads_each;
  s.rows_block = std::max(1, kRotThreads / (s.items * s.head_parts));
  const uint64_t grid = ((uint64_t)a.rows + s.rows_block - 1) / s.rows_block;
  if (a.interleaved)
    hipLaunchKernelGGL((rotary_kernel<T, true>), dim3((uint32_t)grid), dim3(kRotThreads), 0, st, a, s);
  else
    hipLaunchKernelGGL((rotary_kernel<T, false>), dim3((uint32_t)grid), dim3(kRotThreads), 0, st, a, s);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, int32_t dtype, hipStream_t st) {
  if (a.rows == 0) return hipSuccess;
  return dtype == MMBEV_F32 ? rotary_of<float>(a, st) : dtype == MMBEV_F16 ? rotary_of<f16>(a, st) : rotary_of<bf16>(a, st);
}

}  // namespace mmbev
