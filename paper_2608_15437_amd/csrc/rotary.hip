// Rotary positions: pairs of every head turned by position times step.
//
// The phase of a pair is a wrapping 64-bit product, exact at any position; its
// top 32 bits are a signed fraction of a turn.  The nearest quarter turn is
// taken off as an integer, which leaves at most an eighth of a turn (pi/4
// radians) to the Taylor polynomials of sine and cosine: terms to x^11 and
// x^10, whose next terms are below 2^-29.
//
// A thread owns the neighbouring pairs of a 16-byte access (of two, where a
// pair's elements lie apart), works their sines and cosines out once, and turns
// those pairs of several heads
// (the fewer rows, the fewer heads a thread, so that small calls spread out).
// The operator moves bytes: 7 operations a pair and head beside the loads, and
// some 50 a pair for its angle.  213,879 x 16 x 64 bf16: 151 us, 5.8 TB/s.
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

// A thread's elements of a head: one pack of neighbouring pairs, or the packs
// of their first and of their second elements.
template <typename T, bool INTERLEAVED>
struct Turned {
  static constexpr int V = kPackOf<T>, PAIRS = INTERLEAVED ? V / 2 : V;
  Pack<T, V> p, q;

  static __device__ __forceinline__ Pack<T, V> load_one(const T* x, int left, bool past) {
    return past && left >= V ? load_past<T, V>(x) : load_some<T, V>(x, left);
  }
  __device__ __forceinline__ void load(const T* x, int j0, int half, bool past) {
    const int left = half - j0;
    if constexpr (INTERLEAVED) {
      p = load_one(x + 2 * j0, 2 * left, past);
    } else {
      p = load_one(x + j0, left, past);
      q = load_one(x + half + j0, left, past);
    }
  }
  __device__ __forceinline__ void store(T* x, int j0, int half, bool past) const {
    const int left = half - j0;
    if constexpr (INTERLEAVED) {
      store_some<T, V>(x + 2 * j0, p, 2 * left, past);
    } else {
      store_some<T, V>(x + j0, p, left, past);
      store_some<T, V>(x + half + j0, q, left, past);
    }
  }
  __device__ __forceinline__ void turn(const float (&sn)[PAIRS], const float (&cs)[PAIRS]) {
#pragma unroll
    for (int e = 0; e < PAIRS; ++e) {
      const float a = (float)(INTERLEAVED ? p.v[2 * e] : p.v[e]), b = (float)(INTERLEAVED ? p.v[2 * e + 1] : q.v[e]);
      const T u = (T)__builtin_fmaf(a, cs[e], -(b * sn[e])), v = (T)__builtin_fmaf(a, sn[e], b * cs[e]);
      if constexpr (INTERLEAVED) {
        p.v[2 * e] = u;
        p.v[2 * e + 1] = v;
      } else {
        p.v[e] = u;
        q.v[e] = v;
      }
    }
  }
};

template <typename T, bool INTERLEAVED>
__global__ __launch_bounds__(kRotThreads) void rotary_kernel(RotaryArgs a, RotShape s) {
  using Elements = Turned<T, INTERLEAVED>;
  constexpr int V = kPackOf<T>, PAIRS = Elements::PAIRS;
  const int64_t n = rows_in_use(a.row_count, a.rows, a.fault);
  const int per_row = s.items * s.head_parts;
  const int64_t row0 = a.first_row + (int64_t)blockIdx.x * s.rows_block;
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
        store_some<T, V>(out + c, load_some<T, V>(x + c, a.dim - c), a.dim - c, a.past);
      continue;
    }
    const int j0 = item * PAIRS;
    float sn[PAIRS], cs[PAIRS];
#pragma unroll
    for (int e = 0; e < PAIRS; ++e) {
      // pairs past the last turn by its angle; they are not stored
      const int j = min(j0 + e, half - 1);
      const int ax = min((int)a.axis[j], a.axes - 1);
      const uint64_t phase = (uint64_t)(int64_t)a.positions[row * a.position_stride + ax] * a.steps[j];
      sincos_of_phase((uint32_t)(phase >> 32), sn[e], cs[e]);
      if (a.inverse) sn[e] = -sn[e];
    }
    // four heads' loads before their stores: out may be x, so the compiler keeps a load behind the store before it
    int h = h0;
    for (; h + 4 <= h1; h += 4, x += 4 * a.x_head, out += 4 * a.out_head) {
      Elements e[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) e[i].load(x + i * a.x_head, j0, half, a.past);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        e[i].turn(sn, cs);
        e[i].store(out + i * a.out_head, j0, half, a.past);
      }
    }
    for (; h < h1; ++h, x += a.x_head, out += a.out_head) {
      Elements e;
      e.load(x, j0, half, a.past);
      e.turn(sn, cs);
      e.store(out, j0, half, a.past);
    }
  }
}

template <typename T>
hipError_t rotary_of(const RotaryArgs& a, hipStream_t st) {
  RotShape s;
  const int pairs = a.interleaved ? kPackOf<T> / 2 : kPackOf<T>;
  s.turned = (a.rotary_dim / 2 + pairs - 1) / pairs;
  const int rest = a.dim - a.rotary_dim;
  s.items = s.turned + (a.copy_rest ? (rest + kPackOf<T> - 1) / kPackOf<T> : 0);
  // eight heads share an angle unless that leaves the chip under four waves a SIMD
  const int64_t wanted = 256 * 4 * 4 * 64;
  s.heads_each = (int32_t)std::max<int64_t>(1, std::min<int64_t>(8, a.rows * s.items * a.heads / wanted));
  s.head_parts = (a.heads + s.heads_each - 1) / s.heads_each;
  s.rows_block = std::max(1, kRotThreads / (s.items * s.head_parts));
  RotaryArgs part = a;
  for (; part.first_row < a.rows; part.first_row += kMostGroups * s.rows_block) {
    const int64_t groups = std::min((a.rows - part.first_row + s.rows_block - 1) / s.rows_block, kMostGroups);
    if (a.interleaved)
      hipLaunchKernelGGL((rotary_kernel<T, true>), dim3((uint32_t)groups), dim3(kRotThreads), 0, st, part, s);
    else
      hipLaunchKernelGGL((rotary_kernel<T, false>), dim3((uint32_t)groups), dim3(kRotThreads), 0, st, part, s);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, int32_t dtype, hipStream_t st) {
  if (a.rows == 0) return hipSuccess;
  return dtype == MMBEV_F32 ? rotary_of<float>(a, st) : dtype == MMBEV_F16 ? rotary_of<f16>(a, st) : rotary_of<bf16>(a, st);
}

}  // namespace mmbev
