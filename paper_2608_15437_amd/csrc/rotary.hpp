// The angle of a rotary pair.
//
// The phase of a pair is a wrapping 64-bit product, exact at any position; its
// top 32 bits are a signed fraction of a turn.  The nearest quarter turn is
// taken off as an integer, which leaves at most an eighth of a turn (pi/4
// radians) to the Taylor polynomials of sine and cosine: terms to x^11 and
// x^10, whose next terms are below 2^-29.
#pragma once

#include "sequence.hpp"

namespace mmbev {

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

}  // namespace mmbev
