// Sine and cosine of a rotary angle (device code, header-only).
#pragma once

#include "upr_paged.h"

namespace upr {

// cos and sin of pos * quarters quarter turns, times magnitude.  The product
// is formed and reduced to [-1/2, 1/2] quarter turns in 64 bits (a position of
// 2^20 leaves 1e-10 of a turn); there the Taylor series to x^9 and x^10 leave
// less than 2e-9, and their fp32 evaluation about one rounding.
__device__ __forceinline__ void rope_angle(int pos, double quarters, float magnitude, float& c, float& s) {
    const double t = (double)pos * quarters;
    const double n = __builtin_rint(t);
    const float x = (float)((t - n) * 1.5707963267948966);
    const float y = x * x;
    float ps = fmaf(y, 1.f / 362880.f, -1.f / 5040.f);
    ps = fmaf(y, ps, 1.f / 120.f);
    ps = fmaf(y, ps, -1.f / 6.f);
    ps = fmaf(x * y, ps, x);
    float pc = fmaf(y, -1.f / 3628800.f, 1.f / 40320.f);
    pc = fmaf(y, pc, -1.f / 720.f);
    pc = fmaf(y, pc, 1.f / 24.f);
    pc = fmaf(y, pc, -0.5f);
    pc = fmaf(y, pc, 1.f);
    // n mod 4: the low bits of the integer (n is below 2^53 for any position
    // and frequency of use; beyond that every angle is as good as any other)
    const int quadrant = (int)(n - 4.0 * __builtin_floor(n * 0.25));
    const float a = quadrant & 1 ? ps : pc, b = quadrant & 1 ? pc : ps;
    c = ((quadrant + 1) & 2 ? -a : a) * magnitude;
    s = (quadrant & 2 ? -b : b) * magnitude;
}

}  // namespace upr
