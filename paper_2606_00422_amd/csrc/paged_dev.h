// Sine and cosine of a rotary angle, and the user of a work item (device code,
// header-only).
#pragma once

#include "upr_paged.h"

namespace upr {

// cos and sin of pos * quarters quarter turns, times magnitude.  The product
// is formed and reduced to [-1/2, 1/2] quarter turns in 64 bits (a position of
// 2^20 leaves 1e-10 of a turn); there the Taylor series to x^9 and x^10 leave
// less than 2e-9, and their fp32 evaluation about one rounding.
__device__ __forceinline__ void rope_angle(int pos, double quarters, float magnitude, float& c, float& s) {
    // (adding 1.5 * 2^52 rounds to whole quarter turns, whose low bits it leaves
    // in the sum's: the product is below 2^51 for any 32-bit position and the
    // frequencies that the host lets through)
    const double magic = 6755399441055744.0;
    const double t = (double)pos * quarters, n = t + magic;
    const int quadrant = (int)__double2loint(n);
    const float x = (float)((t - (n - magic)) * 1.5707963267948966);
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
    const float a = quadrant & 1 ? ps : pc, b = quadrant & 1 ? pc : ps;
    c = ((quadrant + 1) & 2 ? -a : a) * magnitude;
    s = (quadrant & 2 ? -b : b) * magnitude;
}

// The launch's user that item b belongs to: the last one whose items start at
// or before b.  (One load per lane instead of a search's chain of loads.)
__device__ __forceinline__ int user_of(const PagedUsers& users, int b) {
    const int lane = threadIdx.x & 63;
    int i = 0;
#pragma unroll
    for (int base = 0; base < kPagedUsers; base += 64)
        i += __popcll(__ballot(base + lane < users.n && users.item0[base + lane + 1] <= b));
    return __builtin_amdgcn_readfirstlane(i);
}

}  // namespace upr
