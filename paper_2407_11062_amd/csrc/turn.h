// Cosine and sine of position x frequency, for positions far along.
#pragma once
#include "common.h"

namespace eqat {

// The angle in turns is held in binary64 (a position below 2^31 times a frequency: 2^-22 of a turn at the least, where binary32 would lose the angle at all from 2^24 on),
// its whole turns and quarters are taken off there, and what is left, y of [-1/8, 1/8] turns, goes through the Taylor polynomials of sin and cos about 0: |2 pi y| <= pi / 4, where the
// first terms left out, (pi / 4)^11 / 11! and (pi / 4)^10 / 10!, are 2e-9 and 2.5e-8 of 1.  The sine is odd in y: its error is relative.
__device__ __forceinline__ void cos_sin(int32_t pos, float freq, float &c, float &s)
{
    constexpr double kPerTurn = 0.15915494309189533577;               // 1 / (2 pi)
    const double turns = (double)pos * ((double)freq * kPerTurn), quarters = __builtin_rint(turns * 4.0);
    const float y = (float)__builtin_fma(quarters, -0.25, turns);
    const float x = y * 6.28318530717958647692f, z = x * x;
    // (beyond 2^31 quarters the number itself is too large for 32 bits; its last two bits are what counts)
    const int q = (int)(int64_t)quarters & 3;
    float sp = __builtin_fmaf(z, 2.75573192239858906526e-6f, -1.98412698412698412698e-4f);
    sp = __builtin_fmaf(z, sp, 8.33333333333333333333e-3f);
    sp = __builtin_fmaf(z, sp, -1.66666666666666666667e-1f);
    sp = __builtin_fmaf(x * z, sp, x);
    float cp = __builtin_fmaf(z, 2.48015873015873015873e-5f, -1.38888888888888888889e-3f);
    cp = __builtin_fmaf(z, cp, 4.16666666666666666667e-2f);
    cp = __builtin_fmaf(z, cp, -0.5f);
    cp = __builtin_fmaf(z, cp, 1.0f);
    const float a = q & 1 ? sp : cp, b = q & 1 ? cp : sp;             // quarters: (c, s), (-s, c), (-c, -s), (s, -c)
    c = q == 1 || q == 2 ? -a : a;
    s = q >= 2 ? -b : b;
}

}  // namespace eqat
