// Rotary positions: what the kernels that turn pairs share.
#pragma once
#include "common.h"
#include "kernels.h"

namespace psd {

// magnitude * (cos, sin) of position * frequency; turn = frequency / (2 pi).  The product is taken in fp64 and cut to an eighth of a
// turn either side of the nearest quarter before it is rounded, so that the angle is exact to 2^-25 radians: an fp32 product would be
// off by position * 2^-24 radians, a twentieth of a radian at a million.  Up to pi/4 the series of sin to x^9 (next term 2^-29) and of
// cos to x^10 (2^-33) are as good as fp32.
__device__ __forceinline__ float2 rope_cs(int position, double turn, float magnitude) {
    const double quarters = 4.0 * ((double)position * turn), n = rint(quarters);
    const uint32_t quarter = (uint32_t)(int)(n - 4.0 * floor(0.25 * n));
    const float x = (float)((quarters - n) * 1.57079632679489661923), z = x * x;
    const float s = fmaf(x * z, fmaf(z, fmaf(z, fmaf(z, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), x);
    const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
    const float u = (quarter & 1u) ? s : c, v = (quarter & 1u) ? c : s;
    return make_float2((quarter + 1u) & 2u ? -u * magnitude : u * magnitude, quarter & 2u ? -v * magnitude : v * magnitude);
}
__device__ __forceinline__ void rope_turn(float2 cs, float &x1, float &x2) {
    const float y1 = fmaf(x1, cs.x, -(x2 * cs.y)), y2 = fmaf(x2, cs.x, x1 * cs.y);     // the same in every kernel
    x1 = y1;
    x2 = y2;
}

}  // namespace psd
