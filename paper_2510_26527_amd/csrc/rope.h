// Rotary positions: what the kernels that turn pairs share.
#pragma once
#include "common.h"
#include "kernels.h"

namespace psd {

// magnitude * (cos, sin) of position * frequency; turn = frequency / (2 pi).  The product is taken in fp64 and cut to an eighth of a
// turn either side of the nearest quarter before it is rounded, which leaves it exact to 2^-27 of a turn: an fp32 product would be
// off by position * 2^-24 radians, a twentieth of a radian at a million.
__device__ __forceinline__ float2 rope_cs(int position, double turn, float magnitude) {
    const double quarters = 4.0 * ((double)position * turn), n = rint(quarters);
    const uint32_t quarter = (uint32_t)(int)(n - 4.0 * floor(0.25 * n));
    float s, c;
    sincospif((float)(0.5 * (quarters - n)), &s, &c);
    const float x = (quarter & 1u) ? s : c, y = (quarter & 1u) ? c : s;
    return make_float2((quarter + 1u) & 2u ? -x * magnitude : x * magnitude, quarter & 2u ? -y * magnitude : y * magnitude);
}
__device__ __forceinline__ void rope_turn(float2 cs, float &x1, float &x2) {
    const float y1 = fmaf(x1, cs.x, -(x2 * cs.y)), y2 = fmaf(x2, cs.x, x1 * cs.y);     // the same in every kernel
    x1 = y1;
    x2 = y2;
}

}  // namespace psd
