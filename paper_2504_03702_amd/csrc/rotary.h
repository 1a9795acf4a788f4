// What the kernels that turn rows to their positions share.
#pragma once

#include "device_util.h"

// Cosine and sine of position * frequency.  Whole turns go in 64 bits: a position of 31 bits times a frequency of 24 leaves the fraction all
// a float can hold.
__device__ __forceinline__ float2 turn_of(int32_t position, float frequency) {
    double turns = (double)position * (double)frequency * 0.15915494309189533577;
    turns -= rint(turns);
    float s, c;
    sincospif(2.f * (float)turns, &s, &c);
    return make_float2(c, s);
}
