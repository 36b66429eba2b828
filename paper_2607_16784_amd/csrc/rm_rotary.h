// rm_rotary.h -- angles and pairs of the rotary positions (cache.hip,
// headnorm.hip).  Not part of the C ABI.
#pragma once

#include "rm_decode.h"

namespace rm {

// Turns a position of pair `pair`, fp64.
__device__ inline double turns_of(const float* inv_freq, int pair)
{
    return (double)inv_freq[pair] * 0.15915494309189533577;
}

// Sine and cosine of position * turns whole turns, times scale.  What is left
// of the last turn goes through v_sin_f32 and v_cos_f32, which take turns: off
// by up to 1.3e-7 over [-1/2, 1/2] (measured), against 5e-8 of sincospif, whose
// instructions bound the prompts' append (7600 tokens, the same again and again:
// 47.5 us, 40.3 so, 35.2 without any angle; 51 with inputs that change).  The
// angle's own rounding to fp32 is 9e-8; of a million results in f16 each is the
// exact value's neighbour but for 1.2e-7 around the middle between two.
__device__ inline void turn_of(double turns, int32_t position, float scale, float& cs, float& sn)
{
    const double a = (double)position * turns;
    const float r = (float)(a - rint(a));
    cs = __builtin_amdgcn_cosf(r) * scale;
    sn = __builtin_amdgcn_sinf(r) * scale;
}

// Channels of pair p: the pairs of the layout first, then the pairs of
// neighbours that are copied.
__device__ inline void channels_of(int p, int rot, int layout, int& a, int& b)
{
    const int half = rot >> 1;
    if (p >= half) {
        a = 2 * p;
        b = a + 1;
    } else if (layout == RM_ROTARY_HALF) {
        a = p;
        b = p + half;
    } else {
        a = 2 * p;
        b = a + 1;
    }
}

__device__ inline void turn_pair(float& a, float& b, float cs, float sn)
{
    const float x = a, y = b;
    a = __builtin_fmaf(x, cs, -(y * sn));
    b = __builtin_fmaf(x, sn, y * cs);
}

}  // namespace rm
