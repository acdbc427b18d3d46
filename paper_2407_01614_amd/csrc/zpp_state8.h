// Optimizer moments in 8 bits: codes and scales of a block (formats in zpp.h).
#pragma once

#include "zpp_device.h"
#include "zpp_quant.h"

namespace zpp {

// Decisions of a block, from the bits of its largest |m| or r: codes are 0 and the
// scale as it is where inv is 0.
struct StateScale {
    float scale, inv;
};

__device__ __forceinline__ StateScale first_scale(uint32_t top) {
    const float a = __uint_as_float(top);
    StateScale s{a / 127.0f, 127.0f / a};
    if (top >= 0x7F800000u)
        s = {__uint_as_float(kScaleNaNBits), 0.0f};
    else if (a < 0x1p-100f)
        s = {0.0f, 0.0f};
    return s;
}

__device__ __forceinline__ StateScale second_scale(uint32_t top) {
    const float a = __uint_as_float(top);
    StateScale s{a / 65025.0f, 65025.0f / a};
    if (top >= 0x7F800000u)
        s = {__uint_as_float(kScaleNaNBits), 0.0f};
    else if (top == 0u)
        s = {0.0f, 0.0f};
    return s;
}

// |m inv| <= 127 (1 + 2^-24)^2, so no code needs a clamp.  In a block of Inf or NaN,
// where inv is 0, m inv is 0 or NaN: select rather than multiply.
__device__ __forceinline__ uint32_t first_code(float m, const StateScale &s) {
    return s.inv == 0.0f ? 0u : code_bits(m * s.inv);
}

// The largest c that is 0 or has (c - 1/2)^2 <= t, t = r inv <= 255^2 (1 + 2^-23): near the
// root, which is off by one at most, c^2 -+ c + 1/4 has 18 bits and is exact.
__device__ __forceinline__ uint32_t second_code(float r, const StateScale &s) {
#pragma clang fp contract(off)
    const float t = r * s.inv;
    float c = __builtin_rintf(__builtin_amdgcn_sqrtf(t));
    if (c > 0.0f && __builtin_fmaf(c, c - 1.0f, 0.25f) > t)
        c -= 1.0f;
    if (__builtin_fmaf(c, c + 1.0f, 0.25f) <= t)
        c += 1.0f;
    if (r > 0.0f && c < 1.0f)
        c = 1.0f;
    return s.inv == 0.0f ? 0u : (uint32_t)c;
}

__device__ __forceinline__ float first_value(int32_t code, float scale) {
    return (float)code * scale;
}
__device__ __forceinline__ float second_value(uint32_t code, float scale) {
#pragma clang fp contract(off)
    const float c = (float)code;
    const float r = c * c * scale;
    return r * r;
}

}  // namespace zpp
