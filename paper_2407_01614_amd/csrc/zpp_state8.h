// Optimizer moments in 8 bits: codes and scales of a block (formats in zpp.h).
#pragma once

#include "zpp_act8.h"
#include "zpp_device.h"
#include "zpp_quant.h"

namespace zpp {

// Decisions of a block, the same in all its lanes: codes are 0 and the scale as it is where
// inv is 0.
struct StateScale {
    float scale, inv;
};
// Of both moments: `m` the bits of the largest |m|, `r` those of the largest r (each at least
// Inf's where there is one or a NaN).  The four quotients are one, a lane each.
struct StateScales {
    StateScale m, r;
};
__device__ __forceinline__ StateScales state_scales(uint32_t m, uint32_t r) {
    const uint32_t lane = threadIdx.x;
    const float of = __uint_as_float(lane & 2 ? r : m), whole = lane & 2 ? 65025.0f : 127.0f;
    const float q = (lane & 1 ? whole : of) / (lane & 1 ? of : whole);
    StateScales s{{lane_value(q, 0), lane_value(q, 1)}, {lane_value(q, 2), lane_value(q, 3)}};
    const float nan = __uint_as_float(kScaleNaNBits);
    if (m >= 0x7F800000u)
        s.m = {nan, 0.0f};
    else if (m < 0x0D800000u)  // 2^-100
        s.m = {0.0f, 0.0f};
    if (r >= 0x7F800000u)
        s.r = {nan, 0.0f};
    else if (r == 0u)
        s.r = {0.0f, 0.0f};
    return s;
}

// |m inv| <= 127 (1 + 2^-24)^2, so no code needs a clamp.  (Where inv is 0 the codes mean
// nothing.)
__device__ __forceinline__ uint32_t first_codes(const f32x4 &m, const StateScale &s) {
    return pack_low_bytes(code_bits(m.x * s.inv), code_bits(m.y * s.inv), code_bits(m.z * s.inv),
                          code_bits(m.w * s.inv));
}

// The largest c that is 0 or has (c - 1/2)^2 <= t, t = r inv <= 255^2 (1 + 2^-23): near the
// root, which is off by one at most, c^2 + c + 1/4 has 18 bits and is exact.
__device__ __forceinline__ uint32_t second_code(float r, const StateScale &s) {
#pragma clang fp contract(off)
    const float t = r * s.inv;
    // at least the code below: the root is within 2^-15 of t's
    float c = __builtin_floorf(__builtin_amdgcn_sqrtf(t) + 0.499f);
    c += __builtin_fmaf(c, c + 1.0f, 0.25f) <= t ? 1.0f : 0.0f;
    return (uint32_t)__builtin_fmaxf(c, r > 0.0f ? 1.0f : 0.0f);
}

// Codes of four second moments v of a block, whose roots r are v's rounded to fp32.  The
// roots take most of the arithmetic of a step, so codes come from the hardware's, which are
// within a unit in the last place: r within 2^-23 of itself and half a step for its own
// rounding, t's root within half of that, another step and 2^-24 for the products, below
// 2^-22 together, 2^-14 at 255.  Only where some lane's t has a root within 2^-13 of a border
// (6 in 100 waves) are all taken again from correct ones.  Blocks whose largest is below 2^-96
// too; in others v of less than 2^-126, whose roots the hardware does not have, are of code 1
// or 0: t < 2^-63 / 2^-48 65025 < 2.
__device__ __forceinline__ uint32_t second_codes(const f32x4 &v, uint32_t top,
                                                 const StateScale &s) {
#pragma clang fp contract(off)
    uint32_t codes = 0;
    float off = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float root = __builtin_amdgcn_sqrtf(__builtin_amdgcn_sqrtf(v[e]) * s.inv);
        const float c = __builtin_rintf(root);
        off = __builtin_fmaxf(off, __builtin_fabsf(root - c));
        codes = __builtin_amdgcn_cvt_pk_u8_f32(__builtin_fmaxf(c, v[e] > 0.0f ? 1.0f : 0.0f), e,
                                               codes);
    }
    if (__builtin_expect(__ballot(off > 0.5f - 0x1p-13f) != 0 || top < 0x0F800000u, 0)) {
        codes = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            codes |= second_code(__builtin_sqrtf(v[e]), s) << (8 * e);
    }
    return codes;
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
