// Pieces of the layer operators' kernels: eight elements of a row as a lane's
// share (bf16, fp32 or a checkpoint's codes), the decisions of the 8-bit
// checkpoint, and sums over lanes.
#pragma once

#include <atomic>

#include "zpp_device.h"
#include "zpp_layer.h"
#include "zpp_quant.h"

namespace zpp {

// More than 64 KB of LDS has to be asked for, once on each device; `asked`, a
// kernel's own, has a bit for each of the first 64 where that is done.
inline hipError_t allow_lds(const void *kernel, size_t bytes, std::atomic<uint64_t> &asked) {
    int device = 0;
    hipError_t e = hipGetDevice(&device);
    if (e != hipSuccess)
        return e;
    const uint64_t bit = (unsigned)device < 64 ? (uint64_t)1 << device : 0;
    if (asked.load(std::memory_order_relaxed) & bit)
        return hipSuccess;
    e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e == hipSuccess)
        asked.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

// Eight elements as they are loaded; turned to fp32 only where they are used,
// so that loads in flight hold 4 (bf16), 8 (fp32) or 3 (codes) registers.
template <int TYPE>
struct Chunk;
template <>
struct Chunk<kBf16> {
    u32x4 w;
};
template <>
struct Chunk<kF32> {
    f32x4 lo, hi;
};
template <>
struct Chunk<kI8> {
    u32x2 codes;
    uint32_t exp;
};

// A vector at an address aligned to A bytes, as an ordinary access.
template <class V, int A>
__device__ __forceinline__ V ld_at(const void *p) {
    typedef V U __attribute__((aligned(A)));
    return *reinterpret_cast<const U *>(p);
}
template <class V, int A>
__device__ __forceinline__ void st_at(void *p, V v) {
    typedef V U __attribute__((aligned(A)));
    *reinterpret_cast<U *>(p) = v;
}

// A chunk's elements lie at p: eight in a row, or (APART 32) four and another four
// 32 elements on, so that 8 lanes share a block's fp32 as whole lines.  Its element
// e is at place_at(e).
template <uint32_t APART>
__device__ __forceinline__ constexpr uint32_t place_at(uint32_t e) {
    return e < 4 ? e : APART + e - 4;
}

// The eight elements, `valid` >= 1 of the APART + 4 from p inside the row (what is
// past them reads as the row's last).  A row's last, partial chunk takes single
// loads at clamped places, which do not wait for each other; RAGGED false: there is
// none.  Codes are read as ordinary, temporal loads: 8 bytes a lane, they left half
// of each line's fetch behind as streaming ones (8192x8192 read back: 34.8 us, 29.4
// so).
template <int TYPE, bool RAGGED = true, uint32_t APART = 4>
__device__ __forceinline__ Chunk<TYPE> load_chunk(const Mat &m, size_t off, uint32_t valid,
                                                  size_t block) {
    static_assert(APART == 4 || TYPE != kBf16);
    const bool whole = !RAGGED || valid >= APART + 4;
    Chunk<TYPE> c;
    if constexpr (TYPE == kBf16) {
        const uint16_t *p = reinterpret_cast<const uint16_t *>(m.data) + off;
        if (whole) {
            c.w = ld_nt_at<u32x4, 2>(p);
        } else {
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e)
                c.w[e] = (uint32_t)p[clamped(2 * e, valid)] |
                         ((uint32_t)p[clamped(2 * e + 1, valid)] << 16);
        }
    } else if constexpr (TYPE == kF32) {
        const float *p = reinterpret_cast<const float *>(m.data) + off;
        if (whole) {
            c.lo = ld_nt_at<f32x4, 4>(p);
            c.hi = ld_nt_at<f32x4, 4>(p + APART);
        } else {
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e) {
                c.lo[e] = p[clamped(e, valid)];
                c.hi[e] = p[clamped(APART + e, valid)];
            }
        }
    } else {
        const uint8_t *p = reinterpret_cast<const uint8_t *>(m.data) + off;
        if (whole && APART == 4) {
            c.codes = ld_at<u32x2, 1>(p);
        } else if (whole) {
            c.codes = u32x2{ld_at<uint32_t, 1>(p), ld_at<uint32_t, 1>(p + APART)};
        } else {
            c.codes = u32x2{0, 0};
#pragma unroll
            for (uint32_t e = 0; e < 8; ++e)
                c.codes[e / 4] |= (uint32_t)p[clamped(place_at<APART>(e), valid)] << (8 * (e % 4));
        }
        c.exp = m.exps[block];
    }
    return c;
}

// Keeps what is made of a loaded chunk behind this point: the compiler would
// make it early and hold that in registers instead.
__device__ __forceinline__ void hold(Chunk<kBf16> &c) {
    asm volatile("" : "+v"(c.w.x), "+v"(c.w.y), "+v"(c.w.z), "+v"(c.w.w));
}
__device__ __forceinline__ void hold(Chunk<kF32> &) {}
__device__ __forceinline__ void hold(Chunk<kI8> &c) {
    asm volatile("" : "+v"(c.codes.x), "+v"(c.codes.y), "+v"(c.exp));
}

// The scale of a checkpoint's block.
__device__ __forceinline__ float act_scale(uint32_t exp) {
    return __uint_as_float(exp == 255u ? kScaleNaNBits : exp << 23);
}

__device__ __forceinline__ void chunk_values(const Chunk<kBf16> &c, float (&x)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[2 * e] = bf16_lo(c.w[e]);
        x[2 * e + 1] = bf16_hi(c.w[e]);
    }
}
__device__ __forceinline__ void chunk_values(const Chunk<kF32> &c, float (&x)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[e] = c.lo[e];
        x[e + 4] = c.hi[e];
    }
}
__device__ __forceinline__ void chunk_values(const Chunk<kI8> &c, float (&x)[8]) {
    const float s = act_scale(c.exp);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        x[e] = (float)(int8_t)(c.codes[e / 4] >> (8 * (e % 4))) * s;
}

// Two floats as packed bf16, to nearest even (NaN stays NaN).
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    const bf16x2 v = __builtin_convertvector((f32x2){lo, hi}, bf16x2);
    return __builtin_bit_cast(uint32_t, v);
}

template <int TYPE>
__device__ __forceinline__ Chunk<TYPE> make_chunk(const float (&x)[8]) {
    Chunk<TYPE> c;
    if constexpr (TYPE == kBf16) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            c.w[e] = bf16_pair(x[2 * e], x[2 * e + 1]);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            c.lo[e] = x[e];
            c.hi[e] = x[e + 4];
        }
    }
    return c;
}

// Stores the chunk's elements that are inside the row (`valid` as above).  Eight fp32
// in a row are stored as ordinary, temporal: streaming stores of every other 16
// bytes do not meet in the L2 (a checkpoint read back as 8192x8192 fp32: 91 us, 69
// so, and 48 with the halves apart, whole lines as streaming stores).
template <int TYPE, bool RAGGED = true, uint32_t APART = 4>
__device__ __forceinline__ void store_chunk(const Mat &m, size_t off, uint32_t valid,
                                            const Chunk<TYPE> &c) {
    static_assert(APART == 4 || TYPE != kBf16);
    const bool whole = !RAGGED || valid >= APART + 4;
    if constexpr (TYPE == kBf16) {
        uint16_t *p = reinterpret_cast<uint16_t *>(m.data) + off;
        if (whole) {
            st_nt_at<u32x4, 2>(p, c.w);
        } else {
#pragma unroll
            for (uint32_t e = 0; e < 8; ++e)
                if (e < valid)
                    p[e] = (uint16_t)(c.w[e / 2] >> (16 * (e % 2)));
        }
    } else {
        float *p = reinterpret_cast<float *>(m.data) + off;
        if (whole && APART == 4) {
            st_at<f32x4, 4>(p, c.lo);
            st_at<f32x4, 4>(p + 4, c.hi);
        } else if (whole) {
            st_nt_at<f32x4, 4>(p, c.lo);
            st_nt_at<f32x4, 4>(p + APART, c.hi);
        } else {
#pragma unroll
            for (uint32_t e = 0; e < 8; ++e)
                if (place_at<APART>(e) < valid)
                    p[place_at<APART>(e)] = e < 4 ? c.lo[e] : c.hi[e - 4];
        }
    }
}

// x moved by DPP; every lane has a source lane in these patterns.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true);
}
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
    return __uint_as_float(dpp<CTRL>(__float_as_uint(x)));
}
constexpr int kSwap1 = 0xB1;     // quad_perm 1,0,3,2
constexpr int kSwap2 = 0x4E;     // quad_perm 2,3,0,1
constexpr int kMirror8 = 0x141;  // the other half of 8 lanes, reversed
constexpr int kMirror16 = 0x140; // the other half of 16 lanes, reversed

// Sum of 16 neighbouring lanes, in all of them.
__device__ __forceinline__ float sum16(float x) {
    x += dpp<kSwap1>(x);
    x += dpp<kSwap2>(x);
    x += dpp<kMirror8>(x);
    x += dpp<kMirror16>(x);
    return x;
}
__device__ __forceinline__ float lane_value(float x, int lane) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(x), lane));
}
// Sum of the wave, in its last lane: the rows of 16 lanes, then row 0 to 1 and 2
// to 3, then the lower two to the upper two.
__device__ __forceinline__ float sum64_last(float x) {
    x = sum16(x);
    x += __uint_as_float(
        (uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), 0x142, 0xA, 0xF, false));
    x += __uint_as_float(
        (uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), 0x143, 0xC, 0xF, false));
    return x;
}

// The exponent byte of a block from the bits of its largest magnitude: the
// smallest e with a <= 127 * 2^e.  127 = 1.984375 * 2^6, so with a = m 2^E, e
// is E - 6 up to m = 1.984375 and E - 5 beyond, which adding the distance from
// there to the next power of two makes a carry into the exponent field.  Inf
// and NaN, whose bits are at least 0x7F800000, are 255.
__device__ __forceinline__ uint32_t act_exp(uint32_t absbits) {
    const int e = (int)((absbits + 0x1FFFFu) >> 23) - 6;
    return absbits >= 0x7F800000u ? 255u : (uint32_t)(e < 1 ? 1 : e);
}

// A lane's share of a block's largest magnitude, as fp32 bits, whose order is
// that of the magnitudes, Inf and then NaN above all: of a chunk as loaded (what a
// partial one holds past the row's end is the row's last element again), and of
// values.
__device__ __forceinline__ uint32_t max_bits(const Chunk<kBf16> &c) {
    u16x2 a = absbits2(c.w[0]);
#pragma unroll
    for (int e = 1; e < 4; ++e)
        a = __builtin_elementwise_max(a, absbits2(c.w[e]));
    return (uint32_t)(a.x > a.y ? a.x : a.y) << 16;
}
__device__ __forceinline__ uint32_t max_bits(const float (&x)[8]) {
    uint32_t a = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t b = __float_as_uint(x[e]) & 0x7FFFFFFFu;
        a = b > a ? b : a;
    }
    return a;
}
__device__ __forceinline__ uint32_t max_bits(const Chunk<kF32> &c) {
    const float x[8] = {c.lo.x, c.lo.y, c.lo.z, c.lo.w, c.hi.x, c.hi.y, c.hi.z, c.hi.w};
    return max_bits(x);
}
// Largest of 8 neighbouring lanes' (one block's), in all of them.
__device__ __forceinline__ uint32_t max8(uint32_t a) {
    uint32_t b = dpp<kSwap1>(a);
    a = a > b ? a : b;
    b = dpp<kSwap2>(a);
    a = a > b ? a : b;
    b = dpp<kMirror8>(a);
    return a > b ? a : b;
}

// Codes of eight elements of a block with this exponent byte.  x * 2^-e is
// exact, so the fma with 1.5 * 2^23 rounds it to the integer as rint does.  Its
// magnitude is at most 127, but up to 64 at the largest exponent, where 63 is kept.
__device__ __forceinline__ u32x2 act_codes(const float (&x)[8], uint32_t exp) {
    const float inv = __uint_as_float((254u - exp) << 23);
    uint32_t b[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
        b[e] = __float_as_uint(__builtin_fmaf(x[e], inv, kRoundMagic));
    if (__builtin_expect(exp >= 249u, 0)) {
        // with 255, a block of Inf or NaN, the codes are 0
        const float most = exp == 255u ? 0.0f : 63.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float y = exp == 255u ? 0.0f : x[e] * inv;
            b[e] = code_bits(__builtin_amdgcn_fmed3f(y, -most, most));
        }
    }
    return u32x2{pack_low_bytes(b[0], b[1], b[2], b[3]), pack_low_bytes(b[4], b[5], b[6], b[7])};
}

// Writes the checkpoint of the elements that the 8 lanes of a block hold, `top`
// the lane's largest.  All 8 lanes take part, with `valid` 0 and `top` 0 where a
// lane is past the row's end.
template <bool RAGGED = true, uint32_t APART = 4>
__device__ __forceinline__ void save_chunk(const Mat &m, size_t off, uint32_t valid, size_t block,
                                           uint32_t top, const float (&x)[8]) {
    const uint32_t exp = act_exp(max8(top));
    if (valid) {
        const u32x2 w = act_codes(x, exp);
        uint8_t *p = reinterpret_cast<uint8_t *>(m.data) + off;
        const bool whole = !RAGGED || valid >= APART + 4;
        if (whole && APART == 4) {
            st_nt_at<u32x2, 1>(p, w);
        } else if (whole) {
            st_at<uint32_t, 1>(p, w.x);
            st_at<uint32_t, 1>(p + APART, w.y);
        } else {
#pragma unroll
            for (uint32_t e = 0; e < 8; ++e)
                if (place_at<APART>(e) < valid)
                    p[place_at<APART>(e)] = (uint8_t)(w[e / 4] >> (8 * (e % 4)));
        }
        if ((threadIdx.x & 7) == 0)
            m.exps[block] = (uint8_t)exp;
    }
}

}  // namespace zpp
