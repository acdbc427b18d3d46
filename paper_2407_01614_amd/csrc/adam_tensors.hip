// AdamW over many tensors in one launch, moments in fp32 or in 8 bits, and the
// moments' way between the two (formats in zpp.h).
//
// A wave takes a tile of 256 elements of one tensor, which is also a block of
// the 8-bit moments, so a block's largest values are reductions within the wave
// and nothing is written twice.  Which tensor a tile belongs to is searched in the
// table's levels, 64 first tiles at a time: one load a level, a ballot and a count.
#include "zpp_act8.h"
#include "zpp_adam.h"
#include "zpp_state8.h"
#include "zpp_token.h"

namespace zpp {
namespace {

struct TableArgs {
    const AdamEntry *entries;
    const uint32_t *level[4];  // the search's levels, the widest last
    int levels;
    uint32_t base;  // the launch's first tile
    AdamConsts c;
};

// The tensor of a tile.
__device__ __forceinline__ uint32_t tensor_of(const TableArgs &a, uint32_t tile) {
    uint32_t i = 0;
    for (int l = 0; l < a.levels; ++l) {
        const uint32_t first = a.level[l][i * kSearch + (threadIdx.x & 63)];
        i = i * kSearch + (uint32_t)__builtin_popcountll(__ballot(first <= tile)) - 1;
    }
    return i;
}

// Largest of the wave, the same in all lanes.
__device__ __forceinline__ uint32_t max64(uint32_t a) {
    a = max8(a);
    const uint32_t b = dpp<kMirror16>(a);
    a = a > b ? a : b;
    uint32_t top = 0;
#pragma unroll
    for (int l = 0; l < 64; l += 16) {
        const uint32_t r = (uint32_t)__builtin_amdgcn_readlane((int)a, l);
        top = top > r ? top : r;
    }
    return top;
}

// Four codes of a tile, those past its end 0.
template <bool WHOLE>
__device__ __forceinline__ uint32_t load_codes(const void *p, uint32_t i, uint32_t rest) {
    const uint8_t *b = reinterpret_cast<const uint8_t *>(p);
    if constexpr (WHOLE) {
        return ld_nt_at<uint32_t, 1>(b + i);
    } else {
        uint32_t w = 0;
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e)
            w |= (uint32_t)b[clamped(i + e, rest)] << (8 * e);
        return w;
    }
}

template <bool WHOLE>
__device__ __forceinline__ f32x4 load_bf16(const void *p, uint32_t i, uint32_t rest) {
    const uint16_t *b = reinterpret_cast<const uint16_t *>(p);
    if constexpr (WHOLE) {
        const u32x2 w = ld_nt_at<u32x2, 2>(b + i);
        return f32x4{bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y)};
    } else {
        f32x4 x;
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e)
            x[e] = bf16_lo((uint32_t)b[clamped(i + e, rest)]);
        return x;
    }
}

// Codes and scale of a block's first or second moments, four a lane; `inside`:
// how many of the four are inside the block.
template <int MOMENT, bool WHOLE>
__device__ __forceinline__ void store_state(void *codes, float *scale, uint32_t i, uint32_t rest,
                                            const f32x4 &x) {
    float y[4];
    uint32_t top = 0;
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e) {
        y[e] = MOMENT == 1 ? x[e] : __builtin_sqrtf(x[e]);
        const uint32_t b = __float_as_uint(y[e]) & 0x7FFFFFFFu;
        if (WHOLE || i + e < rest)
            top = top > b ? top : b;
    }
    top = max64(top);
    const StateScale s = MOMENT == 1 ? first_scale(top) : second_scale(top);
    uint32_t c[4];
#pragma unroll
    for (int e = 0; e < 4; ++e)
        c[e] = MOMENT == 1 ? first_code(y[e], s) : second_code(y[e], s);
    store4_i8<WHOLE>(reinterpret_cast<int8_t *>(codes), i, rest,
                     pack_low_bytes(c[0], c[1], c[2], c[3]));
    if ((threadIdx.x & 63) == 0)
        *scale = s.scale;
}

template <int MOMENT>
__device__ __forceinline__ f32x4 state_values(uint32_t codes, float scale) {
    f32x4 x;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        x[e] = MOMENT == 1 ? first_value((int8_t)(codes >> (8 * e)), scale)
                           : second_value((codes >> (8 * e)) & 0xFFu, scale);
    return x;
}

template <bool ADAMW, int STATE, int GRAD, bool WHOLE>
__device__ __forceinline__ void step_tile(const AdamEntry &t, size_t base, uint32_t rest,
                                          const AdamConsts &c) {
    const uint32_t i = 4 * (threadIdx.x & 63);
    f32x4 P = load4<WHOLE>(t.p + base, i, rest), M, V, G;
    const size_t block = base / kAdamTile;
    if constexpr (STATE == kF32) {
        M = load4<WHOLE>((const float *)t.m + base, i, rest);
        V = load4<WHOLE>((const float *)t.v + base, i, rest);
    } else {
        const uint32_t m = load_codes<WHOLE>((const uint8_t *)t.m + base, i, rest);
        const uint32_t v = load_codes<WHOLE>((const uint8_t *)t.v + base, i, rest);
        M = state_values<1>(m, t.m_scales[block]);
        V = state_values<2>(v, t.v_scales[block]);
    }
    if constexpr (GRAD == kF32)
        G = load4<WHOLE>((const float *)t.g + base, i, rest);
    else
        G = load_bf16<WHOLE>((const uint16_t *)t.g + base, i, rest);
    adam_update4<ADAMW>(P, M, V, G, c);
    store4<WHOLE>(t.p + base, i, rest, P);
    if (t.primary)
        store4_bf16<WHOLE>(t.primary + base, i, rest,
                           u32x2{pack_bf16x2(P.x, P.y), pack_bf16x2(P.z, P.w)});
    if constexpr (STATE == kF32) {
        store4<WHOLE>((float *)t.m + base, i, rest, M);
        store4<WHOLE>((float *)t.v + base, i, rest, V);
    } else {
        store_state<1, WHOLE>((uint8_t *)t.m + base, t.m_scales + block, i, rest, M);
        store_state<2, WHOLE>((uint8_t *)t.v + base, t.v_scales + block, i, rest, V);
    }
}

template <bool ADAMW, int STATE, int GRAD>
__global__ __launch_bounds__(64) void adam_tensors_kernel(TableArgs a) {
    const uint32_t tile = a.base + blockIdx.x;
    const AdamEntry &t = a.entries[tensor_of(a, tile)];
    const size_t base = (size_t)(tile - t.first) * kAdamTile;
    AdamConsts c = a.c;
    // the step size times the decay, rounded once, as the host rounds it for one tensor
    c.lr_wd = a.c.lr_wd * t.decay;
    c.wd = t.decay;
    const size_t rest = t.n - base;
    if (__builtin_expect(rest >= kAdamTile, 1))
        step_tile<ADAMW, STATE, GRAD, true>(t, base, kAdamTile, c);
    else
        step_tile<ADAMW, STATE, GRAD, false>(t, base, (uint32_t)rest, c);
}

template <int MOMENT>
__global__ __launch_bounds__(64) void state_save_kernel(const float *x, void *codes, float *scales,
                                                        TileSpan tiles) {
    const size_t block = tiles.first + blockIdx.x, base = block * kAdamTile;
    const uint32_t i = 4 * threadIdx.x;
    uint8_t *p = (uint8_t *)codes + base;
    if (blockIdx.x < tiles.whole)
        store_state<MOMENT, true>(p, scales + block, i, kAdamTile,
                                  load4<true>(x + base, i, kAdamTile));
    else
        store_state<MOMENT, false>(p, scales + block, i, tiles.tail,
                                   load4<false>(x + base, i, tiles.tail));
}

template <int MOMENT>
__global__ __launch_bounds__(64) void state_load_kernel(const void *codes, const float *scales,
                                                        float *out, TileSpan tiles) {
    const size_t block = tiles.first + blockIdx.x, base = block * kAdamTile;
    const uint32_t i = 4 * threadIdx.x;
    const uint8_t *p = (const uint8_t *)codes + base;
    const float s = scales[block];
    if (blockIdx.x < tiles.whole)
        store4<true>(out + base, i, kAdamTile,
                     state_values<MOMENT>(load_codes<true>(p, i, kAdamTile), s));
    else
        store4<false>(out + base, i, tiles.tail,
                      state_values<MOMENT>(load_codes<false>(p, i, tiles.tail), s));
}

template <int STATE, int GRAD>
void launch_step(const TableArgs &a, unsigned grid, hipStream_t stream) {
    if (a.c.adamw)
        hipLaunchKernelGGL((adam_tensors_kernel<true, STATE, GRAD>), dim3(grid), dim3(64), 0, stream,
                           a);
    else
        hipLaunchKernelGGL((adam_tensors_kernel<false, STATE, GRAD>), dim3(grid), dim3(64), 0,
                           stream, a);
}

}  // namespace

hipError_t launch_adam_tensors(const void *table, uint32_t tensors, uint64_t tiles, int state_type,
                               int grad_type, const AdamConsts &c, hipStream_t stream) {
    TableArgs a;
    a.entries = reinterpret_cast<const AdamEntry *>(table);
    a.c = c;
    a.levels = 0;
    const uint32_t *words = reinterpret_cast<const uint32_t *>(a.entries + tensors), *found[4];
    size_t n = tensors;
    do {
        found[a.levels++] = words;
        words += padded_level(n);
        n = (n + kSearch - 1) / kSearch;
    } while (n > 1);
    for (int l = 0; l < a.levels; ++l)
        a.level[l] = found[a.levels - 1 - l];
    constexpr uint64_t kMost = (uint64_t)1 << 25;  // 2^31 work-items a launch
    for (uint64_t t = 0; t < tiles; t += kMost) {
        const unsigned grid = (unsigned)(tiles - t < kMost ? tiles - t : kMost);
        a.base = (uint32_t)t;
        if (state_type == kF32 && grad_type == kF32)
            launch_step<kF32, kF32>(a, grid, stream);
        else if (state_type == kF32)
            launch_step<kF32, kBf16>(a, grid, stream);
        else if (grad_type == kF32)
            launch_step<kI8, kF32>(a, grid, stream);
        else
            launch_step<kI8, kBf16>(a, grid, stream);
    }
    return hipGetLastError();
}

hipError_t launch_adam_state_save(const float *x, size_t n, int moment, void *codes, float *scales,
                                  hipStream_t stream) {
    for_tiles(n, kAdamTile, 1, 64, true, [&](const TileSpan &tiles, unsigned grid) {
        if (moment == 1)
            hipLaunchKernelGGL(state_save_kernel<1>, dim3(grid), dim3(64), 0, stream, x, codes,
                               scales, tiles);
        else
            hipLaunchKernelGGL(state_save_kernel<2>, dim3(grid), dim3(64), 0, stream, x, codes,
                               scales, tiles);
    });
    return hipGetLastError();
}

hipError_t launch_adam_state_load(const void *codes, const float *scales, size_t n, int moment,
                                  float *out, hipStream_t stream) {
    for_tiles(n, kAdamTile, 1, 64, true, [&](const TileSpan &tiles, unsigned grid) {
        if (moment == 1)
            hipLaunchKernelGGL(state_load_kernel<1>, dim3(grid), dim3(64), 0, stream, codes, scales,
                               out, tiles);
        else
            hipLaunchKernelGGL(state_load_kernel<2>, dim3(grid), dim3(64), 0, stream, codes, scales,
                               out, tiles);
    });
    return hipGetLastError();
}

}  // namespace zpp
