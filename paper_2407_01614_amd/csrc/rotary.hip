// Rotary positions (formulas and layouts in zpp.h): one pass over the heads of a
// batch of tokens, forward or backward, in place or into other arrays.
//
// A workgroup takes a few tokens.  Their angles' cosines and sines are computed
// once, a pair a lane, and kept in LDS for all heads: the angle is a product in 64
// bits of which the fraction of a turn is taken there, so that far positions lose
// nothing, and the rest is at most an eighth of a turn, where Taylor's polynomials
// hold.  The heads then pass through registers, P pairs a lane: 16 bytes of u and
// 16 of v of halves, 32 in a row of neighbours.
#include "zpp_act8.h"
#include "zpp_token.h"

namespace zpp {
namespace {

constexpr uint32_t kThreads = 256;
constexpr uint32_t kMostPairs = 2048;  // pairs of a workgroup's tokens, 16 KB of LDS

// x / d for x d < 2^32: with magic = ceil(2^32 / d) the product exceeds x / d by
// less than x / 2^32 < 1 / d.
struct Div {
    uint32_t d, magic;
    __device__ __forceinline__ uint32_t operator()(uint32_t x) const {
        return d == 1 ? x : __umulhi(x, magic);
    }
};
Div make_div(uint32_t d) { return {d, (uint32_t)(0xFFFFFFFFu / d + 1)}; }

struct Args {
    Heads x, out, k, k_out;
    const int64_t *positions;
    const double *turns;
    size_t tokens, base;   // of the batch, and the launch's first
    uint32_t tile;         // tokens of a workgroup
    uint32_t slices;       // workgroups of a tile, each with `share` heads
    uint32_t share, heads, heads_x;
    uint32_t pairs, rot_chunks, copy_chunks, dim, rotated;
    Div by_pairs, by_chunks, by_token, by_group_x, by_group_k;
    float scale, sign;
    bool copy_x, copy_k;
};

// cos and sin of 2 pi t.
__device__ __forceinline__ f32x2 turned(double t) {
    const double f = t - __builtin_rint(t);
    const double q = __builtin_rint(4.0 * f);
    const float a = (float)(__builtin_fma(q, -0.25, f) * 6.283185307179586);
    const float z = a * a;
    // Taylor to a^9 and a^10: at pi / 4 what follows is below 2e-9
    float s = __builtin_fmaf(z, 1.0f / 362880, -1.0f / 5040);
    s = __builtin_fmaf(z, s, 1.0f / 120);
    s = __builtin_fmaf(z, s, -1.0f / 6);
    s = __builtin_fmaf(z * a, s, a);
    float c = __builtin_fmaf(z, -1.0f / 3628800, 1.0f / 40320);
    c = __builtin_fmaf(z, c, -1.0f / 720);
    c = __builtin_fmaf(z, c, 1.0f / 24);
    c = __builtin_fmaf(z, c, -0.5f);
    c = __builtin_fmaf(z, c, 1.0f);
    const int quarter = (int)q & 3;
    const float x = quarter & 1 ? s : c, y = quarter & 1 ? c : s;
    // NaN and Inf, whose quarter means nothing, are NaN here already
    return f32x2{quarter == 1 || quarter == 2 ? -x : x, quarter >= 2 ? -y : y};
}

template <int TYPE>
using Element = std::conditional_t<TYPE == kBf16, uint16_t, float>;

// N elements in a row at p as fp32, and back.
template <int TYPE, int N>
__device__ __forceinline__ void load_row(const Element<TYPE> *p, float (&x)[N]) {
    if constexpr (TYPE == kF32) {
        if constexpr (N % 4 == 0) {
#pragma unroll
            for (int i = 0; i < N; i += 4) {
                const f32x4 v = ld_at<f32x4, 4>(p + i);
                x[i] = v.x, x[i + 1] = v.y, x[i + 2] = v.z, x[i + 3] = v.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                x[i] = p[i];
        }
    } else if constexpr (N >= 2) {
        uint32_t w[N / 2];
        if constexpr (N % 8 == 0) {
#pragma unroll
            for (int i = 0; i < N / 2; i += 4) {
                const u32x4 v = ld_at<u32x4, 2>(p + 2 * i);
                w[i] = v.x, w[i + 1] = v.y, w[i + 2] = v.z, w[i + 3] = v.w;
            }
        } else if constexpr (N == 4) {
            const u32x2 v = ld_at<u32x2, 2>(p);
            w[0] = v.x, w[1] = v.y;
        } else {
            w[0] = ld_at<uint32_t, 2>(p);
        }
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            x[2 * i] = bf16_lo(w[i]);
            x[2 * i + 1] = bf16_hi(w[i]);
        }
    } else {
        x[0] = bf16_lo(p[0]);
    }
}

template <int TYPE, int N>
__device__ __forceinline__ void store_row(Element<TYPE> *p, const float (&x)[N]) {
    if constexpr (TYPE == kF32) {
        if constexpr (N % 4 == 0) {
#pragma unroll
            for (int i = 0; i < N; i += 4)
                st_at<f32x4, 4>(p + i, f32x4{x[i], x[i + 1], x[i + 2], x[i + 3]});
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                p[i] = x[i];
        }
    } else if constexpr (N >= 2) {
        uint32_t w[N / 2];
#pragma unroll
        for (int i = 0; i < N / 2; ++i)
            w[i] = bf16_pair(x[2 * i], x[2 * i + 1]);
        if constexpr (N % 8 == 0) {
#pragma unroll
            for (int i = 0; i < N / 2; i += 4)
                st_at<u32x4, 2>(p + 2 * i, u32x4{w[i], w[i + 1], w[i + 2], w[i + 3]});
        } else if constexpr (N == 4) {
            st_at<u32x2, 2>(p, u32x2{w[0], w[1]});
        } else {
            st_at<uint32_t, 2>(p, w[0]);
        }
    } else {
        p[0] = (uint16_t)bf16_pair(x[0], x[0]);
    }
}

// P pairs of a head from pair i on.
template <int TYPE, bool NEAR, int P>
__device__ __forceinline__ void rotate(const Element<TYPE> *x, Element<TYPE> *out, uint32_t i,
                                       uint32_t pairs, const f32x2 *angle) {
    float u[P], v[P];
    if constexpr (NEAR) {
        float w[2 * P];
        load_row<TYPE>(x + 2 * i, w);
#pragma unroll
        for (int j = 0; j < P; ++j)
            u[j] = w[2 * j], v[j] = w[2 * j + 1];
    } else {
        load_row<TYPE>(x + i, u);
        load_row<TYPE>(x + pairs + i, v);
    }
#pragma unroll
    for (int j = 0; j < P; ++j) {
        const f32x2 a = angle[i + j];
        const float turned_u = u[j] * a.x - v[j] * a.y;
        v[j] = u[j] * a.y + v[j] * a.x;
        u[j] = turned_u;
    }
    if constexpr (NEAR) {
        float w[2 * P];
#pragma unroll
        for (int j = 0; j < P; ++j)
            w[2 * j] = u[j], w[2 * j + 1] = v[j];
        store_row<TYPE>(out + 2 * i, w);
    } else {
        store_row<TYPE>(out + i, u);
        store_row<TYPE>(out + pairs + i, v);
    }
}

constexpr uint32_t kCopied = 8;  // features of a chunk that is copied

template <int TYPE, bool NEAR, int P>
__global__ __launch_bounds__(kThreads) void rotary_kernel(Args a) {
    extern __shared__ f32x2 angles[];  // [tokens of the tile][pairs]
    const uint32_t tile = blockIdx.x / a.slices, slice = blockIdx.x % a.slices;
    const size_t token0 = a.base + (size_t)tile * a.tile;
    const uint32_t tokens = (uint32_t)(a.tokens - token0 < a.tile ? a.tokens - token0 : a.tile);
    for (uint32_t i = threadIdx.x; i < tokens * a.pairs; i += kThreads) {
        const uint32_t t = a.by_pairs(i);
        const f32x2 cs = turned((double)a.positions[token0 + t] * a.turns[i - t * a.pairs]);
        angles[i] = f32x2{cs.x * a.scale, cs.y * a.scale * a.sign};
    }
    __syncthreads();
    const uint32_t head0 = slice * a.share;
    const uint32_t heads = a.heads - head0 < a.share ? a.heads - head0 : a.share;
    const uint32_t chunks = a.rot_chunks + a.copy_chunks;
    // the last slice may have fewer heads: its items are numbered as the others'
    for (uint32_t i = threadIdx.x; i < tokens * a.share * chunks; i += kThreads) {
        const uint32_t t = a.by_token(i), in_token = i - t * a.share * chunks;
        const uint32_t h = a.by_chunks(in_token), chunk = in_token - h * chunks;
        if (h >= heads)
            continue;
        uint32_t head = head0 + h;
        const bool is_x = head < a.heads_x;
        if (!is_x)
            head -= a.heads_x;
        const Heads &from = is_x ? a.x : a.k, &to = is_x ? a.out : a.k_out;
        const uint32_t g = is_x ? a.by_group_x(head) : a.by_group_k(head);
        const uint32_t m = head - g * from.heads;
        const Element<TYPE> *x = reinterpret_cast<const Element<TYPE> *>(from.data) +
                                 (token0 + t) * from.token + g * from.group + m * from.head;
        Element<TYPE> *out = reinterpret_cast<Element<TYPE> *>(to.data) +
                             (token0 + t) * to.token + g * to.group + m * to.head;
        if (chunk < a.rot_chunks) {
            rotate<TYPE, NEAR, P>(x, out, chunk * P, a.pairs, angles + t * a.pairs);
        } else if (is_x ? a.copy_x : a.copy_k) {
            const uint32_t f = a.rotated + (chunk - a.rot_chunks) * kCopied;
            if (f + kCopied <= a.dim) {
                float w[kCopied];
                load_row<TYPE>(x + f, w);
                store_row<TYPE>(out + f, w);
            } else {
                for (uint32_t e = f; e < a.dim; ++e)
                    out[e] = x[e];
            }
        }
    }
}

template <int TYPE, bool NEAR>
void launch_pairs(const Args &a, uint32_t per, unsigned grid, size_t lds, hipStream_t stream) {
    const dim3 g(grid), b(kThreads);
    if (per == 8)
        hipLaunchKernelGGL((rotary_kernel<TYPE, NEAR, 8>), g, b, lds, stream, a);
    else if (per == 4)
        hipLaunchKernelGGL((rotary_kernel<TYPE, NEAR, 4>), g, b, lds, stream, a);
    else if (per == 2)
        hipLaunchKernelGGL((rotary_kernel<TYPE, NEAR, 2>), g, b, lds, stream, a);
    else
        hipLaunchKernelGGL((rotary_kernel<TYPE, NEAR, 1>), g, b, lds, stream, a);
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs &r, int type, hipStream_t stream) {
    Args a;
    a.x = r.x, a.out = r.out, a.k = r.k, a.k_out = r.k_out;
    a.positions = r.positions, a.turns = r.turns, a.tokens = r.tokens;
    a.dim = r.dim, a.rotated = r.rotated, a.pairs = r.rotated / 2;
    a.heads_x = r.x.groups * r.x.heads;
    a.heads = a.heads_x + r.k.groups * r.k.heads;
    a.scale = r.scale, a.sign = r.backward ? -1.0f : 1.0f;
    a.copy_x = r.copy_x, a.copy_k = r.copy_k;
    // pairs of a lane: whole chunks only
    uint32_t per = type == kBf16 ? 8 : 4;
    while (a.pairs % per)
        per /= 2;
    a.rot_chunks = a.pairs / per;
    a.copy_chunks = r.copy_x || r.copy_k ? (r.dim - r.rotated + kCopied - 1) / kCopied : 0;
    const uint32_t chunks = a.rot_chunks + a.copy_chunks;
    if (!chunks)
        return hipSuccess;
    // a workgroup has at most 16384 items (the divisions hold to 65535) and at most
    // kMostPairs angles: tokens, or where one token has more, some of its heads
    constexpr uint32_t kItems = 4 * kThreads;
    a.share = a.heads;
    if ((size_t)a.heads * chunks > kItems) {
        const uint32_t most = kItems / chunks ? kItems / chunks : 1;
        a.slices = (a.heads + most - 1) / most;
        a.share = (a.heads + a.slices - 1) / a.slices;
    }
    // few tokens: a lane an item, so that no lane waits twice
    if (r.tokens < 1024) {
        const uint32_t most = kThreads / chunks ? kThreads / chunks : 1;
        a.share = a.share < most ? a.share : most;
    }
    a.slices = (a.heads + a.share - 1) / a.share;
    const uint32_t items = a.share * chunks;
    a.tile = r.tokens < 1024 || items >= kItems ? 1 : kItems / items;
    if (a.pairs && a.tile > kMostPairs / a.pairs)
        a.tile = kMostPairs / a.pairs;
    a.by_pairs = make_div(a.pairs ? a.pairs : 1);
    a.by_chunks = make_div(chunks);
    a.by_token = make_div(items);
    a.by_group_x = make_div(r.x.heads ? r.x.heads : 1);
    a.by_group_k = make_div(r.k.heads ? r.k.heads : 1);
    const size_t lds = (size_t)a.tile * a.pairs * sizeof(f32x2);
    // 2^22 workgroups a launch
    const size_t most = (((size_t)1 << 22) / a.slices) * a.tile;
    for (a.base = 0; a.base < r.tokens; a.base += most) {
        const size_t left = r.tokens - a.base < most ? r.tokens - a.base : most;
        const unsigned grid = (unsigned)((left + a.tile - 1) / a.tile * a.slices);
        if (type == kBf16 && r.interleaved)
            launch_pairs<kBf16, true>(a, per, grid, lds, stream);
        else if (type == kBf16)
            launch_pairs<kBf16, false>(a, per, grid, lds, stream);
        else if (r.interleaved)
            launch_pairs<kF32, true>(a, per > 4 ? 4 : per, grid, lds, stream);
        else
            launch_pairs<kF32, false>(a, per > 4 ? 4 : per, grid, lds, stream);
    }
    return hipGetLastError();
}

}  // namespace zpp
