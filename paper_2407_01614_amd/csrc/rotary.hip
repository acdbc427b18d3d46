// Rotary positions (formulas and layouts in zpp.h): one pass over the heads of a
// batch of tokens, forward or backward, in place or into other arrays.
//
// A workgroup takes a few tokens.  Their angles' cosines and sines are computed
// once, a pair a lane, and kept in LDS for all heads: the angle is a product in 64
// bits of which the fraction of a turn is taken there, so that far positions lose
// nothing, and the rest is at most an eighth of a turn, where Taylor's polynomials
// hold.  The heads pass through registers, P pairs a lane: 16 bytes of u and 16 of v of
// halves, 16 in a row of neighbours; a lane's first pieces are on their way while the angles
// are computed.  Where P does not divide the pairs, the last P of a head are loaded whole,
// and those of them that are another lane's are not stored.
//
// Whole heads into another array are stored as a stream (4096 tokens of 64 heads of 128 in
// bf16: 22.8 us, 29.0 without; where pieces share lines a stream costs, 55.6 for 39.4 with 20
// of 80 features turning, and in place it gains nothing).
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
template <int TYPE>
constexpr int kSize = TYPE == kBf16 ? 2 : 4;

// N elements in a row at p, as they lie in up to four words, and back.
template <int TYPE, int N>
__device__ __forceinline__ void load_row(const Element<TYPE> *p, uint32_t (&w)[4]) {
    constexpr int kBytes = N * kSize<TYPE>;
    if constexpr (kBytes == 16) {
        const u32x4 v = ld_at<u32x4, kSize<TYPE>>(p);
        w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
    } else if constexpr (kBytes == 8) {
        const u32x2 v = ld_at<u32x2, kSize<TYPE>>(p);
        w[0] = v.x, w[1] = v.y;
    } else if constexpr (kBytes == 4) {
        w[0] = ld_at<uint32_t, kSize<TYPE>>(p);
    } else {
        w[0] = *reinterpret_cast<const uint16_t *>(p);
    }
}
template <int TYPE, int N, bool STREAM = false>
__device__ __forceinline__ void store_row(Element<TYPE> *p, const uint32_t (&w)[4]) {
    constexpr int kBytes = N * kSize<TYPE>;
    if constexpr (kBytes == 16 && STREAM)
        st_nt_at<u32x4, kSize<TYPE>>(p, u32x4{w[0], w[1], w[2], w[3]});
    else if constexpr (kBytes == 16)
        st_at<u32x4, kSize<TYPE>>(p, u32x4{w[0], w[1], w[2], w[3]});
    else if constexpr (kBytes == 8)
        st_at<u32x2, kSize<TYPE>>(p, u32x2{w[0], w[1]});
    else if constexpr (kBytes == 4)
        st_at<uint32_t, kSize<TYPE>>(p, w[0]);
    else
        *reinterpret_cast<uint16_t *>(p) = (uint16_t)w[0];
}
// Elements `from` .. N of them, `from` the same in all lanes: in as few stores as there are
// ones in their number of words.
template <int TYPE, int N>
__device__ __forceinline__ void store_end(Element<TYPE> *p, const uint32_t (&w)[4], uint32_t from) {
    constexpr uint32_t kWords = N * kSize<TYPE> / 4, kIn = 4 / kSize<TYPE>;
    if (from == 0)
        return store_row<TYPE, N>(p, w);
    uint32_t word = (from + kIn - 1) / kIn;
    if constexpr (TYPE == kBf16 && N > 1) {
#pragma unroll
        for (uint32_t i = 0; i < kWords; ++i)
            if (2 * i + 1 == from)
                p[2 * i + 1] = (uint16_t)(w[i] >> 16);
    }
    if constexpr (kWords == 4) {
        if (word == 1)
            st_at<uint32_t, kSize<TYPE>>(p + kIn, w[1]);
        if (word <= 2)
            st_at<u32x2, kSize<TYPE>>(p + 2 * kIn, u32x2{w[2], w[3]});
        if (word == 3)
            st_at<uint32_t, kSize<TYPE>>(p + 3 * kIn, w[3]);
    } else if constexpr (kWords == 2) {
        if (word == 1)
            st_at<uint32_t, kSize<TYPE>>(p + kIn, w[1]);
    }
}
template <int TYPE, int N>
__device__ __forceinline__ void unpack(const uint32_t (&w)[4], float *x) {
#pragma unroll
    for (int i = 0; i < N; ++i)
        x[i] = TYPE == kF32  ? __uint_as_float(w[i])
               : i % 2 == 0 ? bf16_lo(w[i / 2])
                            : bf16_hi(w[i / 2]);
}
template <int TYPE, int N>
__device__ __forceinline__ void pack(const float *x, uint32_t (&w)[4]) {
    if constexpr (TYPE == kF32) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            w[i] = __float_as_uint(x[i]);
    } else if constexpr (N == 1) {
        w[0] = bf16_pair(x[0], x[0]);
    } else {
#pragma unroll
        for (int i = 0; i < N / 2; ++i)
            w[i] = bf16_pair(x[2 * i], x[2 * i + 1]);
    }
}

// Features of a chunk that is copied; fewer are copied one by one.
template <int TYPE>
constexpr uint32_t kCopied = 32 / kSize<TYPE>;

// A lane's part of a head: P pairs that turn, or features that are copied.
template <int TYPE, bool NEAR, int P, bool STREAM>
struct Part {
    static constexpr int kHalf = kCopied<TYPE> / 2;
    uint32_t w[2][4];
    Element<TYPE> *out;
    uint32_t first, skip, token;  // its first pair or feature, pairs not its own, which token
    enum { kNone, kTurn, kCopy, kOne } what;

    // Item i of a workgroup's.
    __device__ __forceinline__ void load(const Args &a, size_t token0, uint32_t tokens,
                                         uint32_t head0, uint32_t heads, uint32_t i) {
        const uint32_t chunks = a.rot_chunks + a.copy_chunks;
        what = kNone;
        token = a.by_token(i);
        const uint32_t in_token = i - token * a.share * chunks;
        const uint32_t h = a.by_chunks(in_token), chunk = in_token - h * chunks;
        // the last slice may have fewer heads: its items are numbered as the others'
        if (token >= tokens || h >= heads)
            return;
        uint32_t head = head0 + h;
        const bool is_x = head < a.heads_x;
        if (!is_x)
            head -= a.heads_x;
        const Heads &from = is_x ? a.x : a.k, &to = is_x ? a.out : a.k_out;
        const uint32_t g = is_x ? a.by_group_x(head) : a.by_group_k(head);
        const uint32_t m = head - g * from.heads;
        const Element<TYPE> *x = reinterpret_cast<const Element<TYPE> *>(from.data) +
                                 (token0 + token) * from.token + g * from.group + m * from.head;
        out = reinterpret_cast<Element<TYPE> *>(to.data) + (token0 + token) * to.token +
              g * to.group + m * to.head;
        if (chunk < a.rot_chunks) {
            what = kTurn;
            first = chunk * P < a.pairs - P ? chunk * P : a.pairs - P;
            skip = chunk * P - first;
            if constexpr (NEAR) {
                load_row<TYPE, 2 * P>(x + 2 * first, w[0]);
            } else {
                load_row<TYPE, P>(x + first, w[0]);
                load_row<TYPE, P>(x + a.pairs + first, w[1]);
            }
        } else if (is_x ? a.copy_x : a.copy_k) {
            first = chunk - a.rot_chunks;
            if (a.dim - a.rotated < kCopied<TYPE>) {
                what = kOne;
                first += a.rotated;
                load_row<TYPE, 1>(x + first, w[0]);
                return;
            }
            // the last is copied whole as well: what it shares with the one before is the same
            what = kCopy;
            first = a.rotated + first * kCopied<TYPE>;
            first = first < a.dim - kCopied<TYPE> ? first : a.dim - kCopied<TYPE>;
            load_row<TYPE, kHalf>(x + first, w[0]);
            load_row<TYPE, kHalf>(x + first + kHalf, w[1]);
        }
    }

    __device__ __forceinline__ void store(const Args &a, const f32x2 *angles) {
        if (what == kTurn) {
            float x[2 * P];
            if constexpr (NEAR) {
                unpack<TYPE, 2 * P>(w[0], x);
            } else {
                unpack<TYPE, P>(w[0], x);
                unpack<TYPE, P>(w[1], x + P);
            }
            const f32x2 *angle = angles + token * a.pairs + first;
#pragma unroll
            for (int j = 0; j < P; ++j) {
                float &u = x[NEAR ? 2 * j : j], &v = x[NEAR ? 2 * j + 1 : P + j];
                const f32x2 c = angle[j];
                const float turned_u = u * c.x - v * c.y;
                v = u * c.y + v * c.x;
                u = turned_u;
            }
            // (the same in all lanes where it is not 0)
            const auto from = [&] { return __builtin_amdgcn_readfirstlane(skip); };
            if constexpr (NEAR) {
                pack<TYPE, 2 * P>(x, w[0]);
                if (STREAM || skip == 0)
                    store_row<TYPE, 2 * P, STREAM>(out + 2 * first, w[0]);
                else
                    store_end<TYPE, 2 * P>(out + 2 * first, w[0], 2 * from());
            } else {
                pack<TYPE, P>(x, w[0]);
                pack<TYPE, P>(x + P, w[1]);
                if (STREAM || skip == 0) {
                    store_row<TYPE, P, STREAM>(out + first, w[0]);
                    store_row<TYPE, P, STREAM>(out + a.pairs + first, w[1]);
                } else {
                    store_end<TYPE, P>(out + first, w[0], from());
                    store_end<TYPE, P>(out + a.pairs + first, w[1], from());
                }
            }
        } else if (what == kCopy) {
            store_row<TYPE, kHalf>(out + first, w[0]);
            store_row<TYPE, kHalf>(out + first + kHalf, w[1]);
        } else if (what == kOne) {
            store_row<TYPE, 1>(out + first, w[0]);
        }
    }
};

template <int TYPE, bool NEAR, int P, bool STREAM>
__global__ __launch_bounds__(kThreads) void rotary_kernel(Args a) {
    extern __shared__ f32x2 angles[];  // [tokens of the tile][pairs]
    const uint32_t tile = blockIdx.x / a.slices, slice = blockIdx.x % a.slices;
    const size_t token0 = a.base + (size_t)tile * a.tile;
    const uint32_t tokens = (uint32_t)(a.tokens - token0 < a.tile ? a.tokens - token0 : a.tile);
    const uint32_t head0 = slice * a.share;
    const uint32_t heads = a.heads - head0 < a.share ? a.heads - head0 : a.share;
    const uint32_t items = tokens * a.share * (a.rot_chunks + a.copy_chunks);
    constexpr int kParts = 2;
    Part<TYPE, NEAR, P, STREAM> part[kParts];
    const auto load = [&](uint32_t first) {
#pragma unroll
        for (int j = 0; j < kParts; ++j)
            part[j].load(a, token0, tokens, head0, heads, first + threadIdx.x + j * kThreads);
    };
    load(0);
    for (uint32_t i = threadIdx.x; i < tokens * a.pairs; i += kThreads) {
        const uint32_t t = a.by_pairs(i);
        const f32x2 cs = turned((double)a.positions[token0 + t] * a.turns[i - t * a.pairs]);
        angles[i] = f32x2{cs.x * a.scale, cs.y * a.scale * a.sign};
    }
    __syncthreads();
    for (uint32_t first = 0;;) {
#pragma unroll
        for (int j = 0; j < kParts; ++j)
            part[j].store(a, angles);
        first += kParts * kThreads;
        if (first >= items)
            break;
        load(first);
    }
}

// Pairs of a lane: 16 bytes of each half, or of both.
template <int TYPE, bool NEAR>
constexpr uint32_t kMostPer = 16 / kSize<TYPE> / (NEAR ? 2 : 1);
uint32_t most_per(int type, bool near) {
    return type == kBf16 ? (near ? kMostPer<kBf16, true> : kMostPer<kBf16, false>)
                         : (near ? kMostPer<kF32, true> : kMostPer<kF32, false>);
}

template <int TYPE, bool NEAR>
void launch_pairs(const Args &a, uint32_t per, bool whole, unsigned grid, size_t lds,
                  hipStream_t stream) {
    constexpr int kMost = kMostPer<TYPE, NEAR>;
    const dim3 g(grid), b(kThreads);
    if (whole)
        hipLaunchKernelGGL((rotary_kernel<TYPE, NEAR, kMost, true>), g, b, lds, stream, a);
    else if (per == kMost)
        hipLaunchKernelGGL((rotary_kernel<TYPE, NEAR, kMost, false>), g, b, lds, stream, a);
    else if (per == 4)
        hipLaunchKernelGGL((rotary_kernel<TYPE, NEAR, kMost < 4 ? kMost : 4, false>), g, b, lds,
                           stream, a);
    else if (per == 2)
        hipLaunchKernelGGL((rotary_kernel<TYPE, NEAR, kMost < 2 ? kMost : 2, false>), g, b, lds,
                           stream, a);
    else
        hipLaunchKernelGGL((rotary_kernel<TYPE, NEAR, 1, false>), g, b, lds, stream, a);
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
    // (or the largest power of two that there are)
    uint32_t per = most_per(type, r.interleaved);
    while (per > 1 && a.pairs < per)
        per /= 2;
    a.rot_chunks = (a.pairs + per - 1) / per;
    const uint32_t rest = r.dim - r.rotated, copied = type == kBf16 ? kCopied<kBf16> : kCopied<kF32>;
    a.copy_chunks = !(r.copy_x || r.copy_k) ? 0
                    : rest < copied        ? rest
                                           : (rest + copied - 1) / copied;
    const uint32_t chunks = a.rot_chunks + a.copy_chunks;
    if (!chunks)
        return hipSuccess;
    // a workgroup has about kItems items, a head's at least (below 4096; the divisions hold to
    // 65535), and at most kMostPairs angles: tokens, or where one token has more, some of its
    // heads
    constexpr uint32_t kItems = 4 * kThreads;
    a.share = a.heads;
    if ((size_t)a.heads * chunks > kItems) {
        const uint32_t most = kItems / chunks ? kItems / chunks : 1;
        const uint32_t slices = (a.heads + most - 1) / most;
        a.share = (a.heads + slices - 1) / slices;
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
    const bool whole = r.rotated == r.dim && a.pairs % most_per(type, r.interleaved) == 0 &&
                       (r.copy_x || !r.x.heads) && (r.copy_k || !r.k.heads);
    const size_t lds = (size_t)a.tile * a.pairs * sizeof(f32x2);
    // 2^22 workgroups a launch
    const size_t most = (((size_t)1 << 22) / a.slices) * a.tile;
    for (a.base = 0; a.base < r.tokens; a.base += most) {
        const size_t left = r.tokens - a.base < most ? r.tokens - a.base : most;
        const unsigned grid = (unsigned)((left + a.tile - 1) / a.tile * a.slices);
        if (type == kBf16 && r.interleaved)
            launch_pairs<kBf16, true>(a, per, whole, grid, lds, stream);
        else if (type == kBf16)
            launch_pairs<kBf16, false>(a, per, whole, grid, lds, stream);
        else if (r.interleaved)
            launch_pairs<kF32, true>(a, per, whole, grid, lds, stream);
        else
            launch_pairs<kF32, false>(a, per, whole, grid, lds, stream);
    }
    return hipGetLastError();
}

}  // namespace zpp
