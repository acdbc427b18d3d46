// Checkpoints of activations in 8 bits, and GELU's forward and backward pass
// with them (the formats and formulas are in zpp.h).
//
// All four are one pass over matrices: eight neighbouring lanes take one block
// of 64 elements of a row, 16 bytes of bf16 a lane, so the block's largest
// magnitude is three DPP steps over values that are in registers anyway.  HBM
// bounds them where matrices are long (a copy here runs at 6.74 TB/s): bf16
// 8192x8192 saved 32.7 us (6.2 TB/s) and read back 33.2 (6.1); GELU of
// 2048x32768 with its checkpoint 56.5 (6.0); back from a checkpoint, its output
// again as well, 4096x18176 80.7 (6.5).  Short ones are bound by their launch.
#include <initializer_list>

#include "zpp_act8.h"

namespace zpp {
namespace {

constexpr uint32_t kThreads = 256;
constexpr uint32_t kGroups = kThreads / 8;  // lane groups, blocks side by side

// Where a lane's eight elements are: row and column, or, where all matrices are
// without gaps and rows are whole blocks (FLAT), the place in one long row.
struct Place {
    size_t row, col, block;
    uint32_t valid;  // elements to the row's end, kApart + 4 at most; 0 past either end
    __device__ __forceinline__ size_t in(const Mat &m) const { return row * m.stride + col; }
};

// The blocks of a [rows, cols] matrix are numbered along its rows.  A
// workgroup's first block is found by one 64-bit division that the whole
// workgroup shares; a lane's own lies less than per_row + 64 blocks further on,
// which the high half of a product divides: with per_row < 2^26 and x < 2^26 + 64,
// magic = ceil(2^58 / per_row) gives x magic / 2^58 - x / per_row < x / 2^58 <
// 1 / per_row, so the quotient is exact.
struct Blocks {
    size_t total;
    uint32_t cols, per_row;
    uint64_t magic;
};

template <bool FLAT, uint32_t APART>
__device__ __forceinline__ Place place_of(const Blocks &b, size_t block0, size_t row0,
                                          uint32_t rem0, uint32_t i) {
    constexpr uint32_t kFull = APART + 4;
    const uint32_t lane = (threadIdx.x & 7) * (APART == 4 ? 8 : 4);
    Place p;
    p.block = block0 + i;
    if constexpr (FLAT) {
        p.row = 0;
        p.col = block0 * kActBlock + (i * kActBlock + lane);
        p.valid = i < b.total - block0 ? kFull : 0;
    } else {
        const uint32_t x = rem0 + i;
        const uint32_t q = (uint32_t)__umul64hi((uint64_t)x << 6, b.magic);
        const uint32_t col = (x - q * b.per_row) * kActBlock + lane;
        p.row = row0 + q;
        p.col = col;
        p.valid = i < b.total - block0 && col < b.cols ? (b.cols - col < kFull ? b.cols - col : kFull) : 0;
    }
    return p;
}

// P(-u) exp(u^2 / 2) for u >= 0 as a polynomial in t = 1 / (1 + 0.304 u), a fit of
// the least largest relative error, 1e-7 at most over 0 <= u <= 14 with the constants
// in fp32 as they are here; then P(-u) is that times exp(-u^2 / 2).  The division by
// u falls to t, so one polynomial serves the middle and the tail, with the tail's
// relative accuracy: in fp32 1.6e-6 up to u = 5, where exp's argument is rounded.
// The density of the backward pass is the same exponential.
struct Normal {
    float tail, density;  // P(-u), p(u)
};
__device__ __forceinline__ Normal normal(float u) {
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.304f, u, 1.0f));
    float q = 0.0366241112f;
    q = __builtin_fmaf(q, t, -0.154349089f);
    q = __builtin_fmaf(q, t, 0.190596193f);
    q = __builtin_fmaf(q, t, -0.0417021737f);
    q = __builtin_fmaf(q, t, 0.122817025f);
    q = __builtin_fmaf(q, t, 0.102640495f);
    q = __builtin_fmaf(q, t, 0.122136578f);
    q = __builtin_fmaf(q, t, 0.121236861f);
    const float e = __builtin_amdgcn_exp2f(u * u * -0.72134752f);  // exp(-u^2 / 2)
    return {q * t * e, 0.39894228f * e};
}
// |u|, kept to 16 where the tail and the density are 0 already, so that Inf, whose
// product with them has no value, takes its limit.  NaN stays.
__device__ __forceinline__ float magnitude(float u) {
    const float a = __builtin_fabsf(u);
    return a > 16.0f ? 16.0f : a;
}
// u P(u) from both sides: u - u P(-u), or -|u| P(-|u|).
__device__ __forceinline__ float gelu(float u, float a, float tail) {
    return __builtin_fmaf(-a, tail, u > 0.0f ? u : 0.0f);
}

struct SaveArgs {
    Mat in, saved;
};
struct LoadArgs {
    Mat saved, out;
};
struct GeluForwardArgs {
    Mat u, a, saved;
};
struct GeluBackwardArgs {
    Mat da, u, du, a;
};

// A lane's eight elements of a block: in a row for bf16, 16 bytes; as fp32 four and
// four that are 32 apart, so that each access of the block's 8 lanes is whole lines
// (fp32 8192x8192, GELU forward with its checkpoint 114 us, 94 so, backward 150 and
// 124).
constexpr uint32_t apart(int type) { return type == kF32 ? 32 : 4; }

// The operators: what a lane loads, and what it makes of it.  kUnroll: blocks a
// lane group takes (GELU's backward pass from bf16, 8192x8192, one / two: 70 / 76
// us; its forward pass 54 / 48).
template <int TYPE>
struct SaveOp {
    static constexpr uint32_t kUnroll = 2, kApart = apart(TYPE);
    typedef SaveArgs Args;
    Chunk<TYPE> x;
    template <bool RAGGED>
    __device__ void load(const Args &a, const Place &p) {
        x = load_chunk<TYPE, RAGGED, kApart>(a.in, p.in(a.in), p.valid, p.block);
    }
    template <bool RAGGED>
    __device__ void store(const Args &a, const Place &p) {
        float v[8];
        chunk_values(x, v);
        save_chunk<RAGGED, kApart>(a.saved, p.in(a.saved), p.valid, p.block, max_bits(x), v);
    }
};

template <int TYPE>
struct LoadOp {
    static constexpr uint32_t kUnroll = 2, kApart = apart(TYPE);
    typedef LoadArgs Args;
    Chunk<kI8> x;
    template <bool RAGGED>
    __device__ void load(const Args &a, const Place &p) {
        x = load_chunk<kI8, RAGGED, kApart>(a.saved, p.in(a.saved), p.valid, p.block);
    }
    template <bool RAGGED>
    __device__ void store(const Args &a, const Place &p) {
        float v[8];
        chunk_values(x, v);
        if (p.valid)
            store_chunk<TYPE, RAGGED, kApart>(a.out, p.in(a.out), p.valid, make_chunk<TYPE>(v));
    }
};

template <int TYPE>
struct GeluForwardOp {
    static constexpr uint32_t kUnroll = 2, kApart = apart(TYPE);
    typedef GeluForwardArgs Args;
    Chunk<TYPE> x;
    template <bool RAGGED>
    __device__ void load(const Args &a, const Place &p) {
        x = load_chunk<TYPE, RAGGED, kApart>(a.u, p.in(a.u), p.valid, p.block);
    }
    template <bool RAGGED>
    __device__ void store(const Args &a, const Place &p) {
        float v[8], y[8];
        chunk_values(x, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float m = magnitude(v[e]);
            y[e] = gelu(v[e], m, normal(m).tail);
        }
        if (p.valid)
            store_chunk<TYPE, RAGGED, kApart>(a.a, p.in(a.a), p.valid, make_chunk<TYPE>(y));
        if (a.saved.data)
            save_chunk<RAGGED, kApart>(a.saved, p.in(a.saved), p.valid, p.block, max_bits(x), v);
    }
};

template <int TYPE, int SAVED>
struct GeluBackwardOp {
    static constexpr uint32_t kUnroll = SAVED == kI8 ? 2 : 1, kApart = apart(TYPE);
    typedef GeluBackwardArgs Args;
    Chunk<TYPE> d;
    Chunk<SAVED> x;
    template <bool RAGGED>
    __device__ void load(const Args &a, const Place &p) {
        d = load_chunk<TYPE, RAGGED, kApart>(a.da, p.in(a.da), p.valid, p.block);
        x = load_chunk<SAVED, RAGGED, kApart>(a.u, p.in(a.u), p.valid, p.block);
    }
    template <bool RAGGED>
    __device__ void store(const Args &a, const Place &p) {
        float v[8], g[8], y[8];
        chunk_values(x, v);
        chunk_values(d, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float m = magnitude(v[e]);
            const Normal n = normal(m);
            // P(u) + u p(u): for u < 0, P(-|u|) - |u| p, otherwise 1 less that
            const float below = __builtin_fmaf(-m, n.density, n.tail);
            g[e] *= v[e] < 0.0f ? below : 1.0f - below;
            y[e] = gelu(v[e], m, n.tail);
        }
        if (p.valid) {
            store_chunk<TYPE, RAGGED, kApart>(a.du, p.in(a.du), p.valid, make_chunk<TYPE>(g));
            if (a.a.data)
                store_chunk<TYPE, RAGGED, kApart>(a.a, p.in(a.a), p.valid, make_chunk<TYPE>(y));
        }
    }
};

template <class Op, bool FLAT>
__global__ __launch_bounds__(kThreads) void blocks_kernel(typename Op::Args args, Blocks b,
                                                          size_t first) {
    constexpr uint32_t kUnroll = Op::kUnroll;
    const size_t block0 = first + (size_t)blockIdx.x * (kGroups * kUnroll);
    size_t row0 = 0;
    uint32_t rem0 = 0;
    if constexpr (!FLAT) {
        row0 = block0 / b.per_row;
        rem0 = (uint32_t)(block0 - row0 * b.per_row);
    }
    Op op[kUnroll];
    Place p[kUnroll];
#pragma unroll
    for (uint32_t i = 0; i < kUnroll; ++i) {
        p[i] = place_of<FLAT, Op::kApart>(b, block0, row0, rem0, i * kGroups + threadIdx.x / 8);
        if (p[i].valid)
            op[i].template load<!FLAT>(args, p[i]);
        else
            op[i] = Op{};
    }
#pragma unroll
    for (uint32_t i = 0; i < kUnroll; ++i)
        op[i].template store<!FLAT>(args, p[i]);
}

// One launch over the matrices; `flat`: none has gaps between its rows.
template <class Op>
hipError_t launch_blocks(const typename Op::Args &args, size_t rows, size_t cols, bool flat,
                         hipStream_t stream) {
    constexpr size_t kPerGroup = (size_t)kGroups * Op::kUnroll;
    Blocks b;
    b.cols = (uint32_t)cols;
    b.per_row = (uint32_t)((cols + kActBlock - 1) / kActBlock);
    b.total = rows * b.per_row;
    // ceil(2^58 / per_row), as the high half of (x << 6) * magic takes it
    b.magic = (((uint64_t)1 << 58) + b.per_row - 1) / b.per_row;
    const size_t most = ((size_t)1 << 22) * kPerGroup;
    for (size_t first = 0; first < b.total; first += most) {
        const size_t count = b.total - first < most ? b.total - first : most;
        const dim3 grid((unsigned)((count + kPerGroup - 1) / kPerGroup));
        if (flat && cols % kActBlock == 0)
            hipLaunchKernelGGL((blocks_kernel<Op, true>), grid, dim3(kThreads), 0, stream, args, b,
                               first);
        else
            hipLaunchKernelGGL((blocks_kernel<Op, false>), grid, dim3(kThreads), 0, stream, args, b,
                               first);
    }
    return hipGetLastError();
}

// Whether the rows of all matrices (those that are given) follow each other.
bool no_gaps(size_t rows, size_t cols, std::initializer_list<const Mat *> mats) {
    for (const Mat *m : mats)
        if (m->data && rows > 1 && m->stride != cols)
            return false;
    return true;
}

}  // namespace

hipError_t launch_checkpoint_save(const Mat &x, const Mat &saved, int type, size_t rows,
                                  size_t cols, hipStream_t stream) {
    const SaveArgs a = {x, saved};
    const bool flat = no_gaps(rows, cols, {&x, &saved});
    return type == kBf16 ? launch_blocks<SaveOp<kBf16>>(a, rows, cols, flat, stream)
                         : launch_blocks<SaveOp<kF32>>(a, rows, cols, flat, stream);
}

hipError_t launch_checkpoint_load(const Mat &saved, const Mat &out, int type, size_t rows,
                                  size_t cols, hipStream_t stream) {
    const LoadArgs a = {saved, out};
    const bool flat = no_gaps(rows, cols, {&saved, &out});
    return type == kBf16 ? launch_blocks<LoadOp<kBf16>>(a, rows, cols, flat, stream)
                         : launch_blocks<LoadOp<kF32>>(a, rows, cols, flat, stream);
}

hipError_t launch_gelu_forward(const Mat &u, const Mat &a, const Mat &saved, int type, size_t rows,
                               size_t cols, hipStream_t stream) {
    const GeluForwardArgs g = {u, a, saved};
    const bool flat = no_gaps(rows, cols, {&u, &a, &saved});
    return type == kBf16 ? launch_blocks<GeluForwardOp<kBf16>>(g, rows, cols, flat, stream)
                         : launch_blocks<GeluForwardOp<kF32>>(g, rows, cols, flat, stream);
}

hipError_t launch_gelu_backward(const Mat &da, const Mat &u, const Mat &du, const Mat &a, int type,
                                int u_type, size_t rows, size_t cols, hipStream_t stream) {
    const GeluBackwardArgs g = {da, u, du, a};
    const bool flat = no_gaps(rows, cols, {&da, &u, &du, &a});
    if (type == kBf16)
        return u_type == kI8
                   ? launch_blocks<GeluBackwardOp<kBf16, kI8>>(g, rows, cols, flat, stream)
                   : launch_blocks<GeluBackwardOp<kBf16, kBf16>>(g, rows, cols, flat, stream);
    return u_type == kI8 ? launch_blocks<GeluBackwardOp<kF32, kI8>>(g, rows, cols, flat, stream)
                         : launch_blocks<GeluBackwardOp<kF32, kF32>>(g, rows, cols, flat, stream);
}

}  // namespace zpp
