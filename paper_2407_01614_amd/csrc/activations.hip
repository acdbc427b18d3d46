// Checkpoints of activations in 8 bits, and GELU's forward and backward pass
// with them (the formats and formulas are in zpp.h).
//
// All four are one pass over matrices: eight neighbouring lanes take one block
// of 64 elements of a row, 16 bytes of bf16 a lane, so the block's largest
// magnitude is three DPP steps over values that are in registers anyway.
#include "zpp_act8.h"

namespace zpp {
namespace {

constexpr uint32_t kThreads = 256;
constexpr uint32_t kUnroll = 2;                              // blocks a lane group takes
constexpr uint32_t kBlocksPerWg = kThreads / 8 * kUnroll;    // blocks of 64 elements

// The blocks of a [rows, cols] matrix are numbered along its rows.  A
// workgroup's first block is found by one 64-bit division that the whole
// workgroup shares; a lane's own lies less than blocks + kBlocksPerWg further on,
// which the high half of a 32-bit product divides: with blocks < 2^26 and x <
// 2^26 + 64, magic = ceil(2^58 / blocks) gives x magic / 2^58 - x / blocks <
// x / 2^58 < 1 / blocks, so the quotient is exact (in 64-bit arithmetic).
struct Blocks {
    size_t rows, total;
    uint32_t cols, per_row;
    uint64_t magic;
};

struct Place {
    size_t row;
    uint32_t col, valid;  // valid: 0 past the row's or the matrix's end
};

__device__ __forceinline__ Place place_of(const Blocks &b, size_t row0, uint32_t rem0, size_t left,
                                          uint32_t i) {
    const uint32_t x = rem0 + i;
    const uint32_t q = (uint32_t)__umul64hi((uint64_t)x << 6, b.magic);
    Place p;
    p.row = row0 + q;
    p.col = (x - q * b.per_row) * kActBlock + (threadIdx.x & 7) * 8;
    p.valid = i < left && p.col < b.cols ? (b.cols - p.col < 8 ? b.cols - p.col : 8) : 0;
    return p;
}

// P(-u) exp(u^2 / 2) for u >= 0 as a polynomial in t = 1 / (1 + 0.3 u), a
// least-squares fit of the relative error, 1.5e-7 at most over 0 <= u <= 14;
// then P(-u) is that times exp(-u^2 / 2).  The division by u falls to t, so one
// polynomial serves the middle and the tail, with the tail's relative accuracy:
// 1.6e-6 up to u = 5, where exp's argument is rounded.  The density of the
// backward pass is the same exponential.
struct Normal {
    float cdf, density;
};
__device__ __forceinline__ Normal normal(float u) {
    const float a = __builtin_fabsf(u);
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3f, a, 1.0f));
    float q = 0.035674769f;
    q = __builtin_fmaf(q, t, -0.15720305f);
    q = __builtin_fmaf(q, t, 0.20635340f);
    q = __builtin_fmaf(q, t, -0.053683549f);
    q = __builtin_fmaf(q, t, 0.12856157f);
    q = __builtin_fmaf(q, t, 0.099913508f);
    q = __builtin_fmaf(q, t, 0.12075396f);
    q = __builtin_fmaf(q, t, 0.11962930f);
    const float e = __builtin_amdgcn_exp2f(a * a * -0.72134752f);  // exp(-u^2 / 2)
    const float tail = q * t * e;
    return {u < 0.0f ? tail : 1.0f - tail, 0.39894228f * e};
}
// u with -Inf (whose product with P = 0 has no value) brought to where P is 0
// already, and its square kept finite.
__device__ __forceinline__ float above_tail(float u) { return u < -16.0f ? -16.0f : u; }

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

template <int TYPE>
struct SaveOp {
    typedef SaveArgs Args;
    Chunk<TYPE> x;
    __device__ void load(const Args &a, const Blocks &b, const Place &p) {
        x = load_chunk<TYPE>(a.in, p.row, p.col, p.valid, b.per_row);
    }
    __device__ void store(const Args &a, const Blocks &b, const Place &p) {
        float v[8];
        chunk_values(x, v);
        save_chunk(a.saved, p.row, p.col, p.valid, b.per_row, v);
    }
};

template <int TYPE>
struct LoadOp {
    typedef LoadArgs Args;
    Chunk<kI8> x;
    __device__ void load(const Args &a, const Blocks &b, const Place &p) {
        x = load_chunk<kI8>(a.saved, p.row, p.col, p.valid, b.per_row);
    }
    __device__ void store(const Args &a, const Blocks &, const Place &p) {
        float v[8];
        chunk_values(x, v);
        if (p.valid)
            store_chunk<TYPE>(a.out, p.row, p.col, p.valid, make_chunk<TYPE>(v));
    }
};

template <int TYPE>
struct GeluForwardOp {
    typedef GeluForwardArgs Args;
    Chunk<TYPE> x;
    __device__ void load(const Args &a, const Blocks &b, const Place &p) {
        x = load_chunk<TYPE>(a.u, p.row, p.col, p.valid, b.per_row);
    }
    __device__ void store(const Args &a, const Blocks &b, const Place &p) {
        float v[8], y[8];
        chunk_values(x, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float u = above_tail(v[e]);
            y[e] = u * normal(u).cdf;
        }
        if (p.valid)
            store_chunk<TYPE>(a.a, p.row, p.col, p.valid, make_chunk<TYPE>(y));
        if (a.saved.data)
            save_chunk(a.saved, p.row, p.col, p.valid, b.per_row, v);
    }
};

template <int TYPE, int SAVED>
struct GeluBackwardOp {
    typedef GeluBackwardArgs Args;
    Chunk<TYPE> d;
    Chunk<SAVED> x;
    __device__ void load(const Args &a, const Blocks &b, const Place &p) {
        d = load_chunk<TYPE>(a.da, p.row, p.col, p.valid, b.per_row);
        x = load_chunk<SAVED>(a.u, p.row, p.col, p.valid, b.per_row);
    }
    __device__ void store(const Args &a, const Blocks &, const Place &p) {
        float v[8], g[8], y[8];
        chunk_values(x, v);
        chunk_values(d, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float u = above_tail(v[e]);
            const Normal n = normal(u);
            // from 16 on the density is 0 in fp32 and u may be Inf
            const float slope = u > 16.0f ? 1.0f : __builtin_fmaf(u, n.density, n.cdf);
            g[e] *= slope;
            y[e] = u * n.cdf;
        }
        if (p.valid) {
            store_chunk<TYPE>(a.du, p.row, p.col, p.valid, make_chunk<TYPE>(g));
            if (a.a.data)
                store_chunk<TYPE>(a.a, p.row, p.col, p.valid, make_chunk<TYPE>(y));
        }
    }
};

template <class Op>
__global__ __launch_bounds__(kThreads) void blocks_kernel(typename Op::Args args, Blocks b,
                                                          size_t first) {
    const size_t block0 = first + (size_t)blockIdx.x * kBlocksPerWg;
    const size_t row0 = block0 / b.per_row;
    const uint32_t rem0 = (uint32_t)(block0 - row0 * b.per_row);
    const size_t left = b.total - block0;
    Op op[kUnroll];
    Place p[kUnroll];
#pragma unroll
    for (uint32_t i = 0; i < kUnroll; ++i) {
        p[i] = place_of(b, row0, rem0, left, (i * kThreads + threadIdx.x) / 8);
        if (p[i].valid)
            op[i].load(args, b, p[i]);
        else
            op[i] = Op{};
    }
#pragma unroll
    for (uint32_t i = 0; i < kUnroll; ++i)
        op[i].store(args, b, p[i]);
}

template <class Op>
hipError_t launch_blocks(const typename Op::Args &args, size_t rows, size_t cols,
                         hipStream_t stream) {
    Blocks b;
    b.rows = rows;
    b.cols = (uint32_t)cols;
    b.per_row = (uint32_t)((cols + kActBlock - 1) / kActBlock);
    b.total = rows * b.per_row;
    // ceil(2^58 / per_row), as the high half of (x << 6) * magic takes it
    b.magic = (((uint64_t)1 << 58) + b.per_row - 1) / b.per_row;
    const size_t most = ((size_t)1 << 22) * kBlocksPerWg;
    for (size_t first = 0; first < b.total; first += most) {
        const size_t count = b.total - first < most ? b.total - first : most;
        const unsigned grid = (unsigned)((count + kBlocksPerWg - 1) / kBlocksPerWg);
        hipLaunchKernelGGL((blocks_kernel<Op>), dim3(grid), dim3(kThreads), 0, stream, args, b,
                           first);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_checkpoint_save(const Mat &x, const Mat &saved, int type, size_t rows,
                                  size_t cols, hipStream_t stream) {
    const SaveArgs a = {x, saved};
    return type == kBf16 ? launch_blocks<SaveOp<kBf16>>(a, rows, cols, stream)
                         : launch_blocks<SaveOp<kF32>>(a, rows, cols, stream);
}

hipError_t launch_checkpoint_load(const Mat &saved, const Mat &out, int type, size_t rows,
                                  size_t cols, hipStream_t stream) {
    const LoadArgs a = {saved, out};
    return type == kBf16 ? launch_blocks<LoadOp<kBf16>>(a, rows, cols, stream)
                         : launch_blocks<LoadOp<kF32>>(a, rows, cols, stream);
}

hipError_t launch_gelu_forward(const Mat &u, const Mat &a, const Mat &saved, int type, size_t rows,
                               size_t cols, hipStream_t stream) {
    const GeluForwardArgs g = {u, a, saved};
    return type == kBf16 ? launch_blocks<GeluForwardOp<kBf16>>(g, rows, cols, stream)
                         : launch_blocks<GeluForwardOp<kF32>>(g, rows, cols, stream);
}

hipError_t launch_gelu_backward(const Mat &da, const Mat &u, const Mat &du, const Mat &a, int type,
                                int u_type, size_t rows, size_t cols, hipStream_t stream) {
    const GeluBackwardArgs g = {da, u, du, a};
    if (type == kBf16)
        return u_type == kI8
                   ? launch_blocks<GeluBackwardOp<kBf16, kI8>>(g, rows, cols, stream)
                   : launch_blocks<GeluBackwardOp<kBf16, kBf16>>(g, rows, cols, stream);
    return u_type == kI8 ? launch_blocks<GeluBackwardOp<kF32, kI8>>(g, rows, cols, stream)
                         : launch_blocks<GeluBackwardOp<kF32, kF32>>(g, rows, cols, stream);
}

}  // namespace zpp
