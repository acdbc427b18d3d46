// Layer norm's forward and backward pass (formulas in zpp.h).
//
// A row of up to 8192 features lives in the registers of one workgroup, eight
// consecutive elements a lane, so HBM is read once and the mean is known before
// the squares are summed.  A row's lanes are as many as it asks for, in whole
// waves (4544 features: 568 chunks on 576 lanes).  Longer rows are read again
// for each sum.
//
// RAGGED: rows whose last chunk of 8 is partial.  Its single loads and stores
// need registers of their own, which a workgroup of 1024 lanes has only 128 of
// each, so the kernels for whole chunks are compiled without them.
#include <type_traits>

#include "zpp_act8.h"

namespace zpp {
namespace {

constexpr uint32_t kMaxThreads = 1024;
constexpr uint32_t kMostRegCols = kMaxThreads * 8;  // features of a row in registers

// Sums of Q values over the workgroup's lanes, the same in every lane.  Two
// buffers in turn: a wave writes a buffer again only after the barrier of the
// call between, which every wave reaches after it has read this one.
template <int Q>
struct GroupSum {
    float part[2][Q][16];
};

// Sum of q over the `waves` waves that a row's lanes make up, first of them
// `wave0` (a workgroup may hold several rows).
template <int Q>
__device__ __forceinline__ void group_sum(float (&q)[Q], GroupSum<Q> &s, uint32_t &turn,
                                          uint32_t wave0, uint32_t waves) {
#pragma unroll
    for (int i = 0; i < Q; ++i)
        q[i] = sum64(q[i]);
    if (waves == 1)
        return;
    if ((threadIdx.x & (kWave - 1)) == 0) {
#pragma unroll
        for (int i = 0; i < Q; ++i)
            s.part[turn][i][threadIdx.x / kWave] = q[i];
    }
    __syncthreads();
    const uint32_t lane = threadIdx.x & 15;
#pragma unroll
    for (int i = 0; i < Q; ++i)
        q[i] = lane_value(sum16(lane < waves ? s.part[turn][i][wave0 + lane] : 0.0f), 0);
    turn ^= 1;
}

// Eight elements of a weight or bias of either type as fp32; 0 past the end.
__device__ __forceinline__ void load_param(const void *p, int type, uint32_t col, uint32_t valid,
                                           float (&x)[8]) {
#pragma unroll
    for (uint32_t e = 0; e < 8; ++e) {
        const uint32_t c = col + clamped(e, valid ? valid : 1);
        x[e] = 0.0f;
        if (p && valid)
            x[e] = type == kF32 ? reinterpret_cast<const float *>(p)[c]
                                : __uint_as_float((uint32_t) reinterpret_cast<const uint16_t *>(p)[c]
                                                  << 16);
    }
}

__device__ __forceinline__ uint32_t valid_at(uint32_t col, uint32_t cols) {
    return col >= cols ? 0 : cols - col < 8 ? cols - col : 8;
}

// Elements past the row's end set to 0.
template <bool RAGGED>
__device__ __forceinline__ void clear_past(float (&x)[8], uint32_t valid) {
    if constexpr (RAGGED) {
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e)
            x[e] = e < valid ? x[e] : 0.0f;
    }
}

// x, or x + residual rounded to the matrices' type (and stored as `total`).
template <int TYPE, bool RAGGED>
__device__ __forceinline__ void norm_input(const NormForwardArgs &a, size_t row, uint32_t col,
                                           uint32_t valid, const Chunk<TYPE> &cx,
                                           const Chunk<TYPE> &cr, bool store, float (&x)[8]) {
    chunk_values(cx, x);
    if (a.residual.data) {
        float r[8];
        chunk_values(cr, r);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            x[e] += r[e];
        const Chunk<TYPE> t = make_chunk<TYPE>(x);
        if (store)
            store_chunk<TYPE, RAGGED>(a.total, row, col, valid, t);
        chunk_values(t, x);
    }
}

// R rows in flight a turn, one lane a chunk; blockDim.x lanes a row.
template <int TYPE, int R, bool RAGGED>
__global__ __launch_bounds__(kMaxThreads) void norm_forward_kernel(NormForwardArgs a) {
    __shared__ GroupSum<R> scratch;
    const uint32_t blocks = (a.cols + kActBlock - 1) / kActBlock;
    const uint32_t waves = blockDim.x / kWave;
    const uint32_t col = threadIdx.x * 8, valid = valid_at(col, a.cols);
    const float per = 1.0f / (float)a.cols;
    uint32_t turn = 0;
    float gamma[8], beta[8];
    load_param(a.gamma, a.param_type, col, valid, gamma);
    load_param(a.beta, a.param_type, col, valid, beta);
    for (size_t row0 = (size_t)blockIdx.x * R; row0 < a.rows; row0 += (size_t)gridDim.x * R) {
        Chunk<TYPE> cx[R] = {}, cr[R] = {};
        if (valid) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const size_t row = row0 + r < a.rows ? row0 + r : a.rows - 1;
                cx[r] = load_chunk<TYPE, RAGGED>(a.x, row, col, valid, blocks);
                if (a.residual.data)
                    cr[r] = load_chunk<TYPE, RAGGED>(a.residual, row, col, valid, blocks);
            }
        }
        float x[R][8], sum[R], mean[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            norm_input<TYPE, RAGGED>(a, row0 + r, col, valid, cx[r], cr[r],
                                     row0 + r < a.rows && valid, x[r]);
            clear_past<RAGGED>(x[r], valid);
            sum[r] = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                sum[r] += x[r][e];
        }
        group_sum(sum, scratch, turn, 0, waves);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            mean[r] = sum[r] * per;
            sum[r] = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float d = x[r][e] - mean[r];
                sum[r] += (RAGGED ? (uint32_t)e < valid : valid != 0) ? d * d : 0.0f;
            }
        }
        group_sum(sum, scratch, turn, 0, waves);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const size_t row = row0 + r;
            if (row >= a.rows)
                break;
            const float rstd = 1.0f / __builtin_sqrtf(sum[r] * per + a.eps);
            if (threadIdx.x == 0) {
                if (a.mean)
                    a.mean[row] = mean[r];
                if (a.rstd)
                    a.rstd[row] = rstd;
            }
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                y[e] = __builtin_fmaf((x[r][e] - mean[r]) * rstd, gamma[e], beta[e]);
            if (valid)
                store_chunk<TYPE, RAGGED>(a.y, row, col, valid, make_chunk<TYPE>(y));
            if (a.saved.data)
                save_chunk<RAGGED>(a.saved, row, col, valid, blocks, x[r]);
        }
    }
}

// Rows too long for registers: three passes over each.
template <int TYPE>
__global__ __launch_bounds__(kMaxThreads) void norm_forward_long_kernel(NormForwardArgs a) {
    __shared__ GroupSum<1> scratch;
    const uint32_t blocks = (a.cols + kActBlock - 1) / kActBlock;
    const uint32_t waves = blockDim.x / kWave;
    const uint32_t turns = (a.cols + 8 * blockDim.x - 1) / (8 * blockDim.x);
    uint32_t turn = 0;
    for (size_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        float sum[1], mean = 0.0f, rstd = 0.0f;
        for (int pass = 0; pass < 3; ++pass) {
            sum[0] = 0.0f;
            for (uint32_t t = 0; t < turns; ++t) {
                const uint32_t col = (t * blockDim.x + threadIdx.x) * 8;
                const uint32_t valid = valid_at(col, a.cols);
                Chunk<TYPE> cx = {}, cr = {};
                if (valid) {
                    cx = load_chunk<TYPE>(a.x, row, col, valid, blocks);
                    if (a.residual.data)
                        cr = load_chunk<TYPE>(a.residual, row, col, valid, blocks);
                }
                float x[8];
                norm_input<TYPE, true>(a, row, col, valid, cx, cr, pass == 2 && valid, x);
                if (pass < 2) {
#pragma unroll
                    for (uint32_t e = 0; e < 8; ++e) {
                        const float d = x[e] - mean;
                        sum[0] += e < valid ? (pass == 0 ? x[e] : d * d) : 0.0f;
                    }
                } else {
                    float gamma[8], beta[8], y[8];
                    load_param(a.gamma, a.param_type, col, valid, gamma);
                    load_param(a.beta, a.param_type, col, valid, beta);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        y[e] = __builtin_fmaf((x[e] - mean) * rstd, gamma[e], beta[e]);
                    if (valid)
                        store_chunk<TYPE>(a.y, row, col, valid, make_chunk<TYPE>(y));
                    if (a.saved.data)
                        save_chunk(a.saved, row, col, valid, blocks, x);
                }
            }
            if (pass == 2)
                break;
            group_sum(sum, scratch, turn, 0, waves);
            if (pass == 0)
                mean = sum[0] / (float)a.cols;
            else
                rstd = 1.0f / __builtin_sqrtf(sum[0] / (float)a.cols + a.eps);
        }
        if (threadIdx.x == 0) {
            if (a.mean)
                a.mean[row] = mean;
            if (a.rstd)
                a.rstd[row] = rstd;
        }
    }
}

// --------------------------------------------------------------------------
// Backward
// --------------------------------------------------------------------------

// The weights' gradients are sums over rows: every workgroup keeps its rows'
// sums in registers and leaves them in the workspace, one pair of arrays
// [2][cols] a workgroup, which a second kernel adds in a fixed order.
struct RowShape {
    uint32_t threads;  // lanes of a row; 0: the row does not fit registers
    uint32_t teams;    // rows side by side in a workgroup of the backward pass
    uint32_t grid;     // its workgroups, pairs of arrays in the workspace
};

constexpr uint32_t kRowsAtOnce = 1;  // rows of a team in flight

RowShape row_shape(size_t rows, size_t cols) {
    RowShape s = {0, 0, 0};
    if (cols > kMostRegCols)
        return s;
    const size_t chunks = (cols + 7) / 8;
    s.threads = (uint32_t)((chunks + kWave - 1) / kWave * kWave);
    s.teams = kMaxThreads / s.threads;
    const size_t groups = (rows + s.teams * kRowsAtOnce - 1) / (s.teams * kRowsAtOnce);
    s.grid = (uint32_t)(groups < 2 * kCus ? groups : 2 * kCus);
    return s;
}

template <int TYPE, int X, int R, bool AGAIN, bool RAGGED>
__global__ __launch_bounds__(kMaxThreads) void norm_backward_kernel(NormBackwardArgs a,
                                                                    uint32_t threads,
                                                                    uint32_t teams) {
    __shared__ GroupSum<2 * R> scratch;
    extern __shared__ float joined[];  // [2][cols] where a workgroup has several teams
    const uint32_t blocks = (a.cols + kActBlock - 1) / kActBlock;
    const uint32_t team = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / threads));
    const uint32_t lane = threadIdx.x - team * threads;
    const uint32_t waves = threads / kWave, wave0 = team * waves;
    const uint32_t col = lane * 8, valid = valid_at(col, a.cols);
    const float per = 1.0f / (float)a.cols;
    uint32_t turn = 0;
    float gamma[8], beta[8], dg[8], db[8];
    load_param(a.gamma, a.param_type, col, valid, gamma);
    if constexpr (AGAIN)
        load_param(a.beta, a.param_type, col, valid, beta);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        dg[e] = db[e] = 0.0f;
    // every team takes as many turns, so that all meet at the barriers
    const size_t step = (size_t)gridDim.x * teams * R;
    for (size_t base = (size_t)blockIdx.x * teams * R; base < a.rows; base += step) {
        const size_t row0 = base + (size_t)team * R;
        Chunk<TYPE> cd[R] = {}, cr[R] = {};
        Chunk<X> cx[R] = {};
        float mean[R], rstd[R];
        if (valid) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const size_t row = row0 + r < a.rows ? row0 + r : a.rows - 1;
                cd[r] = load_chunk<TYPE, RAGGED>(a.dy, row, col, valid, blocks);
                cx[r] = load_chunk<X, RAGGED>(a.x, row, col, valid, blocks);
                if (a.dresidual.data)
                    cr[r] = load_chunk<TYPE, RAGGED>(a.dresidual, row, col, valid, blocks);
            }
        }
        float s[2 * R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const size_t row = row0 + r < a.rows ? row0 + r : a.rows - 1;
            mean[r] = a.mean[row];
            rstd[r] = a.rstd[row];
            // a row past the last, whose values are the last row's, adds nothing
            const uint32_t in = row0 + r < a.rows ? valid : 0;
            float d[8], h[8];
            chunk_values(cd[r], d);
            chunk_values(cx[r], h);
            s[2 * r] = s[2 * r + 1] = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const bool inside = RAGGED ? (uint32_t)e < in : in != 0;
                h[e] = inside ? (h[e] - mean[r]) * rstd[r] : 0.0f;
                d[e] = inside ? d[e] : 0.0f;
                dg[e] = __builtin_fmaf(d[e], h[e], dg[e]);
                db[e] += d[e];
                const float g = d[e] * gamma[e];
                s[2 * r] += g;
                s[2 * r + 1] = __builtin_fmaf(g, h[e], s[2 * r + 1]);
            }
        }
        group_sum(s, scratch, turn, wave0, waves);
        if (!valid)
            continue;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const size_t row = row0 + r;
            if (row >= a.rows)
                break;
            const float c1 = s[2 * r] * per, c2 = s[2 * r + 1] * per;
            float d[8], h[8], y[8];
            chunk_values(cd[r], d);
            chunk_values(cx[r], h);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                h[e] = (h[e] - mean[r]) * rstd[r];
                if constexpr (AGAIN)
                    y[e] = __builtin_fmaf(h[e], gamma[e], beta[e]);
                const float g = __builtin_fmaf(d[e], gamma[e], -c1);
                d[e] = rstd[r] * __builtin_fmaf(-h[e], c2, g);
            }
            if (a.dresidual.data) {
                float past[8];
                chunk_values(cr[r], past);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    d[e] += past[e];
            }
            store_chunk<TYPE, RAGGED>(a.dx, row, col, valid, make_chunk<TYPE>(d));
            if constexpr (AGAIN)
                store_chunk<TYPE, RAGGED>(a.y, row, col, valid, make_chunk<TYPE>(y));
        }
    }
    if (!a.partials)
        return;
    // the teams' sums, one team after the other, then the workgroup's pair
    for (uint32_t t = 0; t < teams; ++t) {
        if (team == t) {
#pragma unroll
            for (uint32_t e = 0; e < 8; ++e)
                if (e < valid) {
                    const uint32_t c = col + e;
                    if (t > 0) {
                        dg[e] += joined[c];
                        db[e] += joined[a.cols + c];
                    }
                    if (t + 1 < teams) {
                        joined[c] = dg[e];
                        joined[a.cols + c] = db[e];
                    } else {
                        float *p = a.partials + (size_t)blockIdx.x * 2 * a.cols;
                        p[c] = dg[e];
                        p[a.cols + c] = db[e];
                    }
                }
        }
        if (t + 1 < teams)
            __syncthreads();
    }
}

// Rows too long for registers: the rows' two sums by one kernel (into the
// workspace's head), then dx and the weights' gradients column strip by strip.
template <int TYPE, int X>
__global__ __launch_bounds__(kMaxThreads) void norm_backward_long_sums(NormBackwardArgs a) {
    __shared__ GroupSum<2> scratch;
    const uint32_t blocks = (a.cols + kActBlock - 1) / kActBlock;
    const uint32_t waves = blockDim.x / kWave;
    const uint32_t turns = (a.cols + 8 * blockDim.x - 1) / (8 * blockDim.x);
    uint32_t turn = 0;
    for (size_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const float mean = a.mean[row], rstd = a.rstd[row];
        float s[2] = {0.0f, 0.0f};
        for (uint32_t t = 0; t < turns; ++t) {
            const uint32_t col = (t * blockDim.x + threadIdx.x) * 8;
            const uint32_t valid = valid_at(col, a.cols);
            if (!valid)
                continue;
            float d[8], h[8], gamma[8];
            chunk_values(load_chunk<TYPE>(a.dy, row, col, valid, blocks), d);
            chunk_values(load_chunk<X>(a.x, row, col, valid, blocks), h);
            load_param(a.gamma, a.param_type, col, valid, gamma);
#pragma unroll
            for (uint32_t e = 0; e < 8; ++e) {
                const float g = e < valid ? d[e] * gamma[e] : 0.0f;
                s[0] += g;
                s[1] += e < valid ? g * ((h[e] - mean) * rstd) : 0.0f;
            }
        }
        group_sum(s, scratch, turn, 0, waves);
        if (threadIdx.x == 0) {
            a.partials[2 * row] = s[0] / (float)a.cols;
            a.partials[2 * row + 1] = s[1] / (float)a.cols;
        }
    }
}

constexpr uint32_t kStripThreads = 64;  // 512 columns a strip

template <int TYPE, int X>
__global__ __launch_bounds__(kStripThreads) void norm_backward_long_kernel(NormBackwardArgs a) {
    const uint32_t blocks = (a.cols + kActBlock - 1) / kActBlock;
    const uint32_t col = (blockIdx.x * kStripThreads + threadIdx.x) * 8;
    const uint32_t valid = valid_at(col, a.cols);
    if (!valid)
        return;
    float gamma[8], beta[8], dg[8], db[8];
    load_param(a.gamma, a.param_type, col, valid, gamma);
    load_param(a.beta, a.param_type, col, valid, beta);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        dg[e] = db[e] = 0.0f;
    for (size_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const float mean = a.mean[row], rstd = a.rstd[row];
        const float c1 = a.partials[2 * row], c2 = a.partials[2 * row + 1];
        float d[8], h[8], y[8], past[8];
        chunk_values(load_chunk<TYPE>(a.dy, row, col, valid, blocks), d);
        chunk_values(load_chunk<X>(a.x, row, col, valid, blocks), h);
        if (a.dresidual.data)
            chunk_values(load_chunk<TYPE>(a.dresidual, row, col, valid, blocks), past);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            h[e] = (h[e] - mean) * rstd;
            dg[e] = __builtin_fmaf(d[e], h[e], dg[e]);
            db[e] += d[e];
            y[e] = __builtin_fmaf(h[e], gamma[e], beta[e]);
            d[e] = rstd * __builtin_fmaf(-h[e], c2, __builtin_fmaf(d[e], gamma[e], -c1));
            if (a.dresidual.data)
                d[e] += past[e];
        }
        store_chunk<TYPE>(a.dx, row, col, valid, make_chunk<TYPE>(d));
        if (a.y.data)
            store_chunk<TYPE>(a.y, row, col, valid, make_chunk<TYPE>(y));
    }
    if (!a.dgamma && !a.dbeta)
        return;
    float *p = a.partials + 2 * a.rows + (size_t)blockIdx.y * 2 * a.cols;
#pragma unroll
    for (uint32_t e = 0; e < 8; ++e)
        if (e < valid) {
            p[col + e] = dg[e];
            p[a.cols + col + e] = db[e];
        }
}

// The workgroups' pairs of arrays added: 64 columns a workgroup, its 16 waves
// taking every 16th pair, joined in order.
constexpr uint32_t kJoinWaves = 16;
__global__ __launch_bounds__(kJoinWaves *kWave) void norm_backward_join(const float *partials,
                                                                        uint32_t count,
                                                                        uint32_t cols,
                                                                        float *dgamma,
                                                                        float *dbeta,
                                                                        int accumulate) {
    __shared__ float part[kJoinWaves][kWave];
    const uint32_t wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    float *out = blockIdx.y ? dbeta : dgamma;
    if (!out)
        return;
    const size_t col = (size_t)blockIdx.x * kWave + lane;
    const float *p = partials + (size_t)blockIdx.y * cols + col;
    float sum = 0.0f;
    if (col < cols)
        for (uint32_t i = wave; i < count; i += kJoinWaves)
            sum += p[(size_t)i * 2 * cols];
    part[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && col < cols) {
#pragma unroll
        for (uint32_t w = 1; w < kJoinWaves; ++w)
            sum += part[w][lane];
        out[col] = accumulate ? out[col] + sum : sum;
    }
}

// Calls f(std::integral_constant<int, type>()).
template <class F>
hipError_t with_type(int type, F &&f) {
    if (type == kBf16)
        f(std::integral_constant<int, kBf16>());
    else
        f(std::integral_constant<int, kF32>());
    return hipGetLastError();
}

uint32_t long_row_groups(size_t rows, size_t cols) {
    const size_t strips = (cols + 8 * kStripThreads - 1) / (8 * kStripThreads);
    const size_t groups = (16 * kCus + strips - 1) / strips;
    return (uint32_t)(groups < rows ? groups : rows);
}

template <int TYPE, int X, bool AGAIN>
void start_backward(const NormBackwardArgs &a, const RowShape &s, hipStream_t stream) {
    const size_t lds = s.teams > 1 ? 2 * sizeof(float) * a.cols : 0;
    const dim3 grid(s.grid), threads(s.threads * s.teams);
    if (a.cols % 8)
        hipLaunchKernelGGL((norm_backward_kernel<TYPE, X, 1, AGAIN, true>), grid, threads, lds,
                           stream, a, s.threads, s.teams);
    else
        hipLaunchKernelGGL((norm_backward_kernel<TYPE, X, kRowsAtOnce, AGAIN, false>), grid,
                           threads, lds, stream, a, s.threads, s.teams);
}

template <int TYPE, int X>
void start_backward(const NormBackwardArgs &a, const RowShape &s, hipStream_t stream) {
    if (s.threads) {
        if (a.y.data)
            start_backward<TYPE, X, true>(a, s, stream);
        else
            start_backward<TYPE, X, false>(a, s, stream);
        return;
    }
    const dim3 strips((a.cols + 8 * kStripThreads - 1) / (8 * kStripThreads),
                      long_row_groups(a.rows, a.cols));
    const unsigned groups = (unsigned)(a.rows < 2 * kCus ? a.rows : 2 * kCus);
    hipLaunchKernelGGL((norm_backward_long_sums<TYPE, X>), dim3(groups), dim3(kMaxThreads), 0,
                       stream, a);
    hipLaunchKernelGGL((norm_backward_long_kernel<TYPE, X>), strips, dim3(kStripThreads), 0, stream,
                       a);
}

}  // namespace

hipError_t launch_norm_forward(const NormForwardArgs &a, int type, hipStream_t stream) {
    const uint32_t threads = row_shape(a.rows, a.cols).threads;
    return with_type(type, [&](auto t) {
        constexpr int T = decltype(t)::value;
        if (!threads) {
            hipLaunchKernelGGL((norm_forward_long_kernel<T>),
                               dim3((unsigned)(a.rows < 2 * kCus ? a.rows : 2 * kCus)),
                               dim3(kMaxThreads), 0, stream, a);
            return;
        }
        // workgroups that fit the GPU's 2048 lanes per CU at once; two rows in
        // flight each where there are rows for all
        const size_t fit = (size_t)kCus * (2048 / threads);
        const dim3 grid((unsigned)(a.rows < fit ? a.rows : fit));
        if (a.cols % 8)
            hipLaunchKernelGGL((norm_forward_kernel<T, 1, true>), grid, dim3(threads), 0, stream, a);
        else if (a.rows < 2 * fit)
            hipLaunchKernelGGL((norm_forward_kernel<T, 1, false>), grid, dim3(threads), 0, stream,
                               a);
        else
            hipLaunchKernelGGL((norm_forward_kernel<T, 2, false>), grid, dim3(threads), 0, stream,
                               a);
    });
}

size_t norm_backward_workspace(size_t rows, size_t cols) {
    if (rows == 0 || cols == 0)
        return 0;
    const RowShape s = row_shape(rows, cols);
    if (s.threads)
        return (size_t)s.grid * 2 * cols * sizeof(float);
    return (2 * rows + (size_t)long_row_groups(rows, cols) * 2 * cols) * sizeof(float);
}

hipError_t launch_norm_backward(const NormBackwardArgs &args, int type, int x_type,
                                hipStream_t stream) {
    const RowShape s = row_shape(args.rows, args.cols);
    NormBackwardArgs a = args;
    const bool weights = a.dgamma || a.dbeta;
    if (s.threads && !weights)
        a.partials = nullptr;
    if (a.rows) {
        const hipError_t e = with_type(type, [&](auto t) {
            constexpr int T = decltype(t)::value;
            if (x_type == kI8)
                start_backward<T, kI8>(a, s, stream);
            else
                start_backward<T, T>(a, s, stream);
        });
        if (e != hipSuccess)
            return e;
    }
    if (!weights)
        return hipSuccess;
    const uint32_t pairs =
        !a.rows ? 0 : s.threads ? s.grid : long_row_groups(a.rows, a.cols);
    const float *partials = args.partials + (s.threads ? 0 : 2 * a.rows);
    hipLaunchKernelGGL(norm_backward_join, dim3((a.cols + kWave - 1) / kWave, 2),
                       dim3(kJoinWaves * kWave), 0, stream, partials, pairs, a.cols, a.dgamma,
                       a.dbeta, a.accumulate);
    return hipGetLastError();
}

}  // namespace zpp
