// Layer norm's forward and backward pass (formulas in zpp.h).
//
// A row of up to 8192 features lives in the registers of one workgroup, eight
// consecutive elements a lane, so HBM is read once and the mean is known before
// the squares are summed.  A row's lanes are as many as it asks for, in whole
// waves (4544 features: 568 chunks on 576 lanes).  Rows of up to 16384 are held
// so with two chunks a lane; longer ones are read again for each sum.  HBM bounds
// long batches (a copy here runs at 6.74 TB/s): 8192x8192 bf16 with residual and
// checkpoint forward 107 us (5.7 TB/s), backward 87 (5.4) and 5 for the join of
// the weights' gradients; 4096x4544 backward 33 (5.1) and 5.  Short ones are
// bound by their launches and first loads.
//
// RAGGED: rows whose last chunk of 8 is partial.  The lane that has it takes the
// row's last 8 elements instead and leaves out those that are the lane's before
// (single loads would need registers of their own, and a workgroup of 1024 lanes
// has 128 of each).  Rows of less than 8 go with the long ones.
#include <type_traits>

#include "zpp_act8.h"

namespace zpp {
namespace {

constexpr uint32_t kMaxThreads = 1024;
constexpr uint32_t kMostRegCols = kMaxThreads * 8;  // features of a row, a chunk a lane

// Sums of Q values over a row's lanes, the same in every lane.  Two buffers in
// turn: a wave writes a buffer again only after the barrier of the call between,
// which every wave reaches after it has read this one.
template <int Q>
struct GroupSum {
    float part[2][16][Q];
};

// Sums of q over the `waves` waves that a row's lanes make up, first of them
// `wave0` (a workgroup may hold several rows).
template <int Q>
__device__ __forceinline__ void group_sum(float (&q)[Q], GroupSum<Q> &s, uint32_t &turn,
                                          uint32_t wave0, uint32_t waves) {
#pragma unroll
    for (int i = 0; i < Q; ++i)
        q[i] = sum64_last(q[i]);
    if (waves == 1) {
#pragma unroll
        for (int i = 0; i < Q; ++i)
            q[i] = lane_value(q[i], kWave - 1);
        return;
    }
    const uint32_t lane = threadIdx.x & (kWave - 1);
    if (lane == kWave - 1) {
#pragma unroll
        for (int i = 0; i < Q; ++i)
            s.part[turn][threadIdx.x / kWave][i] = q[i];
    }
    __syncthreads();
    // every 16 lanes read all of the row's waves
    const uint32_t wave = lane & 15;
    float v[Q];
#pragma unroll
    for (int i = 0; i < Q; ++i)
        v[i] = s.part[turn][wave < waves ? wave0 + wave : wave0][i];
#pragma unroll
    for (int i = 0; i < Q; ++i)
        q[i] = sum16(wave < waves ? v[i] : 0.0f);
    turn ^= 1;
}

// Eight elements of a weight or bias of either type as fp32; 0 past the end.
__device__ __forceinline__ void load_param(const void *p, int type, uint32_t col, uint32_t valid,
                                           float (&x)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
        x[e] = 0.0f;
    if (!p || !valid)
        return;
    uint8_t *at = reinterpret_cast<uint8_t *>(const_cast<void *>(p)) + col * (type == kF32 ? 4 : 2);
    const Mat m = {at, nullptr, 0};
    if (type == kF32)
        chunk_values(load_chunk<kF32>(m, 0, valid, 0), x);
    else
        chunk_values(load_chunk<kBf16>(m, 0, valid, 0), x);
}

__device__ __forceinline__ uint32_t valid_at(uint32_t col, uint32_t cols) {
    return col >= cols ? 0 : cols - col < 8 ? cols - col : 8;
}

// A lane's share of a row.
struct RowLane {
    uint32_t col;    // its 8 elements start here
    uint32_t first;  // of them, those before this one are the lane's before
    uint32_t block;  // the checkpoint's block of its elements
    bool in;         // the row reaches it
};

template <bool RAGGED>
__device__ __forceinline__ RowLane row_lane(uint32_t lane, uint32_t cols) {
    RowLane l;
    l.col = lane * 8;
    l.block = l.col / kActBlock;
    l.in = l.col < cols;
    l.first = 0;
    if (RAGGED && l.in && cols - l.col < 8) {
        l.first = 8 - (cols - l.col);
        l.col = cols - 8;
    }
    return l;
}

// A lane's elements of a row: the row's address is the same in all lanes and stays
// in scalar registers, a lane adds 32 bits.
template <int TYPE>
__device__ __forceinline__ Mat lane_at(const Mat &m, size_t row, const RowLane &l,
                                       uint32_t blocks) {
    constexpr uint32_t kSize = TYPE == kF32 ? 4 : TYPE == kBf16 ? 2 : 1;
    Mat at = m;
    at.data = reinterpret_cast<uint8_t *>(m.data) + row * m.stride * kSize + l.col * kSize;
    if (TYPE == kI8)
        at.exps = m.exps + row * blocks + l.block;
    return at;
}

template <int TYPE>
__device__ __forceinline__ Chunk<TYPE> load_row(const Mat &m, size_t row, const RowLane &l,
                                                uint32_t blocks) {
    return load_chunk<TYPE, false>(lane_at<TYPE>(m, row, l, blocks), 0, 8, 0);
}

template <int TYPE, bool RAGGED>
__device__ __forceinline__ void store_row(const Mat &m, size_t row, const RowLane &l,
                                          const Chunk<TYPE> &c) {
    const Mat at = lane_at<TYPE>(m, row, l, 0);
    if (!RAGGED || l.first == 0) {
        store_chunk<TYPE, false>(at, 0, 8, c);
        return;
    }
#pragma unroll
    for (uint32_t e = 1; e < 8; ++e)
        if (e >= l.first) {
            if constexpr (TYPE == kBf16)
                reinterpret_cast<uint16_t *>(at.data)[e] = (uint16_t)(c.w[e / 2] >> (16 * (e % 2)));
            else
                reinterpret_cast<float *>(at.data)[e] = e < 4 ? c.lo[e] : c.hi[e - 4];
        }
}

// Writes the checkpoint of the elements that the 8 lanes of a block hold, all
// of which take part, `top` each one's largest.
template <bool RAGGED>
__device__ __forceinline__ void save_row(const Mat &m, size_t row, const RowLane &l,
                                         uint32_t blocks, uint32_t top, const float (&x)[8]) {
    const uint32_t exp = act_exp(max8(top));
    if (!l.in)
        return;
    const u32x2 w = act_codes(x, exp);
    const Mat at = lane_at<kI8>(m, row, l, blocks);
    uint8_t *p = reinterpret_cast<uint8_t *>(at.data);
    if (!RAGGED || l.first == 0) {
        st_nt_at<u32x2, 1>(p, w);
    } else {
#pragma unroll
        for (uint32_t e = 1; e < 8; ++e)
            if (e >= l.first)
                p[e] = (uint8_t)(w[e / 4] >> (8 * (e % 4)));
    }
    if ((threadIdx.x & 7) == 0)
        *at.exps = (uint8_t)exp;
}

// Elements that are not the lane's set to 0.
template <bool RAGGED>
__device__ __forceinline__ void clear_others(float (&x)[8], const RowLane &l) {
    if constexpr (RAGGED) {
#pragma unroll
        for (uint32_t e = 0; e < 7; ++e)
            x[e] = e < l.first ? 0.0f : x[e];
    }
}

// x, or x + residual rounded to the matrices' type (and stored as `total`).
template <int TYPE, class Store>
__device__ __forceinline__ void norm_input(const NormForwardArgs &a, const Chunk<TYPE> &cx,
                                           const Chunk<TYPE> &cr, float (&x)[8], Store &&store) {
    chunk_values(cx, x);
    if (a.residual.data) {
        float r[8];
        chunk_values(cr, r);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            x[e] += r[e];
        const Chunk<TYPE> t = make_chunk<TYPE>(x);
        store(t);
        chunk_values(t, x);
    }
}

// 1 / sqrt(v), within an ulp; v below the normal numbers is scaled up first.
__device__ __forceinline__ float inverse_root(float v) {
    const bool tiny = v < 0x1p-96f;
    return __builtin_amdgcn_rsqf(tiny ? v * 0x1p64f : v) * (tiny ? 0x1p32f : 1.0f);
}

// sum / n, rounded: taken up unrounded in some of the differences from it (as the
// product of an fma), it would not be what their mean corrects.
__device__ __forceinline__ float rounded_mean(float sum, float per) {
#pragma clang fp contract(off)
    return sum * per;
}

// A row's mean, made of its sum, may be ulps off by the roundings of the sum and of the
// quotient.  The mean `off` of the differences from it is what it is off by:
//     mean = near + mean(d),  variance = mean(d^2) - mean(d)^2
// Without that a row of 1000 times 700, whose mean then is 700.00006, has y off by
// 0.02 gamma at an eps of 1e-5.  The product is not rounded before it is taken off
// (beyond 2^64 it may pass fp32 where the mean of squares, Inf, stands), and what
// rounding leaves below 0 is 0.
__device__ __forceinline__ float variance(float off, float square) {
    const float var = __builtin_fmaf(-off, off, square);
    return var < 0.0f ? 0.0f : var;
}

// One row a turn, V chunks a lane, the i-th `threads` lanes after the one
// before; the next row is on its way while this one's sums are made.  With V == 1
// gamma and beta stay in registers; two chunks a lane leave none for them, and
// they lie in LDS as fp32, [2][V][2 halves][threads][4] (8192x16384 bf16, read in
// each row instead and the next row fetched after it: 190 us, 92 so).
template <int TYPE, int V, bool RAGGED>
__global__ __launch_bounds__(kMaxThreads) void norm_forward_kernel(NormForwardArgs a) {
    __shared__ GroupSum<1> scratch;
    extern __shared__ float shared[];
    const uint32_t blocks = (a.cols + kActBlock - 1) / kActBlock;
    const uint32_t waves = blockDim.x / kWave;
    const float per = 1.0f / (float)a.cols;
    uint32_t turn = 0;
    RowLane l[V];
    float gamma[8], beta[8];
    f32x4 *const params = reinterpret_cast<f32x4 *>(shared) + threadIdx.x;
    auto params_of = [&](int v) {
        load_param(a.gamma, a.param_type, l[v].col, l[v].in ? 8 : 0, gamma);
        load_param(a.beta, a.param_type, l[v].col, l[v].in ? 8 : 0, beta);
    };
#pragma unroll
    for (int v = 0; v < V; ++v)
        // a row of two chunks a lane has more than kMaxThreads: its last is a second one
        l[v] = v == V - 1 ? row_lane<RAGGED>(v * blockDim.x + threadIdx.x, a.cols)
                          : row_lane<false>(v * blockDim.x + threadIdx.x, a.cols);
    Chunk<TYPE> cx[V] = {}, cr[V] = {};
    auto fetch = [&](size_t row) {
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (l[v].in) {
                cx[v] = load_row<TYPE>(a.x, row, l[v], blocks);
                if (a.residual.data)
                    cr[v] = load_row<TYPE>(a.residual, row, l[v], blocks);
            }
    };
    fetch(blockIdx.x);
    if constexpr (V == 1) {
        params_of(0);
    } else {
        // a lane reads only what it has written
#pragma unroll
        for (int v = 0; v < V; ++v) {
            params_of(v);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int e = 4 * half;
                params[(2 * v + half) * blockDim.x] =
                    f32x4{gamma[e], gamma[e + 1], gamma[e + 2], gamma[e + 3]};
                params[(2 * (V + v) + half) * blockDim.x] =
                    f32x4{beta[e], beta[e + 1], beta[e + 2], beta[e + 3]};
            }
        }
    }
    for (size_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        if constexpr (RAGGED && V > 1) {
            // the masks that follow from `first` are made again in each row: kept,
            // they take more scalar registers than there are (4096x8201 bf16 38.8 us,
            // 34.0 so; with one chunk a lane they fit, and 4096x4550 goes from 17.9 to 19.5)
            asm volatile("" : "+v"(l[V - 1].first));
        }
        float x[V][8], sum[1] = {0.0f};
        uint32_t top[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (!RAGGED)
                top[v] = max_bits(cx[v]);
            norm_input<TYPE>(a, cx[v], cr[v], x[v], [&](const Chunk<TYPE> &t) {
                if (!RAGGED)
                    top[v] = max_bits(t);
                if (l[v].in)
                    store_row<TYPE, RAGGED>(a.total, row, l[v], t);
            });
            clear_others<RAGGED>(x[v], l[v]);
            if (RAGGED)
                top[v] = max_bits(x[v]);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                sum[0] += x[v][e];
        }
        if (row + gridDim.x < a.rows)
            fetch(row + gridDim.x);
        group_sum(sum, scratch, turn, 0, waves);
        const float near = rounded_mean(sum[0], per);
        // differences from the mean, and the lane's sum of f of them
        float mean = near, d[V][8];
        auto lane_sum = [&](auto &&f) {
            sum[0] = 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float part = 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    part += !RAGGED || (uint32_t)e >= l[v].first ? f(d[v][e]) : 0.0f;
                sum[0] += l[v].in ? part : 0.0f;
            }
        };
        auto center = [&] {
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    d[v][e] = x[v][e] - mean;
        };
        center();
        lane_sum([](float q) { return q * q; });
        group_sum(sum, scratch, turn, 0, waves);
        float var = sum[0] * per;
        // What the mean is off by is ulps of the row's magnitude, and no more than
        // roundings of y where the row varies as much as its mean is; only beyond
        // that is it summed (16384x4544 bf16 52 us, 61 where it is for every row).  Every
        // lane of the row has the same sums, to the bit, and takes the same way.
        if (__builtin_amdgcn_readfirstlane(near * near > var)) {
            lane_sum([](float q) { return q; });
            group_sum(sum, scratch, turn, 0, waves);
            const float off = sum[0] * per;
            mean = near + off;
            var = variance(off, var);
            center();
        }
        const float rstd = inverse_root(var + a.eps);
        if (threadIdx.x == 0) {
            if (a.mean)
                a.mean[row] = mean;
            if (a.rstd)
                a.rstd[row] = rstd;
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float y[8];
            if constexpr (V > 1) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const f32x4 w = params[(2 * v + half) * blockDim.x];
                    const f32x4 b = params[(2 * (V + v) + half) * blockDim.x];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        gamma[4 * half + e] = w[e];
                        beta[4 * half + e] = b[e];
                    }
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e)
                y[e] = __builtin_fmaf(d[v][e] * rstd, gamma[e], beta[e]);
            if (l[v].in)
                store_row<TYPE, RAGGED>(a.y, row, l[v], make_chunk<TYPE>(y));
            if (a.saved.data)
                save_row<RAGGED>(a.saved, row, l[v], blocks, top[v], x[v]);
        }
    }
}

// Elements col .. col + 7 of a row, `valid` of them inside it.
template <int TYPE>
__device__ __forceinline__ Chunk<TYPE> load_part(const Mat &m, size_t row, uint32_t col,
                                                 uint32_t valid, uint32_t blocks) {
    return load_chunk<TYPE>(m, row * m.stride + col, valid, row * blocks + col / kActBlock);
}

// Rows too long for registers: three passes over each.
template <int TYPE>
__global__ __launch_bounds__(kMaxThreads) void norm_forward_long_kernel(NormForwardArgs a) {
    __shared__ GroupSum<2> scratch;
    const uint32_t blocks = (a.cols + kActBlock - 1) / kActBlock;
    const uint32_t waves = blockDim.x / kWave;
    const uint32_t turns = (a.cols + 8 * blockDim.x - 1) / (8 * blockDim.x);
    const float per = 1.0f / (float)a.cols;
    uint32_t turn = 0;
    for (size_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        float sum[2], mean = 0.0f, rstd = 0.0f;
        for (int pass = 0; pass < 3; ++pass) {
            sum[0] = sum[1] = 0.0f;
            for (uint32_t t = 0; t < turns; ++t) {
                const uint32_t col = (t * blockDim.x + threadIdx.x) * 8;
                const uint32_t valid = valid_at(col, a.cols);
                Chunk<TYPE> cx = {}, cr = {};
                if (valid) {
                    cx = load_part<TYPE>(a.x, row, col, valid, blocks);
                    if (a.residual.data)
                        cr = load_part<TYPE>(a.residual, row, col, valid, blocks);
                }
                float x[8];
                norm_input<TYPE>(a, cx, cr, x, [&](const Chunk<TYPE> &t) {
                    if (pass == 2 && valid)
                        store_chunk<TYPE>(a.total, row * a.total.stride + col, valid, t);
                });
                if (pass < 2) {
#pragma unroll
                    for (uint32_t e = 0; e < 8; ++e) {
                        // the mean of the first pass is 0
                        const float d = e < valid ? x[e] - mean : 0.0f;
                        sum[0] += d;
                        sum[1] = __builtin_fmaf(d, d, sum[1]);
                    }
                } else {
                    float gamma[8], beta[8], y[8];
                    load_param(a.gamma, a.param_type, col, valid, gamma);
                    load_param(a.beta, a.param_type, col, valid, beta);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        y[e] = __builtin_fmaf((x[e] - mean) * rstd, gamma[e], beta[e]);
                    if (valid)
                        store_chunk<TYPE>(a.y, row * a.y.stride + col, valid, make_chunk<TYPE>(y));
                    if (a.saved.data)
                        save_chunk(a.saved, row * a.saved.stride + col, valid,
                                   row * blocks + col / kActBlock, valid ? max_bits(x) : 0u, x);
                }
            }
            if (pass == 2)
                break;
            group_sum(sum, scratch, turn, 0, waves);
            if (pass == 0) {
                mean = rounded_mean(sum[0], per);
            } else {
                const float off = sum[0] * per;
                mean += off;
                rstd = inverse_root(variance(off, sum[1] * per) + a.eps);
            }
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
    uint32_t chunks;   // chunks of 8 that they hold, one or two each
    uint32_t teams;    // rows side by side in a workgroup of the backward pass
    uint32_t grid;     // its workgroups, pairs of arrays in the workspace
};

RowShape row_shape(size_t rows, size_t cols) {
    RowShape s = {0, 0, 0, 0};
    if (cols > 2 * kMostRegCols || cols < 8)
        return s;
    const uint32_t each = cols > kMostRegCols ? 2 : 1;
    const size_t lanes = ((cols + 7) / 8 + each - 1) / each;
    s.threads = (uint32_t)((lanes + kWave - 1) / kWave * kWave);
    s.chunks = s.threads * each;
    s.teams = kMaxThreads / s.threads;
    const size_t groups = (rows + s.teams - 1) / s.teams;
    s.grid = (uint32_t)(groups < kCus ? groups : kCus);
    return s;
}

// (x - mean) rstd of a lane's element e, 0 for a lane past the row (whose rstd is given
// as 0) and for those that a checkpoint holds as another lane's: such numbers, -mean
// rstd or a code with another block's scale, may pass fp32, and times a dy of 0 they
// would be NaN in the row's sums.
template <int X, bool RAGGED>
__device__ __forceinline__ float normalised(float x, float mean, float rstd, uint32_t e,
                                            const RowLane &l) {
    const float h = (x - mean) * rstd;
    return RAGGED && X == kI8 && e < l.first ? 0.0f : h;
}

// One row of each team a turn; the next turn's are on their way while this one's
// are summed.
template <int TYPE, int X, bool AGAIN, bool RAGGED>
__global__ __launch_bounds__(kMaxThreads) void norm_backward_kernel(NormBackwardArgs a,
                                                                    uint32_t threads,
                                                                    uint32_t teams) {
    __shared__ GroupSum<2> scratch;
    // gamma (and beta) in fp32, then, where a workgroup has several teams, the
    // join of their sums
    extern __shared__ float shared[];
    const uint32_t blocks = (a.cols + kActBlock - 1) / kActBlock;
    const uint32_t team = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / threads));
    const uint32_t lane = threadIdx.x - team * threads;
    const uint32_t waves = threads / kWave, wave0 = team * waves;
    const RowLane l = row_lane<RAGGED>(lane, a.cols);
    const float per = 1.0f / (float)a.cols;
    uint32_t turn = 0;
    float dg[8], db[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
        dg[e] = db[e] = 0.0f;
    // as two halves of four features a lane, so that neighbouring lanes read
    // neighbouring 16 bytes
    f32x4 *const params = reinterpret_cast<f32x4 *>(shared) + lane;
    auto param = [&](int which, float (&v)[8]) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const f32x4 p = params[(2 * which + half) * threads];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[4 * half + e] = p[e];
        }
    };
    Chunk<TYPE> nd = {}, nr = {};
    Chunk<X> nx = {};
    float stat[2] = {0.0f, 0.0f};  // the next row's mean and factor
    // A row past the last is zeros, and so are its mean and factor: it adds nothing
    // to any sum.
    auto fetch = [&](size_t row) {
        if (row < a.rows) {
            if (l.in) {
                nd = load_row<TYPE>(a.dy, row, l, blocks);
                nx = load_row<X>(a.x, row, l, blocks);
                if (a.dresidual.data)
                    nr = load_row<TYPE>(a.dresidual, row, l, blocks);
            }
            stat[0] = a.mean[row];
            stat[1] = a.rstd[row];
        } else {
            nd = Chunk<TYPE>{};
            nx = Chunk<X>{};
            stat[0] = stat[1] = 0.0f;
        }
    };
    // every team takes as many turns, so that all meet at the barriers
    const size_t step = (size_t)gridDim.x * teams;
    fetch((size_t)blockIdx.x * teams + team);
    if (team == 0) {
#pragma unroll
        for (int which = 0; which < (AGAIN ? 2 : 1); ++which) {
            float v[8];
            load_param(which ? a.beta : a.gamma, a.param_type, l.col, l.in ? 8 : 0, v);
            params[2 * which * threads] = f32x4{v[0], v[1], v[2], v[3]};
            params[(2 * which + 1) * threads] = f32x4{v[4], v[5], v[6], v[7]};
        }
    }
    __syncthreads();
    for (size_t base = (size_t)blockIdx.x * teams; base < a.rows; base += step) {
        const size_t row = base + team;
        const Chunk<TYPE> cr = nr;
        const float mean = stat[0], scale = l.in ? stat[1] : 0.0f;
        float s[2] = {0.0f, 0.0f}, d[8], g[8], h[8];
        chunk_values(nd, d);
        clear_others<RAGGED>(d, l);
        chunk_values(nx, h);
        param(0, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            h[e] = normalised<X, RAGGED>(h[e], mean, scale, e, l);
            dg[e] = __builtin_fmaf(d[e], h[e], dg[e]);
            db[e] += d[e];
            g[e] *= d[e];
            s[0] += g[e];
            s[1] = __builtin_fmaf(g[e], h[e], s[1]);
        }
        if (base + step < a.rows)
            fetch(row + step);
        group_sum(s, scratch, turn, wave0, waves);
        if (!l.in || row >= a.rows)
            continue;
        const float c1 = s[0] * per, c2 = s[1] * per;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            d[e] = scale * __builtin_fmaf(-h[e], c2, g[e] - c1);
        if (a.dresidual.data) {
            float past[8];
            chunk_values(cr, past);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                d[e] += past[e];
        }
        store_row<TYPE, RAGGED>(a.dx, row, l, make_chunk<TYPE>(d));
        if constexpr (AGAIN) {
            float w[8], y[8];
            param(0, w);
            param(1, y);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                y[e] = __builtin_fmaf(h[e], w[e], y[e]);
            store_row<TYPE, RAGGED>(a.y, row, l, make_chunk<TYPE>(y));
        }
    }
    if (!a.partials)
        return;
    // The workgroup's pair, laid out as gamma is, [2][2 halves][threads][4]: the
    // teams' sums of one array at a time side by side in LDS, where gamma was, and
    // added in the teams' order.
    const f32x4 v[4] = {{dg[0], dg[1], dg[2], dg[3]},
                        {dg[4], dg[5], dg[6], dg[7]},
                        {db[0], db[1], db[2], db[3]},
                        {db[4], db[5], db[6], db[7]}};
    f32x4 *const out = reinterpret_cast<f32x4 *>(a.partials) + (size_t)blockIdx.x * 4 * threads;
    if (teams == 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            out[i * threads + lane] = v[i];
        return;
    }
    f32x4 *const sums = reinterpret_cast<f32x4 *>(shared);  // [2 halves][teams][threads]
#pragma unroll
    for (uint32_t which = 0; which < 2; ++which) {
        __syncthreads();
        sums[team * threads + lane] = v[2 * which];
        sums[(teams + team) * threads + lane] = v[2 * which + 1];
        __syncthreads();
        if (team < 2) {
            f32x4 sum = sums[team * teams * threads + lane];
            for (uint32_t t = 1; t < teams; ++t)
                sum += sums[(team * teams + t) * threads + lane];
            out[(2 * which + team) * threads + lane] = sum;
        }
    }
}

// Two chunks a lane, in 128 registers: gamma and the rows' sum of dy lie in LDS as
// fp32, the row itself stays as it was loaded and is unpacked again after its
// sums, and beta is read where it is used.  From bf16 the next row is fetched
// ahead (127 registers); bf16 that also writes y leaves none for that (118 without
// it).  fp32 fetches a row when its turn comes: its kernels take 92 to 114, and one
// with a second row in flight has not been measured.  A lane past the row takes the
// row's last chunk, so that no load is in a branch, and clears it.  8192x12288, dx
// and the weights' gradients: bf16 108 us, fp32 247; as long rows, read twice, 212
// and 440.
template <int TYPE, int X, bool AGAIN, bool RAGGED>
__global__ __launch_bounds__(kMaxThreads) void norm_backward_wide_kernel(NormBackwardArgs a) {
    constexpr bool kAhead = TYPE == kBf16 && !AGAIN;
    constexpr bool kEarly = TYPE == kBf16;  // dresidual is fetched before the sums
    __shared__ GroupSum<2> scratch;
    // gamma, then the sum of dy, [2][2 halves][2 chunks][kMaxThreads][4]
    extern __shared__ float shared[];
    const uint32_t blocks = (a.cols + kActBlock - 1) / kActBlock;
    const uint32_t threads = blockDim.x, waves = threads / kWave;
    const float per = 1.0f / (float)a.cols;
    uint32_t turn = 0;
    RowLane l[2];
    float dg[2][8];
    // the row has more chunks than kMaxThreads: every first chunk is whole
    l[0] = row_lane<false>(threadIdx.x, a.cols);
    l[0].in = true;
    l[1] = row_lane<RAGGED>(threads + threadIdx.x, a.cols);
    if (!l[1].in) {
        l[1].col = a.cols - 8;
        l[1].block = l[1].col / kActBlock;
    }
#pragma unroll
    for (int v = 0; v < 2; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            dg[v][e] = 0.0f;
    // a lane reads only what it has written
    f32x4 *const params = reinterpret_cast<f32x4 *>(shared) + threadIdx.x;
    auto param = [&](int v, float (&p)[8]) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const f32x4 q = params[(2 * half + v) * kMaxThreads];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                p[4 * half + e] = q[e];
        }
    };
    Chunk<TYPE> nd[2], cd[2], cr[2];
    Chunk<X> nx[2], cx[2];
    float stat[2];
    auto fence = [] { __builtin_amdgcn_sched_barrier(0); };
    auto fetch = [&](size_t row) {
#pragma unroll
        for (int v = 0; v < 2; ++v) {
            nd[v] = load_row<TYPE>(a.dy, row, l[v], blocks);
            nx[v] = load_row<X>(a.x, row, l[v], blocks);
        }
        stat[0] = a.mean[row];
        stat[1] = a.rstd[row];
    };
    if (kAhead)
        fetch(blockIdx.x);
#pragma unroll
    for (int v = 0; v < 2; ++v) {
        float p[8];
        load_param(a.gamma, a.param_type, l[v].col, l[v].in ? 8 : 0, p);
        params[v * kMaxThreads] = f32x4{p[0], p[1], p[2], p[3]};
        params[(2 + v) * kMaxThreads] = f32x4{p[4], p[5], p[6], p[7]};
        params[(4 + v) * kMaxThreads] = params[(6 + v) * kMaxThreads] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    for (size_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        // addresses and masks are made again in each row: kept, they take registers
#pragma unroll
        for (int v = 0; v < 2; ++v)
            asm volatile("" : "+v"(l[v].col), "+v"(l[v].block));
        asm volatile("" : "+v"(l[1].first));
        if (!kAhead)
            fetch(row);
        const float mean = stat[0], scale = stat[1];
        float s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int v = 0; v < 2; ++v) {
            float d[8], g[8], h[8];
            cd[v] = l[v].in ? nd[v] : Chunk<TYPE>{};
            cx[v] = l[v].in ? nx[v] : Chunk<X>{};
            fence();
            chunk_values(cd[v], d);
            clear_others<RAGGED>(d, l[v]);
            chunk_values(cx[v], h);
            params[(4 + v) * kMaxThreads] += f32x4{d[0], d[1], d[2], d[3]};
            params[(6 + v) * kMaxThreads] += f32x4{d[4], d[5], d[6], d[7]};
            param(v, g);
            const float inside = l[v].in ? scale : 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                h[e] = normalised<X, RAGGED>(h[e], mean, inside, e, l[v]);
                dg[v][e] = __builtin_fmaf(d[e], h[e], dg[v][e]);
                g[e] *= d[e];
                s[0] += g[e];
                s[1] = __builtin_fmaf(g[e], h[e], s[1]);
            }
        }
        fence();
        if (kEarly && a.dresidual.data) {
#pragma unroll
            for (int v = 0; v < 2; ++v)
                cr[v] = load_row<TYPE>(a.dresidual, row, l[v], blocks);
        }
        if (kAhead && row + gridDim.x < a.rows)
            fetch(row + gridDim.x);
        group_sum(s, scratch, turn, 0, waves);
        const float c1 = s[0] * per, c2 = s[1] * per;
#pragma unroll
        for (int v = 0; v < 2; ++v) {
            if (!l[v].in)
                continue;
            fence();
            hold(cd[v]);
            hold(cx[v]);
            float d[8], g[8], h[8];
            chunk_values(cd[v], d);
            chunk_values(cx[v], h);
            param(v, g);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                h[e] = (h[e] - mean) * scale;
                d[e] = scale * __builtin_fmaf(-h[e], c2, g[e] * d[e] - c1);
            }
            if (a.dresidual.data) {
                float past[8];
                if (!kEarly)
                    cr[v] = load_row<TYPE>(a.dresidual, row, l[v], blocks);
                chunk_values(cr[v], past);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    d[e] += past[e];
            }
            store_row<TYPE, RAGGED>(a.dx, row, l[v], make_chunk<TYPE>(d));
            if constexpr (AGAIN) {
                fence();
                float y[8];
                load_param(a.beta, a.param_type, l[v].col, 8, y);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    y[e] = __builtin_fmaf(h[e], g[e], y[e]);
                store_row<TYPE, RAGGED>(a.y, row, l[v], make_chunk<TYPE>(y));
            }
        }
    }
    if (!a.partials)
        return;
    f32x4 *const out =
        reinterpret_cast<f32x4 *>(a.partials) + (size_t)blockIdx.x * 8 * threads + threadIdx.x;
#pragma unroll
    for (int v = 0; v < 2; ++v) {
        out[v * threads] = f32x4{dg[v][0], dg[v][1], dg[v][2], dg[v][3]};
        out[(2 + v) * threads] = f32x4{dg[v][4], dg[v][5], dg[v][6], dg[v][7]};
        out[(4 + v) * threads] = params[(4 + v) * kMaxThreads];
        out[(6 + v) * threads] = params[(6 + v) * kMaxThreads];
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
            chunk_values(load_part<TYPE>(a.dy, row, col, valid, blocks), d);
            chunk_values(load_part<X>(a.x, row, col, valid, blocks), h);
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
    Chunk<TYPE> nd, nr = {};
    Chunk<X> nx;
    auto fetch = [&](size_t row) {
        nd = load_part<TYPE>(a.dy, row, col, valid, blocks);
        nx = load_part<X>(a.x, row, col, valid, blocks);
        if (a.dresidual.data)
            nr = load_part<TYPE>(a.dresidual, row, col, valid, blocks);
    };
    fetch(blockIdx.y);
    for (size_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const float mean = a.mean[row], rstd = a.rstd[row];
        const float c1 = a.partials[2 * row], c2 = a.partials[2 * row + 1];
        float d[8], h[8], y[8], past[8];
        chunk_values(nd, d);
        chunk_values(nx, h);
        chunk_values(nr, past);
        if (row + gridDim.y < a.rows)
            fetch(row + gridDim.y);
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
        store_chunk<TYPE>(a.dx, row * a.dx.stride + col, valid, make_chunk<TYPE>(d));
        if (a.y.data)
            store_chunk<TYPE>(a.y, row * a.y.stride + col, valid, make_chunk<TYPE>(y));
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
// taking every 16th pair, joined in order.  An array holds `width` columns, in
// their order (chunks == 0) or as the register kernels lay them out.
constexpr uint32_t kJoinWaves = 16;
__global__ __launch_bounds__(kJoinWaves *kWave) void norm_backward_join(
    const float *partials, uint32_t count, uint32_t width, uint32_t chunks, uint32_t cols,
    float *dgamma, float *dbeta, int accumulate) {
    __shared__ float part[kJoinWaves][kWave];
    const uint32_t wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    float *out = blockIdx.y ? dbeta : dgamma;
    if (!out)
        return;
    const uint32_t at = blockIdx.x * kWave + lane;
    uint32_t col = at;
    bool in = at < width;
    if (chunks && in) {
        const uint32_t half = at / (4 * chunks), i = at % (4 * chunks);
        const uint32_t e = 4 * half + i % 4, start = i / 4 * 8;
        // a last, partial chunk holds the row's last 8 columns
        in = start < cols;
        col = start + e;
        if (in && cols - start < 8) {
            col = cols - 8 + e;
            in = col >= start;
        }
    }
    const float *p = partials + (size_t)blockIdx.y * width + at;
    float sum = 0.0f;
    if (in) {
        // sixteen loads at a time; those past the last are not added
        for (uint32_t i = wave; i < count; i += 16 * kJoinWaves) {
            float v[16];
#pragma unroll
            for (uint32_t u = 0; u < 16; ++u) {
                const uint32_t pair = i + u * kJoinWaves;
                v[u] = p[(size_t)(pair < count ? pair : count - 1) * 2 * width];
            }
#pragma unroll
            for (uint32_t u = 0; u < 16; ++u)
                sum += i + u * kJoinWaves < count ? v[u] : 0.0f;
        }
    }
    part[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && in) {
#pragma unroll
        for (uint32_t w = 1; w < kJoinWaves; ++w)
            sum += part[w][lane];
        out[col] = accumulate ? out[col] + sum : sum;
    }
}

// f(std::integral_constant<int, type>()).
template <class F>
hipError_t with_type(int type, F &&f) {
    return type == kBf16 ? f(std::integral_constant<int, kBf16>())
                         : f(std::integral_constant<int, kF32>());
}

uint32_t long_row_groups(size_t rows, size_t cols) {
    const size_t strips = (cols + 8 * kStripThreads - 1) / (8 * kStripThreads);
    const size_t groups = (16 * kCus + strips - 1) / strips;
    return (uint32_t)(groups < rows ? groups : rows);
}

template <int TYPE, int X, bool AGAIN, bool RAGGED>
hipError_t start_backward(const NormBackwardArgs &a, const RowShape &s, hipStream_t stream) {
    const dim3 grid(s.grid), threads(s.threads * s.teams);
    if (s.chunks > s.threads) {
        constexpr size_t kLds = 2 * 2 * 2 * kMaxThreads * sizeof(f32x4);
        static std::atomic<uint64_t> asked{0};
        const hipError_t e = allow_lds(
            reinterpret_cast<const void *>(norm_backward_wide_kernel<TYPE, X, AGAIN, RAGGED>), kLds,
            asked);
        if (e != hipSuccess)
            return e;
        hipLaunchKernelGGL((norm_backward_wide_kernel<TYPE, X, AGAIN, RAGGED>), grid, threads, kLds,
                           stream, a);
        return hipGetLastError();
    }
    const size_t params = (AGAIN ? 2 : 1) * 2 * sizeof(f32x4) * s.threads;
    const size_t sums = s.teams > 1 ? 2 * sizeof(f32x4) * s.teams * s.threads : 0;
    if constexpr (AGAIN) {
        // gamma and beta of 1024 lanes are 64 KB, and the rows' sums come on top
        constexpr size_t kLds = 2 * 2 * sizeof(f32x4) * kMaxThreads;
        static std::atomic<uint64_t> asked{0};
        const hipError_t e = allow_lds(
            reinterpret_cast<const void *>(norm_backward_kernel<TYPE, X, AGAIN, RAGGED>), kLds,
            asked);
        if (e != hipSuccess)
            return e;
    }
    hipLaunchKernelGGL((norm_backward_kernel<TYPE, X, AGAIN, RAGGED>), grid, threads,
                       params > sums ? params : sums, stream, a, s.threads, s.teams);
    return hipGetLastError();
}

template <int TYPE, int X>
hipError_t start_backward(const NormBackwardArgs &a, const RowShape &s, hipStream_t stream) {
    if (s.threads) {
        if (a.cols % 8)
            return a.y.data ? start_backward<TYPE, X, true, true>(a, s, stream)
                            : start_backward<TYPE, X, false, true>(a, s, stream);
        return a.y.data ? start_backward<TYPE, X, true, false>(a, s, stream)
                        : start_backward<TYPE, X, false, false>(a, s, stream);
    }
    const dim3 strips((a.cols + 8 * kStripThreads - 1) / (8 * kStripThreads),
                      long_row_groups(a.rows, a.cols));
    const unsigned groups = (unsigned)(a.rows < 2 * kCus ? a.rows : 2 * kCus);
    hipLaunchKernelGGL((norm_backward_long_sums<TYPE, X>), dim3(groups), dim3(kMaxThreads), 0,
                       stream, a);
    hipLaunchKernelGGL((norm_backward_long_kernel<TYPE, X>), strips, dim3(kStripThreads), 0, stream,
                       a);
    return hipGetLastError();
}

}  // namespace

namespace {

template <int TYPE, int V, bool RAGGED>
hipError_t start_forward(const NormForwardArgs &a, dim3 grid, uint32_t threads,
                         hipStream_t stream) {
    const size_t lds = V > 1 ? (size_t)threads * V * 2 * 8 * sizeof(float) : 0;
    if constexpr (V > 1) {
        static std::atomic<uint64_t> asked{0};
        const hipError_t e =
            allow_lds(reinterpret_cast<const void *>(norm_forward_kernel<TYPE, V, RAGGED>),
                      (size_t)kMaxThreads * V * 2 * 8 * sizeof(float), asked);
        if (e != hipSuccess)
            return e;
    }
    hipLaunchKernelGGL((norm_forward_kernel<TYPE, V, RAGGED>), grid, dim3(threads), lds, stream, a);
    return hipGetLastError();
}

template <int TYPE, int V>
hipError_t start_forward(const NormForwardArgs &a, hipStream_t stream) {
    const size_t lanes = ((size_t)a.cols + 8 * V - 1) / (8 * V);
    const uint32_t threads = (uint32_t)((lanes + kWave - 1) / kWave * kWave);
    // The workgroups that the GPU holds at once, by a SIMD's waves: 8 of up to 64
    // registers (bf16), 6 of up to 80 (fp32), 4 with two chunks a lane.  A workgroup
    // of more than 4 waves is counted with its fullest SIMD's, so that no part of the
    // grid waits for a second round: 10 waves, of which a CU's lanes hold three times,
    // fit twice (4096x5120 bf16 with three counted 22.8 us, 18.0 with two; 2048x4544
    // fp32 with 8 waves a SIMD 23.4, 18.8 so).  bf16 rows with a partial chunk are
    // counted as the others, though their kernel's 104 scalar registers leave 7 waves:
    // rows of 6 to 8 waves then have a second round and would gain by 7 (8192x4001
    // 35.2 -> 29.6 us), narrower ones would lose (16384x1001 19.1 -> 20.3, 8192x2501
    // 19.7 -> 21.0).
    constexpr uint32_t kWaves = V == 2 ? 4 : TYPE == kF32 ? 6 : 8;
    const uint32_t waves = threads / kWave;
    const size_t fit = (size_t)kCus * (waves > 4 ? kWaves / ((waves + 3) / 4) : kWaves * 4 / waves);
    const dim3 grid((unsigned)(a.rows < fit ? a.rows : fit));
    return a.cols % 8 ? start_forward<TYPE, V, true>(a, grid, threads, stream)
                      : start_forward<TYPE, V, false>(a, grid, threads, stream);
}

}  // namespace

hipError_t launch_norm_forward(const NormForwardArgs &a, int type, hipStream_t stream) {
    return with_type(type, [&](auto t) {
        constexpr int T = decltype(t)::value;
        if (a.cols >= 8 && a.cols <= 2 * kMostRegCols)
            return a.cols <= kMostRegCols ? start_forward<T, 1>(a, stream)
                                          : start_forward<T, 2>(a, stream);
        hipLaunchKernelGGL((norm_forward_long_kernel<T>),
                           dim3((unsigned)(a.rows < 2 * kCus ? a.rows : 2 * kCus)),
                           dim3(kMaxThreads), 0, stream, a);
        return hipGetLastError();
    });
}

size_t norm_backward_workspace(size_t rows, size_t cols) {
    if (rows == 0 || cols == 0)
        return 0;
    const RowShape s = row_shape(rows, cols);
    if (s.threads)
        return (size_t)s.grid * 2 * s.chunks * 8 * sizeof(float);
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
            return x_type == kI8 ? start_backward<T, kI8>(a, s, stream)
                                 : start_backward<T, T>(a, s, stream);
        });
        if (e != hipSuccess)
            return e;
    }
    if (!weights)
        return hipSuccess;
    const uint32_t pairs =
        !a.rows ? 0 : s.threads ? s.grid : long_row_groups(a.rows, a.cols);
    const float *partials = args.partials + (s.threads ? 0 : 2 * a.rows);
    const uint32_t width = s.threads ? s.chunks * 8 : a.cols;
    hipLaunchKernelGGL(norm_backward_join, dim3((width + kWave - 1) / kWave, 2),
                       dim3(kJoinWaves * kWave), 0, stream, partials, pairs, width, s.chunks,
                       a.cols, a.dgamma, a.dbeta, a.accumulate);
    return hipGetLastError();
}

}  // namespace zpp
