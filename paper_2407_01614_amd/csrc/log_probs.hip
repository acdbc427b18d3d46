// Log probabilities of given tokens with entropy, the most probable tokens, and the
// gradient of the logits (formulas in zpp.h).
//
// The softmax is one pass: every lane keeps its own running maximum r, sum s of
// e^(x - r) and sum w of e^(x - r) (x - r), rescaled where a batch of its elements
// has a larger one, and lanes, waves and slices of a row are joined at the end:
//     s = sum s_i e^(r_i - r);  w = sum (w_i + (r_i - r) s_i) e^(r_i - r)
//     lse = r + ln s;  entropy = ln s - w / s
// r starts at the lowest finite number, so that masked elements add e^-Inf = 0; a
// row of nothing else ends with s = 0.  Inf or NaN make s NaN.
#include "zpp_act8.h"
#include "zpp_token.h"

namespace zpp {
namespace {

constexpr uint32_t kThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLowest = -3.402823466e38f;
// e^kFar is 0, and 0 times it is 0: in place of -Inf where it is multiplied
constexpr float kFar = -1e4f;

__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }
__device__ __forceinline__ float infinity() { return __uint_as_float(0x7F800000u); }
__device__ __forceinline__ float not_a_number() { return __uint_as_float(kScaleNaNBits); }

struct Sums {
    float r, s, w;
};
__device__ __forceinline__ Sums no_sums() { return {kLowest, 0.0f, 0.0f}; }

// Both as one.
__device__ __forceinline__ Sums joined(const Sums &a, float r) {
    const float d = __builtin_fmaxf(a.r - r, kFar), f = exp_of(d);
    return {r, a.s * f, __builtin_fmaf(d, a.s, a.w) * f};
}
__device__ __forceinline__ Sums join2(const Sums &a, const Sums &b) {
    const float r = __builtin_fmaxf(a.r, b.r);
    const Sums x = joined(a, r), y = joined(b, r);
    return {r, x.s + y.s, x.w + y.w};
}

__device__ __forceinline__ float max_wave(float x) {
    x = __builtin_fmaxf(x, dpp<kSwap1>(x));
    x = __builtin_fmaxf(x, dpp<kSwap2>(x));
    x = __builtin_fmaxf(x, dpp<kMirror8>(x));
    x = __builtin_fmaxf(x, dpp<kMirror16>(x));
    return __builtin_fmaxf(__builtin_fmaxf(lane_value(x, 0), lane_value(x, 16)),
                           __builtin_fmaxf(lane_value(x, 32), lane_value(x, 48)));
}
__device__ __forceinline__ float sum_wave(float x) {
    x = sum16(x);
    return (lane_value(x, 0) + lane_value(x, 16)) + (lane_value(x, 32) + lane_value(x, 48));
}
__device__ __forceinline__ Sums join_wave(const Sums &a) {
    const Sums x = joined(a, max_wave(a.r));
    return {x.r, sum_wave(x.s), sum_wave(x.w)};
}

// The workgroup's, in all lanes; `shared` holds one for each wave.
template <uint32_t THREADS>
__device__ __forceinline__ Sums join_workgroup(Sums a, Sums *shared) {
    a = join_wave(a);
    if constexpr (THREADS > 64) {
        if ((threadIdx.x & 63) == 0)
            shared[threadIdx.x / 64] = a;
        __syncthreads();
        a = shared[0];
#pragma unroll
        for (uint32_t w = 1; w < THREADS / 64; ++w)
            a = join2(a, shared[w]);
    }
    return a;
}

// A row's elements as chunks of eight: chunk i of a row begins at column
// column(i), its second half follows at once (bf16) or 32 columns on (fp32, where
// eight lanes take whole lines so).
template <int TYPE>
constexpr uint32_t kApart = TYPE == kBf16 ? 4 : 32;
template <int TYPE>
__device__ __forceinline__ uint32_t column(uint32_t i) {
    return TYPE == kBf16 ? i * 8 : (i / 8) * 64 + (i % 8) * 4;
}
// Elements from a chunk's column to the row's end, as load_chunk takes them.
template <int TYPE>
__device__ __forceinline__ uint32_t valid_of(uint32_t col, uint32_t end) {
    const uint32_t n = col < end ? end - col : 0;
    return n < kApart<TYPE> + 4 ? n : kApart<TYPE> + 4;
}

// The chunk as loaded, -Inf past the row's end.
template <int TYPE>
__device__ __forceinline__ Chunk<TYPE> load_valid(const Mat &m, size_t off, uint32_t valid) {
    constexpr uint32_t kWhole = kApart<TYPE> + 4;
    Chunk<TYPE> c;
    if constexpr (TYPE == kBf16)
        c.w = u32x4{0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u};
    else
        c.lo = c.hi = f32x4{-infinity(), -infinity(), -infinity(), -infinity()};
    if (valid >= kWhole) {
        c = load_chunk<TYPE, false, kApart<TYPE>>(m, off, valid, 0);
    } else if (valid) {
        const Chunk<TYPE> some = load_chunk<TYPE, true, kApart<TYPE>>(m, off, valid, 0);
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e)
            if (place_at<kApart<TYPE>>(e) < valid) {
                if constexpr (TYPE == kBf16) {
                    const uint32_t half = 0xFFFFu << (16 * (e % 2));
                    c.w[e / 2] = (c.w[e / 2] & ~half) | (some.w[e / 2] & half);
                } else if (e < 4) {
                    c.lo[e] = some.lo[e];
                } else {
                    c.hi[e - 4] = some.hi[e - 4];
                }
            }
    }
    return c;
}

__device__ __forceinline__ float max_of(const float (&x)[8]) {
    return __builtin_fmaxf(__builtin_fmaxf(__builtin_fmaxf(x[0], x[1]), __builtin_fmaxf(x[2], x[3])),
                           __builtin_fmaxf(__builtin_fmaxf(x[4], x[5]), __builtin_fmaxf(x[6], x[7])));
}

// Eight elements added to the sums, none above a.r.
template <bool ENTROPY>
__device__ __forceinline__ void add(Sums &a, const float (&x)[8]) {
    float s = 0.0f, w = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float d = x[e] - a.r, p = exp_of(d);
        s += p;
        if (ENTROPY)
            w = __builtin_fmaf(p, __builtin_fmaxf(d, kFar), w);
    }
    a.s += s;
    a.w += w;
}

struct RowArgs {
    Mat x;
    const int64_t *targets;
    float *log_probs, *lse, *entropies;
    size_t rows, base;  // of the batch, and the launch's first
    uint32_t vocab;
    uint32_t splits, slice;  // slices of a row, and their columns
    Sums *partials;          // [row][split]
    unsigned long long *keys;  // [row][split][top]
    uint32_t top;
    int32_t *top_ids;
    float *top_log_probs;
};

template <int TYPE>
__device__ __forceinline__ float element(const Mat &m, size_t off) {
    return TYPE == kBf16 ? bf16_lo(reinterpret_cast<const uint16_t *>(m.data)[off])
                         : reinterpret_cast<const float *>(m.data)[off];
}

// x - lse with lse = r + ln s, in 64 bits: where the token is nearly certain, the
// difference is far smaller than its terms.
__device__ __forceinline__ float log_prob(float x, const Sums &a, float ln) {
    if (a.s == 0.0f)
        return -infinity();
    return (float)((double)x - (double)a.r - (double)ln);
}

// A row's results, by one lane.
__device__ __forceinline__ void store_sums(const RowArgs &a, size_t row, const Sums &t, float ln) {
    if (a.lse)
        a.lse[row] = t.s == 0.0f ? -infinity() : (float)((double)t.r + (double)ln);
    if (a.entropies)
        a.entropies[row] = t.s == 0.0f ? 0.0f : ln - t.w / t.s;
}
template <int TYPE>
__device__ __forceinline__ void finish(const RowArgs &a, size_t row, const Sums &t, float ln) {
    const int64_t target = a.targets[row];
    float lp = 0.0f;
    if (target >= (int64_t)a.vocab)
        lp = not_a_number();
    else if (target >= 0)
        lp = log_prob(element<TYPE>(a.x, row * a.x.stride + (size_t)target), t, ln);
    a.log_probs[row] = lp;
    store_sums(a, row, t, ln);
}

// THREADS lanes a row or slice: a wave, four rows to a workgroup, or the workgroup.
constexpr uint32_t kBatch = 4;  // chunks of a lane in flight
template <int TYPE, uint32_t THREADS, bool ENTROPY>
__global__ __launch_bounds__(kThreads) void forward_kernel(RowArgs a) {
    __shared__ Sums shared[kThreads / 64];
    const uint32_t lane = threadIdx.x % THREADS;
    const size_t task = (size_t)blockIdx.x * (kThreads / THREADS) + threadIdx.x / THREADS;
    const size_t row = a.base + task / a.splits;
    const uint32_t split = (uint32_t)(task % a.splits);
    if (THREADS == 64 && row >= a.rows)
        return;
    const uint32_t begin = split * a.slice;
    const uint32_t end = a.vocab - begin < a.slice ? a.vocab : begin + a.slice;
    const size_t off = row * a.x.stride;
    Sums t = no_sums();
    for (uint32_t i = lane; begin + column<TYPE>(i - lane) < end; i += kBatch * THREADS) {
        Chunk<TYPE> c[kBatch];
#pragma unroll
        for (uint32_t b = 0; b < kBatch; ++b) {
            const uint32_t col = begin + column<TYPE>(i + b * THREADS);
            c[b] = load_valid<TYPE>(a.x, off + col, valid_of<TYPE>(col, end));
        }
        float x[kBatch][8], r = t.r;
#pragma unroll
        for (uint32_t b = 0; b < kBatch; ++b) {
            chunk_values(c[b], x[b]);
            r = __builtin_fmaxf(r, max_of(x[b]));
        }
        t = joined(t, r);
#pragma unroll
        for (uint32_t b = 0; b < kBatch; ++b)
            add<ENTROPY>(t, x[b]);
    }
    t = join_workgroup<THREADS>(t, shared);
    if (lane == 0) {
        if (a.splits > 1)
            a.partials[row * a.splits + split] = t;
        else
            finish<TYPE>(a, row, t, logf(t.s));
    }
}

// The slices of a row joined by a wave, in the same order each time.
__device__ __forceinline__ Sums join_slices(const RowArgs &a, size_t row) {
    Sums t = no_sums();
    for (uint32_t i = threadIdx.x & 63; i < a.splits; i += 64)
        t = join2(t, a.partials[row * a.splits + i]);
    return join_wave(t);
}

template <int TYPE>
__global__ __launch_bounds__(64) void join_kernel(RowArgs a) {
    const size_t row = a.base + blockIdx.x;
    const Sums t = join_slices(a, row);
    if (threadIdx.x == 0)
        finish<TYPE>(a, row, t, logf(t.s));
}

// --------------------------------------------------------------------------
// The most probable tokens.  An element is one 64-bit key: its value as an integer
// of the same order, and below it its column, inverted, so that of equals the lower
// comes first and no two keys are alike.  Every lane finds its largest key; 128
// groups of two lanes put theirs into LDS, and the k-th largest of these is a
// threshold that at least k elements reach, few more among them: all are in the k
// groups whose largest key reaches it.  They are listed, and each one's rank counted.
// --------------------------------------------------------------------------
typedef unsigned long long Key;
constexpr uint32_t kGroupsOfTop = kThreads / 2;
constexpr uint32_t kTopPerLane = 32;  // keys of a lane at most

__device__ __forceinline__ Key key_of(float x, uint32_t col) {
    const uint32_t b = __float_as_uint(x + 0.0f);  // both zeros are one
    const uint32_t order = b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
    return (Key)order << 32 | (0xFFFFFFFFu - col);
}
__device__ __forceinline__ float value_of(Key k) {
    const uint32_t order = (uint32_t)(k >> 32);
    return __uint_as_float(order & 0x80000000u ? order ^ 0x80000000u : ~order);
}
__device__ __forceinline__ uint32_t column_of(Key k) { return 0xFFFFFFFFu - (uint32_t)k; }

// The workgroup's `top` largest keys.  each(f) calls f with every key of the lane,
// at most kTopPerLane; write(rank, key) stores one.  Returns how many there were, if
// fewer than `top`.  list: 2 kTopPerLane top keys of LDS.
template <class Each, class Write>
__device__ __forceinline__ uint32_t select_top(uint32_t top, Key *list, Each &&each,
                                               Write &&write) {
    __shared__ Key groups[kGroupsOfTop];
    __shared__ Key threshold;
    __shared__ uint32_t listed;
    Key best = 0;  // below every key
    each([&](Key k) { best = k > best ? k : best; });
    const Key beside = (Key)dpp<kSwap1>((uint32_t)(best >> 32)) << 32 | dpp<kSwap1>((uint32_t)best);
    const Key group = best > beside ? best : beside;
    if (threadIdx.x % 2 == 0)
        groups[threadIdx.x / 2] = group;
    if (threadIdx.x == 0) {
        threshold = 1;  // fewer than `top` groups with a key: all their keys
        listed = 0;
    }
    __syncthreads();
    uint32_t above = 0;
#pragma unroll 8
    for (uint32_t j = 0; j < kGroupsOfTop / 2; ++j)
        above += groups[(threadIdx.x % 2) * (kGroupsOfTop / 2) + j] > group;
    above += dpp<kSwap1>(above);
    if (threadIdx.x % 2 == 0 && group && above == top - 1)
        threshold = group;
    __syncthreads();
    const Key least = threshold;
    if (best >= least)
        each([&](Key k) {
            if (k >= least)
                list[atomicAdd(&listed, 1u)] = k;
        });
    __syncthreads();
    const uint32_t n = listed;
    for (uint32_t i = threadIdx.x; i < n; i += kThreads) {
        const Key k = list[i];
        uint32_t rank = 0;
        for (uint32_t j = 0; j < n; ++j)
            rank += list[j] > k;
        if (rank < top)
            write(rank, k);
    }
    return n;
}

// A slice of a row, C chunks a lane: sums and its most probable tokens.
template <int TYPE, uint32_t C>
__global__ __launch_bounds__(kThreads) void top_kernel(RowArgs a) {
    extern __shared__ Key list[];
    __shared__ Sums shared[kThreads / 64];
    const size_t row = a.base + blockIdx.x / a.splits;
    const uint32_t split = blockIdx.x % a.splits, begin = split * a.slice;
    const uint32_t end = a.vocab - begin < a.slice ? a.vocab : begin + a.slice;
    const size_t off = row * a.x.stride;
    Chunk<TYPE> c[C];
    uint32_t valid[C];
#pragma unroll
    for (uint32_t b = 0; b < C; ++b) {
        const uint32_t col = begin + column<TYPE>(threadIdx.x + b * kThreads);
        valid[b] = valid_of<TYPE>(col, end);
        c[b] = load_valid<TYPE>(a.x, off + col, valid[b]);
    }
    float x[C][8];
    Sums t = no_sums();
#pragma unroll
    for (uint32_t b = 0; b < C; ++b) {
        chunk_values(c[b], x[b]);
        t.r = __builtin_fmaxf(t.r, max_of(x[b]));
    }
#pragma unroll
    for (uint32_t b = 0; b < C; ++b)
        add<true>(t, x[b]);
    t = join_workgroup<kThreads>(t, shared);
    if (threadIdx.x == 0)
        a.partials[row * a.splits + split] = t;
    Key *out = a.keys + (row * a.splits + split) * a.top;
    const auto each = [&](auto &&f) {
#pragma unroll
        for (uint32_t b = 0; b < C; ++b)
#pragma unroll
            for (uint32_t e = 0; e < 8; ++e)
                if (place_at<kApart<TYPE>>(e) < valid[b])
                    f(key_of(x[b][e], begin + column<TYPE>(threadIdx.x + b * kThreads) +
                                          place_at<kApart<TYPE>>(e)));
    };
    const uint32_t n =
        select_top(a.top, list, each, [&](uint32_t rank, Key k) { out[rank] = k; });
    for (uint32_t i = n + threadIdx.x; i < a.top; i += kThreads)
        out[i] = 0;
}

// The slices joined: sums, and the most probable of the slices' most probable.
template <int TYPE>
__global__ __launch_bounds__(kThreads) void top_join_kernel(RowArgs a) {
    extern __shared__ Key list[];
    const size_t row = a.base + blockIdx.x;
    const Sums t = join_slices(a, row);
    const float ln = logf(t.s);
    if (threadIdx.x == 0)
        finish<TYPE>(a, row, t, ln);
    const Key *keys = a.keys + row * a.splits * a.top;
    const uint32_t n = a.splits * a.top;
    select_top(
        a.top, list,
        [&](auto &&f) {
            for (uint32_t i = threadIdx.x; i < n; i += kThreads)
                f(keys[i]);
        },
        [&](uint32_t rank, Key k) {
            a.top_ids[row * a.top + rank] = (int32_t)column_of(k);
            a.top_log_probs[row * a.top + rank] = log_prob(value_of(k), t, ln);
        });
}

// --------------------------------------------------------------------------
// The gradient
// --------------------------------------------------------------------------
struct GradArgs {
    Mat x, dx;
    const int64_t *targets;
    const float *lse, *entropies, *dlog_probs, *dentropies;
    size_t rows, base;
    uint32_t vocab, per_row;  // waves of a row
};

// What a row's elements share: p = e^(x - r - ln), dx = p (c - h max(x - r, kFar)) with
// c = h (ln - entropy) - g; g once more at the target's column.
struct RowGrad {
    float r, ln, c, h, g;
    uint32_t target;
};
// No column, and not one past a row's end either.
constexpr uint32_t kNoTarget = UINT32_MAX;
__device__ __forceinline__ RowGrad row_grad(float r, float ln, bool empty, float entropy,
                                            float dlog_prob, float h, int64_t target,
                                            uint32_t vocab) {
    RowGrad q;
    q.target = target >= 0 && target < (int64_t)vocab ? (uint32_t)target : kNoTarget;
    q.g = target < 0 ? 0.0f : target < (int64_t)vocab ? dlog_prob : not_a_number();
    q.r = r, q.ln = ln, q.h = h;
    if (empty) {
        // e^-Inf = 0: no element has a share, and none gets a gradient
        q.r = kLowest, q.ln = 0.0f, q.target = kNoTarget;
        q.h = 0.0f;
        q.g = q.g == q.g ? 0.0f : q.g;
    }
    q.c = __builtin_fmaf(q.h, q.ln - (empty ? 0.0f : entropy), -q.g);
    return q;
}

// Eight elements' gradients; found(x): with the target's logit, by the lane that has it.
template <int TYPE, bool ENTROPY, class F>
__device__ __forceinline__ Chunk<TYPE> grad_chunk(const RowGrad &q, const Chunk<TYPE> &chunk,
                                                  uint32_t col, F &&found) {
    float x[8];
    chunk_values(chunk, x);
    const bool near = q.target - col < kApart<TYPE> + 4;
    if (near) {
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e)
            if (q.target == col + place_at<kApart<TYPE>>(e))
                found(x[e]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float d = x[e] - q.r, p = exp_of(d - q.ln);
        float c = q.c;
        if (ENTROPY)
            c = __builtin_fmaf(-q.h, __builtin_fmaxf(d, kFar), c);
        x[e] = p * c;
    }
    if (near) {
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e)
            x[e] += q.target == col + place_at<kApart<TYPE>>(e) ? q.g : 0.0f;
    }
    return make_chunk<TYPE>(x);
}

// A wave takes kBatch chunks a lane of one row.
template <int TYPE, bool ENTROPY>
__global__ __launch_bounds__(kThreads) void backward_kernel(GradArgs a) {
    const size_t wave = (size_t)blockIdx.x * (kThreads / 64) + threadIdx.x / 64;
    const size_t row = a.base + wave / a.per_row;
    if (row >= a.rows)
        return;
    const uint32_t first = (uint32_t)(wave % a.per_row) * 64 * kBatch + threadIdx.x % 64;
    Chunk<TYPE> c[kBatch];
#pragma unroll
    for (uint32_t b = 0; b < kBatch; ++b) {
        const uint32_t col = column<TYPE>(first + b * 64);
        c[b] = load_valid<TYPE>(a.x, row * a.x.stride + col, valid_of<TYPE>(col, a.vocab));
    }
    const float lse = a.lse[row];
    const RowGrad q =
        row_grad(lse, 0.0f, lse == -infinity(), ENTROPY ? a.entropies[row] : 0.0f,
                 a.dlog_probs[row], ENTROPY ? a.dentropies[row] : 0.0f, a.targets[row], a.vocab);
#pragma unroll
    for (uint32_t b = 0; b < kBatch; ++b) {
        const uint32_t col = column<TYPE>(first + b * 64), valid = valid_of<TYPE>(col, a.vocab);
        if (valid)
            store_chunk<TYPE, true, kApart<TYPE>>(a.dx, row * a.dx.stride + col, valid,
                                                  grad_chunk<TYPE, ENTROPY>(q, c[b], col, [](float) {}));
    }
}

struct TrainArgs {
    RowArgs f;
    Mat dx;
    const float *dlog_probs, *dentropies;
};

// A row held in registers, C chunks a lane: read once, its sums, then its gradient.
template <int TYPE, uint32_t THREADS, uint32_t C, bool ENTROPY>
__global__ __launch_bounds__(THREADS < kThreads ? kThreads : THREADS) void train_kernel(
    TrainArgs a) {
    constexpr uint32_t kGroup = THREADS < kThreads ? kThreads : THREADS;
    __shared__ Sums shared[kGroup / 64];
    const uint32_t lane = threadIdx.x % THREADS;
    const size_t row = a.f.base + (size_t)blockIdx.x * (kGroup / THREADS) + threadIdx.x / THREADS;
    if (THREADS == 64 && row >= a.f.rows)
        return;
    const size_t off = row * a.f.x.stride;
    Chunk<TYPE> c[C];
#pragma unroll
    for (uint32_t b = 0; b < C; ++b) {
        const uint32_t col = column<TYPE>(lane + b * THREADS);
        c[b] = load_valid<TYPE>(a.f.x, off + col, valid_of<TYPE>(col, a.f.vocab));
    }
    const int64_t target = a.f.targets[row];
    const float g = a.dlog_probs[row], h = ENTROPY && a.dentropies ? a.dentropies[row] : 0.0f;
    Sums t = no_sums();
#pragma unroll
    for (uint32_t b = 0; b < C; ++b) {
        float x[8];
        chunk_values(c[b], x);
        t.r = __builtin_fmaxf(t.r, max_of(x));
    }
#pragma unroll
    for (uint32_t b = 0; b < C; ++b) {
        float x[8];
        hold(c[b]);
        chunk_values(c[b], x);
        add<ENTROPY>(t, x);
    }
    t = join_workgroup<THREADS>(t, shared);
    const float ln = logf(t.s);
    if (lane == 0) {
        store_sums(a.f, row, t, ln);
        // the lane that holds the target's logit stores the others: dx may be x
        if (target < 0)
            a.f.log_probs[row] = 0.0f;
        else if (target >= (int64_t)a.f.vocab)
            a.f.log_probs[row] = not_a_number();
        else if (t.s == 0.0f)
            a.f.log_probs[row] = -infinity();
    }
    const RowGrad q = row_grad(t.r, ln, t.s == 0.0f, ln - t.w / t.s, g, h, target, a.f.vocab);
#pragma unroll
    for (uint32_t b = 0; b < C; ++b) {
        const uint32_t col = column<TYPE>(lane + b * THREADS);
        const uint32_t valid = valid_of<TYPE>(col, a.f.vocab);
        hold(c[b]);
        if (valid)
            store_chunk<TYPE, true, kApart<TYPE>>(a.dx, row * a.dx.stride + col, valid,
                                                  grad_chunk<TYPE, ENTROPY>(q, c[b], col, [&](float v) {
                                                      a.f.log_probs[row] = log_prob(v, t, ln);
                                                  }));
    }
}

// --------------------------------------------------------------------------
// Launches
// --------------------------------------------------------------------------

// How a batch's rows are cut: splits slices of `slice` columns each.
struct Cut {
    uint32_t splits, slice;
};

// With `top` a slice is 1, 2 or 4 chunks a lane of a workgroup: the least that makes
// no more than kFill workgroups.
constexpr size_t kFill = 1024;
Cut cut_of(size_t rows, uint32_t vocab, uint32_t top) {
    if (top) {
        uint32_t slice = kThreads * 8;
        while (slice < kThreads * 8 * 4 &&
               (rows * ((vocab + slice - 1) / slice) > kFill ||
                (size_t)((vocab + slice - 1) / slice) * top > kThreads * kTopPerLane / 2))
            slice *= 2;
        return {(vocab + slice - 1) / slice, slice};
    }
    const uint32_t least = kThreads * 8;
    if (vocab <= 2 * least || rows >= kFill / 2)
        return {1, vocab};
    uint32_t splits = (uint32_t)(kFill / (rows ? rows : 1));
    const uint32_t most = (vocab + least - 1) / least;
    splits = splits < most ? splits : most;
    uint32_t slice = (vocab + splits - 1) / splits;
    slice = (slice + least - 1) / least * least;
    return {(vocab + slice - 1) / slice, slice};
}

// Rows a launch, so that its work-items stay below 2^31.
constexpr size_t kMostWorkgroups = (size_t)1 << 22;

RowArgs row_args(const LogProbsArgs &a, const Cut &cut) {
    RowArgs r{};
    r.x = a.x;
    r.targets = a.targets;
    r.log_probs = a.log_probs, r.lse = a.lse, r.entropies = a.entropies;
    r.rows = a.rows;
    r.vocab = a.vocab;
    r.splits = cut.splits, r.slice = cut.slice;
    r.partials = reinterpret_cast<Sums *>(a.workspace);
    const size_t sums = (a.rows * cut.splits * sizeof(Sums) + 15) / 16 * 16;
    r.keys = reinterpret_cast<unsigned long long *>(reinterpret_cast<char *>(a.workspace) + sums);
    r.top = a.top, r.top_ids = a.top_ids, r.top_log_probs = a.top_log_probs;
    return r;
}

// launch(workgroups) for rows base .. of RowArgs or GradArgs, `per_row` workgroups
// each, or `rows_per` rows to a workgroup.
template <class A, class F>
void for_rows(A &a, size_t per_row, size_t rows_per, F &&launch) {
    const size_t rows = a.rows;
    size_t most = kMostWorkgroups / per_row * rows_per;
    if (!most)
        most = 1;
    for (size_t r = 0; r < rows; r += most) {
        const size_t left = rows - r < most ? rows - r : most;
        a.base = r;
        a.rows = r + left;
        launch((unsigned)((left * per_row + rows_per - 1) / rows_per));
    }
    a.rows = rows;
}

template <int TYPE>
void forward_typed(const LogProbsArgs &args, hipStream_t stream) {
    const Cut cut = cut_of(args.rows, args.vocab, args.top);
    RowArgs a = row_args(args, cut);
    if (args.top) {
        const size_t lds = 2 * kTopPerLane * args.top * sizeof(Key);
        const uint32_t chunks = cut.slice / (kThreads * 8);
        for_rows(a, cut.splits, 1, [&](unsigned grid) {
            if (chunks == 1)
                hipLaunchKernelGGL((top_kernel<TYPE, 1>), dim3(grid), dim3(kThreads), lds, stream,
                                   a);
            else if (chunks == 2)
                hipLaunchKernelGGL((top_kernel<TYPE, 2>), dim3(grid), dim3(kThreads), lds, stream,
                                   a);
            else
                hipLaunchKernelGGL((top_kernel<TYPE, 4>), dim3(grid), dim3(kThreads), lds, stream,
                                   a);
        });
        for_rows(a, 1, 1, [&](unsigned grid) {
            hipLaunchKernelGGL(top_join_kernel<TYPE>, dim3(grid), dim3(kThreads), lds, stream, a);
        });
        return;
    }
    // a wave a row where that is enough lanes for it
    if (cut.splits == 1 && args.vocab <= 2048) {
        for_rows(a, 1, kThreads / 64, [&](unsigned grid) {
            if (a.entropies)
                hipLaunchKernelGGL((forward_kernel<TYPE, 64, true>), dim3(grid), dim3(kThreads), 0,
                                   stream, a);
            else
                hipLaunchKernelGGL((forward_kernel<TYPE, 64, false>), dim3(grid), dim3(kThreads), 0,
                                   stream, a);
        });
        return;
    }
    for_rows(a, cut.splits, 1, [&](unsigned grid) {
        if (a.entropies)
            hipLaunchKernelGGL((forward_kernel<TYPE, kThreads, true>), dim3(grid), dim3(kThreads),
                               0, stream, a);
        else
            hipLaunchKernelGGL((forward_kernel<TYPE, kThreads, false>), dim3(grid), dim3(kThreads),
                               0, stream, a);
    });
    if (cut.splits > 1)
        for_rows(a, 1, 1, [&](unsigned grid) {
            hipLaunchKernelGGL(join_kernel<TYPE>, dim3(grid), dim3(64), 0, stream, a);
        });
}

template <int TYPE>
void backward_typed(const LogProbsArgs &args, hipStream_t stream) {
    GradArgs a{args.x,         args.dx,         args.targets,    args.lse, args.entropies,
               args.dlog_probs, args.dentropies, args.rows,      0,        args.vocab, 0};
    const uint32_t wave = 64 * 8 * kBatch;
    a.per_row = (a.vocab + wave - 1) / wave;
    // whole rows a launch, four waves to a workgroup
    for_rows(a, a.per_row, kThreads / 64, [&](unsigned grid) {
        if (args.dentropies)
            hipLaunchKernelGGL((backward_kernel<TYPE, true>), dim3(grid), dim3(kThreads), 0, stream,
                               a);
        else
            hipLaunchKernelGGL((backward_kernel<TYPE, false>), dim3(grid), dim3(kThreads), 0,
                               stream, a);
    });
}

template <int TYPE, uint32_t THREADS, uint32_t C>
void launch_train(const LogProbsArgs &args, hipStream_t stream) {
    TrainArgs a{row_args(args, {1, args.vocab}), args.dx, args.dlog_probs, args.dentropies};
    constexpr uint32_t kGroup = THREADS < kThreads ? kThreads : THREADS;
    for_rows(a.f, 1, kGroup / THREADS, [&](unsigned grid) {
        if (args.entropies)
            hipLaunchKernelGGL((train_kernel<TYPE, THREADS, C, true>), dim3(grid), dim3(kGroup), 0,
                               stream, a);
        else
            hipLaunchKernelGGL((train_kernel<TYPE, THREADS, C, false>), dim3(grid), dim3(kGroup), 0,
                               stream, a);
    });
}

// Rows that fit a workgroup's registers are read once; longer ones take the two
// passes, and so do rows that are few and long, which these cut into slices.
constexpr uint32_t kMostTrain = 1024 * 8 * 8;
bool one_pass(size_t, uint32_t vocab) { return vocab <= kMostTrain; }

template <int TYPE>
void train_typed(const LogProbsArgs &args, hipStream_t stream) {
    if (args.vocab <= 64 * 8 * 2)
        launch_train<TYPE, 64, 2>(args, stream);
    else if (args.vocab <= 64 * 8 * 4)
        launch_train<TYPE, 64, 4>(args, stream);
    else if (args.vocab <= 256 * 8 * 4)
        launch_train<TYPE, 256, 4>(args, stream);
    else if (args.vocab <= 256 * 8 * 8)
        launch_train<TYPE, 256, 8>(args, stream);
    else if (args.vocab <= 1024 * 8 * 4)
        launch_train<TYPE, 1024, 4>(args, stream);
    else
        launch_train<TYPE, 1024, 8>(args, stream);
}

}  // namespace

size_t log_probs_workspace(size_t rows, size_t vocab, uint32_t top) {
    if (!rows || !vocab)
        return 0;
    const Cut cut = cut_of(rows, (uint32_t)vocab, top);
    size_t bytes = 0;
    if (cut.splits > 1 || top)
        bytes = (rows * cut.splits * sizeof(Sums) + 15) / 16 * 16 +
                rows * cut.splits * top * sizeof(Key);
    return bytes;
}

hipError_t launch_log_probs_forward(const LogProbsArgs &a, int type, hipStream_t stream) {
    if (type == kBf16)
        forward_typed<kBf16>(a, stream);
    else
        forward_typed<kF32>(a, stream);
    return hipGetLastError();
}

hipError_t launch_log_probs_backward(const LogProbsArgs &a, int type, hipStream_t stream) {
    if (type == kBf16)
        backward_typed<kBf16>(a, stream);
    else
        backward_typed<kF32>(a, stream);
    return hipGetLastError();
}

hipError_t launch_log_probs_train(const LogProbsArgs &a, int type, hipStream_t stream) {
    if (!one_pass(a.rows, a.vocab)) {
        const hipError_t e = launch_log_probs_forward(a, type, stream);
        return e == hipSuccess ? launch_log_probs_backward(a, type, stream) : e;
    }
    if (type == kBf16)
        train_typed<kBf16>(a, stream);
    else
        train_typed<kF32>(a, stream);
    return hipGetLastError();
}

}  // namespace zpp
