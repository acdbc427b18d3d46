// Weight gradient of a linear layer, dw[i][j] (+)= sum_t dy[t][i] x[t][j] (zpp.h),
// on the matrix cores.
//
// Both operands lie along features while the sum runs over tokens, and an MFMA
// lane wants eight tokens of one feature.  So each lane fetches 4 tokens by 8
// features, turns them in registers (byte permutes pair the tokens; a
// checkpoint's codes are scaled on the way, exactly) and lays them into LDS
// feature by feature, from where a lane reads its 16 bytes at once.
#include "zpp_act8.h"

namespace zpp {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr uint32_t kStep = 64;  // tokens a turn

struct WeightGradArgs {
    Mat dy, x;
    float *out;         // dw, or the workspace's [splits][n][k]
    size_t out_stride;  // between rows
    size_t out_split;   // between splits
    size_t rows, split_rows;
    uint32_t n, k, tiles_k;
    int accumulate;
};

// 4 tokens by 8 features as fetched.
template <int TYPE>
struct Piece {
    Chunk<TYPE> t[4];
};

template <int TYPE>
__device__ __forceinline__ void fetch(Piece<TYPE> &p, const Mat &m, size_t row, size_t rows,
                                      uint32_t col, uint32_t cols, uint32_t blocks) {
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
        p.t[i] = Chunk<TYPE>{};
        if (row + i < rows && col < cols)
            p.t[i] = load_chunk<TYPE>(m, row + i, col, cols - col, blocks);
    }
}

// The piece with its tokens side by side: word pair e holds feature e's four
// tokens as bf16.
__device__ __forceinline__ void turn(const Piece<kBf16> &p, u32x2 (&w)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t sel = e % 2 ? 0x07060302u : 0x05040100u;
        w[e].x = __builtin_amdgcn_perm(p.t[1].w[e / 2], p.t[0].w[e / 2], sel);
        w[e].y = __builtin_amdgcn_perm(p.t[3].w[e / 2], p.t[2].w[e / 2], sel);
    }
}
__device__ __forceinline__ void turn(const Piece<kI8> &p, u32x2 (&w)[8]) {
    float x[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        chunk_values(p.t[i], x[i]);
    // code * 2^e is a bf16 number: its high half is all of it
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        w[e].x = __builtin_amdgcn_perm(__float_as_uint(x[1][e]), __float_as_uint(x[0][e]),
                                       0x07060302u);
        w[e].y = __builtin_amdgcn_perm(__float_as_uint(x[3][e]), __float_as_uint(x[2][e]),
                                       0x07060302u);
    }
}

// LDS holds a tile as [feature][64 tokens] bf16, 128 bytes a feature, in 16-byte
// units of 8 tokens.  Unit u of feature f lies at place u ^ f % 8 ^ f / 8 % 8:
// lanes that read one unit of 8 features in a row, and lanes that write one
// feature of 8 neighbouring pieces, meet 8 different places.
__device__ __forceinline__ uint32_t unit_at(uint32_t f, uint32_t u) {
    return f * (kStep * 2) + ((u ^ f ^ (f >> 3)) & 7) * 16;
}

template <int X, int TILE, int WAVES_N, int WAVES_K>
__global__ __launch_bounds__(WAVES_N *WAVES_K *kWave) void weight_grad_kernel(WeightGradArgs a) {
    constexpr int MN = TILE / WAVES_N / 32, MK = TILE / WAVES_K / 32;
    constexpr uint32_t kChunks = TILE / 8;
    static_assert(WAVES_N * WAVES_K * kWave == kChunks * kStep / 4, "one piece a lane");
    __shared__ __attribute__((aligned(16))) uint8_t lds[2][TILE * kStep * 2];
    const uint32_t tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    const uint32_t tile_n = blockIdx.x / a.tiles_k, tile_k = blockIdx.x - tile_n * a.tiles_k;
    const uint32_t n0 = tile_n * TILE, k0 = tile_k * TILE;
    const uint32_t blocks = (a.k + kActBlock - 1) / kActBlock;
    const size_t begin = (size_t)blockIdx.y * a.split_rows;
    const size_t end = begin + a.split_rows < a.rows ? begin + a.split_rows : a.rows;

    // the lane's piece: neighbouring lanes take the two halves of a unit
    const uint32_t chunk = tid / 2 % kChunks, group = tid % 2 + 2 * (tid / (2 * kChunks));
    const uint32_t wn = wave / WAVES_K * (TILE / WAVES_N), wk = wave % WAVES_K * (TILE / WAVES_K);

    f32x16 acc[MN][MK];
#pragma unroll
    for (int i = 0; i < MN; ++i)
#pragma unroll
        for (int j = 0; j < MK; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                acc[i][j][e] = 0.0f;

    Piece<kBf16> pd;
    Piece<X> px;
    fetch(pd, a.dy, begin + group * 4, end, n0 + chunk * 8, a.n, 0);
    fetch(px, a.x, begin + group * 4, end, k0 + chunk * 8, a.k, blocks);
    for (size_t row = begin; row < end; row += kStep) {
        u32x2 w[8];
        __syncthreads();
        turn(pd, w);
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e)
            *reinterpret_cast<u32x2 *>(&lds[0][unit_at(chunk * 8 + e, group / 2) + group % 2 * 8]) =
                w[e];
        turn(px, w);
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e)
            *reinterpret_cast<u32x2 *>(&lds[1][unit_at(chunk * 8 + e, group / 2) + group % 2 * 8]) =
                w[e];
        __syncthreads();
        if (row + kStep < end) {
            fetch(pd, a.dy, row + kStep + group * 4, end, n0 + chunk * 8, a.n, 0);
            fetch(px, a.x, row + kStep + group * 4, end, k0 + chunk * 8, a.k, blocks);
        }
#pragma unroll
        for (uint32_t kk = 0; kk < kStep / 16; ++kk) {
            bf16x8 fd[MN], fx[MK];
            const uint32_t unit = kk * 2 + lane / 32;
#pragma unroll
            for (int i = 0; i < MN; ++i)
                fd[i] = *reinterpret_cast<const bf16x8 *>(
                    &lds[0][unit_at(wn + i * 32 + lane % 32, unit)]);
#pragma unroll
            for (int j = 0; j < MK; ++j)
                fx[j] = *reinterpret_cast<const bf16x8 *>(
                    &lds[1][unit_at(wk + j * 32 + lane % 32, unit)]);
#pragma unroll
            for (int i = 0; i < MN; ++i)
#pragma unroll
                for (int j = 0; j < MK; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fd[i], fx[j], acc[i][j], 0,
                                                                        0, 0);
        }
    }

    // lane l holds column l % 32 and, in register r, row 8 (r / 4) + 4 (l / 32) + r % 4
    float *out = a.out + (size_t)blockIdx.y * a.out_split;
#pragma unroll
    for (int j = 0; j < MK; ++j) {
        const uint32_t col = k0 + wk + j * 32 + lane % 32;
        if (col >= a.k)
            continue;
#pragma unroll
        for (int i = 0; i < MN; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const uint32_t row = n0 + wn + i * 32 + 8 * (r / 4) + 4 * (lane / 32) + r % 4;
                if (row < a.n) {
                    float *p = out + (size_t)row * a.out_stride + col;
                    *p = a.accumulate ? *p + acc[i][j][r] : acc[i][j][r];
                }
            }
    }
}

// dw (+)= the splits' sums, in order; also writes zeros where there is nothing
// to sum.
__global__ __launch_bounds__(256) void weight_grad_join(const float *parts, uint32_t splits,
                                                        uint32_t n, uint32_t k, float *dw,
                                                        size_t stride, int accumulate) {
    const size_t total = (size_t)n * k;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < total;
         i += (size_t)gridDim.x * 256) {
        float sum = 0.0f;
        for (uint32_t s = 0; s < splits; ++s)
            sum += parts[s * total + i];
        float *p = dw + i / k * stride + i % k;
        *p = accumulate ? *p + sum : sum;
    }
}

struct GradShape {
    uint32_t tile, splits;
    size_t split_rows;
};

GradShape grad_shape(size_t rows, size_t n, size_t k) {
    (void)n;
    (void)k;
    return {128, 1, (rows + kStep - 1) / kStep * kStep};
}

}  // namespace

size_t weight_grad_workspace(size_t rows, size_t n, size_t k) {
    const GradShape s = grad_shape(rows, n, k);
    return s.splits > 1 ? s.splits * n * k * sizeof(float) : 0;
}

hipError_t launch_weight_grad(const Mat &dy, const Mat &x, int x_type, size_t rows, size_t n,
                              size_t k, const Mat &dw, int accumulate, void *workspace,
                              hipStream_t stream) {
    const size_t total = n * k;
    const unsigned join_grid = (unsigned)(total / 256 < 8 * kCus ? total / 256 + 1 : 8 * kCus);
    float *out = reinterpret_cast<float *>(dw.data);
    if (rows == 0) {
        if (!accumulate)
            hipLaunchKernelGGL(weight_grad_join, dim3(join_grid), dim3(256), 0, stream, nullptr, 0u,
                               (uint32_t)n, (uint32_t)k, out, dw.stride, 0);
        return hipGetLastError();
    }
    const GradShape s = grad_shape(rows, n, k);
    WeightGradArgs a;
    a.dy = dy;
    a.x = x;
    a.out = s.splits > 1 ? reinterpret_cast<float *>(workspace) : out;
    a.out_stride = s.splits > 1 ? k : dw.stride;
    a.out_split = total;
    a.rows = rows;
    a.split_rows = s.split_rows;
    a.n = (uint32_t)n;
    a.k = (uint32_t)k;
    a.tiles_k = (uint32_t)((k + s.tile - 1) / s.tile);
    a.accumulate = s.splits > 1 ? 0 : accumulate;
    const dim3 grid((unsigned)((n + s.tile - 1) / s.tile * a.tiles_k), s.splits);
    if (x_type == kI8)
        hipLaunchKernelGGL((weight_grad_kernel<kI8, 128, 2, 2>), grid, dim3(256), 0, stream, a);
    else
        hipLaunchKernelGGL((weight_grad_kernel<kBf16, 128, 2, 2>), grid, dim3(256), 0, stream, a);
    if (s.splits > 1)
        hipLaunchKernelGGL(weight_grad_join, dim3(join_grid), dim3(256), 0, stream,
                           reinterpret_cast<const float *>(workspace), s.splits, (uint32_t)n,
                           (uint32_t)k, out, dw.stride, accumulate);
    return hipGetLastError();
}

}  // namespace zpp
