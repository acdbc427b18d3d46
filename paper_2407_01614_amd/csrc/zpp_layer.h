// Internal launchers of the layer operators (layer norm, GELU, checkpoints in
// 8 bits, weight gradient).  Arguments are already validated; each launcher
// only enqueues its kernels on `stream` and returns the launch error.
#pragma once

#include <hip/hip_runtime_api.h>
#include <stddef.h>
#include <stdint.h>

namespace zpp {

// Elements of a checkpoint's block: one power of two as their scale.
constexpr uint32_t kActBlock = 64;
// Element types, the values of zpp_type.
constexpr int kBf16 = 0, kF32 = 1, kI8 = 2;

constexpr uint32_t kCus = 256;

// A matrix argument of a kernel; data == nullptr: not given.
struct Mat {
    void *data;
    uint8_t *exps;
    size_t stride;
};

struct NormForwardArgs {
    Mat x, residual, y, total, saved;
    const void *gamma, *beta;
    float *mean, *rstd;
    size_t rows;
    uint32_t cols;
    int param_type;
    float eps;
};

struct NormBackwardArgs {
    Mat dy, x, dresidual, dx, y;
    const void *gamma, *beta;
    const float *mean, *rstd;
    float *dgamma, *dbeta;
    float *partials;  // the workspace
    size_t rows;
    uint32_t cols;
    int param_type;
    int accumulate;
};

hipError_t launch_norm_forward(const NormForwardArgs &a, int type, hipStream_t stream);
size_t norm_backward_workspace(size_t rows, size_t cols);
hipError_t launch_norm_backward(const NormBackwardArgs &a, int type, int x_type,
                                hipStream_t stream);

hipError_t launch_checkpoint_save(const Mat &x, const Mat &saved, int type, size_t rows,
                                  size_t cols, hipStream_t stream);
hipError_t launch_checkpoint_load(const Mat &saved, const Mat &out, int type, size_t rows,
                                  size_t cols, hipStream_t stream);
hipError_t launch_gelu_forward(const Mat &u, const Mat &a, const Mat &saved, int type, size_t rows,
                               size_t cols, hipStream_t stream);
hipError_t launch_gelu_backward(const Mat &da, const Mat &u, const Mat &du, const Mat &a, int type,
                                int u_type, size_t rows, size_t cols, hipStream_t stream);

size_t weight_grad_workspace(size_t rows, size_t n, size_t k);
hipError_t launch_weight_grad(const Mat &dy, const Mat &x, int x_type, size_t rows, size_t n,
                              size_t k, const Mat &dw, int accumulate, void *workspace,
                              hipStream_t stream);

}  // namespace zpp
