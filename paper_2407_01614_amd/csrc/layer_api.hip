// C ABI of the layer operators (declared in include/zpp.h): argument checks,
// stream ordering with events, and dispatch to the kernels.
#include <math.h>
#include <stdint.h>

#include "zpp.h"
#include "zpp_arguments.h"

namespace {

using zpp::Arguments;
using zpp::kBf;
using zpp::kCode;
using zpp::kFl;
using zpp::kMostCols;
using zpp::kMostElems;
using zpp::Mat;
using zpp::plain_type;
using zpp::run;
using zpp::type_size;
using zpp::valid_param;

constexpr size_t kMostNormCols = (size_t)1 << 26;  // exclusive; the join's grid

}  // namespace

extern "C" {

ZPP_API zpp_status zpp_checkpoint_save(const zpp_matrix *x, const zpp_matrix *saved, size_t rows,
                                       size_t cols, hipStream_t stream, hipEvent_t wait_before,
                                       hipEvent_t done_after) {
    Arguments args(rows, cols);
    const Mat mx = args.matrix(x, kBf | kFl, true, false);
    const Mat ms = args.matrix(saved, kCode, true, true);
    const zpp_status st = args.check();
    if (st != ZPP_OK)
        return st;
    return run(stream, wait_before, done_after, !args.empty(), [&] {
        return zpp::launch_checkpoint_save(mx, ms, x->type, rows, cols, stream);
    });
}

ZPP_API zpp_status zpp_checkpoint_load(const zpp_matrix *saved, const zpp_matrix *out, size_t rows,
                                       size_t cols, hipStream_t stream, hipEvent_t wait_before,
                                       hipEvent_t done_after) {
    Arguments args(rows, cols);
    const Mat ms = args.matrix(saved, kCode, true, false);
    const Mat mo = args.matrix(out, kBf | kFl, true, true);
    const zpp_status st = args.check();
    if (st != ZPP_OK)
        return st;
    return run(stream, wait_before, done_after, !args.empty(), [&] {
        return zpp::launch_checkpoint_load(ms, mo, out->type, rows, cols, stream);
    });
}

ZPP_API zpp_status zpp_layer_norm_forward(const zpp_matrix *x, const zpp_matrix *residual,
                                          const void *gamma, const void *beta, int32_t param_type,
                                          size_t rows, size_t cols, float eps, const zpp_matrix *y,
                                          const zpp_matrix *total, const zpp_matrix *saved,
                                          float *mean, float *rstd, hipStream_t stream,
                                          hipEvent_t wait_before, hipEvent_t done_after) {
    Arguments args(rows, cols);
    if (!isfinite(eps) || eps < 0.0f || !valid_param(param_type) || !residual != !total ||
        cols >= kMostNormCols)
        args.fail(ZPP_EINVAL);
    const unsigned type = plain_type(x);
    zpp::NormForwardArgs a;
    a.x = args.matrix(x, type, true, false);
    a.residual = args.matrix(residual, type, false, false);
    a.y = args.matrix(y, type, true, true);
    a.total = args.matrix(total, type, false, true);
    a.saved = args.matrix(saved, kCode, false, true);
    if (!args.empty()) {
        args.vector(gamma, cols, type_size(param_type), true, false);
        args.vector(beta, cols, type_size(param_type), false, false);
        args.vector(mean, rows, 4, false, true);
        args.vector(rstd, rows, 4, false, true);
    }
    const zpp_status st = args.check();
    if (st != ZPP_OK)
        return st;
    a.gamma = gamma;
    a.beta = beta;
    a.mean = mean;
    a.rstd = rstd;
    a.rows = rows;
    a.cols = (uint32_t)cols;
    a.param_type = param_type;
    a.eps = eps;
    return run(stream, wait_before, done_after, !args.empty(),
               [&] { return zpp::launch_norm_forward(a, x->type, stream); });
}

ZPP_API size_t zpp_layer_norm_backward_workspace(size_t rows, size_t cols) {
    if (cols >= kMostNormCols || (cols && rows > kMostElems / cols))
        return 0;
    return zpp::norm_backward_workspace(rows, cols);
}

ZPP_API zpp_status zpp_layer_norm_backward(const zpp_matrix *dy, const zpp_matrix *x,
                                           const void *gamma, const void *beta, int32_t param_type,
                                           const float *mean, const float *rstd,
                                           const zpp_matrix *dresidual, size_t rows, size_t cols,
                                           const zpp_matrix *dx, const zpp_matrix *y,
                                           float *dgamma, float *dbeta, int32_t accumulate,
                                           void *workspace, size_t workspace_bytes,
                                           hipStream_t stream, hipEvent_t wait_before,
                                           hipEvent_t done_after) {
    Arguments args(rows, cols);
    if (!valid_param(param_type) || cols >= kMostNormCols)
        args.fail(ZPP_EINVAL);
    const unsigned type = plain_type(dy);
    zpp::NormBackwardArgs a;
    a.dy = args.matrix(dy, type, true, false);
    a.x = args.matrix(x, type | kCode, true, false);
    a.dresidual = args.matrix(dresidual, type, false, false);
    a.dx = args.matrix(dx, type, true, true);
    a.y = args.matrix(y, type, false, true);
    if (!args.empty()) {
        args.vector(gamma, cols, type_size(param_type), true, false);
        args.vector(beta, cols, type_size(param_type), false, false);
        args.vector(mean, rows, 4, true, false);
        args.vector(rstd, rows, 4, true, false);
    }
    args.vector(dgamma, cols, 4, false, true);
    args.vector(dbeta, cols, 4, false, true);
    args.workspace(workspace, workspace_bytes, zpp_layer_norm_backward_workspace(rows, cols));
    const zpp_status st = args.check();
    if (st != ZPP_OK)
        return st;
    a.gamma = gamma;
    a.beta = beta;
    a.mean = mean;
    a.rstd = rstd;
    a.dgamma = dgamma;
    a.dbeta = dbeta;
    a.partials = reinterpret_cast<float *>(workspace);
    a.rows = rows;
    a.cols = (uint32_t)cols;
    a.param_type = param_type;
    a.accumulate = accumulate;
    // without rows the weights' gradients are sums of nothing: zeros
    const bool work = cols && (rows || (!accumulate && (dgamma || dbeta)));
    return run(stream, wait_before, done_after, work, [&] {
        return zpp::launch_norm_backward(a, dy->type, x->type, stream);
    });
}

ZPP_API zpp_status zpp_gelu_forward(const zpp_matrix *u, size_t rows, size_t cols,
                                    const zpp_matrix *a, const zpp_matrix *saved,
                                    hipStream_t stream, hipEvent_t wait_before,
                                    hipEvent_t done_after) {
    Arguments args(rows, cols);
    const unsigned type = plain_type(u);
    const Mat mu = args.matrix(u, type, true, false);
    const Mat ma = args.matrix(a, type, true, true);
    const Mat ms = args.matrix(saved, kCode, false, true);
    const zpp_status st = args.check();
    if (st != ZPP_OK)
        return st;
    return run(stream, wait_before, done_after, !args.empty(), [&] {
        return zpp::launch_gelu_forward(mu, ma, ms, u->type, rows, cols, stream);
    });
}

ZPP_API zpp_status zpp_gelu_backward(const zpp_matrix *da, const zpp_matrix *u, size_t rows,
                                     size_t cols, const zpp_matrix *du, const zpp_matrix *a,
                                     hipStream_t stream, hipEvent_t wait_before,
                                     hipEvent_t done_after) {
    Arguments args(rows, cols);
    const unsigned type = plain_type(da);
    const Mat md = args.matrix(da, type, true, false);
    const Mat mu = args.matrix(u, type | kCode, true, false);
    const Mat mo = args.matrix(du, type, true, true);
    const Mat ma = args.matrix(a, type, false, true);
    const zpp_status st = args.check();
    if (st != ZPP_OK)
        return st;
    return run(stream, wait_before, done_after, !args.empty(), [&] {
        return zpp::launch_gelu_backward(md, mu, mo, ma, da->type, u->type, rows, cols, stream);
    });
}

ZPP_API size_t zpp_weight_grad_workspace(size_t rows, size_t n, size_t k) {
    if (rows >= kMostCols || n >= kMostCols || k >= kMostCols || rows == 0 || n == 0 || k == 0)
        return 0;
    return zpp::weight_grad_workspace(rows, n, k);
}

ZPP_API zpp_status zpp_weight_grad(const zpp_matrix *dy, const zpp_matrix *x, size_t rows,
                                   size_t n, size_t k, const zpp_matrix *dw, int32_t accumulate,
                                   void *workspace, size_t workspace_bytes, hipStream_t stream,
                                   hipEvent_t wait_before, hipEvent_t done_after) {
    if (rows >= kMostCols || n >= kMostCols || k >= kMostCols)
        return ZPP_EINVAL;
    Arguments tokens(rows, n > k ? n : k), weights(n, k);
    const Mat md = tokens.matrix(dy, kBf, true, false, n);
    const Mat mx = tokens.matrix(x, kBf | kCode, true, false, k);
    const Mat mw = weights.matrix(dw, kFl, true, true);
    // one list, so that outputs are held against all
    tokens.take(weights);
    tokens.workspace(workspace, workspace_bytes, zpp_weight_grad_workspace(rows, n, k));
    const zpp_status st = tokens.check();
    if (st != ZPP_OK)
        return st;
    const bool work = n && k && (rows || !accumulate);
    return run(stream, wait_before, done_after, work, [&] {
        return zpp::launch_weight_grad(md, mx, x->type, rows, n, k, mw, accumulate, workspace,
                                       stream);
    });
}

}  // extern "C"
