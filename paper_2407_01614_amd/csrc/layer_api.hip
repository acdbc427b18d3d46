// C ABI of the layer operators (declared in include/zpp.h): argument checks,
// stream ordering with events, and dispatch to the kernels.
#include <math.h>
#include <stdint.h>

#include "zpp.h"
#include "zpp_abi.h"
#include "zpp_layer.h"

namespace {

using zpp::aligned;
using zpp::hip_fail;
using zpp::Mat;
using zpp::record;
using zpp::wait_on;

// Sizes whose byte offsets cannot overflow a size_t.
constexpr size_t kMostElems = SIZE_MAX / 32;
constexpr size_t kMostCols = (size_t)1 << 31;      // exclusive; column indices are 32 bits
constexpr size_t kMostNormCols = (size_t)1 << 26;  // exclusive; the join's grid

size_t type_size(int32_t type) { return type == ZPP_F32 ? 4 : type == ZPP_BF16 ? 2 : 1; }

// The memory of one argument: `rows` pieces of `bytes`, `stride` apart.
struct Range {
    const void *p;
    size_t rows, bytes, stride;
};

// Do the two share a byte?  Pieces the same distance apart, as column ranges of
// one wider matrix are, may lie between each other's.
bool share(const Range &a, const Range &b) {
    if (!a.p || !b.p || !a.rows || !b.rows || !a.bytes || !b.bytes)
        return false;
    const uintptr_t a0 = (uintptr_t)a.p, b0 = (uintptr_t)b.p;
    const uintptr_t a1 = a0 + (a.rows - 1) * a.stride + a.bytes;
    const uintptr_t b1 = b0 + (b.rows - 1) * b.stride + b.bytes;
    if (a0 >= b1 || b0 >= a1)
        return false;
    if (a.stride != b.stride || a.stride == 0)
        return true;
    // where b's pieces start within a's stride
    const size_t d = b0 >= a0 ? (b0 - a0) % a.stride : (a.stride - (a0 - b0) % a.stride) % a.stride;
    return d < a.bytes || d + b.bytes > a.stride;
}

// The arguments of one call: checks each as it is added, then outputs against
// all.
class Arguments {
  public:
    Arguments(size_t rows, size_t cols) : rows_(rows), cols_(cols) {
        if (cols >= kMostCols || (cols && rows > kMostElems / cols))
            status_ = ZPP_EINVAL;
    }

    // A matrix of `cols` columns (0: the call's) with one of the types of the
    // mask.  `needed`: NULL is an error.
    Mat matrix(const zpp_matrix *m, unsigned types, bool needed, bool output, size_t cols) {
        Mat none = {nullptr, nullptr, 0};
        if (!m) {
            if (needed)
                fail(ZPP_EINVAL);
            return none;
        }
        if (m->type < ZPP_BF16 || m->type > ZPP_I8 || !((types >> m->type) & 1u)) {
            fail(ZPP_EINVAL);
            return none;
        }
        if (rows_ == 0 || cols == 0)
            return none;
        if (!m->data || (m->type == ZPP_I8 && !m->exps) ||
            (rows_ > 1 && (m->stride < cols || m->stride > kMostElems / rows_))) {
            fail(ZPP_EINVAL);
            return none;
        }
        const size_t size = type_size(m->type);
        if (!aligned(m->data, size))
            fail(ZPP_EALIGN);
        const size_t stride = rows_ > 1 ? m->stride : cols;
        add({m->data, rows_, cols * size, stride * size}, output);
        if (m->type == ZPP_I8) {
            const size_t blocks = (cols + zpp::kActBlock - 1) / zpp::kActBlock;
            add({m->exps, 1, rows_ * blocks, 0}, output);
        }
        return {m->data, m->type == ZPP_I8 ? m->exps : nullptr, stride};
    }
    Mat matrix(const zpp_matrix *m, unsigned types, bool needed, bool output) {
        return matrix(m, types, needed, output, cols_);
    }

    void vector(const void *p, size_t elems, size_t size, bool needed, bool output) {
        if (!elems)
            return;
        if (!p) {
            if (needed)
                fail(ZPP_EINVAL);
            return;
        }
        if (!aligned(p, size))
            fail(ZPP_EALIGN);
        add({p, 1, elems * size, 0}, output);
    }

    void workspace(const void *p, size_t bytes, size_t needed) {
        if (!needed)
            return;
        if (!p || bytes < needed) {
            fail(ZPP_EINVAL);
            return;
        }
        if (!aligned(p, 16))
            fail(ZPP_EALIGN);
        add({p, 1, needed, 0}, true);
    }

    void fail(zpp_status s) {
        // the first kind in the order EINVAL, EALIGN, EOVERLAP
        if (status_ == ZPP_OK || s < status_)
            status_ = s;
    }

    zpp_status check() const {
        if (status_ != ZPP_OK)
            return status_;
        for (int x = 0; x < count_; ++x)
            for (int y = 0; y < count_; ++y)
                if (x != y && output_[x] && share(ranges_[x], ranges_[y]))
                    return ZPP_EOVERLAP;
        return ZPP_OK;
    }

    // Another list's arguments and failures as well.
    void take(const Arguments &other) {
        if (other.status_ != ZPP_OK)
            fail(other.status_);
        for (int x = 0; x < other.count_; ++x)
            add(other.ranges_[x], other.output_[x]);
    }

    bool empty() const { return rows_ == 0 || cols_ == 0; }

  private:
    void add(const Range &r, bool output) {
        ranges_[count_] = r;
        output_[count_++] = output;
    }
    size_t rows_, cols_;
    zpp_status status_ = ZPP_OK;
    int count_ = 0;
    Range ranges_[20];
    bool output_[20] = {};
};

constexpr unsigned kBf = 1u << ZPP_BF16, kFl = 1u << ZPP_F32, kCode = 1u << ZPP_I8;

// The type that a call's plain matrices share, as a mask (0: not a plain type).
unsigned plain_type(const zpp_matrix *m) {
    return m && m->type == ZPP_BF16 ? kBf : m && m->type == ZPP_F32 ? kFl : 0;
}

bool valid_param(int32_t type) { return type == ZPP_BF16 || type == ZPP_F32; }

// Waits, launches where there is work, records.
template <class F>
zpp_status run(hipStream_t stream, hipEvent_t wait_before, hipEvent_t done_after, bool work,
               F &&launch) {
    const zpp_status st = wait_on(stream, wait_before);
    if (st != ZPP_OK)
        return st;
    if (work) {
        const hipError_t e = launch();
        if (e != hipSuccess)
            return hip_fail(e);
    }
    return record(stream, done_after);
}

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
