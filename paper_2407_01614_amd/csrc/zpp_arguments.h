// The arguments of the layer and token operators' C entry points: checks of each,
// outputs held against all others, and the order of waits, launch and record.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "zpp.h"
#include "zpp_abi.h"
#include "zpp_layer.h"

namespace zpp {

// Sizes whose byte offsets cannot overflow a size_t.
constexpr size_t kMostElems = SIZE_MAX / 32;
constexpr size_t kMostCols = (size_t)1 << 31;  // exclusive; column indices are 32 bits

inline size_t type_size(int32_t type) { return type == ZPP_F32 ? 4 : type == ZPP_BF16 ? 2 : 1; }

// The memory of one argument: `rows` pieces of `bytes`, `stride` apart.
struct Range {
    const void *p;
    size_t rows, bytes, stride;
};

// Do the two share a byte?  Pieces the same distance apart, as column ranges of
// one wider matrix are, may lie between each other's.
inline bool share(const Range &a, const Range &b) {
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
            const size_t blocks = (cols + kActBlock - 1) / kActBlock;
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
inline unsigned plain_type(const zpp_matrix *m) {
    return m && m->type == ZPP_BF16 ? kBf : m && m->type == ZPP_F32 ? kFl : 0;
}

inline bool valid_param(int32_t type) { return type == ZPP_BF16 || type == ZPP_F32; }

// Waits, launches where there is work, records.
template <class F>
inline zpp_status run(hipStream_t stream, hipEvent_t wait_before, hipEvent_t done_after, bool work,
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

}  // namespace zpp
