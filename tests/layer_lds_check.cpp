// Every launch of the layer operators that takes more than 64 KB of LDS has asked
// for it, on the device that it runs on: hipFuncSetAttribute for that kernel with
// as much.  The library's host code as built, with the HIP calls that it makes on
// the way to a launch answered here (a program's own definitions come before a
// library's); nothing is launched, addresses are made up and no device is needed.
// Test infrastructure of tests/test_layer_lds.py.
#include <hip/hip_runtime_api.h>
#include <stdio.h>

#include <map>
#include <utility>

#include "zpp.h"

static int device = 0, launches = 0, large = 0, failures = 0;
static const char *now = "";
static size_t now_rows, now_cols;
static std::map<std::pair<const void *, int>, int> asked;
static dim3 next_grid, next_block;
static size_t next_lds;
static hipStream_t next_stream;

// LDS that kernels declare beside what a launch asks for: the sums of a row's waves
// (256 bytes).  The joins' 4 KB stand alone.
static const size_t kMostStatic = 256, kPlain = 64 << 10, kMost = 160 << 10;

extern "C" {
hipError_t hipGetDevice(int *d) {
    *d = device;
    return hipSuccess;
}
hipError_t hipGetLastError(void) { return hipSuccess; }
hipError_t hipFuncSetAttribute(const void *kernel, hipFuncAttribute what, int value) {
    if (what == hipFuncAttributeMaxDynamicSharedMemorySize)
        asked[{kernel, device}] = value;
    return hipSuccess;
}
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t stream) {
    next_grid = grid;
    next_block = block;
    next_lds = lds;
    next_stream = stream;
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *lds, hipStream_t *stream) {
    *grid = next_grid;
    *block = next_block;
    *lds = next_lds;
    *stream = next_stream;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void *kernel, dim3, dim3, void **, size_t lds, hipStream_t) {
    ++launches;
    const auto found = asked.find({kernel, device});
    const size_t allowed = found == asked.end() ? 0 : (size_t)found->second;
    if (lds + kMostStatic > kPlain) {
        ++large;
        if (lds > allowed || lds + kMostStatic > kMost) {
            if (++failures <= 8)
                printf("%s, %zux%zu, device %d: %zu bytes of LDS where %zu are asked for\n", now,
                       now_rows, now_cols, device, lds, allowed);
        }
    }
    return hipSuccess;
}
}

static void *dev(unsigned k) { return (void *)(uintptr_t)((16ull << 30) + ((uint64_t)k << 30)); }
static zpp_matrix mat(unsigned k, int type, size_t stride) {
    return {dev(k), type == ZPP_I8 ? (uint8_t *)dev(k + 40) : nullptr, stride, type};
}
static void run(const char *what, size_t rows, size_t cols, zpp_status st) {
    if (st != ZPP_OK) {
        printf("%s, %zux%zu: status %d\n", what, rows, cols, (int)st);
        ++failures;
    }
}

static void norm(size_t rows, size_t cols, int type, int x_type) {
    now_rows = rows;
    now_cols = cols;
    const zpp_matrix x = mat(0, type, cols), r = mat(1, type, cols), y = mat(2, type, cols),
                     t = mat(3, type, cols), s = mat(4, ZPP_I8, cols), from = mat(5, x_type, cols);
    float *const f = (float *)dev(8);
    now = "norm forward";
    run(now, rows, cols,
        zpp_layer_norm_forward(&x, &r, dev(9), dev(10), ZPP_F32, rows, cols, 1e-5f, &y, &t, &s, f,
                               (float *)dev(11), nullptr, nullptr, nullptr));
    for (int again = 0; again < 2; ++again) {
        now = again ? "norm backward with y" : "norm backward";
        run(now, rows, cols,
            zpp_layer_norm_backward(&x, &from, dev(9), dev(10), ZPP_F32, f, (float *)dev(11), &r,
                                    rows, cols, &y, again ? &t : nullptr, (float *)dev(12),
                                    (float *)dev(13), 0, dev(14),
                                    zpp_layer_norm_backward_workspace(rows, cols), nullptr, nullptr,
                                    nullptr));
    }
}

int main() {
    // the second device's kernels are asked for as well
    for (device = 0; device < 2; ++device) {
        const size_t step = device ? 513 : 61;
        for (int type : {ZPP_BF16, ZPP_F32})
            for (int x_type : {type, (int)ZPP_I8}) {
                for (size_t cols = 1; cols < 17000; cols += step)
                    norm(300, cols, type, x_type);
                for (size_t cols : {7680, 7681, 8184, 8191, 8192, 8193, 16383, 16384, 16385})
                    norm(5, cols, type, x_type);
            }
        for (int x_type : {ZPP_BF16, ZPP_I8})
            for (size_t n : {70, 300, 4544, 8192})
                for (size_t rows : {1, 100, 4096}) {
                    now = "weight gradient";
                    now_rows = rows;
                    now_cols = n;
                    const zpp_matrix dy = mat(0, ZPP_BF16, n), x = mat(1, x_type, n),
                                     dw = mat(2, ZPP_F32, n);
                    run(now, rows, n,
                        zpp_weight_grad(&dy, &x, rows, n, n, &dw, 0, dev(14),
                                        zpp_weight_grad_workspace(rows, n, n), nullptr, nullptr,
                                        nullptr));
                }
    }
    printf("%d launches, %d with more than 64 KB of LDS, %d failures\n", launches, large, failures);
    return failures || !large ? 1 : 0;
}
