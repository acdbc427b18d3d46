// The layer operators' host code (csrc/layer_api.hip) under AddressSanitizer and
// UndefinedBehaviorSanitizer: every entry point with arguments that validation
// settles, with extreme sizes and addresses, and with good ones, which have to
// reach the launcher (a stand-in here that counts) with what they were given.
// Test infrastructure of tests/test_layers_abi.py; addresses are never
// dereferenced and no device is needed.
#include <stdio.h>

#include "zpp.h"
#include "zpp_layer.h"

static int launches = 0;
static zpp::NormForwardArgs seen_forward;
static zpp::NormBackwardArgs seen_backward;
static zpp::Mat seen[4];

namespace zpp {
hipError_t launch_norm_forward(const NormForwardArgs &a, int, hipStream_t) {
    seen_forward = a;
    ++launches;
    return hipSuccess;
}
size_t norm_backward_workspace(size_t, size_t cols) { return 8 * cols; }
hipError_t launch_norm_backward(const NormBackwardArgs &a, int, int, hipStream_t) {
    seen_backward = a;
    ++launches;
    return hipSuccess;
}
hipError_t launch_checkpoint_save(const Mat &x, const Mat &s, int, size_t, size_t, hipStream_t) {
    seen[0] = x;
    seen[1] = s;
    ++launches;
    return hipSuccess;
}
hipError_t launch_checkpoint_load(const Mat &, const Mat &, int, size_t, size_t, hipStream_t) {
    ++launches;
    return hipSuccess;
}
hipError_t launch_gelu_forward(const Mat &, const Mat &, const Mat &, int, size_t, size_t,
                               hipStream_t) {
    ++launches;
    return hipErrorInvalidConfiguration;
}
hipError_t launch_gelu_backward(const Mat &, const Mat &, const Mat &, const Mat &a, int, int,
                                size_t, size_t, hipStream_t) {
    seen[3] = a;
    ++launches;
    return hipSuccess;
}
size_t weight_grad_workspace(size_t, size_t, size_t) { return 64; }
hipError_t launch_weight_grad(const Mat &, const Mat &, int, size_t, size_t, size_t, const Mat &w,
                              int, void *, hipStream_t) {
    seen[2] = w;
    ++launches;
    return hipSuccess;
}
}  // namespace zpp

static int failures = 0;
#define EXPECT(cond)                                                  \
    do {                                                              \
        if (!(cond)) {                                                \
            printf("%s:%d: %s\n", __FILE__, __LINE__, #cond);         \
            ++failures;                                               \
        }                                                             \
    } while (0)

static void *dev(unsigned k, size_t off = 0) {
    return (void *)(uintptr_t)((16ull << 30) + ((uint64_t)k << 30) + off);
}
static zpp_matrix mat(unsigned k, int type, size_t stride, size_t off = 0) {
    return {dev(k, off), type == ZPP_I8 ? (uint8_t *)dev(k, 512u << 20) : nullptr, stride, type};
}

int main() {
    const size_t R = 7, C = 1001;
    const zpp_matrix x = mat(0, ZPP_BF16, 1100), s = mat(1, ZPP_I8, C), o = mat(2, ZPP_BF16, C);
    EXPECT(zpp_checkpoint_save(&x, &s, R, C, nullptr, nullptr, nullptr) == ZPP_OK);
    EXPECT(launches == 1 && seen[0].data == x.data && seen[0].stride == 1100 &&
           seen[1].exps == s.exps);
    EXPECT(zpp_checkpoint_load(&s, &o, R, C, nullptr, nullptr, nullptr) == ZPP_OK && launches == 2);
    // one row: its stride does not matter
    zpp_matrix one = mat(0, ZPP_BF16, 0);
    EXPECT(zpp_checkpoint_save(&one, &s, 1, C, nullptr, nullptr, nullptr) == ZPP_OK);
    EXPECT(launches == 3 && seen[0].stride == C);
    // a launch that fails is told
    EXPECT(zpp_gelu_forward(&x, R, C, &o, nullptr, nullptr, nullptr, nullptr) == ZPP_EHIP);
    EXPECT(zpp::launch_gelu_forward({}, {}, {}, 0, 0, 0, nullptr) == hipErrorInvalidConfiguration);
    launches = 0;
    // column ranges of one wide matrix beside each other
    const zpp_matrix left = mat(3, ZPP_BF16, 300), right = mat(3, ZPP_BF16, 300, 2 * 100),
                     last = mat(3, ZPP_BF16, 300, 2 * 200);
    EXPECT(zpp_gelu_backward(&left, &s, R, 100, &right, &last, nullptr, nullptr, nullptr) == ZPP_OK);
    EXPECT(launches == 1 && seen[3].data == last.data);
    EXPECT(zpp_gelu_backward(&left, &s, R, 101, &right, nullptr, nullptr, nullptr, nullptr) ==
           ZPP_EOVERLAP);
    // layer norm, everything given and as little as possible
    const zpp_matrix r = mat(4, ZPP_BF16, C), y = mat(5, ZPP_BF16, C), t = mat(6, ZPP_BF16, C);
    EXPECT(zpp_layer_norm_forward(&x, &r, dev(7), dev(8), ZPP_F32, R, C, 0.0f, &y, &t, &s,
                                  (float *)dev(9), (float *)dev(10), nullptr, nullptr,
                                  nullptr) == ZPP_OK);
    EXPECT(seen_forward.total.data == t.data && seen_forward.saved.exps == s.exps &&
           seen_forward.param_type == ZPP_F32 && seen_forward.cols == C);
    EXPECT(zpp_layer_norm_forward(&x, nullptr, dev(7), nullptr, ZPP_BF16, R, C, 1e-5f, &y, nullptr,
                                  nullptr, nullptr, nullptr, nullptr, nullptr, nullptr) == ZPP_OK);
    EXPECT(!seen_forward.residual.data && !seen_forward.total.data && !seen_forward.saved.data &&
           !seen_forward.mean && !seen_forward.beta);
    launches = 0;
    EXPECT(zpp_layer_norm_backward(&x, &s, dev(7), dev(8), ZPP_BF16, (float *)dev(9),
                                   (float *)dev(10), &r, R, C, &y, &t, (float *)dev(11),
                                   (float *)dev(12), 1, dev(13), 8 * C, nullptr, nullptr,
                                   nullptr) == ZPP_OK);
    EXPECT(launches == 1 && seen_backward.partials == dev(13) && seen_backward.accumulate == 1);
    // no rows: zeros are written, unless the sums are added to what is there
    EXPECT(zpp_layer_norm_backward(&x, &s, dev(7), nullptr, ZPP_BF16, nullptr, nullptr, nullptr, 0,
                                   C, &y, nullptr, (float *)dev(11), nullptr, 0, dev(13), 8 * C,
                                   nullptr, nullptr, nullptr) == ZPP_OK);
    EXPECT(launches == 2);
    EXPECT(zpp_layer_norm_backward(&x, &s, dev(7), nullptr, ZPP_BF16, nullptr, nullptr, nullptr, 0,
                                   C, &y, nullptr, (float *)dev(11), nullptr, 1, dev(13), 8 * C,
                                   nullptr, nullptr, nullptr) == ZPP_OK);
    EXPECT(launches == 2);
    const zpp_matrix w = mat(7, ZPP_F32, 70);
    EXPECT(zpp_weight_grad(&x, &s, R, 50, 60, &w, 0, dev(8), 64, nullptr, nullptr, nullptr) ==
           ZPP_OK);
    EXPECT(launches == 3 && seen[2].stride == 70);
    EXPECT(zpp_weight_grad(&x, &x, R, 50, 60, &w, 0, dev(8), 64, nullptr, nullptr, nullptr) ==
           ZPP_OK);
    EXPECT(zpp_weight_grad(&x, &s, 0, 50, 60, &w, 0, nullptr, 0, nullptr, nullptr, nullptr) ==
           ZPP_OK);
    EXPECT(launches == 5);
    EXPECT(zpp_weight_grad(&x, &s, R, 50, 60, &w, 0, dev(8), 63, nullptr, nullptr, nullptr) ==
           ZPP_EINVAL);
    // extreme sizes: no overflow on the way to the refusal
    const size_t huge[] = {(size_t)1 << 31, (size_t)1 << 62, SIZE_MAX, SIZE_MAX / 64};
    for (size_t a : huge)
        for (size_t b : huge) {
            zpp_matrix h = mat(0, ZPP_BF16, b);
            EXPECT(zpp_checkpoint_save(&h, &s, a, b, nullptr, nullptr, nullptr) == ZPP_EINVAL);
            EXPECT(zpp_gelu_forward(&h, 7, 5, &o, nullptr, nullptr, nullptr, nullptr) != ZPP_OK);
            EXPECT(zpp_weight_grad(&h, &s, a, b, 5, &w, 0, nullptr, 0, nullptr, nullptr, nullptr) ==
                   ZPP_EINVAL);
            EXPECT(zpp_layer_norm_backward_workspace(a, b) == 0);
            EXPECT(zpp_weight_grad_workspace(a, b, 3) == 0);
        }
    if (failures)
        return 1;
    printf("sanitized layer abi run ok\n");
    return 0;
}
