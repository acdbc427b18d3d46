// The token operators' host code (csrc/token_api.hip) under AddressSanitizer and
// UndefinedBehaviorSanitizer: arguments that validation settles, extreme sizes, and
// good ones, which have to reach the launcher (a stand-in here that counts) with what
// they were given.  Test infrastructure of tests/test_tokens_abi.py; addresses are
// never dereferenced and no device is needed.
#include <stdio.h>
#include <string.h>

#include <vector>

#include "zpp.h"
#include "zpp_token.h"

static int launches = 0;
static zpp::RotaryArgs seen_rotary;
static zpp::LogProbsArgs seen_logits;
static zpp::AdamConsts seen_consts;

namespace zpp {
hipError_t launch_rotary(const RotaryArgs &a, int, hipStream_t) {
    seen_rotary = a;
    ++launches;
    return hipSuccess;
}
size_t log_probs_workspace(size_t, size_t, uint32_t top) { return 64 + top; }
hipError_t launch_log_probs_forward(const LogProbsArgs &a, int, hipStream_t) {
    seen_logits = a;
    ++launches;
    return hipSuccess;
}
hipError_t launch_log_probs_backward(const LogProbsArgs &a, int, hipStream_t) {
    seen_logits = a;
    ++launches;
    return hipErrorInvalidConfiguration;
}
hipError_t launch_log_probs_train(const LogProbsArgs &a, int, hipStream_t) {
    seen_logits = a;
    ++launches;
    return hipSuccess;
}
hipError_t launch_adam_tensors(const void *, uint32_t, uint64_t, int, int, const AdamConsts &c,
                               hipStream_t) {
    seen_consts = c;
    ++launches;
    return hipSuccess;
}
hipError_t launch_adam_state_save(const float *, size_t, int, void *, float *, hipStream_t) {
    ++launches;
    return hipSuccess;
}
hipError_t launch_adam_state_load(const void *, const float *, size_t, int, float *, hipStream_t) {
    ++launches;
    return hipSuccess;
}
}  // namespace zpp

static int failures = 0;
#define EXPECT(cond)                                          \
    do {                                                      \
        if (!(cond)) {                                        \
            printf("%s:%d: %s\n", __FILE__, __LINE__, #cond); \
            ++failures;                                       \
        }                                                     \
    } while (0)

static void *dev(unsigned k, size_t off = 0) {
    return (void *)(uintptr_t)((16ull << 30) + ((uint64_t)k << 30) + off);
}

static zpp_status turn(const zpp_heads &x, const zpp_heads &out, const zpp_heads *k,
                       const zpp_heads *k_out, size_t tokens, uint32_t dim, uint32_t rotated) {
    return zpp_rotary_forward(&x, &out, k, k_out, ZPP_BF16, tokens, dim, rotated,
                              (const int64_t *)dev(20), (const double *)dev(21), 0, 1.0f, nullptr,
                              nullptr, nullptr);
}

static void rotary() {
    const zpp_heads x{dev(0), 512, 0, 64, 1, 8}, out{dev(1), 512, 0, 64, 1, 8};
    EXPECT(turn(x, out, nullptr, nullptr, 10, 64, 64) == ZPP_OK && launches == 1);
    EXPECT(seen_rotary.copy_x && !seen_rotary.copy_k && seen_rotary.x.heads == 8);
    EXPECT(turn(x, x, nullptr, nullptr, 10, 64, 64) == ZPP_OK && !seen_rotary.copy_x);
    // one more element down the row: shares, and is not in place
    zpp_heads moved = x;
    moved.data = dev(0, 2);
    EXPECT(turn(x, moved, nullptr, nullptr, 10, 64, 64) == ZPP_EOVERLAP);
    // query and key columns of one fused buffer, both in place
    const zpp_heads q{dev(2), 1024, 0, 64, 1, 8}, k{dev(2, 2 * 512), 1024, 0, 64, 1, 4};
    EXPECT(turn(q, q, &k, &k, 10, 64, 64) == ZPP_OK);
    zpp_heads near = k;
    near.data = dev(2, 2 * 511);
    EXPECT(turn(q, q, &near, &near, 10, 64, 64) == ZPP_EOVERLAP);
    // a key's head behind its group's queries: pieces at one distance, and with a gap after
    // every token, where they are enumerated
    for (size_t gap : {0, 8}) {
        const size_t token = 3 * 6 * 64 + gap;
        const zpp_heads gq{dev(3), token, 6 * 64, 64, 3, 4}, gk{dev(3, 2 * 256), token, 6 * 64, 64, 3, 1};
        EXPECT(turn(gq, gq, &gk, &gk, 10, 64, 64) == ZPP_OK);
        zpp_heads bad = gk;
        bad.data = dev(3, 2 * 255);
        EXPECT(turn(gq, gq, &bad, &bad, 10, 64, 64) == ZPP_EOVERLAP);
        bad.data = dev(3, 2 * (6 * 64 - 63));  // reaches into the next group
        EXPECT(turn(gq, gq, &bad, &bad, 10, 64, 64) == ZPP_EOVERLAP);
    }
    // outputs whose elements share a place
    zpp_heads same_place = out;
    same_place.head_stride = 63;
    EXPECT(turn(x, same_place, nullptr, nullptr, 10, 64, 64) == ZPP_EINVAL);
    same_place.head_stride = 0;
    EXPECT(turn(x, same_place, nullptr, nullptr, 10, 64, 64) == ZPP_EINVAL);
    // heads before tokens; inputs may repeat
    const zpp_heads turned{dev(1), 64, 0, 640, 1, 8}, spread{dev(0), 512, 0, 0, 1, 8};
    EXPECT(turn(spread, turned, nullptr, nullptr, 10, 64, 64) == ZPP_OK);
    // one token: its stride does not matter
    zpp_heads one = x;
    one.token_stride = SIZE_MAX;
    EXPECT(turn(one, out, nullptr, nullptr, 1, 64, 64) == ZPP_OK);
    // nothing to do
    zpp_heads none = x;
    none.heads = 0;
    launches = 0;
    EXPECT(turn(none, none, nullptr, nullptr, 10, 64, 64) == ZPP_OK && launches == 0);
    EXPECT(turn(x, out, nullptr, nullptr, 0, 64, 64) == ZPP_OK && launches == 0);
    EXPECT(turn(x, out, &k, nullptr, 10, 64, 64) == ZPP_EINVAL);
    EXPECT(turn(x, out, nullptr, nullptr, 10, 64, 63) == ZPP_EINVAL);
    EXPECT(turn(x, out, nullptr, nullptr, 10, 64, 66) == ZPP_EINVAL);
    EXPECT(turn(x, out, nullptr, nullptr, 10, 16385, 64) == ZPP_EINVAL);
    EXPECT(turn(x, out, nullptr, nullptr, 10, 8192, 4098) == ZPP_EINVAL);
    // positions inside an output
    const zpp_heads over{dev(20), 512, 0, 64, 1, 8};
    EXPECT(turn(x, over, nullptr, nullptr, 10, 64, 64) == ZPP_EOVERLAP);
    EXPECT(turn(x, over, nullptr, nullptr, 10, 64, 0) == ZPP_OK);
    const size_t huge[] = {(size_t)1 << 31, (size_t)1 << 62, SIZE_MAX, SIZE_MAX / 64};
    for (size_t a : huge)
        for (size_t b : huge) {
            zpp_heads h{dev(0), a, b, a, 3, 5};
            EXPECT(turn(h, h, nullptr, nullptr, 10, 64, 64) != ZPP_OK || a == b || a < 1u << 31);
            EXPECT(turn(x, out, nullptr, nullptr, a, 64, 64) != ZPP_OK || a == huge[0]);
        }
    zpp_heads many = x;
    many.groups = many.heads = 1u << 31;
    EXPECT(turn(many, many, nullptr, nullptr, 10, 64, 64) == ZPP_EINVAL);
}

static void log_probs() {
    launches = 0;
    const size_t R = 9, V = 1000;
    const zpp_matrix x{dev(0), nullptr, 1100, ZPP_BF16}, dx{dev(1), nullptr, V, ZPP_BF16};
    const int64_t *t = (const int64_t *)dev(2);
    float *lp = (float *)dev(3), *lse = (float *)dev(4), *h = (float *)dev(5), *g = (float *)dev(6);
    float *dh = (float *)dev(7), *tlp = (float *)dev(9);
    int32_t *ids = (int32_t *)dev(8);
    const auto forward = [&](const zpp_matrix *m, uint32_t top, size_t v, size_t ws) {
        return zpp_log_probs_forward(m, R, v, t, lp, lse, h, top, ids, tlp, dev(10), ws, nullptr,
                                     nullptr, nullptr);
    };
    EXPECT(forward(&x, 0, V, 64) == ZPP_OK && launches == 1 && seen_logits.vocab == V);
    EXPECT(forward(&x, 20, V, 84) == ZPP_OK && seen_logits.top == 20 && seen_logits.top_ids == ids);
    EXPECT(forward(&x, 20, V, 83) == ZPP_EINVAL);
    EXPECT(forward(&x, 65, V, 1000) == ZPP_EINVAL);
    EXPECT(forward(&x, 20, 19, 1000) == ZPP_EINVAL);
    EXPECT(forward(&x, 0, 0, 1000) == ZPP_EINVAL);
    zpp_matrix wide{dev(0), nullptr, 600000, ZPP_F32};
    EXPECT(forward(&wide, 0, 600000, 64) == ZPP_OK);
    EXPECT(forward(&wide, 1, 600000, 1000) == ZPP_EINVAL);
    const auto train = [&](const zpp_matrix *o, float *e, const float *de) {
        return zpp_log_probs_train(&x, R, V, t, lp, lse, e, g, de, o, dev(10), 64, nullptr, nullptr,
                                   nullptr);
    };
    EXPECT(train(&dx, h, dh) == ZPP_OK && seen_logits.dx.data == dx.data);
    EXPECT(train(&x, h, dh) == ZPP_OK && seen_logits.dx.data == x.data);  // in place
    EXPECT(train(&x, nullptr, dh) == ZPP_EINVAL);
    zpp_matrix other = x;
    other.stride = 1101;
    EXPECT(train(&other, h, dh) == ZPP_EOVERLAP);
    other = x;
    other.type = ZPP_F32;
    EXPECT(train(&other, h, dh) == ZPP_EINVAL);
    EXPECT(zpp_log_probs_backward(&x, R, V, t, lse, g, nullptr, nullptr, &x, nullptr, nullptr,
                                  nullptr) == ZPP_EHIP);
    EXPECT(zpp_log_probs_backward(&x, R, V, t, lse, g, h, nullptr, &x, nullptr, nullptr, nullptr) ==
           ZPP_EINVAL);
    const size_t huge[] = {(size_t)1 << 31, (size_t)1 << 62, SIZE_MAX, SIZE_MAX / 64};
    for (size_t a : huge)
        for (size_t b : huge) {
            EXPECT(zpp_log_probs_forward(&x, a, b, t, lp, lse, h, 0, ids, tlp, dev(10), 64, nullptr,
                                         nullptr, nullptr) == ZPP_EINVAL);
            EXPECT(zpp_log_probs_workspace(a, b, 0) == 0);
        }
}

static void adam() {
    launches = 0;
    const size_t counts[] = {0, 1, 63, 64, 65, 4096, 4097, 5000};
    for (size_t n : counts)
        for (int32_t type : {(int32_t)ZPP_F32, (int32_t)ZPP_I8}) {
            std::vector<zpp_adam_tensor> t(n);
            for (size_t i = 0; i < n; ++i)
                t[i] = {(float *)dev(0, 8192 * i), dev(10, 8192 * i), dev(20, 8192 * i),
                        (float *)dev(30, 64 * i), (float *)dev(31, 64 * i), dev(40, 8192 * i),
                        (uint16_t *)dev(50, 8192 * i), (size_t)(i % 3 ? 300 : i % 2 ? 0 : 1000), 0.1f};
            const size_t bytes = zpp_adam_tensors_table_bytes(n);
            std::vector<uint64_t> table(bytes / 8 + 1);  // as long as told, to a word
            zpp_adam_table list;
            EXPECT(zpp_adam_tensors_table(t.data(), n, type, ZPP_F32, table.data(), bytes, &list) ==
                   ZPP_OK);
            uint64_t tiles = 0;
            size_t full = 0;
            for (const zpp_adam_tensor &x : t)
                tiles += (x.n + 255) / 256, full += x.n != 0;
            EXPECT(list.tiles == tiles && list.tensors == full && !list.table);
            if (!n)
                continue;
            // every tile's tensor by the levels, as the kernel searches them
            const zpp::AdamEntry *e = (const zpp::AdamEntry *)table.data();
            std::vector<const uint32_t *> level;
            const uint32_t *w = (const uint32_t *)(e + full);
            for (size_t m = full;;) {
                level.push_back(w);
                w += zpp::padded_level(m);
                m = (m + 63) / 64;
                if (m <= 1)
                    break;
            }
            for (uint32_t tile = 0; tile < tiles; tile += 1 + tile / 7) {
                uint32_t i = 0;
                for (size_t l = level.size(); l--;) {
                    uint32_t reached = 0;
                    for (uint32_t lane = 0; lane < 64; ++lane)
                        reached += level[l][i * 64 + lane] <= tile;
                    i = i * 64 + reached - 1;
                }
                EXPECT(i < full && e[i].first <= tile &&
                       tile < e[i].first + (e[i].n + 255) / 256);
            }
            EXPECT(zpp_adam_tensors_table(t.data(), n, type, ZPP_F32, table.data(), bytes - 1,
                                          &list) == ZPP_EINVAL);
            if (n > 1) {
                zpp_adam_tensor kept = t[1];
                t[1].master = t[0].master;  // the same array twice
                EXPECT(zpp_adam_tensors_table(t.data(), n, type, ZPP_F32, table.data(), bytes,
                                              &list) == ZPP_EOVERLAP);
                t[1] = kept;
                t[1].grad = t[0].grad;      // a gradient of two
                EXPECT(zpp_adam_tensors_table(t.data(), n, type, ZPP_F32, table.data(), bytes,
                                              &list) == ZPP_OK);
                t[1].grad = t[0].master;
                EXPECT(zpp_adam_tensors_table(t.data(), n, type, ZPP_F32, table.data(), bytes,
                                              &list) == ZPP_EOVERLAP);
            }
        }
    zpp_adam_table list{dev(0), 5, 2, ZPP_I8, ZPP_F32};
    zpp_adam_hparams hp{0.5f, 0.9f, 0.95f, 1e-8f, 0.0f, 1, 3};
    EXPECT(zpp_adam_tensors_step(&list, &hp, nullptr, nullptr, nullptr) == ZPP_OK && launches == 1 &&
           seen_consts.lr_wd == 0.5f);
    hp.weight_decay = 0.1f;
    EXPECT(zpp_adam_tensors_step(&list, &hp, nullptr, nullptr, nullptr) == ZPP_EINVAL);
    hp.weight_decay = 0.0f;
    list.table = nullptr;
    EXPECT(zpp_adam_tensors_step(&list, &hp, nullptr, nullptr, nullptr) == ZPP_EINVAL);
    list.table = dev(0, 8);
    EXPECT(zpp_adam_tensors_step(&list, &hp, nullptr, nullptr, nullptr) == ZPP_EALIGN);
    list = {nullptr, 0, 0, ZPP_F32, ZPP_BF16};
    EXPECT(zpp_adam_tensors_step(&list, &hp, nullptr, nullptr, nullptr) == ZPP_OK && launches == 1);
    zpp_adam_tensor big{(float *)dev(0), dev(1), dev(2), nullptr, nullptr, dev(3), nullptr, SIZE_MAX,
                        0.0f};
    std::vector<uint64_t> table(100);
    EXPECT(zpp_adam_tensors_table(&big, 1, ZPP_F32, ZPP_F32, table.data(), 800, &list) == ZPP_EINVAL);
    big.n = (size_t)1 << 40;
    EXPECT(zpp_adam_tensors_table(&big, 1, ZPP_F32, ZPP_F32, table.data(), 800, &list) == ZPP_EINVAL);
    EXPECT(zpp_adam_tensors_table_bytes(SIZE_MAX) == 0);
    EXPECT(zpp_adam_tensors_table(nullptr, SIZE_MAX, ZPP_F32, ZPP_F32, nullptr, 0, &list) ==
           ZPP_EINVAL);
    launches = 0;
    EXPECT(zpp_adam_state_save((float *)dev(0), 1000, 1, dev(1), (float *)dev(2), nullptr, nullptr,
                               nullptr) == ZPP_OK);
    EXPECT(zpp_adam_state_load(dev(1), (float *)dev(2), 1000, 2, (float *)dev(0), nullptr, nullptr,
                               nullptr) == ZPP_OK && launches == 2);
    EXPECT(zpp_adam_state_load(dev(1), (float *)dev(2), 1000, 3, (float *)dev(0), nullptr, nullptr,
                               nullptr) == ZPP_EINVAL);
    EXPECT(zpp_adam_state_save((float *)dev(0), SIZE_MAX, 1, dev(1), (float *)dev(2), nullptr,
                               nullptr, nullptr) == ZPP_EINVAL);
    EXPECT(zpp_adam_state_save((float *)dev(0), 1000, 1, dev(0, 3999), (float *)dev(2), nullptr,
                               nullptr, nullptr) == ZPP_EOVERLAP);
    EXPECT(zpp_adam_state_save((float *)dev(0), 1000, 1, dev(1), (float *)dev(1, 996), nullptr,
                               nullptr, nullptr) == ZPP_EOVERLAP);
}

int main() {
    rotary();
    log_probs();
    adam();
    if (failures)
        return 1;
    printf("sanitized token abi run ok\n");
    return 0;
}
