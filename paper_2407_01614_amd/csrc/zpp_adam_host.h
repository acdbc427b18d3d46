// Hyperparameters of a step on the host: their checks and the constants that the
// kernels take.
#pragma once

#include <math.h>

#include "zpp.h"
#include "zpp_launch.h"

namespace zpp {

inline zpp_status check_hparams(const zpp_adam_hparams *hp) {
    if (!hp)
        return ZPP_EINVAL;
    if (!isfinite(hp->lr) || !isfinite(hp->beta1) || !isfinite(hp->beta2) ||
        !isfinite(hp->eps) || !isfinite(hp->weight_decay))
        return ZPP_EINVAL;
    if (hp->beta1 < 0.0f || hp->beta1 >= 1.0f || hp->beta2 < 0.0f || hp->beta2 >= 1.0f ||
        hp->eps < 0.0f || hp->step < 1)
        return ZPP_EINVAL;
    return ZPP_OK;
}

// Step-dependent constants, folded on the host in double and rounded once.
inline AdamConsts adam_consts(const zpp_adam_hparams &hp) {
    AdamConsts c;
    const double b1 = hp.beta1, b2 = hp.beta2, lr = hp.lr, wd = hp.weight_decay;
    const double bc1 = 1.0 - pow(b1, (double)hp.step);
    const double bc2 = 1.0 - pow(b2, (double)hp.step);
    c.lr_wd = (float)(lr * wd);
    c.wd = hp.weight_decay;
    c.beta1 = hp.beta1;
    c.one_minus_beta1 = (float)(1.0 - b1);
    c.beta2 = hp.beta2;
    c.one_minus_beta2 = (float)(1.0 - b2);
    c.step_size = (float)(lr / bc1);
    c.inv_bc2 = (float)(1.0 / bc2);
    c.eps = hp.eps;
    c.adamw = hp.adamw ? 1 : 0;
    return c;
}

}  // namespace zpp
