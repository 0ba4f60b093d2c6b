// What the optimizer steps share: AdamW's arguments and the constants of a step (internal header).
#pragma once

#include <cmath>

#include "common.h"

namespace pcm {

struct AdamConst {
    float beta1, beta2, one_minus_beta1, one_minus_beta2;
    float decay;            // 1 - lr * weight_decay
    float step_size;        // lr / (1 - beta1^t)
    float inv_sqrt_bc2;     // 1 / sqrt(1 - beta2^t)
    float eps;
};

inline bool adam_arguments_ok(int64_t step, double lr, double beta1, double beta2, double eps, double weight_decay, double max_grad_norm) {
    return step >= 1 && lr >= 0.0 && beta1 >= 0.0 && beta1 < 1.0 && beta2 >= 0.0 && beta2 < 1.0 && eps > 0.0 && weight_decay >= 0.0 &&
           max_grad_norm > 0.0;
}
inline AdamConst adam_const(int64_t step, double lr, double beta1, double beta2, double eps, double weight_decay) {
    AdamConst c;
    c.beta1 = (float)beta1; c.beta2 = (float)beta2;
    c.one_minus_beta1 = (float)(1.0 - beta1); c.one_minus_beta2 = (float)(1.0 - beta2);
    c.decay = (float)(1.0 - lr * weight_decay);
    c.step_size = (float)(lr / (1.0 - pow(beta1, (double)step)));
    c.inv_sqrt_bc2 = (float)(1.0 / sqrt(1.0 - pow(beta2, (double)step)));
    c.eps = (float)eps;
    return c;
}

}  // namespace pcm
