// AdamW update of one element, shared by the kernels on packed rows and those on many tensors.
#pragma once
#include "common.cuh"

namespace {

// The ViT runs of the paper train with AdamW (lr 5e-4, weight decay 0.01).  Decoupled form:
//   x <- x (1 - lr wd);  m <- m + (1 - b1)(g - m);  v <- b2 v + (1 - b2) g^2;
//   x <- x - [lr / (1 - b1^t)] m / ( sqrt(v) / sqrt(1 - b2^t) + eps )
// The step-dependent factors are formed on the host in double and passed as floats.

struct AdamArgs {
    float *m1;   // exp_avg      [M, ld]
    float *m2;   // exp_avg_sq   [M, ld]
    const float *g;
    float decay, one_minus_b1, b2, one_minus_b2, step_size, inv_sqrt_bc2, eps;
};

__device__ __forceinline__ void adamw1(float &x, float &m1, float &m2, float g, const AdamArgs &p) {
    x = __fmul_rn(x, p.decay);
    m1 = __fmaf_rn(p.one_minus_b1, __fsub_rn(g, m1), m1);
    m2 = __fmaf_rn(p.b2, m2, __fmul_rn(p.one_minus_b2, __fmul_rn(g, g)));
    const float denom = __fmaf_rn(__fsqrt_rn(m2), p.inv_sqrt_bc2, p.eps);
    x = __fmaf_rn(-p.step_size, __fdiv_rn(m1, denom), x);
}

}  // namespace
