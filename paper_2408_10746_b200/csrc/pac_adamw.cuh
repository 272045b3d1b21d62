#pragma once
#include "pac_common.cuh"

namespace pac {

// One element of the update, shared by every kernel that applies AdamW so that fused and
// separate updates are bit-identical.
// The arithmetic of one element: returns the new parameter, updates mi / vi in place.
__device__ __forceinline__ float adamw_math(float th, float& mi, float& vi, float gi, bool decays, const pac_adamw& hp,
                                            float bc1, float bc2) {
    // every rounding is spelled out (no contraction into FMAs), in the order the update is written:
    // m = b1 m + (1-b1) g;  v = b2 v + ((1-b2) g) g;  theta = (theta - lr wd theta) - (lr mhat)/(sqrt(vhat)+eps)
    mi = __fadd_rn(__fmul_rn(hp.beta1, mi), __fmul_rn(__fsub_rn(1.f, hp.beta1), gi));
    vi = __fadd_rn(__fmul_rn(hp.beta2, vi), __fmul_rn(__fmul_rn(__fsub_rn(1.f, hp.beta2), gi), gi));
    const float mhat = __fdiv_rn(mi, bc1), vhat = __fdiv_rn(vi, bc2);
    const float decay = decays ? __fmul_rn(__fmul_rn(hp.lr, hp.weight_decay), th) : 0.f;
    return __fsub_rn(__fsub_rn(th, decay), __fdiv_rn(__fmul_rn(hp.lr, mhat), __fadd_rn(__fsqrt_rn(vhat), hp.eps)));
}

}  // namespace pac
