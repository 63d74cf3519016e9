// What follows the product in one output of the layer,
//   y = act(v + bias[n]) * multiplier + residual,
// evaluated in fp32 on the fp32 sum v and rounded once, as it is stored.
#ifndef SHIFTADD_EPILOGUE_H
#define SHIFTADD_EPILOGUE_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "shiftadd.h"

namespace sa_epi {

struct Epilogue {
    const float* bias;       // [N] or null
    const void* multiplier;  // [rows][N] of y's type, or null
    const void* residual;    // [rows][N] of y's type, or null; may be y itself
    void* y;                 // [rows][N] binary16 (half) or fp32
    int act;                 // sa_activation
    int half;
};

// 1 / (1 + exp(-z)) by the hardware's exponential and reciprocal (1 ulp each): the
// rounding of z log2(e) is a relative error of |z| 2^-24 of exp(-z), and v times the
// result is off by at most 2^-23 |v| either way.
__device__ inline float sigmoid(float z) {
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504088896341f * z));
}

__device__ inline float activate(float v, int act) {
    switch (act) {
        case SA_ACT_RELU: return v < 0.0f ? 0.0f : v;  // a NaN stays one
        // the upper tail, not 1 + erf: no cancellation for negative v
        case SA_ACT_GELU: return 0.5f * v * erfcf(-0.70710678118654752f * v);
        // 0.5 (1 + tanh u) = sigmoid(2 u)
        case SA_ACT_GELU_TANH:
            return v * sigmoid(1.59576912160573071f * fmaf(0.044715f * v, v * v, v));
        case SA_ACT_SILU: return v * sigmoid(v);
        default: return v;
    }
}

__device__ inline float load(const void* p, int64_t i, int half) {
    return half ? (float)static_cast<const _Float16*>(p)[i] : static_cast<const float*>(p)[i];
}

__device__ inline void store(void* p, int64_t i, float v, int half) {
    if (half) static_cast<_Float16*>(p)[i] = (_Float16)v;
    else static_cast<float*>(p)[i] = v;
}

// One output: element i = row * N + n.
__device__ inline void finish(const Epilogue& e, int64_t i, int n, float v) {
    if (e.bias) v += e.bias[n];
    v = activate(v, e.act);
    if (e.multiplier) v *= load(e.multiplier, i, e.half);
    if (e.residual) v += load(e.residual, i, e.half);
    store(e.y, i, v, e.half);
}

}  // namespace sa_epi

#endif
