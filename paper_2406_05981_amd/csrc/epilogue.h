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

template <int V>
__device__ inline void activate(float (&v)[V], int act) {
    switch (act) {
        case SA_ACT_RELU:
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = v[j] < 0.0f ? 0.0f : v[j];  // a NaN stays one
            break;
        case SA_ACT_GELU:
            // the upper tail, not 1 + erf: no cancellation for negative v
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = 0.5f * v[j] * erfcf(-0.70710678118654752f * v[j]);
            break;
        case SA_ACT_GELU_TANH:
            // 0.5 (1 + tanh u) = sigmoid(2 u)
#pragma unroll
            for (int j = 0; j < V; ++j)
                v[j] *= sigmoid(1.59576912160573071f * fmaf(0.044715f * v[j], v[j] * v[j], v[j]));
            break;
        case SA_ACT_SILU:
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] *= sigmoid(v[j]);
            break;
        default: break;
    }
}

__device__ inline float load(const void* p, int64_t i, int half) {
    return half ? (float)static_cast<const _Float16*>(p)[i] : static_cast<const float*>(p)[i];
}

__device__ inline void store(void* p, int64_t i, float v, int half) {
    if (half) static_cast<_Float16*>(p)[i] = (_Float16)v;
    else static_cast<float*>(p)[i] = v;
}

// V (4 or 8) consecutive outputs of one row from element i, a multiple of V.
template <int V>
__device__ inline void load_vector(const void* p, int64_t i, int half, float (&out)[V]) {
    typedef _Float16 halfv_t __attribute__((ext_vector_type(V)));
    typedef float floatv_t __attribute__((ext_vector_type(V)));
    if (half) {
        const halfv_t h = *reinterpret_cast<const halfv_t*>(static_cast<const _Float16*>(p) + i);
#pragma unroll
        for (int j = 0; j < V; ++j) out[j] = (float)h[j];
    } else {
        const floatv_t f = *reinterpret_cast<const floatv_t*>(static_cast<const float*>(p) + i);
#pragma unroll
        for (int j = 0; j < V; ++j) out[j] = f[j];
    }
}

template <int V>
__device__ inline void finish_vector(const Epilogue& e, int64_t i, int n, float (&v)[V]) {
    typedef _Float16 halfv_t __attribute__((ext_vector_type(V)));
    typedef float floatv_t __attribute__((ext_vector_type(V)));
    float z[V];
    if (e.bias) {
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] += e.bias[n + j];
    }
    activate(v, e.act);
    if (e.multiplier) {
        load_vector<V>(e.multiplier, i, e.half, z);
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] *= z[j];
    }
    if (e.residual) {
        load_vector<V>(e.residual, i, e.half, z);
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] += z[j];
    }
    if (e.half) {
        halfv_t h;
#pragma unroll
        for (int j = 0; j < V; ++j) h[j] = (_Float16)v[j];
        *reinterpret_cast<halfv_t*>(static_cast<_Float16*>(e.y) + i) = h;
    } else {
        floatv_t f;
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = v[j];
        *reinterpret_cast<floatv_t*>(static_cast<float*>(e.y) + i) = f;
    }
}

// The first `count` of V consecutive outputs of one row from element i.
template <int V>
__device__ inline void finish_some(const Epilogue& e, int64_t i, int n, int count, float (&v)[V]) {
    if (e.bias) {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (j < count) v[j] += e.bias[n + j];
    }
    activate(v, e.act);
#pragma unroll
    for (int j = 0; j < V; ++j) {
        if (j >= count) break;
        if (e.multiplier) v[j] *= load(e.multiplier, i + j, e.half);
        if (e.residual) v[j] += load(e.residual, i + j, e.half);
        store(e.y, i + j, v[j], e.half);
    }
}

// One output: element i = row * N + n.
__device__ inline void finish(const Epilogue& e, int64_t i, int n, float v) {
    float one[1] = {v};
    finish_some(e, i, n, 1, one);
}

}  // namespace sa_epi

#endif
