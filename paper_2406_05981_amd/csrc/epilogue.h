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

// 1 / (1 + exp(-z)) by the hardware's exponential and reciprocal (1 ulp each).  Measured
// over 4 million v in each of 13 ranges within +-100: v times the result is off by at most
// 2.6 * 2^-24 |v|, SILU and GELU_TANH.  Small results of negative v are off by more relative
// to themselves, since the rounding of z log2(e) is a relative error of |z| 2^-24 of
// exp(-z): 4e-7 of SILU and 3e-6 of GELU_TANH at -5..-3, 1e-6 and 1.4e-5 at -13..-8.
__device__ inline float sigmoid(float z) {
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504088896341f * z));
}

// v Phi(v) = v / 2 erfc(-v / sqrt 2).  erfc(z) = exp(-z^2) t P(t), t = 1 / (1 + z / 2), z >= 0, P
// the polynomial of degree 8 closest to erfcx(z) / t (a least-squares fit, reweighted
// towards equal relative errors: 3.2e-8); for v > 0 from the other tail, 2 - erfc.  The
// result, measured as above: off by at most 4.1 * 2^-24 |v| (at |v| < 0.1); relative to
// itself 5e-7 above -1, 1.4e-6 at -3..-1, 7e-6 at -8..-5, 1.7e-5 at -13..-8.  The library's
// erfcf has branches for every range: 45 million outputs after a prompt's product cost 48 us
// with it.
__device__ inline float gelu(float v) {
    const float z = 0.70710678118654752f * fabsf(v);
    const float t = __builtin_amdgcn_rcpf(fmaf(0.5f, z, 1.0f));
    float p = -0.0555105545f;
    p = fmaf(p, t, 0.266813397f);
    p = fmaf(p, t, -0.449434638f);
    p = fmaf(p, t, 0.233498693f);
    p = fmaf(p, t, 0.00522376923f);
    p = fmaf(p, t, 0.188610703f);
    p = fmaf(p, t, 0.246851534f);
    p = fmaf(p, t, 0.281826973f);
    p = fmaf(p, t, 0.282120109f);
    const float tail = p * t * __builtin_amdgcn_exp2f(-1.44269504088896341f * z * z);
    return 0.5f * v * (v > 0.0f ? 2.0f - tail : tail);
}

template <int V>
__device__ inline void activate(float (&v)[V], int act) {
    switch (act) {
        case SA_ACT_RELU:
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = v[j] < 0.0f ? 0.0f : v[j];  // a NaN stays one
            break;
        case SA_ACT_GELU:
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = gelu(v[j]);
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

// 8 consecutive outputs of one row from element i.  Their operands are requested as they
// lie in memory (rows of odd lengths begin at any element) and unpacked when they are used.
typedef _Float16 half8_t __attribute__((ext_vector_type(8), aligned(2)));
typedef float float8_t __attribute__((ext_vector_type(8), aligned(4)));
struct Operands8 {
    half8_t multiplier_h, residual_h;
    float8_t multiplier_f, residual_f;
};
__device__ inline void fetch(const Epilogue& e, int64_t i, Operands8* o) {
    if (e.half) {
        if (e.multiplier)
            o->multiplier_h =
                *reinterpret_cast<const half8_t*>(static_cast<const _Float16*>(e.multiplier) + i);
        if (e.residual)
            o->residual_h =
                *reinterpret_cast<const half8_t*>(static_cast<const _Float16*>(e.residual) + i);
    } else {
        if (e.multiplier)
            o->multiplier_f =
                *reinterpret_cast<const float8_t*>(static_cast<const float*>(e.multiplier) + i);
        if (e.residual)
            o->residual_f =
                *reinterpret_cast<const float8_t*>(static_cast<const float*>(e.residual) + i);
    }
}

__device__ inline void finish(const Epilogue& e, int64_t i, const float (&bias)[8],
                              const Operands8& o, float (&v)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += bias[j];
    activate(v, e.act);
    if (e.half) {
        half8_t h;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (e.multiplier) v[j] *= (float)o.multiplier_h[j];
            if (e.residual) v[j] += (float)o.residual_h[j];
            h[j] = (_Float16)v[j];
        }
        *reinterpret_cast<half8_t*>(static_cast<_Float16*>(e.y) + i) = h;
    } else {
        float8_t f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (e.multiplier) v[j] *= o.multiplier_f[j];
            if (e.residual) v[j] += o.residual_f[j];
            f[j] = v[j];
        }
        *reinterpret_cast<float8_t*>(static_cast<float*>(e.y) + i) = f;
    }
}

// The first `count` of 8 such outputs.
__device__ inline void finish_some(const Epilogue& e, int64_t i, const float (&bias)[8], int count,
                                   float (&v)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += bias[j];
    activate(v, e.act);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if (j >= count) break;
        if (e.multiplier) v[j] *= load(e.multiplier, i + j, e.half);
        if (e.residual) v[j] += load(e.residual, i + j, e.half);
        store(e.y, i + j, v[j], e.half);
    }
}

// One output: what it needs besides its sum may be requested before the sum is there.
struct Operands {
    float bias, multiplier, residual;
};
__device__ inline Operands fetch(const Epilogue& e, int64_t i, int n) {
    return {e.bias ? e.bias[n] : 0.0f, e.multiplier ? load(e.multiplier, i, e.half) : 1.0f,
            e.residual ? load(e.residual, i, e.half) : 0.0f};
}
__device__ inline void finish(const Epilogue& e, int64_t i, const Operands& o, float v) {
    float z[1] = {v + o.bias};
    activate(z, e.act);
    store(e.y, i, fmaf(z[0], o.multiplier, o.residual), e.half);
}

}  // namespace sa_epi

#endif
