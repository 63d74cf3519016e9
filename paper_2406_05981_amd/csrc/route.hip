// A router's choice of experts and the sum of the experts' rows.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "checks.h"
#include "epilogue.h"
#include "keys.h"

namespace {

// ---------------------------------------------------------------- choice
//
// A wave takes a token at a time, each lane PER consecutive experts.  The k largest
// logits come one after the other: a maximum over the wave, the lowest lane that
// holds it, its lowest expert.  Logits are compared as unsigned numbers of the same
// order; 0 stands for -inf, NaN and what was chosen before.
//
// The lists.  Tokens are dealt to at most kMaxBlocks workgroups in ranges of whole
// 32-token steps.  Each workgroup counts its choices by expert (k_choose); a second
// launch (k_place) adds up the counts of the workgroups before it and of all experts
// below, and gives every choice its place: a step's choices of an expert are one bit a
// token in a 32-bit mask, the place is the number of bits below.  Nothing depends on
// the order of atomics.  Up to kOneBlock tokens one workgroup does both.
constexpr int kStep = 32;         // tokens of a step
constexpr int kMaxBlocks = 256;
constexpr int kWaves = 16;
constexpr int kThreads = 64 * kWaves;
constexpr int kOneBlock = 64;     // tokens

struct Route {
    const float* logits;
    int tokens, experts, k, normalize;
    int32_t* ids;
    float* weights;
    int32_t* offsets;
    int32_t* row_of;
    int32_t* slot_of;
    int32_t* counts;  // [blocks][experts]
    int per_block;    // tokens of a workgroup
};

__device__ inline uint32_t order_of(float v) {
    if (!(v > -__builtin_inff())) return 0u;
    const uint32_t b = __builtin_bit_cast(uint32_t, v + 0.0f);  // -0 counts as 0
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ inline float logit_of(uint32_t o) {
    return __builtin_bit_cast(float, o & 0x80000000u ? o & 0x7fffffffu : ~o);
}

// The largest of the wave's values, the same in every lane: within 16 lanes, then across.
__device__ inline uint32_t wave_max(uint32_t v) {
    auto from = [&](auto control) {
        return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, decltype(control)::value, 0xf, 0xf,
                                                     false);
    };
    v = max(v, from(std::integral_constant<int, 0xB1>{}));   // lanes 1, 0, 3, 2
    v = max(v, from(std::integral_constant<int, 0x4E>{}));   // lanes 2, 3, 0, 1
    v = max(v, from(std::integral_constant<int, 0x141>{}));  // halves of 8 mirrored
    v = max(v, from(std::integral_constant<int, 0x140>{}));  // 16 mirrored
    v = max(v, from(std::integral_constant<int, 0x142>{}));  // the 16 lanes before
    v = max(v, from(std::integral_constant<int, 0x143>{}));  // the 32 lanes before
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

__device__ inline float wave_sum(float v) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
    return v;
}

// Token t's choices: lane j < k returns the expert of choice j, or -1.
template <int PER>
__device__ inline int choose(const Route& a, int t) {
    const int lane = threadIdx.x & 63;
    const float* l = a.logits + (int64_t)t * a.experts;
    uint32_t o[PER];
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        const int e = PER * lane + p;
        o[p] = e < a.experts ? order_of(l[e]) : 0u;
    }
    uint32_t best = 0;
#pragma unroll
    for (int p = 0; p < PER; ++p) best = max(best, o[p]);
    const uint32_t first = wave_max(best);
    const float peak = first ? logit_of(first) : 0.0f;
    float total = 0.0f;
    if (!a.normalize) {
#pragma unroll
        for (int p = 0; p < PER; ++p)
            if (o[p]) total += expf(logit_of(o[p]) - peak);
        total = wave_sum(total);
    }
    int id = -1;
    float w = 0.0f;
    uint32_t top = first;
    for (int j = 0; j < a.k && top; ++j) {
        const int from = __builtin_ctzll(__ballot(best == top));
        int e = 0;
        bool open = lane == from;
        uint32_t rest = 0;
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            if (open && o[p] == top) {
                e = PER * lane + p;
                o[p] = 0;
                open = false;
            }
            rest = max(rest, o[p]);
        }
        best = rest;
        e = __builtin_amdgcn_readlane(e, from);
        if (lane == j) {
            id = e;
            w = expf(logit_of(top) - peak);
        }
        top = wave_max(best);
    }
    if (a.normalize) total = wave_sum(w);
    if (lane < a.k) {
        const int64_t i = (int64_t)t * a.k + lane;
        a.ids[i] = id;
        a.weights[i] = id < 0 ? 0.0f : w / total;
    }
    return id;
}

// Places of the tokens [t0, t1): base[e] holds the first free slot of expert e.
__device__ inline void place(const Route& a, int t0, int t1, int* base, uint32_t* mask) {
    for (int s = t0; s < t1; s += kStep) {
        for (int e = threadIdx.x; e < a.experts; e += kThreads) mask[e] = 0u;
        __syncthreads();
        const int items = imin(kStep, t1 - s) * a.k;
        const int64_t i0 = (int64_t)s * a.k;
        for (int i = threadIdx.x; i < items; i += kThreads) {
            const int e = a.ids[i0 + i];
            if (e >= 0) atomicOr(&mask[e], 1u << (i / a.k));
        }
        __syncthreads();
        for (int i = threadIdx.x; i < items; i += kThreads) {
            const int e = a.ids[i0 + i], t = i / a.k;
            int slot = -1;
            if (e >= 0) {
                slot = base[e] + __popc(mask[e] & ((1u << t) - 1u));
                a.row_of[slot] = s + t;
            }
            a.slot_of[i0 + i] = slot;
        }
        __syncthreads();
        for (int e = threadIdx.x; e < a.experts; e += kThreads) base[e] += __popc(mask[e]);
        __syncthreads();
    }
}

// base[e] += the choices of the experts below e; returns the choices of all.
// total[e] holds those of expert e.
__device__ inline int add_below(int experts, const int* total, int* base, int* offsets) {
    const int lane = threadIdx.x & 63;
    int before = 0;
    // every wave runs the scan; the first one writes
    for (int e0 = 0; e0 < experts; e0 += 64) {
        const int e = e0 + lane;
        const int v = e < experts ? total[e] : 0;
        int sum = v;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int u = __shfl_up(sum, d);
            if (lane >= d) sum += u;
        }
        if (threadIdx.x < 64 && e < experts) {
            base[e] += before + sum - v;
            if (offsets) offsets[e] = before + sum - v;
        }
        before += __shfl(sum, 63);
    }
    if (offsets && threadIdx.x == 0) offsets[experts] = before;
    return before;
}

template <int PER, bool ALL>
__global__ __launch_bounds__(kThreads) void k_choose(Route a) {
    __shared__ int counts[64 * PER];
    __shared__ int base[ALL ? 64 * PER : 1];
    __shared__ uint32_t mask[ALL ? 64 * PER : 1];
    const int wave = threadIdx.x >> 6;
    for (int e = threadIdx.x; e < a.experts; e += kThreads) {
        counts[e] = 0;
        if constexpr (ALL) base[e] = 0;
    }
    __syncthreads();
    const int t0 = (int)blockIdx.x * a.per_block, t1 = imin(t0 + a.per_block, a.tokens);
    for (int t = t0 + wave; t < t1; t += kWaves) {
        const int id = choose<PER>(a, t);
        if (id >= 0) atomicAdd(&counts[id], 1);
    }
    __syncthreads();
    if constexpr (ALL) {
        const int all = add_below(a.experts, counts, base, a.offsets);
        __syncthreads();
        place(a, 0, a.tokens, base, mask);
        for (int i = all + threadIdx.x; i < a.tokens * a.k; i += kThreads) a.row_of[i] = -1;
    } else {
        for (int e = threadIdx.x; e < a.experts; e += kThreads)
            a.counts[(int64_t)blockIdx.x * a.experts + e] = counts[e];
    }
}

__global__ __launch_bounds__(kThreads) void k_place(Route a) {
    __shared__ int total[SA_MAX_EXPERTS];
    __shared__ int base[SA_MAX_EXPERTS];
    __shared__ uint32_t mask[SA_MAX_EXPERTS];
    const int blocks = (int)gridDim.x;
    for (int e = threadIdx.x; e < a.experts; e += kThreads) base[e] = total[e] = 0;
    __syncthreads();
    // the threads of an expert share the workgroups' counts (integers: any order)
    const int shares = imax(1, kThreads / a.experts);
    for (int i = threadIdx.x; i < shares * a.experts; i += kThreads) {
        const int e = i % a.experts;
        int below = 0, all = 0;
#pragma unroll 4
        for (int b = i / a.experts; b < blocks; b += shares) {
            const int v = a.counts[(int64_t)b * a.experts + e];
            below += b < (int)blockIdx.x ? v : 0;
            all += v;
        }
        atomicAdd(&base[e], below);
        atomicAdd(&total[e], all);
    }
    __syncthreads();
    const int all = add_below(a.experts, total, base, blockIdx.x == 0 ? a.offsets : nullptr);
    __syncthreads();
    const int t0 = (int)blockIdx.x * a.per_block, t1 = imin(t0 + a.per_block, a.tokens);
    place(a, t0, t1, base, mask);
    const int64_t n = (int64_t)a.tokens * a.k;
    for (int64_t i = all + (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n;
         i += (int64_t)blocks * kThreads)
        a.row_of[i] = -1;
}

// Tokens of a workgroup and workgroups.
int route_blocks(int tokens, int* per_block) {
    if (tokens <= kOneBlock) {
        *per_block = tokens;
        return 1;
    }
    const int steps = (tokens + kStep - 1) / kStep;
    const int per = (steps + kMaxBlocks - 1) / kMaxBlocks;
    *per_block = kStep * per;
    return (steps + per - 1) / per;
}

bool route_sizes(int tokens, int experts, int k) {
    return tokens >= 0 && tokens <= SA_MAX_ROWS && experts >= 1 && experts <= SA_MAX_EXPERTS &&
           k >= 1 && k <= experts && k <= SA_MAX_CHOICES;
}

template <int PER>
void launch_route(const Route& a, int blocks, hipStream_t s) {
    if (blocks == 1) {
        hipLaunchKernelGGL((k_choose<PER, true>), dim3(1), dim3(kThreads), 0, s, a);
        return;
    }
    hipLaunchKernelGGL((k_choose<PER, false>), dim3(blocks), dim3(kThreads), 0, s, a);
    hipLaunchKernelGGL(k_place, dim3(blocks), dim3(kThreads), 0, s, a);
}

// ---------------------------------------------------------------- combination

struct Combine {
    const void* h;
    const int32_t* slot_of;
    const float* weights;
    const void* residual;
    void* y;
    int slots, k, N, half;
};

// A workgroup takes kCols columns of one token, a thread 8 consecutive ones: four rows are
// requested at a time.  Bound by memory: every row of h is read once.
constexpr int kCols = 2048;

template <typename T>
__device__ inline void combine(const Combine& a, int64_t t, int n) {
    typedef T vec_t __attribute__((ext_vector_type(8), aligned(sizeof(T))));
    const T* h = static_cast<const T*>(a.h);
    const int64_t at = t * a.N + n;
    const int count = imin(8, a.N - n);
    auto load = [&](const T* p) {
        vec_t v;
        if (count == 8) {
            v = *reinterpret_cast<const vec_t*>(p);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = j < count ? p[j] : (T)0;
        }
        return v;
    };
    float sum[8] = {};
    if (a.residual) {
        const vec_t r = load(static_cast<const T*>(a.residual) + at);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] = (float)r[j];
    }
    for (int j0 = 0; j0 < a.k; j0 += 4) {
        vec_t row[4];
        float w[4];
        bool live[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int j = imin(j0 + u, a.k - 1);
            const int slot = a.slot_of[t * a.k + j];
            live[u] = j0 + u < a.k && slot >= 0 && slot < a.slots;
            w[u] = a.weights[t * a.k + j];
            if (live[u]) row[u] = load(h + (int64_t)slot * a.N + n);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (live[u])
#pragma unroll
                for (int j = 0; j < 8; ++j) sum[j] = fmaf(w[u], (float)row[u][j], sum[j]);
    }
    T* y = static_cast<T*>(a.y) + at;
    if (count == 8) {
        vec_t v;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = (T)sum[j];
        *reinterpret_cast<vec_t*>(y) = v;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < count) y[j] = (T)sum[j];
    }
}

__global__ __launch_bounds__(256) void k_combine(Combine a, int pieces) {
    const int64_t t = blockIdx.x / (unsigned)pieces;
    const int n = (int)(blockIdx.x % (unsigned)pieces) * kCols + 8 * (int)threadIdx.x;
    if (n >= a.N) return;
    if (a.half) combine<_Float16>(a, t, n);
    else combine<float>(a, t, n);
}

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

}  // namespace

extern "C" {

SA_API size_t sa_route_workspace_bytes(int tokens, int experts, int k) {
    if (!route_sizes(tokens, experts, k)) return 0;
    int per;
    const int blocks = route_blocks(tokens, &per);
    return blocks > 1 ? sizeof(int32_t) * (size_t)blocks * (size_t)experts : 0;
}

SA_API int sa_route_experts(const float* logits, int tokens, int experts, int k, int normalize,
                            int32_t* ids, float* weights, int32_t* offsets, int32_t* row_of,
                            int32_t* slot_of, void* workspace, size_t workspace_bytes,
                            void* stream) {
    if (!offsets || (tokens != 0 && (!logits || !ids || !weights || !row_of || !slot_of)))
        return SA_ERR_NULL;
    if (!route_sizes(tokens, experts, k)) return SA_ERR_SHAPE;
    const size_t need = sa_route_workspace_bytes(tokens, experts, k);
    if (need && !workspace) return SA_ERR_NULL;
    if (workspace_bytes < need) return SA_ERR_SHAPE;
    if (!aligned4(logits) || !aligned4(ids) || !aligned4(weights) || !aligned4(offsets) ||
        !aligned4(row_of) || !aligned4(slot_of) || (need && !aligned16(workspace)))
        return SA_ERR_ALIGN;
    Route a = {logits, tokens, experts, k, normalize, ids, weights, offsets, row_of, slot_of,
               static_cast<int32_t*>(workspace), 0};
    const int blocks = route_blocks(tokens, &a.per_block);
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const int per = (experts + 63) / 64;
    if (per == 1) launch_route<1>(a, blocks, s);
    else if (per == 2) launch_route<2>(a, blocks, s);
    else if (per <= 4) launch_route<4>(a, blocks, s);
    else if (per <= 8) launch_route<8>(a, blocks, s);
    else launch_route<16>(a, blocks, s);
    return launch_status();
}

SA_API int sa_combine_experts(const void* h, const int32_t* slot_of, const float* weights,
                              int slots, int tokens, int k, int N, const void* residual, int half,
                              void* y, void* stream) {
    if (tokens != 0 && (!slot_of || !weights || !y || (slots != 0 && !h))) return SA_ERR_NULL;
    if (tokens < 0 || tokens > SA_MAX_ROWS || slots < 0 || slots > SA_MAX_ROWS || k < 1 ||
        k > SA_MAX_CHOICES || N < 1 || (int64_t)tokens * N > (int64_t)1 << 34 ||
        (int64_t)slots * N > (int64_t)1 << 34)
        return SA_ERR_SHAPE;
    if (!aligned16(h) || !aligned16(y) || !aligned16(residual) || !aligned4(slot_of) ||
        !aligned4(weights))
        return SA_ERR_ALIGN;
    if (tokens == 0) return SA_OK;
    const Combine a = {h, slot_of, weights, residual, y, slots, k, N, half};
    const int pieces = (int)(((int64_t)N + kCols - 1) / kCols);
    hipLaunchKernelGGL(k_combine, dim3((unsigned)tokens * (unsigned)pieces), dim3(256), 0,
                       reinterpret_cast<hipStream_t>(stream), a, pieces);
    return launch_status();
}

}  // extern "C"
