// A router's choice of experts and the sum of the experts' rows.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "checks.h"
#include "epilogue.h"
#include "keys.h"

namespace {

// ---------------------------------------------------------------- choice
//
// A token belongs to 16 lanes (up to 256 experts) or to a wave, each lane PER
// consecutive experts.  The k largest logits come one after the other: a maximum over
// the lanes, then the lowest expert that holds it.  Logits are compared as unsigned
// numbers of the same order; 0 stands for -inf, NaN and what was chosen before.
//
// The lists.  Tokens are dealt to at most kMaxBlocks workgroups in ranges of whole
// 32-token steps.  Each workgroup counts its choices by expert (k_choose); a second
// launch (k_place) adds up the counts of the workgroups before it and of all experts
// below, and gives every choice its place: a step's choices of an expert are one bit a
// token in a 32-bit mask, the place is the number of bits below.  Nothing depends on
// the order of atomics.  Up to kOneBlock tokens one workgroup does both.
//
// Bound by latency, not by its bytes: 8192 tokens of 128 experts, 8 choices, 11.3 us for two
// launches of 6 (a wave a token 16.5, lane exchanges through LDS 50); 4 tokens 2.7 us.
constexpr int kStep = 32;         // tokens of a step
constexpr int kMaxBlocks = 256;
constexpr int kThreads = 512;
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

// op over the 16 lanes of a row, or over the wave, in every lane: quads, halves of 8 and 16
// mirrored, then the rows in order.
template <int LANES, typename T, typename F>
__device__ inline T reduce(T v, F op) {
    auto moved = [&](auto control) {
        return __builtin_bit_cast(
            T, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), decltype(control)::value, 0xf, 0xf,
                                        true));
    };
    v = op(v, moved(std::integral_constant<int, 0xB1>{}));
    v = op(v, moved(std::integral_constant<int, 0x4E>{}));
    v = op(v, moved(std::integral_constant<int, 0x141>{}));
    v = op(v, moved(std::integral_constant<int, 0x140>{}));
    if constexpr (LANES == 64) {
        T r[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            r[i] = __builtin_bit_cast(
                T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 16 * i));
        v = op(op(r[0], r[1]), op(r[2], r[3]));
    }
    return v;
}

// Token t's choices by LANES lanes, this one `lane` of them: lane j < k returns the expert
// of choice j, or -1.  All lanes call it; live = false: no token.
template <int LANES, int PER>
__device__ inline int choose(const Route& a, int t, int lane, bool live) {
    const auto larger = [](uint32_t x, uint32_t y) { return max(x, y); };
    const auto smaller = [](int x, int y) { return min(x, y); };
    const auto plus = [](float x, float y) { return x + y; };
    const float* l = a.logits + (int64_t)t * a.experts;
    uint32_t o[PER];
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        const int e = PER * lane + p;
        o[p] = live && e < a.experts ? order_of(l[e]) : 0u;
    }
    uint32_t best = 0;
#pragma unroll
    for (int p = 0; p < PER; ++p) best = max(best, o[p]);
    uint32_t top = reduce<LANES>(best, larger);
    const float peak = top ? logit_of(top) : 0.0f;
    float total = 0.0f;
    if (!a.normalize) {
#pragma unroll
        for (int p = 0; p < PER; ++p)
            if (o[p]) total += expf(logit_of(o[p]) - peak);
        total = reduce<LANES>(total, plus);
    }
    int id = -1;
    uint32_t mine = 0;
    for (int j = 0; j < a.k; ++j) {
        // the lowest expert that holds it; none left: every expert is past the last
        int e = a.experts;
#pragma unroll
        for (int p = PER - 1; p >= 0; --p)
            if (top && o[p] == top) e = PER * lane + p;
        e = reduce<LANES>(e, smaller);
        if (lane == j && top) {
            id = e;
            mine = top;
        }
        best = 0;
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            o[p] = PER * lane + p == e ? 0u : o[p];
            best = max(best, o[p]);
        }
        top = reduce<LANES>(best, larger);
    }
    const float w = mine ? expf(logit_of(mine) - peak) : 0.0f;
    if (a.normalize) total = reduce<LANES>(w, plus);
    if (live && lane < a.k) {
        const int64_t i = (int64_t)t * a.k + lane;
        a.ids[i] = id;
        a.weights[i] = id < 0 ? 0.0f : w / total;
    }
    return live ? id : -1;
}

// The expert of this thread's choice in the step of tokens [s, t1), or -1.
static_assert(kStep * SA_MAX_CHOICES <= kThreads, "one choice a thread and step");
__device__ inline int choice_of(const Route& a, int s, int t1) {
    const int items = imin(kStep, t1 - s) * a.k;
    return (int)threadIdx.x < items ? a.ids[(int64_t)s * a.k + threadIdx.x] : -1;
}

// Places of the tokens [t0, t1): base[e] holds the first free slot of expert e, `e` this
// thread's choice of the first step.
__device__ inline void place(const Route& a, int t0, int t1, int e, int* base, uint32_t* mask) {
    const int t = (int)threadIdx.x / a.k;
    for (int s = t0; s < t1; s += kStep) {
        for (int i = threadIdx.x; i < a.experts; i += kThreads) mask[i] = 0u;
        __syncthreads();
        if (e >= 0) atomicOr(&mask[e], 1u << t);
        __syncthreads();
        if ((int)threadIdx.x < imin(kStep, t1 - s) * a.k) {
            int slot = -1;
            if (e >= 0) {
                slot = base[e] + __popc(mask[e] & ((1u << t) - 1u));
                a.row_of[slot] = s + t;
            }
            a.slot_of[(int64_t)s * a.k + threadIdx.x] = slot;
        }
        if (s + kStep >= t1) break;
        e = choice_of(a, s + kStep, t1);
        __syncthreads();
        for (int i = threadIdx.x; i < a.experts; i += kThreads) base[i] += __popc(mask[i]);
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

template <int LANES, int PER, bool ALL>
__global__ __launch_bounds__(kThreads) void k_choose(Route a) {
    __shared__ int counts[LANES * PER];
    __shared__ int base[ALL ? LANES * PER : 1];
    __shared__ uint32_t mask[ALL ? LANES * PER : 1];
    for (int e = threadIdx.x; e < a.experts; e += kThreads) {
        counts[e] = 0;
        if constexpr (ALL) base[e] = 0;
    }
    __syncthreads();
    const int t0 = (int)blockIdx.x * a.per_block, t1 = imin(t0 + a.per_block, a.tokens);
    for (int s = t0; s < t1; s += kThreads / LANES) {
        const int t = s + (int)threadIdx.x / LANES;
        const int id = choose<LANES, PER>(a, imin(t, t1 - 1), (int)threadIdx.x % LANES, t < t1);
        if (id >= 0) atomicAdd(&counts[id], 1);
    }
    __syncthreads();
    if constexpr (ALL) {
        const int all = add_below(a.experts, counts, base, a.offsets);
        __syncthreads();
        place(a, 0, a.tokens, choice_of(a, 0, a.tokens), base, mask);
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
    const int t0 = (int)blockIdx.x * a.per_block, t1 = imin(t0 + a.per_block, a.tokens);
    const int first = choice_of(a, t0, t1);
    for (int e = threadIdx.x; e < a.experts; e += kThreads) base[e] = total[e] = 0;
    __syncthreads();
    // the threads of an expert share the workgroups' counts (integers: any order)
    const int shares = imax(1, kThreads / a.experts);
    for (int i = threadIdx.x; i < shares * a.experts; i += kThreads) {
        const int e = i % a.experts;
        int below = 0, all = 0;
#pragma unroll 16
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
    place(a, t0, t1, first, base, mask);
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

template <int LANES, int PER>
void launch_route(const Route& a, int blocks, hipStream_t s) {
    if (blocks == 1) {
        hipLaunchKernelGGL((k_choose<LANES, PER, true>), dim3(1), dim3(kThreads), 0, s, a);
        return;
    }
    hipLaunchKernelGGL((k_choose<LANES, PER, false>), dim3(blocks), dim3(kThreads), 0, s, a);
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
// requested at a time.  Bound by memory: 4095 tokens of 4 rows of 4096 in binary16 38 us,
// 5.1 TB/s (a device copy 4.9; one column a thread 110 us).
constexpr int kCols = 2048;

template <typename T>
__device__ inline void combine(const Combine& a, int64_t t, int64_t n) {
    typedef T vec_t __attribute__((ext_vector_type(8), aligned(sizeof(T))));
    const T* h = static_cast<const T*>(a.h);
    const int64_t at = t * a.N + n;
    const int count = a.N - n < 8 ? (int)(a.N - n) : 8;
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
    const int64_t n = (int64_t)(blockIdx.x % (unsigned)pieces) * kCols + 8 * threadIdx.x;
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
    if (experts <= 16) launch_route<16, 1>(a, blocks, s);
    else if (experts <= 64) launch_route<16, 4>(a, blocks, s);
    else if (experts <= 128) launch_route<16, 8>(a, blocks, s);
    else if (experts <= 256) launch_route<16, 16>(a, blocks, s);
    else if (experts <= 512) launch_route<64, 8>(a, blocks, s);
    else launch_route<64, 16>(a, blocks, s);
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
