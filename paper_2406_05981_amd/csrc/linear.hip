// The layer with its epilogue for any number of rows, and for experts with ragged
// rows:
//
//   y[r][n] = act(sum_k W[n][k] x[r][k] + bias[n]) * multiplier[r][n] + residual[r][n],
//   W[n][k] = sum_i 2^e[i][n][k / G] s_i[n][k].
#include <hip/hip_runtime.h>

#include "checks.h"
#include "epilogue.h"
#include "keys.h"

namespace {

using sa_epi::Epilogue;

struct Layer {
    const uint16_t* x;      // activations [x_rows][K]
    const uint8_t* packed;  // planes of the first layer
    const int8_t* exps;     // [q][N][K/G] of the first layer
    const int32_t* row_of;  // row of x of each row of y, or null: the row itself
    const int32_t* offsets; // experts: rows of y of each; null: one layer, all rows
    int q, N, K, G;
    int rows;     // rows of y
    int x_rows;   // rows of x
    int experts;  // layers
    Epilogue epi;
};

// The `tile`-th tile of `height` rows, counted over the experts' rows: its expert and
// rows [first, end).  Every lane of a wave calls it; false past the last tile.
__device__ inline bool find_tile(const Layer& a, int height, int tile, int* expert, int* first,
                                 int* end) {
    if (!a.offsets) {
        *expert = 0;
        *first = tile * height;
        *end = a.rows;
        return *first < a.rows;
    }
    const int lane = threadIdx.x & 63;
    int before = 0;  // tiles of the experts below e0
    for (int e0 = 0; e0 < a.experts; e0 += 64) {
        const int e = e0 + lane;
        int lo = 0, hi = 0;
        if (e < a.experts) {
            lo = imin(max(a.offsets[e], 0), a.rows);
            hi = imin(max(a.offsets[e + 1], lo), a.rows);
        }
        const int tiles = (hi - lo + height - 1) / height;
        int sum = tiles;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int v = __shfl_up(sum, d);
            if (lane >= d) sum += v;
        }
        const int total = __shfl(sum, 63);
        if (tile < before + total) {
            const int l = __builtin_ctzll(__ballot(tile < before + sum));
            const int f = __shfl(lo, l) + height * (tile - before - __shfl(sum - tiles, l));
            *expert = __builtin_amdgcn_readfirstlane(e0 + l);
            *first = __builtin_amdgcn_readfirstlane(f);
            *end = __builtin_amdgcn_readfirstlane(__shfl(hi, l));
            return true;
        }
        before += total;
    }
    return false;
}

// Tiles of `height` rows that any split of `rows` rows over the experts can have.
int64_t most_tiles(int rows, int experts, int height) {
    const int64_t t = ((int64_t)rows + (int64_t)experts * (height - 1)) / height;
    return t < rows ? t : rows;
}

constexpr int kThreads = 256;
constexpr int kRows = 8;

// One output column a thread, kRows rows of y: every chunk's signed sum is shifted
// by its factor and added.
__global__ __launch_bounds__(kThreads) void k_linear(Layer a, int cols) {
    int expert, first, end;
    if (!find_tile(a, kRows, (int)(blockIdx.x / (unsigned)cols), &expert, &first, &end)) return;
    const int n = (int)(blockIdx.x % (unsigned)cols) * kThreads + (int)threadIdx.x;
    if (n >= a.N) return;
    const int C = a.K >> 3, NG = a.K / a.G, gc = a.G >> 3;
    const uint8_t* packed = a.packed + (int64_t)expert * a.q * a.N * C;
    const int8_t* exps = a.exps + (int64_t)expert * a.q * a.N * NG;
    const int count = imin(kRows, end - first);
    int from[kRows];
    bool live[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const int row = first + imin(r, count - 1);
        const int v = a.row_of ? a.row_of[row] : row;
        live[r] = r < count && v >= 0 && v < a.x_rows;
        from[r] = live[r] ? v : 0;
    }
    float sum[kRows] = {};
    for (int c = 0; c < C; ++c) {
        float x[kRows][8];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const uint4 v = *reinterpret_cast<const uint4*>(a.x + (int64_t)from[r] * a.K + 8 * c);
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int j = 0; j < 8; ++j)
                x[r][j] = (float)__builtin_bit_cast(_Float16, (uint16_t)(w[j >> 1] >> (16 * (j & 1))));
        }
        for (int i = 0; i < a.q; ++i) {
            const uint32_t key = packed[layout_offset(i, n, c, a.N, C)];
            const int e = exps[((int64_t)i * a.N + n) * NG + c / gc];
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                float s = 0.0f;
#pragma unroll
                for (int j = 0; j < 8; ++j) s += (key >> j) & 1u ? x[r][j] : -x[r][j];
                sum[r] += ldexpf(s, e);
            }
        }
    }
    Epilogue epi = a.epi;
    if (epi.bias) epi.bias += (int64_t)expert * a.N;
#pragma unroll
    for (int r = 0; r < kRows; ++r)
        if (live[r]) sa_epi::finish(epi, (int64_t)(first + r) * a.N + n, n, sum[r]);
}

// What both entry points check of their sizes; rows of y, 0 allowed.
int check_layer(int q, int N, int K, int group, int rows, int activation) {
    const int st = check_dims(q, N, K);
    if (st != SA_OK) return st;
    if (rows < 0 || rows > SA_MAX_ROWS || (int64_t)rows * N > (int64_t)1 << 34) return SA_ERR_SHAPE;
    if (activation < SA_ACT_NONE || activation > SA_ACT_SILU) return SA_ERR_SHAPE;
    if (group < 8 || (group & 7) || (K % group)) return SA_ERR_GROUP;
    return SA_OK;
}

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

int run(const Layer& a, hipStream_t s) {
    const int64_t tiles = a.offsets ? most_tiles(a.rows, a.experts, kRows)
                                    : (a.rows + kRows - 1) / kRows;
    const int64_t cols = ((int64_t)a.N + kThreads - 1) / kThreads;
    hipLaunchKernelGGL(k_linear, dim3((unsigned)(cols * tiles)), dim3(kThreads), 0, s, a, (int)cols);
    return launch_status();
}

}  // namespace

extern "C" {

SA_API int sa_shiftadd_gemm_epilogue(const uint16_t* x, const uint8_t* packed_bits,
                                     const int8_t* exps, int q, int N, int K, int group, int rows,
                                     const float* bias, int activation, const void* multiplier,
                                     const void* residual, int out_half, void* y, void* stream) {
    if (rows != 0 && (!x || !packed_bits || !exps || !y)) return SA_ERR_NULL;
    const int st = check_layer(q, N, K, group, rows, activation);
    if (st != SA_OK || rows == 0) return st;
    if (!aligned16(x) || !aligned16(packed_bits) || !aligned16(y) || !aligned16(multiplier) ||
        !aligned16(residual) || !aligned4(bias))
        return SA_ERR_ALIGN;
    const Layer a = {x, packed_bits, exps, nullptr, nullptr, q, N, K, group, rows, rows, 1,
                     {bias, multiplier, residual, y, activation, out_half}};
    return run(a, reinterpret_cast<hipStream_t>(stream));
}

SA_API int sa_shiftadd_gemm_experts(const uint16_t* x, int x_rows, const int32_t* row_of,
                                    const int32_t* offsets, const uint8_t* packed_bits,
                                    const int8_t* exps, int q, int N, int K, int group,
                                    int experts, int slots, const float* bias, int activation,
                                    const void* multiplier, int out_half, void* y, void* stream) {
    if (slots != 0 && (!offsets || !packed_bits || !exps || !y)) return SA_ERR_NULL;
    const int st = check_layer(q, N, K, group, slots, activation);
    if (st != SA_OK) return st;
    if (experts < 1 || experts > SA_MAX_EXPERTS || x_rows < 0 || x_rows > SA_MAX_ROWS ||
        (!row_of && x_rows < slots))
        return SA_ERR_SHAPE;
    if (slots == 0 || x_rows == 0) return SA_OK;  // no slot has a row
    if (!x) return SA_ERR_NULL;
    if (!aligned16(x) || !aligned16(packed_bits) || !aligned16(y) || !aligned16(multiplier) ||
        !aligned4(bias) || !aligned4(row_of) || !aligned4(offsets))
        return SA_ERR_ALIGN;
    const Layer a = {x, packed_bits, exps, row_of, offsets, q, N, K, group, slots, x_rows, experts,
                     {bias, multiplier, nullptr, y, activation, out_half}};
    return run(a, reinterpret_cast<hipStream_t>(stream));
}

}  // extern "C"
