// The layer with its epilogue, on one layer or on experts with ragged rows: what the
// kernels of linear.hip and panel.hip share.
#ifndef SHIFTADD_LINEAR_H
#define SHIFTADD_LINEAR_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "epilogue.h"
#include "keys.h"

namespace sa_linear {

struct Layer {
    const uint16_t* x;       // activations [x_rows][K]
    const uint8_t* packed;   // planes of the first layer
    const int8_t* exps;      // [q][N][K/G] of the first layer
    const int32_t* row_of;   // row of x of each row of y, or null: the row itself
    const int32_t* offsets;  // experts: rows of y of each; null: one layer, all rows
    int q, N, K, G;
    int rows;     // rows of y
    int x_rows;   // rows of x
    int experts;  // layers
    int few;      // experts of at most this many rows are left out
    sa_epi::Epilogue epi;
};

// The `tile`-th tile of `height` rows, counted over the experts' rows: whole tiles of all
// experts first, then those at their ends of more than half the height, then the others (the
// shortest run last).  Its expert and rows [first, end).  Every lane of a wave calls it;
// false past the last tile.
__device__ inline bool find_tile(const Layer& a, int height, int tile, int* expert, int* first,
                                 int* end) {
    if (!a.offsets) {
        *expert = 0;
        *first = tile * height;
        *end = a.rows;
        return *first < a.rows;
    }
    const int lane = threadIdx.x & 63;
    int before = 0;  // tiles counted
    for (int kind = 0; kind < 3; ++kind)
        for (int e0 = 0; e0 < a.experts; e0 += 64) {
            const int e = e0 + lane;
            int lo = 0, hi = 0;
            if (e < a.experts) {
                lo = imin(imax(a.offsets[e], 0), a.rows);
                hi = imin(imax(a.offsets[e + 1], lo), a.rows);
            }
            const int rows = hi - lo > a.few ? hi - lo : 0;
            const int rest = rows % height;
            const int tiles = kind == 0   ? rows / height
                              : kind == 1 ? (int)(2 * rest > height)
                                          : (int)(rest > 0 && 2 * rest <= height);
            if (kind) lo += rows - rest;
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

// The row of x of row `row` of y, or -1: none.
__device__ inline int source_row(const Layer& a, int row) {
    if (!a.row_of) return row;
    const int v = a.row_of[row];
    return v >= 0 && v < a.x_rows ? v : -1;
}

// Tiles of `height` rows that any split of the rows over the experts can have.
inline int64_t most_tiles(const Layer& a, int height) {
    if (!a.offsets) return ((int64_t)a.rows + height - 1) / height;
    const int64_t t = ((int64_t)a.rows + (int64_t)a.experts * (height - 1)) / height;
    return t < a.rows ? t : a.rows;
}

}  // namespace sa_linear

// One row of one layer, group % 128 == 0 (shiftadd.hip).
namespace sa_rows {
void launch(const sa_linear::Layer& a, hipStream_t s);
}  // namespace sa_rows

// 2 to 8 rows of one layer as `plan` says, and the experts of 1 to kExpertRows rows
// (false: not this layer); up to 4 planes, group % 128 == 0 (gemm_mx.hip).
namespace sa_mx {
constexpr int kExpertRows = 8;
void launch(const sa_linear::Layer& a, const sa_matrix_plan& plan, hipStream_t s);
bool launch_experts(const sa_linear::Layer& a, hipStream_t s);
}  // namespace sa_mx

// The kernel of a few rows whose waves share the columns, one layer, up to 4 planes,
// group % 128 == 0: estimated time (us) and call (gemm_mfma.hip).
namespace sa_mfma {
double plan_split(const sa_linear::Layer& a, sa_matrix_plan* plan);
void launch(const sa_linear::Layer& a, const sa_matrix_plan& plan, hipStream_t s);
}  // namespace sa_mfma

// Any rows, groups and planes (panel.hip).
namespace sa_panel {
double estimate(const sa_linear::Layer& a);  // us
void launch(const sa_linear::Layer& a, hipStream_t s);
}  // namespace sa_panel

#endif
