// The layer with its epilogue for any number of rows, and for experts with ragged
// rows:
//
//   y[r][n] = act(sum_k W[n][k] x[r][k] + bias[n]) * multiplier[r][n] + residual[r][n],
//   W[n][k] = sum_i 2^e[i][n][k / G] s_i[n][k].
#include <hip/hip_runtime.h>

#include "checks.h"
#include "gemm_matrix.h"
#include "linear.h"

namespace {

using sa_linear::Layer;

// What both entry points check of their sizes; rows of y, 0 allowed.  The kernels count
// activations in 16-byte words of 32 bits, and a grid has fewer than 2^32 threads: tiles
// of at least 32 x 32 outputs, 512 threads each.
int check_layer(int q, int N, int K, int group, int rows, int x_rows, int experts,
                int activation) {
    const int st = check_dims(q, N, K);
    if (st != SA_OK) return st;
    if (experts < 1 || experts > SA_MAX_EXPERTS || rows < 0 || rows > SA_MAX_ROWS || x_rows < 0 ||
        x_rows > SA_MAX_ROWS || (int64_t)x_rows * K > (int64_t)1 << 35 ||
        ((rows + 31) / 32 + (int64_t)experts) * (((int64_t)N + 31) / 32) >= (int64_t)1 << 23)
        return SA_ERR_SHAPE;
    if (activation < SA_ACT_NONE || activation > SA_ACT_SILU) return SA_ERR_SHAPE;
    if (group < 8 || (group & 7) || (K % group)) return SA_ERR_GROUP;
    return SA_OK;
}

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// One layer of 2 to kFewRows rows: the kernel with the least estimated time.  Measured (us,
// weights rotated over 320 MB): 4096x4096 q=3 4 rows 7.1 block-scaled, 12.1 panel; 16 rows
// 8.7 columns shared by waves, 12.0 panel; 8192x28672 q=3 8 rows 48 block-scaled, 64 panel.
constexpr int kFewRows = 64;

void run_few(const Layer& a, hipStream_t s) {
    sa_matrix_plan mx, split;
    const double panel = sa_panel::estimate(a);
    const double mx_us = a.rows <= 8 ? sa_mx::plan(a.q, a.N, a.K, a.G, a.rows, 0, &mx)
                                     : sa_matrix::kNever;
    const double split_us = sa_mfma::plan_split(a, &split);
    if (mx_us < split_us && mx_us < panel) sa_mx::launch(a, mx, s);
    else if (split_us < panel) sa_mfma::launch(a, split, s);
    else sa_panel::launch(a, s);
}

// Experts of a few rows and the others by kernels of their own, up to a mean of kFewMean rows.
// Measured (us, that kernel first, the panel kernel alone second; the rows spread evenly over
// the experts, and falling with the expert's rank): 8 experts 11008x4096 q=3 mean 2 60 and 87,
// 52 and 68; mean 4 60 and 82, 69 and 82; mean 5 99 and 82, 76 and 81; mean 8 104 and 82, 90
// and 82.  16 experts 4096x11008 q=2 mean 2 79 and 104, 81 and 75; mean 4 91 and 105, 115 and
// 104; mean 8 160 and 111, 142 and 122.  128 experts 768x2048 q=2 mean 4 43 and 52, 47 and 44.
// Small layers lose by it: 8 experts 1024x1024 q=3 mean 2 11.4 and 10.0, 15.4 and 10.2.
constexpr int kFewMean = 4;

int run(Layer& a, hipStream_t s) {
    if (a.offsets) {
        if (a.rows <= kFewMean * a.experts && sa_mx::launch_experts(a, s))
            a.few = sa_mx::kExpertRows;
        if (a.rows > a.few) sa_panel::launch(a, s);
    } else if (a.rows == 1 && a.G % 128 == 0) {
        sa_rows::launch(a, s);
    } else if (a.rows <= kFewRows && a.q <= 4 && a.G % 128 == 0) {
        run_few(a, s);
    } else {
        sa_panel::launch(a, s);
    }
    return launch_status();
}

}  // namespace

extern "C" {

SA_API int sa_shiftadd_gemm_epilogue(const uint16_t* x, const uint8_t* packed_bits,
                                     const int8_t* exps, int q, int N, int K, int group, int rows,
                                     const float* bias, int activation, const void* multiplier,
                                     const void* residual, int out_half, void* y, void* stream) {
    if (rows != 0 && (!x || !packed_bits || !exps || !y)) return SA_ERR_NULL;
    const int st = check_layer(q, N, K, group, rows, rows, 1, activation);
    if (st != SA_OK || rows == 0) return st;
    if (!aligned16(x) || !aligned16(packed_bits) || !aligned16(y) || !aligned16(multiplier) ||
        !aligned16(residual) || !aligned4(bias))
        return SA_ERR_ALIGN;
    Layer a = {x, packed_bits, exps, nullptr, nullptr, q, N, K, group, rows, rows, 1, 0,
               {bias, multiplier, residual, y, activation, out_half}};
    return run(a, reinterpret_cast<hipStream_t>(stream));
}

SA_API int sa_shiftadd_gemm_experts(const uint16_t* x, int x_rows, const int32_t* row_of,
                                    const int32_t* offsets, const uint8_t* packed_bits,
                                    const int8_t* exps, int q, int N, int K, int group,
                                    int experts, int slots, const float* bias, int activation,
                                    const void* multiplier, int out_half, void* y, void* stream) {
    if (slots != 0 && (!offsets || !packed_bits || !exps || !y)) return SA_ERR_NULL;
    const int st = check_layer(q, N, K, group, slots, x_rows, experts, activation);
    if (st != SA_OK) return st;
    if (!row_of && x_rows < slots) return SA_ERR_SHAPE;
    if (slots == 0 || x_rows == 0) return SA_OK;  // no slot has a row
    if (!x) return SA_ERR_NULL;
    if (!aligned16(x) || !aligned16(packed_bits) || !aligned16(y) || !aligned16(multiplier) ||
        !aligned4(bias) || !aligned4(row_of) || !aligned4(offsets))
        return SA_ERR_ALIGN;
    Layer a = {x, packed_bits, exps, row_of, offsets, q, N, K, group, slots, x_rows, experts,
               0, {bias, multiplier, nullptr, y, activation, out_half}};
    return run(a, reinterpret_cast<hipStream_t>(stream));
}

}  // extern "C"
