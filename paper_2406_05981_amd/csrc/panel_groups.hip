// The layer for many rows (panel.h) whose groups are 8 to 64 columns, a power of two: a row's
// 16 keys and the 16 exponents from a block's first on load at once (4096x4096, 3 planes,
// group 64: 16 rows 57 -> 22 us, 1024 rows 222 -> 79 against a byte a chunk; k_gemm_generic
// 268 at 1 to 4 rows); what is left over group 128 (8.7 and 50 us) is a factor a chunk and step.
#include "panel.h"

namespace sa_panel {

// panel_chunks.hip
void launch_chunks(const sa_linear::Layer& a, int ct, int kw, hipStream_t s);

void launch_groups(const sa_linear::Layer& a, int ct, int kw, hipStream_t s) {
    // the groups of a block begin at its first column
    if (a.G >= 128 || 16 % (a.G / 8) != 0) {
        launch_chunks(a, ct, kw, s);
        return;
    }
    Args pa = other_args(a);
    const Form f = {ct, kw, 0, 0, 0, 0, 0, 0};
    if (a.q <= 2) start_form<2, kPart>(pa, f, s);
    else if (a.q == 3) start_form<3, kPart>(pa, f, s);
    else if (a.q == 4) start_form<4, kPart>(pa, f, s);
    else start_form<8, kPart>(pa, f, s);
}

}  // namespace sa_panel
