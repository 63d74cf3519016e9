// The layer for many rows (panel.h) where the groups are not whole blocks of 128 columns or
// the columns end inside a block.
#include "panel.h"

namespace sa_panel {

void launch_groups(const sa_linear::Layer& a, int ct, int kw, hipStream_t s) {
    Args pa{};
    pa.a = a;
    pa.byte_offsets = (int64_t)a.x_rows * a.K < (int64_t)1 << 31;
    const Form f = {ct, kw, 0, 0, 0, 0, 0, 0};
    // the groups of a block begin at its first column
    if (a.G < 128 && 16 % (a.G / 8) == 0) {
        if (a.q <= 2) start_form<2, kPart>(pa, f, s);
        else if (a.q == 3) start_form<3, kPart>(pa, f, s);
        else if (a.q == 4) start_form<4, kPart>(pa, f, s);
        else start_form<8, kPart>(pa, f, s);
    } else if (a.q <= 4) {
        start_form<4, kAny>(pa, ct > 2 ? Form{2, 2, 0, 0, 0, 0, 0, 0} : f, s);
    } else {
        start_form<8, kAny>(pa, f, s);
    }
}

}  // namespace sa_panel
