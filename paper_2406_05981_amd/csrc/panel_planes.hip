// The layer for many rows (panel.h) of 4 to 8 planes, groups of whole blocks of 128 columns:
// a file of its own, so that it compiles beside panel.hip.
#include "panel.h"

namespace sa_panel {

void launch_planes(const sa_linear::Layer& a, int ct, int kw, hipStream_t s) {
    Args pa = whole_args(a);
    const Form f = {ct, kw, 0, 0, 0, 0, 0, 0};
    if (a.q == 4) start_form<4, kWhole>(pa, f, s);
    else if (a.q <= 6) start_form<6, kWhole>(pa, f, s);
    else start_form<8, kWhole>(pa, f, s);
}

}  // namespace sa_panel
