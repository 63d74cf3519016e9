// The layer for many rows (panel.h) with any other groups, or more than 2^22 columns: a key and
// an exponent byte a chunk.  A file of its own, so that it compiles beside panel_groups.hip.
#include "panel.h"

namespace sa_panel {

void launch_chunks(const sa_linear::Layer& a, int ct, int kw, hipStream_t s) {
    Args pa = other_args(a);
    const Form f = {ct, kw, 0, 0, 0, 0, 0, 0};
    if (a.q <= 4) start_form<4, kAny>(pa, ct > 2 ? Form{2, 2, 0, 0, 0, 0, 0, 0} : f, s);
    else start_form<8, kAny>(pa, f, s);
}

}  // namespace sa_panel
