// The layer for many rows (panel.h): the choice of tiles, and layers whose groups are
// whole blocks of 128 columns.
#include "panel.h"

namespace sa_panel {

// panel_groups.hip
void launch_groups(const sa_linear::Layer& a, int ct, int kw, hipStream_t s);
// panel_planes.hip
void launch_planes(const sa_linear::Layer& a, int ct, int kw, hipStream_t s);

namespace {

// The estimates (us) are fitted to every form's time on 550 drawn layers of N 64..28672,
// K 128..28672, q 1..4, 2..8192 rows, weights rotated over 320 MB (5th and 95th percentile
// of estimate / measured 0.8 and 1.4): a base; a workgroup alone, per 128-column block of a
// share a fixed part and one per plane, and an end; rounds of workgroups over the CUs, the
// same, a partial round 0.7 of a whole one besides its share.  The form of least estimate
// takes 1.01 times the best form's time in the mean, 1.18 at the 99th percentile.  More
// than 4 planes (registers) and groups that are not multiples of 128 have fewer forms.
constexpr Form kForms[] = {{8, 1, 2.4, 0.0, 0.0, 2.57, 0.41, 15.5},
                           {4, 1, 0.0, 0.0, 0.0, 1.19, 0.43, 8.9},
                           {4, 2, 0.8, 0.0, 0.10, 1.45, 0.385, 5.2},
                           {2, 2, 2.6, 0.68, 0.03, 0.54, 0.49, 2.2},
                           {2, 4, 1.9, 0.0, 0.535, 1.07, 0.36, 2.1},
                           {1, 4, 2.7, 0.43, 0.39, 0.44, 0.35, 0.6},
                           {1, 8, 1.9, 0.64, 0.36, 0.96, 0.355, 1.5}};

// (blocks to groups by multiplication: up to 2^22 columns)
bool whole_groups(const Layer& a) { return a.G % 128 == 0 && a.K <= (1 << 22); }

// Row tiles of the largest form that fits the registers.
int most_row_tiles(const Layer& a) {
    if (a.q > 4) return 2;
    return whole_groups(a) ? 8 : 16 % imax(a.G / 8, 1) == 0 ? 4 : 2;
}

double choose(const Layer& a, const Form** best) {
    const int blocks = (a.K + 127) / 128;
    // rows of an expert, as if all had the same
    const int64_t per = a.offsets ? (a.rows + a.experts - 1) / a.experts : a.rows;
    double least = 1e30;
    for (const Form& f : kForms) {
        if (f.ct > most_row_tiles(a)) continue;
        const int64_t tall = (per + 32 * f.ct - 1) / (32 * f.ct) *
                             (a.offsets ? imin(a.experts, a.rows) : 1);
        const double r = (double)(tall * ((a.N + 256 / f.kw - 1) / (256 / f.kw))) / 256;
        const double rounds = 0.3 * r + 0.7 * (double)(int64_t)(r + 0.999999);
        const int steps = imin(2 * (((blocks + 1) / 2 + f.kw - 1) / f.kw), blocks);
        const double alone = steps * (f.alone + f.alone_q * a.q) + f.end;
        const double shared = rounds * (steps * (f.shared + f.shared_q * a.q) + f.end);
        const double us = f.base + (alone > shared ? alone : shared);
        if (us < least) {
            least = us;
            *best = &f;
        }
    }
    return least;
}

}  // namespace

double estimate(const Layer& a) {
    const Form* f;
    return choose(a, &f);
}

void launch(const Layer& a, hipStream_t s) {
    const Form* f;
    choose(a, &f);
    if (!whole_groups(a)) {
        launch_groups(a, f->ct, f->kw, s);
        return;
    }
    if (a.q > 3) {
        launch_planes(a, f->ct, f->kw, s);
        return;
    }
    Args pa = whole_args(a);
    switch (a.q) {
        case 1: start_form<1, kWhole>(pa, *f, s); break;
        case 2: start_form<2, kWhole>(pa, *f, s); break;
        default: start_form<3, kWhole>(pa, *f, s); break;
    }
}

}  // namespace sa_panel
