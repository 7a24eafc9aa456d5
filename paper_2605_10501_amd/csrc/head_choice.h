// Which tile the gradients of an lm_head and its hidden states take, and in how many parts the latter are summed.  Plain C++ without HIP.
#pragma once
#include "launch_plan.h"

// d_h [rows, d] = e w sums over the vocabulary, which is long, in few workgroups if there are few rows: 512 rows at d = 1536 are 12 tiles of 256 x 256 with 2374
// K tiles each, beside the 3564 short workgroups of d_w.  So the vocabulary is cut into parts, whose sums are added when d_h is rounded: as many as give the
// least time by the estimate of ms_choose_pair, plus what the parts cost to write and read (4.5 TB/s).
struct HeadChoice { int tile, parts, wgrad_first; double us; };
inline HeadChoice head_choose(long rows, long cw, long d, bool d_h, bool d_w) {
    const int ktd = (int)((cw + 63) / 64), ktw = (int)((rows + 63) / 64);
    HeadChoice best = {T128, 1, 0, 1e30};
    for (int i = 0; i < kNumTiles; ++i) {
        const MsTile &t = kTiles[i];
        const MsPairTimes &c = kPairTimes[i];
        const long nd = d_h ? ms_tiles(t, rows, d) : 0, nw = d_w ? ms_tiles(t, cw, d) : 0, slots = 256L * t.per_cu;
        for (int parts = 1; parts <= 64 && (parts == 1 || (d_h && ktd / parts >= 8)); parts *= 2) {
            const long wgs = nd * parts + nw;
            const double dd = (ktd + parts - 1) / parts * ms_ktile_us(c.d, t.per_cu, wgs) + c.us_round + c.us_out * 4 * t.bm * t.bn / 65536.0;
            const double dw = ktw * ms_ktile_us(c.w, t.per_cu, wgs) + c.us_round_w;
            const bool wf = dw > dd;
            const double us = c.us_call + (wf ? ms_two_kinds(slots, nw, dw, nd * parts, dd) : ms_two_kinds(slots, nd * parts, dd, nw, dw)) + (d_w ? c.us_c * 1e-6 * cw * d : 0.0) +
                              (d_h ? 8.0 * parts * rows * d / 4.5e6 : 0.0);
            const int per = (ktd + parts - 1) / parts;
            if (us < best.us) best = {i, (ktd + per - 1) / per, wf, us};
        }
    }
    return best;
}
