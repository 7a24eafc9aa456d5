// Which tile the gradients of an lm_head and its hidden states take, and in how many parts the latter are summed.  Plain C++ without HIP.
#pragma once
#include "launch_plan.h"

// Bytes of a matrix, with 256 rows more than it has, that the bf16 products reach by 32-bit offsets: what they read and what they write, which for gradients are fp32 numbers
constexpr long kHeadReach = (1L << 32) - (1L << 20);

// d_h [rows, d] = e w sums over the vocabulary, which is long, in few workgroups if there are few rows: 512 rows at d = 1536 are 12 tiles of 256 x 256 with 2374
// K tiles each, beside the 3564 short workgroups of d_w.  So the vocabulary is cut into parts, whose sums are added when d_h is rounded: as many as give the
// least time by the estimate of ms_choose_pair, plus what the parts cost to write and read (4.5 TB/s).  How many of the rows count is known on the device only, so it is the
// sum of the times for all of them and for half (chosen for all 8192 tokens of pairs half of which was scored, V = 151936: d_h in one part, 3.85 ms; now in two, 3.2).
// The parts' sums take 2^25 numbers at most (128 MB), so that the workspace grows with the rows.
constexpr long kHeadMostParts = 64, kHeadPartsRoom = 1L << 25;
struct HeadChoice { int tile, parts, wgrad_first; double us; };
inline double head_backward_us(int tile, long rows, long cw, long d, int parts, bool *wgrad_first) {
    const MsTile &t = kTiles[tile];
    const MsPairTimes &c = kPairTimes[tile];
    const int ktd = (int)((cw + 63) / 64), ktw = (int)((rows + 63) / 64);
    const long nd = ms_tiles(t, rows, d) * parts, nw = ms_tiles(t, cw, d), slots = 256L * t.per_cu;
    const double dd = (ktd + parts - 1) / parts * ms_ktile_us(c.d, t.per_cu, nd + nw) + c.us_round + c.us_out * 4 * t.bm * t.bn / 65536.0;
    const double dw = ktw * ms_ktile_us(c.w, t.per_cu, nd + nw) + c.us_round_w;
    *wgrad_first = dw > dd;
    return c.us_call + (dw > dd ? ms_two_kinds(slots, nw, dw, nd, dd) : ms_two_kinds(slots, nd, dd, nw, dw)) + c.us_c * 1e-6 * cw * d +
           8.0 * parts * rows * d / 4.5e6;
}
inline HeadChoice head_choose(long rows, long cw, long d, int forced) {
    const int ktd = (int)((cw + 63) / 64);
    HeadChoice best = {T128, 1, 0, 1e30};
    for (int i = 0; i < kNumTiles; ++i) {
        if (!ms_tile_allowed(i, forced, true)) continue;
        for (int parts = 1; parts <= kHeadMostParts && (parts == 1 || (ktd / parts >= 8 && parts * rows * d <= kHeadPartsRoom)); parts *= 2) {
            bool first = false, half_first = false;
            const double us = head_backward_us(i, (rows + 1) / 2, cw, d, parts, &half_first) + head_backward_us(i, rows, cw, d, parts, &first);
            const int per = (ktd + parts - 1) / parts;
            if (us < best.us) best = {i, (ktd + per - 1) / per, first, us};
        }
    }
    return best;
}

// The tile of the logits' product, by the same two numbers of rows
inline int head_logits_tile(long rows, long cw, int kt, double out_bytes, int forced) {
    int best = T256;
    double best_us = 1e30;
    for (int i = 0; i < kNumTiles; ++i) {
        if (!ms_tile_allowed(i, forced, true)) continue;
        double us = 0;
        for (int half = 0; half < 2; ++half) us += ms_tile_time(kTiles[i], kTiles[i].lin, ms_tiles(kTiles[i], half ? (rows + 1) / 2 : rows, cw), kt, out_bytes);
// (the estimate is of the two-stage kernel; here it is the ping-pong one, and the tile that gains most where a few of the rows do not count: 1031 tokens, 1000 of
        // which do, 1024 x 32000: 69 us, 85 with 128 x 128.  100 .. 4100 rows of that and of 1536 x 151936 that all count: the best of six tiles or 5 % behind, once 14)
        if (i == T256) us *= 0.9;
        if (us < best_us) best_us = us, best = i;
    }
    return best;
}
