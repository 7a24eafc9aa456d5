// Host-side choice of the workgroup tile of the 8-bit products.  Plain C++ without HIP, so that it can be compiled and checked without a GPU.
#pragma once
#include <stddef.h>

// Tile codes: token rows * 1000 + outputs, + 1 for the form with four LDS stages
enum { F256 = 256256, F128 = 128128, F128R = 128129, F64x128 = 64128, F64x128R = 64129, F64 = 64064, FDIRECT = 16016 };

// us_per_ktile: per K tile of 128 with one workgroup per CU, few and all CUs busy, then with two per CU, few and all CUs with a second one;
// us_round: prologue and epilogue of a round; us_call: once.  Fits to sweeps on MI355X with operands that have left the caches: 13 weight
// matrices (256 x 688 .. 22016 x 4096) x 21 token counts (24 .. 16384) for 8-bit sums, 7 x 13 for fp32 sums, 4 x 16 for SwiGLU; K tiles are rounded
// up to the kernel's stages.  The chosen tile is 0.3 % (fp32 sums 0.1, SwiGLU 0.1) slower than the best one in the mean, in 5 of the 428 cases
// more than 6 % (us: 300 x 22016 x 4096 62, best 50; 1500 x 11008 x 2048 with SwiGLU 61, best 57).  Each tile is the best one of some
// shapes: 256 x 256 of 60 of the 273, 128 x 128 of 43 and 35, 64 x 128 of 10 and 20, 64 x 64 of 105.
struct Fp8Tile { int code, bm, bn, per_cu, stages; double us_per_ktile[4], us_round, us_call; };
constexpr Fp8Tile kFp8Fast[] = {{F256, 256, 256, 1, 2, {1.12, 1.51, 0, 0}, 6.7, 0.0},          {F128, 128, 128, 2, 2, {0.564, 0.758, 0.829, 0.939}, 2.7, 1.6},
                                {F128R, 128, 128, 1, 4, {0.334, 0.483, 0, 0}, 2.6, 1.8},       {F64x128, 64, 128, 2, 2, {0.480, 0.598, 0.678, 0.715}, 1.0, 2.4},
                                {F64x128R, 64, 128, 1, 4, {0.296, 0.349, 0, 0}, 2.6, 1.6},     {F64, 64, 64, 2, 4, {0.183, 0.227, 0.377, 0.386}, 1.3, 2.1}};
constexpr Fp8Tile kFp8Precise[] = {{F128, 128, 128, 2, 2, {0.864, 1.217, 1.593, 1.812}, 3.6, 2.5}, {F128R, 128, 128, 1, 4, {0.707, 0.963, 0, 0}, 5.7, 1.7},
                                   {F64x128, 64, 128, 2, 2, {0.644, 0.855, 1.261, 1.094}, 2.4, 1.3}, {F64x128R, 64, 128, 1, 4, {0.524, 0.638, 0, 0}, 3.7, 1.9},
                                   {F64, 64, 64, 2, 4, {0.333, 0.432, 0.663, 0.663}, 1.9, 2.2}};
// (bn: weight rows, half of them gate rows)
constexpr Fp8Tile kFp8Swiglu[] = {{F256, 256, 256, 1, 2, {1.15, 1.44, 0, 0}, 9.0, 1.0}, {F128, 128, 256, 1, 2, {1.046, 1.082, 0, 0}, 2.7, 2.1},
                                  {F64x128, 64, 256, 1, 2, {0.786, 0.916, 0, 0}, 0.9, 2.6}};

// Estimated time (us): full rounds of the chip, then the rest
inline double fp8_tile_us(const Fp8Tile &t, long M, long N, long kb) {
    const long wgs = ((M + t.bm - 1) / t.bm) * ((N + t.bn - 1) / t.bn), slots = 256L * t.per_cu, full = wgs / slots, rest = wgs % slots;
    const double kt = (double)((kb + t.stages - 1) / t.stages * t.stages), *u = t.us_per_ktile;
    double us = t.us_call + full * (kt * u[2 * t.per_cu - 1] + t.us_round);
    if (rest > 256) us += kt * (u[2] + (u[3] - u[2]) * (rest - 256) / 256) + t.us_round;
    else if (rest > 0) us += kt * (u[0] + (u[1] - u[0]) * rest / 256) + t.us_round;
    return us;
}
template <size_t N> inline int fp8_choose(const Fp8Tile (&tiles)[N], long m, long n, long kb) {
    int best = 0;
    double us = 1e30;
    for (const Fp8Tile &t : tiles) {
        const double e = fp8_tile_us(t, m, n, kb);
        if (e < us) { us = e; best = t.code; }
    }
    return best;
}

// The kernel without tiles in LDS: up to 16 rows, and up to 64 while the workgroups are all there at once, because each 16 rows read the
// weights again (32 rows, us, without / with tiles: 4096 x 4096 8.5 / 9.6, 22016 x 4096 40 / 25)
constexpr int kFp8DirectRows = 64;
inline bool fp8_direct(long M, long N) { return M <= 16 || (M <= kFp8DirectRows && (M + 15) / 16 * ((N + 31) / 32) <= 256); }
