// Host-side choice of the workgroup tile of the 8-bit products.  Plain C++ without HIP, so that it can be compiled and checked without a GPU.
#pragma once
#include <stddef.h>

// Tile codes: token rows * 1000 + outputs, + 1 for the form with four LDS stages
enum { F256 = 256256, F192 = 256192, F128 = 128128, F128R = 128129, F64x128 = 64128, F64x128R = 64129, F64 = 64064, FDIRECT = 16016 };

// us_per_ktile: per K tile of 128 with one workgroup per CU, few and all CUs busy, then with two per CU, few and all CUs with a second one;
// us_round: prologue and epilogue of a round; us_call: once.  Fits to sweeps on MI355X with operands that have left the caches: 13 weight
// matrices (256 x 688 .. 22016 x 4096) x 21 token counts (24 .. 16384) for 8-bit sums, 7 x 13 for fp32 sums, 4 x 16 for SwiGLU, and 7 x 10 (896 x 4096 ..
// 22016 x 4096, 65 .. 6000 tokens) for the 256-row tiles of 8-bit sums; K tiles are rounded up to the kernel's stages.  Over those 70 the chosen tile is
// 0.1 % slower than the best tile (the kernel without tiles left out) in the mean and 5 % at most (before there was one of 192 outputs, which fills last rounds that the others leave
// half empty: 3.6 % and 48 %).  Each is the best one of some: 256 x 192 of 14 (4096 x 6144 x 4096: 89 us, 128 x 128 and 256 x 256 100), 256 x 256,
// 128 x 128 and its ring of 12 each, 64 x 64 of 13, the ring of 64 x 128 of 7; 64 x 128 with two stages of some of the larger sweep.
struct Fp8Tile { int code, bm, bn, per_cu, stages; double us_per_ktile[4], us_round, us_call; };
constexpr Fp8Tile kFp8Fast[] = {{F256, 256, 256, 1, 2, {1.04, 1.42, 0, 0}, 9.2, 0.1},          {F192, 256, 192, 1, 2, {0.80, 1.11, 0, 0}, 7.9, 0.0},
                                {F128, 128, 128, 2, 2, {0.564, 0.758, 0.829, 0.939}, 2.7, 1.6}, {F128R, 128, 128, 1, 4, {0.334, 0.483, 0, 0}, 2.6, 1.8},
                                {F64x128, 64, 128, 2, 2, {0.480, 0.598, 0.678, 0.715}, 1.0, 2.4},  {F64x128R, 64, 128, 1, 4, {0.296, 0.349, 0, 0}, 2.6, 1.6},
                                {F64, 64, 64, 2, 4, {0.183, 0.227, 0.377, 0.386}, 1.3, 2.1}};
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
// weights again (32 rows, us, without / with tiles: 4096 x 4096 8.5 / 9.6, 22016 x 4096 41 / 25).  Above 64 rows it is still the faster one for small
// matrices: 65 x 896 x 4096 9.2 / 10.5, 200 x 688 x 256 3.6 / 4.4, 600 x 688 x 256 4.9 / 4.5, in fp32 sums 293 x 256 x 688 3.8 / 7.0, 600 x 256 x 688 4.7 / 7.1; but there a row's bits
// would depend on how many share the call.
constexpr int kFp8DirectRows = 64;
constexpr int kFp8DirectMost = 65535 * 16;       // rows of a launch
inline bool fp8_direct(long M, long N) { return M <= 16 || (M <= kFp8DirectRows && (M + 15) / 16 * ((N + 31) / 32) <= 256); }
