// Exports of csrc/fp8_plan.h for tests/test_fp8_plan.py
#include "fp8_plan.h"

template <size_t N> static double us_of(const Fp8Tile (&tiles)[N], int code, long m, long n, long kb) {
    for (const Fp8Tile &t : tiles)
        if (t.code == code) return fp8_tile_us(t, m, n, kb);
    return -1;
}

extern "C" int fp8_plan_tile(int kind, long m, long n, long kb) {
    return kind == 0 ? fp8_choose(kFp8Fast, m, n, kb) : kind == 1 ? fp8_choose(kFp8Precise, m, n, kb) : fp8_choose(kFp8Swiglu, m, n, kb);
}
extern "C" double fp8_plan_us(int kind, int code, long m, long n, long kb) {
    return kind == 0 ? us_of(kFp8Fast, code, m, n, kb) : kind == 1 ? us_of(kFp8Precise, code, m, n, kb) : us_of(kFp8Swiglu, code, m, n, kb);
}
extern "C" int fp8_plan_direct(long m, long n) { return fp8_direct(m, n); }
