// fp32 logits of many rows.  The fp32 product of small sections (gemm_f32_kernel) splits K over the waves of a 32 x 32 tile and reads its operands past LDS: made for a few hundred rows, 38 TFLOP/s at
// 30000 x 1024 x 128.  Here tiles of 64 x 64 or 128 x 128 go through LDS, and a wave has 32 x 32 or 64 x 64 of them: 84 TFLOP/s there (203 -> 93 us; the matrix unit alone would take 50),
// 2500 x 1024 x 128 25 -> 16 us, 1200 rows 15 -> 13.  Fewer tiles than CUs wait for their loads, K after K: 293 x 1024 x 256 9.5 us, 7.4 split over waves.  128 x 128 from two
// workgroups a CU on, which is what their LDS allows.  (Two tiles on their way in registers instead of one: no faster at 64, 4 % slower at 128.)
//
// v_mfma_f32_32x32x2_f32 (64 cycles of a SIMD) takes one float of each operand per lane, lanes 0 .. 31 the first k, 32 .. 63 the second.  Of eight k, the lower half of a wave takes
// 0 .. 3 and the upper 4 .. 7, so that an operand is one 16-byte read per lane for four instructions.  Every element has one accumulator, which for a long K
// is added to a total every 1024 k: the order of a sum depends on K only.
#include "common.h"
#include "head_f32.h"
#include "launch.h"
#include "launch_plan.h"

namespace {

constexpr int kDepth = 32;                           // k of a tile in LDS
constexpr int kChunk = 1024;                         // k of an accumulator (LONG)
constexpr int kLd = kDepth + 4;                      // floats of a row: sixteen lanes' 16 bytes of rows 144 bytes apart have different banks

struct F32Logits {
    const float *h, *w;
    float *z;
    long ldz;
    int rows, cols, d, tiles_n, tiles;
};

// BT rows of kDepth k, on their way from memory to LDS
template <int BT> struct Tile {
    static constexpr int kLoads = BT * kDepth / 4 / 256;
    float4 v[kLoads];
    __device__ __forceinline__ void fetch(const float *p, int row0, int rows, int k0, int d) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int q = threadIdx.x + 256 * i, row = row0 + q / (kDepth / 4), k = k0 + q % (kDepth / 4) * 4;
            v[i] = row < rows && k < d ? *(const float4 *)(p + (long)row * d + k) : make_float4(0.f, 0.f, 0.f, 0.f);        // (d is a multiple of eight)
        }
    }
    __device__ __forceinline__ void store(float *lds) const {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int q = threadIdx.x + 256 * i;
            *(float4 *)(lds + q / (kDepth / 4) * kLd + q % (kDepth / 4) * 4) = v[i];
        }
    }
};

template <int BT, bool LONG>
__global__ __launch_bounds__(256) void head_f32_logits_kernel(F32Logits p) {
    constexpr int W = BT / 64, kB = BT * kLd, kStage = 2 * kB;                   // a wave's blocks of 32 in either direction
    __shared__ __align__(16) float lds[2 * kStage];
    // neighbouring tiles, which share their rows of h, go to one XCD
    const int each = p.tiles >> 3, b0 = blockIdx.x, tile = b0 < each * 8 ? (b0 & 7) * each + (b0 >> 3) : b0;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m0 = tile / p.tiles_n * BT, n0 = tile % p.tiles_n * BT;
    const int wm = (wave >> 1) * 32 * W, wn = (wave & 1) * 32 * W, row = lane & 31, half = lane >> 5;
    f32x16 acc[W][W], total[LONG ? W : 1][LONG ? W : 1];
    auto clear = [&](auto &v) __attribute__((always_inline)) {
        for (auto &x : v)
            for (auto &y : x)
#pragma unroll
                for (int r = 0; r < 16; ++r) y[r] = 0.f;
    };
    clear(acc);
    clear(total);
    auto collect = [&]() __attribute__((always_inline)) {
        if constexpr (LONG) {
#pragma unroll
            for (int i = 0; i < W; ++i)
#pragma unroll
                for (int j = 0; j < W; ++j)
#pragma unroll
                    for (int r = 0; r < 16; ++r) total[i][j][r] += acc[i][j][r];
            clear(acc);
        }
    };
    Tile<BT> a, b;
    a.fetch(p.h, m0, p.rows, 0, p.d);
    b.fetch(p.w, n0, p.cols, 0, p.d);
    a.store(lds);
    b.store(lds + kB);
    __syncthreads();
    for (int k = 0, stage = 0; k < p.d; k += kDepth, stage ^= 1) {
        const bool more = k + kDepth < p.d;
        if (more) {
            a.fetch(p.h, m0, p.rows, k + kDepth, p.d);
            b.fetch(p.w, n0, p.cols, k + kDepth, p.d);
        }
        const float *la = lds + stage * kStage + (wm + row) * kLd + 4 * half, *lb = lds + stage * kStage + kB + (wn + row) * kLd + 4 * half;
#pragma unroll
        for (int kk = 0; kk < kDepth; kk += 8) {
            f32x4 x[W], y[W];
#pragma unroll
            for (int i = 0; i < W; ++i) x[i] = *(const f32x4 *)(la + 32 * i * kLd + kk);
#pragma unroll
            for (int j = 0; j < W; ++j) y[j] = *(const f32x4 *)(lb + 32 * j * kLd + kk);
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int i = 0; i < W; ++i)
#pragma unroll
                    for (int j = 0; j < W; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[i][c], y[j][c], acc[i][j], 0, 0, 0);
        }
        if (more) {                                                              // (the other stage was last read before the barrier that ended the step before this)
            a.store(lds + (stage ^ 1) * kStage);
            b.store(lds + (stage ^ 1) * kStage + kB);
        }
        if (LONG && (k & (kChunk - 1)) == kChunk - kDepth) collect();
        __syncthreads();
    }
    collect();
    // register r of a block: row 8 (r / 4) + 4 (lane / 32) + r % 4, column lane % 32
#pragma unroll
    for (int i = 0; i < W; ++i)
#pragma unroll
        for (int j = 0; j < W; ++j) {
            const int col = n0 + wn + 32 * j + row;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int m = m0 + wm + 32 * i + 8 * (r >> 2) + 4 * half + (r & 3);
                if (m < p.rows && col < p.cols) p.z[(long)m * p.ldz + col] = LONG ? total[LONG ? i : 0][LONG ? j : 0][r] : acc[i][j][r];
            }
        }
}

}  // namespace

bool head_f32_logits_tiled(long rows, long vocab) { return (rows + 63) / 64 * ((vocab + 63) / 64) >= 256; }

ms_status head_f32_logits(int rows, int cw, int d, const float *h, const float *w, float *z, long ldz, hipStream_t s) {
    const bool large = d <= kChunk && (long)ms_cdiv(rows, 128) * ms_cdiv(cw, 128) >= 512;       // (with totals 128 x 128 keeps one workgroup a CU: 93 -> 121 us in the first example)
    const int bt = large ? 128 : 64, tiles_n = ms_cdiv(cw, bt);
    const long tiles = (long)ms_cdiv(rows, bt) * tiles_n;
    if (!ms_launch_fits(tiles, 256)) return ms_fail(MS_ERR_UNSUPPORTED, "head: %d x %d logits in one launch", rows, cw);
    const F32Logits p = {h, w, z, ldz, rows, cw, d, tiles_n, (int)tiles};
    ProfScope ps(0, 2.0 * rows * cw * d, s);
    if (large) head_f32_logits_kernel<128, false><<<(unsigned)tiles, 256, 0, s>>>(p);
    else if (d <= kChunk) head_f32_logits_kernel<64, false><<<(unsigned)tiles, 256, 0, s>>>(p);
    else head_f32_logits_kernel<64, true><<<(unsigned)tiles, 256, 0, s>>>(p);
    MS_LAUNCH_CHECK();
    return MS_OK;
}
