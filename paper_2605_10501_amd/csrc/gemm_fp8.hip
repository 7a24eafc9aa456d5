// Products in 8-bit floating point with a power-of-two scale for each block of 128 (fp8_quantize.h):
//   C[m, n] (+ residual) = sum over blocks b of 2^(ea[m, b] + ew[n / 128, b]) sum_{k in b} a[m, k] w[n, k]
// on v_mfma_scale_f32_16x16x128_f8f6f4, whose contraction is one block deep and which takes both exponents as operands: a block's scale costs
// no vector instruction, and the sum stays in the fp32 accumulator.  (The instruction has a scale per 32; the four of a block are
// the same byte.  With all of them equal, any permutation of a block's k that both operands share gives the same result.)
//
// The weights are the instruction's row operand, so that a lane ends up with four consecutive outputs n of one token m.  Weight
// rows are dealt to a wave's NI fragment blocks so that those of all blocks join up: row r of block j is output 4 NI (r / 4) + 4 j + r % 4, and a
// lane holds 4 NI consecutive outputs, which leave in 16-byte stores straight from the accumulators.
// SwiGLU: half of the blocks are gate rows, the others the up rows of the same columns.
//
// Precision: the instruction sums eight consecutive k on a grid 2^-13 of the largest product's power of two and cuts off what lies below;
// the sums of eight are added in fp32 (measured with single products: a second one 2^-14 of the first is lost among the same eight, not
// among others).  On normal data that is 1.5e-5 of the result, a hundredth of the rounding to bf16, and results in bf16 and SwiGLU's codes
// are computed so unless the caller asks for more.  An fp32 result is computed on v_mfma_f32_16x16x32_bf16 instead, half the rate, from the codes
// widened to bf16 (exact): fp32 sums throughout; unless the caller asks for the fast ones.
//
//   * gemm_fp8_big_kernel: 256 tokens x 256 or 192 outputs, operands through LDS;
//   * gemm_fp8_ring_kernel: smaller tiles through LDS, for grids that do not fill the chip with the large ones, and fp32 results;
//   * gemm_fp8_direct_kernel: up to 64 tokens, fragments straight from global memory, K split over the waves of a workgroup.
// All but the last add up K in ascending order, one accumulator per output, so they give the same bits.
#include <atomic>
#include <utility>

#include "fp8_plan.h"
#include "fp8_quantize.h"
#include "launch.h"
#include "launch_plan.h"
#include "mfma_tiles.h"

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int kBlk = 128;             // K tile = scale block, in codes = bytes
constexpr int kPanel = 112, kSegment = 108;   // K tiles whose scales a workgroup has room for in LDS, and takes at a time

struct Fp8Params {
    const uint8_t *A, *sA, *W, *sW;
    long lda, ldsa, ldw, ldsw;
    void *C;
    const void *R;
    long ldc, ldr;
    int c_fp32, r_fp32, vec;          // vec: 16-byte accesses to C and R
    uint8_t *sC;                      // SwiGLU: scales of the codes in C
    long ldsc;
    int M, N, K, F;                   // N: weight rows; SwiGLU: N = 2 F
    int kb, tiles_m, tiles_n;
};

// W, A: which byte of sw, sa has the exponents
// The same with the accumulators bound to accumulation registers, where the compiler would copy them to and fro for a kernel that needs all 256.  It does
// not see what the instruction needs around it: whoever reads the sums waits first, and w, a, sw and sa are results of LDS reads as they come (a vector
// instruction's result needs two idle states before it; in front of every product they cost 2 %, so they stand at the head of a K tile only,
// where the compiler may put copies).  The build looks through the compiled kernels for what stands too close (mfma_check.py).
template <int W, int A> __device__ __forceinline__ void mfma_acc(const i32x8 &w, const i32x8 &a, f32x4 &c, int sw, int sa) {
    asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[%5,%6,0] op_sel_hi:[%7,%8,0]"
        : "+a"(c) : "v"(w), "v"(a), "v"(sw), "v"(sa), "n"(W & 1), "n"(A & 1), "n"(W >> 1), "n"(A >> 1));
}
template <int W, int A> __device__ __forceinline__ f32x4 mfma(const i32x8 &w, const i32x8 &a, const f32x4 &c, int sw, int sa) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, a, c, 0, 0, W, sw, A, sa);
}
// f(0), f(1), ... with the index as a constant
template <class F, int... I> __device__ __forceinline__ void each(std::integer_sequence<int, I...>, F f) { (f(std::integral_constant<int, I>{}), ...); }
template <int N, class F> __device__ __forceinline__ void each(F f) { each(std::make_integer_sequence<int, N>{}, f); }
// The same in fp32 sums: 8 k of each lane at a time.  (Codes times scale are bf16 numbers, subnormal ones among them, from 2^-124, of which 2^-9 is the
// smallest code's, to 2^119, of which 448 is the largest's.  Outside, a block would need a sum of its own that is scaled afterwards: that form
// beside this one took the 128 x 128 kernel from 202 to 425 registers, one workgroup per CU instead of two, for blocks below 2^-115 and above 3.29e38.)
__device__ __forceinline__ bf16x8 widen8(int a, int b, float scale) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false), q = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true);
    const bf16x2 u = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false), v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true);
    return bf16x8{p[0], p[1], q[0], q[1], u[0], u[1], v[0], v[1]};
}
__device__ __forceinline__ float scale_of(int byte) { return __uint_as_float((unsigned)(byte & 255) << 23); }
__device__ __forceinline__ i32x8 join(const i32x4 &lo, const i32x4 &hi) { return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7); }

// NV consecutive outputs of a row
template <int NV> __device__ __forceinline__ void store_row(const Fp8Params &p, int m, int n, float *v) {
    if (m >= p.M || n >= p.N) return;
    if (p.vec) {                                         // (N is a multiple of 16: all of them are there)
        if (p.R) {
            if (p.r_fp32) {
                const float4 *r = (const float4 *)((const float *)p.R + m * p.ldr + n);
#pragma unroll
                for (int q = 0; q < NV / 4; ++q) {
                    const float4 t = r[q];
                    v[4 * q] += t.x; v[4 * q + 1] += t.y; v[4 * q + 2] += t.z; v[4 * q + 3] += t.w;
                }
            } else {
#pragma unroll
                for (int q = 0; q < NV / 8; ++q) {
                    const Vec16<bf16_t> t = ldv((const bf16_t *)p.R + m * p.ldr + n + 8 * q);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[8 * q + e] += to_f32(t.v[e]);
                }
            }
        }
        if (p.c_fp32) {
            float4 *c = (float4 *)((float *)p.C + m * p.ldc + n);
#pragma unroll
            for (int q = 0; q < NV / 4; ++q) c[q] = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
        } else {
#pragma unroll
            for (int q = 0; q < NV / 8; ++q) {
                Vec16<bf16_t> t;
#pragma unroll
                for (int e = 0; e < 8; ++e) t.v[e] = from_f32<bf16_t>(v[8 * q + e]);
                stv((bf16_t *)p.C + m * p.ldc + n + 8 * q, t);
            }
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < NV; ++e) {
        if (n + e < p.N) {
            float f = v[e];
            if (p.R) f += p.r_fp32 ? ((const float *)p.R)[m * p.ldr + n + e] : to_f32(((const bf16_t *)p.R)[m * p.ldr + n + e]);
            if (p.c_fp32) ((float *)p.C)[m * p.ldc + n + e] = f;
            else ((bf16_t *)p.C)[m * p.ldc + n + e] = from_f32<bf16_t>(f);
        }
    }
}

// ------------------------------------------------------------------ up to 64 tokens
// 16 tokens x 16 NI weight rows per workgroup; wave w takes the K tiles w, w + 8, ...: together the waves read 1 KB pieces of the rows.
// D tiles are requested before the first is used.  The weights stream from HBM and bound it; a token row is read again by every
// workgroup, from L2.  us on cold weights, NI = 1 / 2 / 4: 4096 x 4096 5.3 / 6.3 / 9.7, 6144 x 4096 7.5 / 6.8 / 9.9, 22016 x 4096 19.1 / 18.6 / 26.4.
constexpr int kDirectWaves = 8;
template <int NI, int D, bool PRECISE>
__global__ __launch_bounds__(64 * kDirectWaves) void gemm_fp8_direct_kernel(Fp8Params p) {
    constexpr int COLS = 16 * NI, LDR = COLS + 4;
    __shared__ __align__(16) float red[kDirectWaves][16][LDR];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 15, g = lane >> 4;
    const int m0 = blockIdx.y * 16;
    const long n0 = (long)blockIdx.x * COLS;
    const long rows_w = p.N - n0 < COLS ? p.N - n0 : COLS, rows_a = p.M - m0 < 16 ? p.M - m0 : 16;
    const __amdgpu_buffer_rsrc_t rw = make_rsrc(p.W + n0 * p.ldw, (rows_w - 1) * p.ldw + p.K);
    const __amdgpu_buffer_rsrc_t ra = make_rsrc(p.A + (long)m0 * p.lda, (rows_a - 1) * p.lda + p.K);
    const uint8_t *sw_row = p.sW + n0 / kBlk * p.ldsw;                   // (a tile lies within one block of 128 rows)
    const uint8_t *sa_row = p.sA + (long)(m0 + (r < rows_a ? r : 0)) * p.ldsa;
    unsigned wo[NI];
#pragma unroll
    for (int j = 0; j < NI; ++j) {
        const int row = 4 * NI * (r >> 2) + 4 * j + (r & 3);
        wo[j] = row < rows_w ? (unsigned)(row * p.ldw + 16 * g) : kOob;
    }
    const unsigned ao = r < rows_a ? (unsigned)(r * p.lda + 16 * g) : kOob;
    f32x4 acc[NI];
#pragma unroll
    for (int j = 0; j < NI; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int kt = wave; kt < p.kb; kt += kDirectWaves * D) {
        i32x4 w[D][NI][2], a[D][2];
        int sa[D], sw[D];
#pragma unroll
        for (int u = 0; u < D; ++u) {
            const int t = kt + u * kDirectWaves;
            const bool in = t < p.kb;                                    // a tile past the end: zeros, scaled by 1
            const int k0 = in ? t * kBlk : 0;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const unsigned inv = in && k0 + 16 * g + 64 * h < p.K ? 0u : kOob;      // (K is a multiple of 16)
#pragma unroll
                for (int j = 0; j < NI; ++j) w[u][j][h] = (i32x4)__builtin_amdgcn_raw_buffer_load_b128(rw, (wo[j] + 64 * h) | inv, k0, 0);
                a[u][h] = (i32x4)__builtin_amdgcn_raw_buffer_load_b128(ra, (ao + 64 * h) | inv, k0, 0);
            }
            sw[u] = in ? sw_row[t] : 127;
            sa[u] = in && r < rows_a ? sa_row[t] : 127;
        }
#pragma unroll
        for (int u = 0; u < D; ++u) {
            if constexpr (PRECISE) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const bf16x8 x = widen8(a[u][q >> 1][2 * (q & 1)], a[u][q >> 1][2 * (q & 1) + 1], scale_of(sa[u]));
#pragma unroll
                    for (int j = 0; j < NI; ++j)
                        acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(w[u][j][q >> 1][2 * (q & 1)], w[u][j][q >> 1][2 * (q & 1) + 1], scale_of(sw[u])), x,
                                                                         acc[j], 0, 0, 0);
                }
            } else {
#pragma unroll
                for (int j = 0; j < NI; ++j) acc[j] = mfma<0, 0>(join(w[u][j][0], w[u][j][1]), join(a[u][0], a[u][1]), acc[j], sw[u], sa[u]);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < NI; ++j) *(f32x4 *)&red[wave][r][4 * NI * g + 4 * j] = acc[j];
    __syncthreads();
    if (tid < 16 * COLS) {
        const int ml = tid / COLS, nl = tid % COLS;
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < kDirectWaves; ++w) s += red[w][ml][nl];
        const long m = m0 + ml, n = n0 + nl;
        if (m < p.M && n < p.N) {
            if (p.R) s += p.r_fp32 ? ((const float *)p.R)[m * p.ldr + n] : to_f32(((const bf16_t *)p.R)[m * p.ldr + n]);
            if (p.c_fp32) ((float *)p.C)[m * p.ldc + n] = s;
            else ((bf16_t *)p.C)[m * p.ldc + n] = from_f32<bf16_t>(s);
        }
    }
}

// ------------------------------------------------------------------ operands through LDS
// An LDS tile row is the 128 codes of a block, eight 16-byte pieces in the swizzled order of mfma_tiles.h.  A fragment is the pieces g and
// 4 + g of a row (g = lane / 16) for both operands.
__device__ __forceinline__ int piece_off(int row, int piece) { return row * kBlk + (swz(row, piece) << 4); }

// Byte offset of LDS row 8 lg + lr of a wave's NI weight blocks (lr = lane / 8, lg counts 8-row groups of the blocks): the lane's part and the group's
template <int NI> __device__ __forceinline__ int weight_row_lane(int lr) { return 4 * NI * (lr >> 2) + (lr & 3); }
template <int NI> __device__ __forceinline__ int weight_row_group(int lg) { return 8 * NI * (lg & 1) + 4 * (lg >> 1); }

// Scales of a workgroup's BM tokens and NW weight blocks for up to kPanel K tiles from tile t0 on.  pa: per K tile the bytes of the G fragment
// blocks that a wave works on together, side by side, for each of their 16 rows: one read gets a lane's scales.  Tiles past the end get 1: their codes
// arrive as zeros, and a scale may not turn those into NaN.
template <int BM, int G, int NW, int THREADS, class WBLK>
__device__ __forceinline__ void stage_scales(const Fp8Params &p, uint8_t *pa, uint8_t *pw, int m0, WBLK wblk, int t0, int nt, int tid) {
    const int words = (nt + 3) >> 2;                     // four K tiles each
    for (int i = tid; i < words * (BM + NW); i += THREADS) {
        const int row = i / words, q = i % words, t = t0 + 4 * q;
        unsigned v = 0x7f7f7f7fu;
        if (row < BM) {
            if (m0 + row < p.M) v = *(const unsigned *)(p.sA + (long)(m0 + row) * p.ldsa + t);
        } else {
            v = *(const unsigned *)(p.sW + (long)wblk(row - BM) * p.ldsw + t);
        }
        const int left = p.kb - t;
        if (left < 4) v = (v & ((1u << (8 * left)) - 1)) | (0x7f7f7f7fu << (8 * left));
        const int step = row < BM ? BM : NW;
        uint8_t *d = row < BM ? pa + 4 * q * BM + (row / (16 * G) * 16 + row % 16) * G + row / 16 % G : pw + 4 * q * NW + row - BM;
        d[0] = (uint8_t)v;
        d[step] = (uint8_t)(v >> 8);
        d[2 * step] = (uint8_t)(v >> 16);
        d[3 * step] = (uint8_t)(v >> 24);
    }
}

// Most calls want bf16 without a residual.  The kernels have that by itself: store_row's other forms, unrolled over the accumulators, are ten
// times the code, more than the instruction cache holds (256 x 256 tile, 32768 x 22016 x 4096: 2.60 ms with one form for all, 2.45 so).  Onto the fp32 stream, as
// a section's output and down projections go, a product reads and writes 8 bytes per output instead of 2, the reads with nothing beside them: 32768 x 4096 x 11008
// 1.10 ms in bf16, 1.18 into fp32, 1.28 onto an fp32 residual; 32768 x 4096 x 4096 0.45, 0.50, 0.65; 777 x 2048 x 5504 18.2 us, 20.9, 20.9.
__device__ __forceinline__ bool plain_rows(const Fp8Params &p) { return p.vec && !p.c_fp32 && !p.R; }
template <int NV> __device__ __forceinline__ void store_plain(const Fp8Params &p, int m, int n, const float *v) {
    if (m >= p.M || n >= p.N) return;
#pragma unroll
    for (int q = 0; q < NV / 8; ++q) {
        Vec16<bf16_t> t;
#pragma unroll
        for (int e = 0; e < 8; ++e) t.v[e] = from_f32<bf16_t>(v[8 * q + e]);
        stv((bf16_t *)p.C + m * p.ldc + n + 8 * q, t);
    }
}

// Which tile a workgroup has: each XCD (every eighth workgroup) works on a contiguous range of tiles, ordered in groups of `gm` rows of
// tiles x all columns, so that it shares operand panels in its L2
__device__ __forceinline__ void tile_of(const Fp8Params &p, int gm, int bm, int bn, int *m0, int *n0) {
    const int nb = gridDim.x, b = blockIdx.x, per = nb >> 3, rem = nb & 7, x = b & 7, q = b >> 3;
    const int pid = x * per + (x < rem ? x : rem) + q, width = gm * p.tiles_n;
    const int first = pid / width * gm, rows = p.tiles_m - first < gm ? p.tiles_m - first : gm;
    *m0 = (first + pid % width % rows) * bm;
    *n0 = pid % width / rows * bn;
}

// SwiGLU tile of 128 activation columns: the first half of the accumulator blocks is gate, the second up of the lane's 2 NJ consecutive columns; the
// tile's width is their scale block, so its maximum needs the wave columns' maxima (mx: LDS, [WN][BM])
template <int MI, int BM, int NJ, class ROW>
__device__ __forceinline__ void swiglu_epilogue(const Fp8Params &p, const f32x4 (&acc)[MI][NJ], unsigned *mx, int m0, int n0, int wn, int g, ROW row) {
    constexpr int NV = 2 * NJ, WN = kBlk / (4 * NV);     // a lane's consecutive columns, wave columns
    float v[MI][NV];
    const int n = n0 + wn * 4 * NV + NV * g;
#pragma unroll
    for (int i = 0; i < MI; ++i) {
        unsigned m = 0;
#pragma unroll
        for (int j = 0; j < NJ / 2; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[i][4 * j + e] = fp8_silu_mul(acc[i][j][e], acc[i][NJ / 2 + j][e]);
                m = max(m, __float_as_uint(v[i][4 * j + e]) & 0x7fffffffu);
            }
        if (__builtin_expect(__any(m >= 0x7f800000u), 0)) {
            m = 0;
#pragma unroll
            for (int e = 0; e < NV; ++e) m = max(m, fp8_finite_bits(v[i][e]));
        }
        m = max(m, (unsigned)__shfl_xor((int)m, 16, 64));
        m = max(m, (unsigned)__shfl_xor((int)m, 32, 64));
        if (g == 0) mx[wn * BM + row(i)] = m;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < MI; ++i) {
        const int ml = row(i), m = m0 + ml;
        unsigned most = mx[ml];
#pragma unroll
        for (int w = 1; w < WN; ++w) most = max(most, mx[w * BM + ml]);
        const int byte = fp8_scale_byte(most);
        const float is = fp8_inverse_scale(byte);
        if (m < p.M) {
            unsigned c[NV / 4];
#pragma unroll
            for (int q = 0; q < NV / 4; ++q) c[q] = fp8_pack4(v[i][4 * q] * is, v[i][4 * q + 1] * is, v[i][4 * q + 2] * is, v[i][4 * q + 3] * is);
            __builtin_memcpy(__builtin_assume_aligned((uint8_t *)p.C + (long)m * p.ldc + n, NV), c, NV);
            if (wn == 0 && g == 0) {
                const int b = n0 / kBlk, blocks = p.F / kBlk;
                uint8_t *s = p.sC + (long)m * p.ldsc + b;
                s[0] = (uint8_t)byte;
                if (b + 1 == blocks)
                    for (int q = blocks; q & 3; ++q) s[q - b] = 127;
            }
        }
    }
}

// Tile of 256 tokens x BN = 256 or 192 outputs: four waves, one per SIMD, wave tile 128 tokens x BN / 2 outputs as four quarters (token half, weight
// half).  At full load the chip's power bounds this kernel (a K tile of 256 x 256 takes 1.15 us on a few CUs, 1.5 us on all), so what counts is work
// per operand byte out of LDS: 128 KB of reads per K tile, where eight waves of 128 x 64 read 192 KB (32768 x 22016 x 4096 with SwiGLU 2.32 -> 2.24
// ms, 32768 x 4096 x 11008 1.13 -> 1.10).  Persistent workgroups that fetch the next tile behind their stores were no faster for the same reason.
//   * The quarters follow (A0 F)(A0 S)(A1 S)(A1 F), F / S = the weight half used first / second, which swap roles every K tile: one operand
//     half changes at a time.  The fragments of A0 are replaced by those of A1 one by one, each behind the last MFMAs that read it, A1's by
//     the next tile's A0; S is free in the last quarter, F in the first.
//   * An operand tile is two halves with an LDS slot each and two stages.  Two barriers per K tile, in the first and third quarters behind a
//     quarter of their MFMAs, when the reads before them are done; each hands over the slots that have been read, to loads of K tile t + 2, and
//     what has landed: every half is requested 1.5 K tiles before it is read, and the waits are for all but the youngest loads of a wave, those
//     of four halves.  Reads and loads are dealt out between the MFMAs: nothing else fills a SIMD's gaps.
//   * Half h of the weights is BN / 4 rows of either wave column; with SwiGLU gate and up.  A lane's outputs are 8 consecutive ones of every 32, so that
//     the four lanes of a row store 64 bytes side by side (scale blocks of 192-wide tiles' columns change between such 32, hence a scale byte
//     for each); with SwiGLU 16 consecutive ones, a byte each.
//   * BN = 192 is for last rounds that 256 leaves half empty: 4096 x 6144 x 4096 102 -> 89 us, 777 x 22016 x 4096 99 -> 84.
template <int BN, bool SWIGLU, bool TAIL>
__device__ __forceinline__ void fp8_big_body(const Fp8Params &p) {
    constexpr int NB = BN / 64, LOADS = 4 + NB;          // weight blocks of a quarter; a wave's loads of an A and a B half
    static_assert(BN % 64 == 0 && NB <= 4 && (!SWIGLU || BN == 256), "tile");
    constexpr int HA = 128 * kBlk, HB = BN / 2 * kBlk, NW = SWIGLU ? 4 : 8;       // (scales: gate, up and the same again: a word; or a byte per wave column and 32 outputs)
    __shared__ __align__(16) uint8_t A00[HA], A01[HA], A10[HA], A11[HA], B00[HB], B01[HB], B10[HB], B11[HB];
    __shared__ __align__(16) uint8_t pa[kPanel * 256], pw[kPanel * NW];
    const int tid = threadIdx.x, lane = tid & 63, lr = lane >> 3;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave >> 1, wn = wave & 1;
    int m0, n0;
    tile_of(p, 4, 256, SWIGLU ? 128 : BN, &m0, &n0);
    const long rows_a = p.M - m0 < 256 ? p.M - m0 : 256, rows_b = SWIGLU ? p.N - n0 : (p.N - n0 < BN ? p.N - n0 : BN);
    const __amdgpu_buffer_rsrc_t ra = make_rsrc(p.A + (long)m0 * p.lda, (rows_a - 1) * p.lda + p.K);
    const __amdgpu_buffer_rsrc_t rb = make_rsrc(p.W + (long)n0 * p.ldw, (rows_b - 1) * p.ldw + p.K);
    const int x = (lane & 7) ^ swz_row(lr);
    const unsigned lda = (unsigned)p.lda, ldw = (unsigned)p.ldw;
    // A wave fetches every fourth 8-row group of a half: 32 rows apart, so the lane's piece and its part of the offsets are the same in all
    const int piece = x ^ swz_row(8 * wave);
    const unsigned al = (unsigned)lr * lda + (piece << 4), bl = (unsigned)weight_row_lane<SWIGLU ? 4 : 2>(lr) * ldw + (piece << 4);
    const int nk = p.kb;
    int base = 0;                                        // first K tile of the panel of scales
    auto invalid = [&](int kt) __attribute__((always_inline)) {
        unsigned inv = kt < nk ? 0u : kOob;
        if (TAIL) inv |= kt * kBlk + piece * 16 < p.K ? 0u : kOob;
        return inv;
    };
    // request half h of K tile kt (a tile past the end arrives as zeros)
    auto load_a = [&](int kt, int h, int i, uint8_t *slot) __attribute__((always_inline)) {
        const int lg = wave + 4 * i;
        unsigned row = (unsigned)(h * 128 + lg * 8) * lda;
        asm volatile("" : "+s"(row));                    // (added in the loop: the sums would fill the lane's registers)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_void *)(slot + lg * 8 * kBlk), 16, (al + row) | invalid(kt), kt < nk ? kt * kBlk : 0, 0, 0);
    };
    auto load_b = [&](int kt, int h, int i, uint8_t *slot) __attribute__((always_inline)) {
        const int lg = wave + 4 * i, w = lg / (2 * NB), lw = lg % (2 * NB), block = h * NB + (lw >> 1);      // block: of the wave column
        unsigned row = (SWIGLU ? (unsigned)(h * p.F + w * 64 + weight_row_group<4>(lw)) : (unsigned)(w * (BN / 2) + (block >> 1) * 32 + weight_row_group<2>((block & 1) * 2 + (lw & 1)))) * ldw;
        asm volatile("" : "+s"(row));
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (lds_void *)(slot + lg * 8 * kBlk), 16, (bl + row) | invalid(kt), kt < nk ? kt * kBlk : 0, 0, 0);
    };
    auto fetch_a = [&](int kt, int h, uint8_t *slot) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) load_a(kt, h, i, slot);
    };
    auto fetch_b = [&](int kt, int h, uint8_t *slot) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NB; ++i) load_b(kt, h, i, slot);
    };

    f32x4 acc[8][2 * NB];                                     // [16-token block: 4 half + b][weight block]
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 2 * NB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    i32x8 af[4], bf[2 * NB];                                  // the present token half's blocks; weights
    int sa[2], sw = 0;                                   // scales: a byte for each of a token half's four blocks; of the weights (SwiGLU: gate, up; else per 32 outputs)
    int fo[2][2], fb[2][2];                              // [block parity][piece g / 4 + g]; of the wave's blocks of weights
    const int r16 = lane & 15, g = lane >> 4;
#pragma unroll
    for (int par = 0; par < 2; ++par)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            fo[par][q] = piece_off(par * 16 + r16, q * 4 + g) - par * 16 * kBlk;
            const int pb = (par + wn * NB) & 1;
            fb[par][q] = piece_off(pb * 16 + r16, q * 4 + g) - pb * 16 * kBlk;
        }
    auto frag = [&](const uint8_t *slot, int blk) __attribute__((always_inline)) {
        const uint8_t *s = slot + (wm * 64 + blk * 16) * kBlk;
        return join(*(const i32x4 *)(s + fo[blk & 1][0]), *(const i32x4 *)(s + fo[blk & 1][1]));
    };
    auto frag_b = [&](const uint8_t *slot, int blk) __attribute__((always_inline)) {
        const uint8_t *s = slot + (wn * NB + blk) * 16 * kBlk;
        return join(*(const i32x4 *)(s + fb[blk & 1][0]), *(const i32x4 *)(s + fb[blk & 1][1]));
    };
    auto read_b = [&](auto half, const uint8_t *slot) __attribute__((always_inline)) {
        constexpr int h = decltype(half)::value;
#pragma unroll
        for (int c = 0; c < NB; ++c) bf[NB * h + c] = frag_b(slot, c);
    };
    auto read_sa = [&](auto half, int kt) __attribute__((always_inline)) {
        constexpr int h = decltype(half)::value;
        sa[h] = *(const int *)(pa + (kt - base) * 256 + ((h * 2 + wm) * 16 + r16) * 4);
    };
    auto weight_scale = [&](int kt) __attribute__((always_inline)) -> int {
        return *(const int *)(pw + kt * NW + (SWIGLU ? 0 : wn * 4));
    };
    auto mul = [&](auto ah, auto bh, auto block, auto col) __attribute__((always_inline)) {
        constexpr int h = decltype(ah)::value, q = decltype(bh)::value, b = decltype(block)::value, c = decltype(col)::value;
        mfma_acc<SWIGLU ? q : (NB * q + c) / 2, b>(bf[NB * q + c], af[b], acc[4 * h + b][NB * q + c], sw, sa[h]);
        __builtin_amdgcn_sched_barrier(0);
    };
    auto mul_row = [&](auto ah, auto bh, auto block) __attribute__((always_inline)) { each<NB>([&](auto c) __attribute__((always_inline)) { mul(ah, bh, block, c); }); };
    auto hand_over = [&]() __attribute__((always_inline)) {
        __builtin_amdgcn_sched_barrier(0);
        wait_vmcnt_lgkm0<2 * LOADS>();
        lds_barrier();
        __builtin_amdgcn_sched_barrier(0);
    };
    using I0 = std::integral_constant<int, 0>;
    using I1 = std::integral_constant<int, 1>;
    using I2 = std::integral_constant<int, 2>;
    using I3 = std::integral_constant<int, 3>;
    // K tile kt (parity = fh = its first weight half) in stage slots a0, a1, f, s; nb / na: the next tile's first halves
    auto tile = [&](int kt, auto F, uint8_t *a0, uint8_t *a1, uint8_t *f, uint8_t *s, const uint8_t *nb, const uint8_t *na) __attribute__((always_inline)) {
        constexpr int fh = decltype(F)::value;
        using FH = std::integral_constant<int, fh>;
        using SH = std::integral_constant<int, 1 - fh>;
        asm volatile("s_nop 1");
        mul_row(I0{}, FH{}, I0{});
        hand_over();                                     // a0 and f have been read; a1 and s have landed
        each<3 * NB>([&](auto step) __attribute__((always_inline)) {
            constexpr int t = decltype(step)::value, l = t - (3 * NB - LOADS);
            mul(I0{}, FH{}, std::integral_constant<int, 1 + t / NB>{}, std::integral_constant<int, t % NB>{});
            if (t < NB) bf[NB * SH::value + t % NB] = frag_b(s, t % NB);
            if (t == NB) read_sa(I1{}, kt);
            if (l >= 0 && l < NB) load_b(kt + 2, fh, l, f);
            if (l >= NB) load_a(kt + 2, 0, l - NB, a0);
            __builtin_amdgcn_sched_barrier(0);
        });
        each<4>([&](auto b) __attribute__((always_inline)) {
            mul_row(I0{}, SH{}, b);
            af[b] = frag(a1, b);
            __builtin_amdgcn_sched_barrier(0);
        });
        mul_row(I1{}, SH{}, I0{});
        hand_over();                                     // a1 and s have been read; the next tile's first halves have landed
        int sw1 = 0;
        each<3 * NB>([&](auto step) __attribute__((always_inline)) {
            constexpr int t = decltype(step)::value;
            mul(I1{}, SH{}, std::integral_constant<int, 1 + t / NB>{}, std::integral_constant<int, t % NB>{});
            if (t == 0) read_sa(I0{}, kt + 1);
            if (t == 1) sw1 = weight_scale(kt + 1 - base);
            if (t < NB) load_b(kt + 2, 1 - fh, t, s);
            if (t >= NB && t < LOADS) load_a(kt + 2, 1, t - NB, a1);
            __builtin_amdgcn_sched_barrier(0);
        });
        each<4>([&](auto b) __attribute__((always_inline)) {
            each<NB>([&](auto c) __attribute__((always_inline)) {
                mul(I1{}, FH{}, b, c);
                if (b == 0) bf[NB * SH::value + c] = frag_b(nb, c);
            });
            af[b] = frag(na, b);
            __builtin_amdgcn_sched_barrier(0);
        });
        sw = sw1;
    };
    auto wblk = [&](int i) __attribute__((always_inline)) {
        if (SWIGLU) return i & 1 ? (p.F + n0) / kBlk : n0 / kBlk;
        const int n = n0 + (i >> 2) * (BN / 2) + (i & 3) * 32;
        return (n < p.N ? n : p.N - 1) / kBlk;
    };
    fetch_b(0, 0, B00); fetch_a(0, 0, A00); fetch_b(0, 1, B01); fetch_a(0, 1, A01);           // in the loop's order
    fetch_b(1, 1, B11); fetch_a(1, 0, A10); fetch_b(1, 0, B10); fetch_a(1, 1, A11);
    stage_scales<256, 4, NW, 256>(p, pa, pw, m0, wblk, 0, nk < kPanel ? nk : kPanel, tid);
    wait_vmcnt_lgkm0<3 * LOADS>();
    lds_barrier();
    read_b(I0{}, B00);
#pragma unroll
    for (int b = 0; b < 4; ++b) af[b] = frag(A00, b);
    read_sa(I0{}, 0);
    sw = weight_scale(0);
    for (int kt = 0; kt < nk; kt += 2) {                 // an odd count is rounded up with a tile of zeros
        if (kt - base == kSegment) {                     // the next panel of scales (this tile's first ones have been read from the old one, which goes further)
            base = kt;
            __syncthreads();
            stage_scales<256, 4, NW, 256>(p, pa, pw, m0, wblk, base, nk - base < kPanel ? nk - base : kPanel, tid);
            __syncthreads();
        }
        tile(kt, I0{}, A00, A01, B00, B01, B11, A10);
        tile(kt + 1, I1{}, A10, A11, B11, B10, B00, A00);
    }
    asm volatile("s_nop 15\n\ts_nop 15");               // the last products are there before anything reads them (the compiler does not see mfma_acc's latency)
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 2 * NB; ++j) asm volatile("" : "+a"(acc[i][j]));
    dma_publish_barrier();                               // what is still in flight must land before LDS is used again
    const int mrow = m0 + wm * 64 + r16;
    if constexpr (!SWIGLU) {
        auto rows = [&](auto store) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                int m = mrow + (i >> 2) * 128 + (i & 3) * 16;
                asm volatile("" : "+v"(m));              // (row after row: together their copies and conditions would not fit the registers)
#pragma unroll
                for (int j = 0; j < 2 * NB; ++j) asm volatile("" : "+a"(acc[i][j]));
#pragma unroll
                for (int q = 0; q < NB; ++q) {
                    float v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = acc[i][2 * q + (e >> 2)][e & 3];
                    store(m, n0 + wn * (BN / 2) + 32 * q + 8 * g, v);
                }
            }
        };
        if (plain_rows(p)) rows([&](int m, int n, float (&v)[8]) __attribute__((always_inline)) { store_plain<8>(p, m, n, v); });
        else rows([&](int m, int n, float (&v)[8]) __attribute__((always_inline)) { store_row<8>(p, m, n, v); });
    } else {
        swiglu_epilogue<8, 256>(p, acc, (unsigned *)A00, m0, n0, wn, g, [&](int i) { return wm * 64 + (i >> 2) * 128 + (i & 3) * 16 + r16; });
    }
}
template <int BN, bool SWIGLU, bool TAIL>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 1))) void gemm_fp8_big_kernel(Fp8Params p) { fp8_big_body<BN, SWIGLU, TAIL>(p); }

// Scheduling pattern: R LDS reads and V loads dealt to the first half of the MFMAs
template <int R, int V, int... I> __device__ __forceinline__ void spread_over_mfmas(std::integer_sequence<int, I...>) {
    constexpr int H = (int)sizeof...(I) / 2, RP = (R + H - 1) / H, VP = (V + H - 1) / H;
    ((__builtin_amdgcn_sched_group_barrier(0x008, 1, 0), I < H ? __builtin_amdgcn_sched_group_barrier(0x100, RP, 0) : (void)0,
      I < H ? __builtin_amdgcn_sched_group_barrier(0x020, VP, 0) : (void)0), ...);
}

// The tile template's LDS stages as objects of their own (mfma_tiles.h, FastLds in gemm.hip, on why)
template <int BM, int BN, int WM, int WN, int NST, bool SWIGLU, bool PRECISE>
__device__ __forceinline__ void fp8_ring_body(const Fp8Params &p) {
    constexpr int NW = WM * WN, THREADS = 64 * NW, NI = BN / WN / 16, MI = BM / WM / 16, LA = BM / 8 / NW, LB = BN / 8 / NW;
    constexpr int NB = BN > kBlk || SWIGLU ? 2 : 1;      // weight scale blocks of a tile
    static_assert(NST == 2 || NST == 4, "the parity of a K tile is that of its stage");
    static_assert(LA * 8 * NW == BM && LB * 8 * NW == BN && NI == 4 && (!SWIGLU || BN == 256), "tile and waves");
    constexpr bool RING = NST == 4;
    __shared__ __align__(16) uint8_t A0[BM * kBlk], A1[BM * kBlk], A2[RING ? BM * kBlk : 16], A3[RING ? BM * kBlk : 16];
    __shared__ __align__(16) uint8_t B0[BN * kBlk], B1[BN * kBlk], B2[RING ? BN * kBlk : 16], B3[RING ? BN * kBlk : 16];
    __shared__ __align__(16) uint8_t pa[kPanel * BM], pw[kPanel * NB];
    uint8_t *const As[4] = {A0, A1, A2, A3}, *const Bs[4] = {B0, B1, B2, B3};
    const int tid = threadIdx.x, lane = tid & 63, lr = lane >> 3, r16 = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / WN, wn = wave % WN;
    int m0, n0;
    tile_of(p, 8, BM, SWIGLU ? BN / 2 : BN, &m0, &n0);
    const long rows_a = p.M - m0 < BM ? p.M - m0 : BM, rows_b = SWIGLU ? p.N - n0 : (p.N - n0 < BN ? p.N - n0 : BN);
    const __amdgpu_buffer_rsrc_t ra = make_rsrc(p.A + (long)m0 * p.lda, (rows_a - 1) * p.lda + p.K);
    const __amdgpu_buffer_rsrc_t rb = make_rsrc(p.W + (long)n0 * p.ldw, (rows_b - 1) * p.ldw + p.K);
    const int x = (lane & 7) ^ swz_row(lr);
    const unsigned alane = (unsigned)(lr * p.lda), blane = (unsigned)(weight_row_lane<SWIGLU ? 2 : NI>(lr) * p.ldw);
    const unsigned lda = (unsigned)p.lda, ldw = (unsigned)p.ldw;
    int kt0 = 0, nk = 0;
    auto fetch = [&](int kt, uint8_t *as, uint8_t *bs) __attribute__((always_inline)) {
        const int soff = kt < nk ? (kt0 + kt) * kBlk : 0;
        auto invalid = [&](int piece) { return kt < nk && (kt0 + kt) * kBlk + piece * 16 < p.K ? 0u : kOob; };
#pragma unroll
        for (int i = 0; i < LA; ++i) {
            const int lg = wave * LA + i, piece = x ^ swz_row(8 * lg);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_void *)(as + lg * 8 * kBlk), 16, (alane + (unsigned)(lg * 8) * lda + (piece << 4)) | invalid(piece), soff, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < LB; ++i) {
            const int lg = wave * LB + i, piece = x ^ swz_row(8 * lg), w = lg / (2 * NI), lw = lg % (2 * NI);
            const unsigned row = SWIGLU ? (unsigned)((lw >> 2) * p.F + w * 32 + weight_row_group<2>(lw & 3)) : (unsigned)(w * 16 * NI + weight_row_group<NI>(lw));
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (lds_void *)(bs + lg * 8 * kBlk), 16, (blane + row * ldw + (piece << 4)) | invalid(piece), soff, 0, 0);
        }
    };
    f32x4 acc[MI][NI];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int arow = wm * MI * 16, brow = wn * NI * 16;
    auto piece_of = [&](const uint8_t *tile, int row, int q) __attribute__((always_inline)) { return *(const i32x4 *)(tile + piece_off(row + r16, q * 4 + g)); };
    // fragments and scales of a K tile, two sets: the next tile's are read while the matrix cores work on the present one
    i32x4 a[2][MI][2], b[2][NI][2];
    int sa[2], sw[2];                                    // (sa: a byte per token block, sw: SwiGLU: gate and up)
    using word = std::conditional_t<MI == 4, int, std::conditional_t<MI == 2, uint16_t, uint8_t>>;
    auto read = [&](auto parity, int kt, const uint8_t *as, const uint8_t *bs) __attribute__((always_inline)) {
        constexpr int par = decltype(parity)::value;
#pragma unroll
        for (int j = 0; j < NI; ++j) { b[par][j][0] = piece_of(bs, brow + j * 16, 0); b[par][j][1] = piece_of(bs, brow + j * 16, 1); }
#pragma unroll
        for (int i = 0; i < MI; ++i) { a[par][i][0] = piece_of(as, arow + i * 16, 0); a[par][i][1] = piece_of(as, arow + i * 16, 1); }
        sa[par] = *(const word *)(pa + kt * BM + (wm * 16 + r16) * MI);
        if (SWIGLU) sw[par] = *(const uint16_t *)(pw + kt * NB);
        else sw[par] = pw[kt * NB + (NB == 2 ? wn * 16 * NI / kBlk : 0)];
    };
    auto step = [&](auto parity) __attribute__((always_inline)) {
        constexpr int par = decltype(parity)::value;
        if constexpr (PRECISE) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                bf16x8 y[NI];
#pragma unroll
                for (int j = 0; j < NI; ++j) y[j] = widen8(b[par][j][q >> 1][2 * (q & 1)], b[par][j][q >> 1][2 * (q & 1) + 1], scale_of(sw[par]));
#pragma unroll
                for (int i = 0; i < MI; ++i) {
                    const bf16x8 v = widen8(a[par][i][q >> 1][2 * (q & 1)], a[par][i][q >> 1][2 * (q & 1) + 1], scale_of(sa[par] >> (8 * i)));
#pragma unroll
                    for (int j = 0; j < NI; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y[j], v, acc[i][j], 0, 0, 0);
                }
            }
        } else {
            each<MI>([&](auto block) __attribute__((always_inline)) {
                constexpr int i = decltype(block)::value;
                each<NI>([&](auto col) __attribute__((always_inline)) {
                    constexpr int j = decltype(col)::value;
                    acc[i][j] = mfma<SWIGLU && j >= NI / 2, i>(join(b[par][j][0], b[par][j][1]), join(a[par][i][0], a[par][i][1]), acc[i][j], sw[par], sa[par]);
                });
            });
        }
    };
    using I0 = std::integral_constant<int, 0>;
    using I1 = std::integral_constant<int, 1>;
    auto wblk = [&](int i) __attribute__((always_inline)) {
        return i == 0 ? n0 / kBlk : SWIGLU ? (p.F + n0) / kBlk : ((n0 / kBlk + 1) * kBlk < p.N ? n0 / kBlk + 1 : n0 / kBlk);
    };
    for (; kt0 < p.kb; kt0 += kSegment) {
        nk = p.kb - kt0 < kSegment ? p.kb - kt0 : kSegment;
#pragma unroll
        for (int k = 0; k < NST; ++k) fetch(k, As[k], Bs[k]);
        stage_scales<BM, MI, NB, THREADS>(p, pa, pw, m0, wblk, kt0, nk, tid);
        wait_vmcnt_lgkm0<(NST - 1) * (LA + LB)>();
        lds_barrier();
        read(I0{}, 0, A0, B0);
        for (int kt = 0; kt < nk; kt += NST) {           // rounded up with tiles of zeros: a single loop exit keeps the accumulators in place
#pragma unroll
            for (int k = 0; k < NST; ++k) {
                // the next tile has landed (own loads, then everybody's), and everybody has read this one: its stage takes new loads
                wait_vmcnt_lgkm0<(NST - 2) * (LA + LB)>();
                lds_barrier();
                __builtin_amdgcn_sched_barrier(0);
                constexpr int kn[4] = {1, NST == 2 ? 0 : 2, 3, 0};
                if (k & 1) read(I0{}, kt + k + 1, As[kn[k]], Bs[kn[k]]); else read(I1{}, kt + k + 1, As[kn[k]], Bs[kn[k]]);
                fetch(kt + k + NST, As[k], Bs[k]);
                if (k & 1) step(I1{}); else step(I0{});
                // the reads and loads between the MFMAs, spread over the first of them
                if constexpr (!PRECISE) spread_over_mfmas<2 * (MI + NI), LA + LB>(std::make_integer_sequence<int, MI * NI>{});
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        dma_publish_barrier();
    }
    if constexpr (!SWIGLU) {
        auto rows = [&](auto store) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                float v[4 * NI];
#pragma unroll
                for (int j = 0; j < NI; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[4 * j + e] = acc[i][j][e];
                store(m0 + arow + i * 16 + r16, n0 + brow + 4 * NI * g, v);
            }
        };
        if (plain_rows(p)) rows([&](int m, int n, float (&v)[4 * NI]) __attribute__((always_inline)) { store_plain<4 * NI>(p, m, n, v); });
        else rows([&](int m, int n, float (&v)[4 * NI]) __attribute__((always_inline)) { store_row<4 * NI>(p, m, n, v); });
    } else {
        swiglu_epilogue<MI, BM>(p, acc, (unsigned *)A0, m0, n0, wn, g, [&](int i) { return arow + i * 16 + r16; });
    }
}
template <int BM, int BN, int WM, int WN, int NST, bool SWIGLU, bool PRECISE>
__global__ __launch_bounds__(64 * WM * WN) void gemm_fp8_ring_kernel(Fp8Params p) { fp8_ring_body<BM, BN, WM, WN, NST, SWIGLU, PRECISE>(p); }

// (named here because the host pass does not define all launch stubs of templates that only the launchers below use)
#define MS_FP8_RING(BM, BN, WM, WN, NST)                                                    \
    template __global__ void gemm_fp8_ring_kernel<BM, BN, WM, WN, NST, false, false>(Fp8Params); \
    template __global__ void gemm_fp8_ring_kernel<BM, BN, WM, WN, NST, false, true>(Fp8Params)
MS_FP8_RING(128, 128, 2, 2, 2);
MS_FP8_RING(128, 128, 4, 2, 4);
MS_FP8_RING(64, 128, 2, 2, 2);
MS_FP8_RING(64, 128, 2, 2, 4);
MS_FP8_RING(64, 64, 4, 1, 4);
template __global__ void gemm_fp8_ring_kernel<128, 256, 2, 4, 2, true, false>(Fp8Params);
template __global__ void gemm_fp8_ring_kernel<64, 256, 2, 4, 2, true, false>(Fp8Params);
#undef MS_FP8_RING
template __global__ void gemm_fp8_big_kernel<256, false, false>(Fp8Params);
template __global__ void gemm_fp8_big_kernel<256, false, true>(Fp8Params);
template __global__ void gemm_fp8_big_kernel<192, false, false>(Fp8Params);
template __global__ void gemm_fp8_big_kernel<192, false, true>(Fp8Params);
template __global__ void gemm_fp8_big_kernel<256, true, false>(Fp8Params);
template __global__ void gemm_fp8_big_kernel<256, true, true>(Fp8Params);

bool aligned(const void *p, int to) { return ((uintptr_t)p & (to - 1)) == 0; }

ms_status check(const char *who, int M, int N, int K, const void *A, long lda, const void *sA, long ldsa, const void *W, long ldw, const void *sW, long ldsw) {
    if (!A || !sA || !W || !sW || M < 0 || N <= 0 || K <= 0) return ms_fail(MS_ERR_INVALID_ARG, "%s: null pointer or bad size", who);
    if (K % 16) return ms_fail(MS_ERR_UNSUPPORTED, "%s: K=%d is not a multiple of 16", who, K);
    const long words = (K + 511L) / 512 * 4;
    if (lda < K || ldw < K || ldsa < words || ldsw < words) return ms_fail(MS_ERR_SHAPE, "%s: a row stride is less than a row", who);
    if (lda % 16 || ldw % 16 || ldsa % 4 || ldsw % 4 || !aligned(A, 16) || !aligned(W, 16) || !aligned(sA, 4) || !aligned(sW, 4))
        return ms_fail(MS_ERR_UNSUPPORTED, "%s: codes must have 16-byte, scales 4-byte aligned rows", who);
    if (!ms_buffer_range_ok(256, K, lda, 1) || !ms_buffer_range_ok(256, K, ldw, 1)) return ms_fail(MS_ERR_UNSUPPORTED, "%s: rows are too far apart", who);
    return MS_OK;
}

template <int NI, bool PRECISE> void launch_direct(const Fp8Params &p, hipStream_t s) {
    // D = 4 where that requests no more tiles past the end than 2 does (4096 deep: 5.3 us against 6.1, 8960 deep 8.1 against 7.4)
    const int t = ms_cdiv(p.kb, kDirectWaves);
    const dim3 grid(ms_cdiv(p.N, 16 * NI), ms_cdiv(p.M, 16));
    if ((t + 3) / 4 * 2 == (t + 1) / 2) gemm_fp8_direct_kernel<NI, 4, PRECISE><<<grid, 64 * kDirectWaves, 0, s>>>(p);
    else gemm_fp8_direct_kernel<NI, 2, PRECISE><<<grid, 64 * kDirectWaves, 0, s>>>(p);
}
template <bool PRECISE> void launch_direct(const Fp8Params &p, hipStream_t s) {
    if (p.N <= 4096 && p.M <= 16) launch_direct<1, PRECISE>(p, s); else launch_direct<2, PRECISE>(p, s);
}
// tiles of a launch, or 0 if they do not fit one
int tiles_of(Fp8Params &p, int bm, int bn, int cols, int threads) {
    p.tiles_m = ms_cdiv(p.M, bm);
    p.tiles_n = ms_cdiv(cols, bn);
    const long tiles = (long)p.tiles_m * p.tiles_n;
    return ms_launch_fits(tiles, threads) ? (int)tiles : 0;
}
template <int BM, int BN, int WM, int WN, int NST, bool SWIGLU, bool PRECISE> bool launch_ring(Fp8Params &p, hipStream_t s) {
    const int tiles = tiles_of(p, BM, SWIGLU ? BN / 2 : BN, SWIGLU ? p.F : p.N, 64 * WM * WN);
    if (tiles) gemm_fp8_ring_kernel<BM, BN, WM, WN, NST, SWIGLU, PRECISE><<<tiles, 64 * WM * WN, 0, s>>>(p);
    return tiles != 0;
}
template <int BN, bool SWIGLU> bool launch_big(Fp8Params &p, hipStream_t s) {
    const int tiles = tiles_of(p, 256, SWIGLU ? 128 : BN, SWIGLU ? p.F : p.N, 256);
    if (tiles && p.K % kBlk) gemm_fp8_big_kernel<BN, SWIGLU, true><<<tiles, 256, 0, s>>>(p);
    else if (tiles) gemm_fp8_big_kernel<BN, SWIGLU, false><<<tiles, 256, 0, s>>>(p);
    return tiles != 0;
}

// The tile that measurements and tests ask for (0: by shape), as in ms_k_gemm_config
std::atomic<int> g_tile{0};

template <bool PRECISE> bool launch_tile(int tile, Fp8Params &p, hipStream_t s) {
    if (tile == F128) return launch_ring<128, 128, 2, 2, 2, false, PRECISE>(p, s);
    if (tile == F128R) return launch_ring<128, 128, 4, 2, 4, false, PRECISE>(p, s);
    if (tile == F64x128) return launch_ring<64, 128, 2, 2, 2, false, PRECISE>(p, s);
    if (tile == F64x128R) return launch_ring<64, 128, 2, 2, 4, false, PRECISE>(p, s);
    if (tile == F64) return launch_ring<64, 64, 4, 1, 4, false, PRECISE>(p, s);
    return false;
}
// rows: of the whole call, which may be a part of
ms_status launch_gemm(Fp8Params p, int rows, bool precise, hipStream_t s) {
    ProfScope ps(0, 2.0 * p.M * p.N * p.K, s);
    bool fits = true;
    const int forced = g_tile.load();
    if (forced ? forced == FDIRECT : fp8_direct(rows, p.N)) {
        fits = p.M <= kFp8DirectMost;
        if (fits && precise) launch_direct<true>(p, s);
        else if (fits) launch_direct<false>(p, s);
    } else {
        const int tile = forced && !(precise && (forced == F256 || forced == F192)) ? forced : precise ? fp8_choose(kFp8Precise, p.M, p.N, p.kb) : fp8_choose(kFp8Fast, p.M, p.N, p.kb);
        fits = !precise && tile == F256 ? launch_big<256, false>(p, s) : !precise && tile == F192 ? launch_big<192, false>(p, s) : precise ? launch_tile<true>(tile, p, s) : launch_tile<false>(tile, p, s);
    }
    if (!fits) return ms_fail(MS_ERR_UNSUPPORTED, "gemm_fp8: %d x %d is too large for one launch", p.M, p.N);
    MS_LAUNCH_CHECK();
    return MS_OK;
}

// SwiGLU in the epilogue: gate and up rows of a tile's columns have to lie in whole blocks of 128 weight rows
bool swiglu_fused(int M, int F, int K, long ldw) { return M > kFp8DirectRows && F % kBlk == 0 && ms_buffer_range_ok(2L * F, K, ldw, 1); }
bool launch_swiglu(Fp8Params &p, hipStream_t s) {
    const int forced = g_tile.load(), tile = forced ? forced : fp8_choose(kFp8Swiglu, p.M, p.N, p.kb);
    if (tile == F256 || tile == F192) return launch_big<256, true>(p, s);
    if (tile == F128 || tile == F128R) return launch_ring<128, 256, 2, 4, 2, true, false>(p, s);
    return launch_ring<64, 256, 2, 4, 2, true, false>(p, s);
}

}  // namespace

extern "C" ms_status ms_k_gemm_fp8_config(int32_t tile) {
    if (tile != 0 && tile != F256 && tile != F192 && tile != F128 && tile != F128R && tile != F64x128 && tile != F64x128R && tile != F64 && tile != FDIRECT)
        return ms_fail(MS_ERR_INVALID_ARG, "gemm_fp8_config: unknown tile %d", tile);
    g_tile = tile;
    return MS_OK;
}

extern "C" ms_status ms_k_gemm_fp8(int32_t M, int32_t N, int32_t K, const void *A, int64_t lda, const void *sA, int64_t ldsa, const void *W,
                                   int64_t ldw, const void *sW, int64_t ldsw, void *C, int64_t ldc, int32_t c_fp32, const void *residual,
                                   int64_t ldr, int32_t residual_fp32, void *stream) {
    if (M == 0) return MS_OK;
    MS_TRY(check("gemm_fp8", M, N, K, A, lda, sA, ldsa, W, ldw, sW, ldsw));
    if (!C || c_fp32 < 0 || c_fp32 > 3) return ms_fail(MS_ERR_INVALID_ARG, "gemm_fp8: null pointer or bad c_fp32");
    if (ldc < N || (residual && ldr < N)) return ms_fail(MS_ERR_SHAPE, "gemm_fp8: a row stride is less than a row");
    const bool f32 = c_fp32 == 1 || c_fp32 == 2, precise = c_fp32 & 1;
    const int ec = f32 ? 4 : 2, er = residual_fp32 ? 4 : 2;
    if (!aligned(C, ec) || (residual && !aligned(residual, er))) return ms_fail(MS_ERR_UNSUPPORTED, "gemm_fp8: C or residual is not aligned to its type");
    if (residual && !(residual == C && ldr == ldc && er == ec) && !ms_apart(C, ldc * ec, (long)N * ec, residual, ldr * er, (long)N * er, M))
        return ms_fail(MS_ERR_INVALID_ARG, "gemm_fp8: the residual is neither C nor apart from it");
    Fp8Params p = {};
    p.A = (const uint8_t *)A; p.sA = (const uint8_t *)sA; p.W = (const uint8_t *)W; p.sW = (const uint8_t *)sW;
    p.lda = lda; p.ldsa = ldsa; p.ldw = ldw; p.ldsw = ldsw;
    p.C = C; p.ldc = ldc; p.R = residual; p.ldr = ldr; p.c_fp32 = f32; p.r_fp32 = residual_fp32 != 0;
    p.vec = N % 16 == 0 && ldc * ec % 16 == 0 && aligned(C, 16) && (!residual || (ldr * er % 16 == 0 && aligned(residual, 16)));
    p.M = M; p.N = N; p.K = K; p.kb = ms_cdiv(K, kBlk);
    return launch_gemm(p, M, precise, (hipStream_t)stream);
}

extern "C" size_t ms_k_gemm_fp8_swiglu_scratch_bytes(int32_t M, int32_t F, int32_t K) {
    if (M <= 0 || F <= 0 || K <= 0) return 0;
    const int rows = swiglu_fused(M, F, K, K) && M > kFp8DirectRows ? kFp8DirectRows : M;       // never less than for fewer rows
    return ms_align_up((size_t)rows * 2 * F * sizeof(float));
}

extern "C" ms_status ms_k_gemm_fp8_swiglu(int32_t M, int32_t F, int32_t K, const void *A, int64_t lda, const void *sA, int64_t ldsa, const void *W,
                                          int64_t ldw, const void *sW, int64_t ldsw, void *q, int64_t ldq, void *scales, int64_t lds,
                                          void *scratch, size_t scratch_bytes, void *stream) {
    if (M == 0) return MS_OK;
    if (F <= 0 || F > 0x3fffffff) return ms_fail(MS_ERR_INVALID_ARG, "gemm_fp8_swiglu: bad size");
    MS_TRY(check("gemm_fp8_swiglu", M, 2 * F, K, A, lda, sA, ldsa, W, ldw, sW, ldsw));
    if (!q || !scales) return ms_fail(MS_ERR_INVALID_ARG, "gemm_fp8_swiglu: null pointer");
    if (F % 16) return ms_fail(MS_ERR_UNSUPPORTED, "gemm_fp8_swiglu: F=%d is not a multiple of 16", F);
    if (ldq < F || lds < (F + 511L) / 512 * 4) return ms_fail(MS_ERR_SHAPE, "gemm_fp8_swiglu: a row stride is less than a row");
    if (ldq % 16 || lds % 4 || !aligned(q, 16) || !aligned(scales, 4)) return ms_fail(MS_ERR_UNSUPPORTED, "gemm_fp8_swiglu: codes must have 16-byte, scales 4-byte aligned rows");
    Fp8Params p = {};
    p.A = (const uint8_t *)A; p.sA = (const uint8_t *)sA; p.W = (const uint8_t *)W; p.sW = (const uint8_t *)sW;
    p.lda = lda; p.ldsa = ldsa; p.ldw = ldw; p.ldsw = ldsw;
    p.M = M; p.N = 2 * F; p.K = K; p.F = F; p.kb = ms_cdiv(K, kBlk);
    hipStream_t s = (hipStream_t)stream;
    if (swiglu_fused(M, F, K, ldw)) {
        p.C = q; p.ldc = ldq; p.sC = (uint8_t *)scales; p.ldsc = lds;
        ProfScope ps(0, 4.0 * M * F * K, s);
        if (!launch_swiglu(p, s)) return ms_fail(MS_ERR_UNSUPPORTED, "gemm_fp8_swiglu: %d x %d is too large for one launch", M, F);
        MS_LAUNCH_CHECK();
        return MS_OK;
    }
    // Gate and up in fp32 first: the same numbers before the same activation.  As many rows at a time as the scratch has room for, which is all of
    // them unless only the weights' row stride keeps the call from the kernels above.
    const size_t row = (size_t)2 * F * sizeof(float), need = ms_k_gemm_fp8_swiglu_scratch_bytes(M, F, K);
    if (!scratch || scratch_bytes < need) return ms_fail(MS_ERR_WORKSPACE, "gemm_fp8_swiglu: scratch %zu < %zu bytes", scratch_bytes, need);
    if (!aligned(scratch, 16)) return ms_fail(MS_ERR_UNSUPPORTED, "gemm_fp8_swiglu: scratch must be 16-byte aligned");
    const size_t room = scratch_bytes / row;
    const int rows = room < (size_t)M ? (int)room : M;
    p.C = scratch; p.ldc = 2L * F; p.c_fp32 = 1; p.vec = 1;
    for (int m = 0; m < M; m += rows) {
        p.M = M - m < rows ? M - m : rows;
        p.A = (const uint8_t *)A + (long)m * lda;
        p.sA = (const uint8_t *)sA + (long)m * ldsa;
        MS_TRY(launch_gemm(p, M, false, s));
        MS_TRY(ms_k_swiglu_fp8(MS_F32, p.M, F, scratch, 2L * F, (uint8_t *)q + (long)m * ldq, ldq, (uint8_t *)scales + (long)m * lds, lds, stream));
        if (M - m <= rows) break;                        // (m + rows could pass 2^31)
    }
    return MS_OK;
}
