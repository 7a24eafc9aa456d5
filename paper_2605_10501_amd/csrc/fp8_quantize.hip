// 8-bit operands: e4m3 codes and one power-of-two scale per block of 128 columns of a row (activations) or of 128 x 128 (weights),
// from a matrix as it is, from RMSNorm and from SwiGLU.  HBM bounds all of them: each element is read once and its code written
// once; norm and activation are evaluated in registers and rounded only to their codes.
// A wave's step is 512 columns of a row: 8 per lane, 16 lanes per block, four blocks, whose scales leave as one word.
#include "fp8_quantize.h"
#include "launch.h"
#include "launch_plan.h"

namespace {

// SWIGLU: x holds [gate | up] of k columns each and silu(gate) * up is quantised
template <class T, bool SWIGLU>
__global__ __launch_bounds__(256) void fp8_rows_kernel(const T *__restrict__ x, long ldx, uint8_t *__restrict__ q, long ldq, uint8_t *__restrict__ s, long lds,
                                                       int k, int groups, long steps) {
    const int lane = threadIdx.x & 63, blocks = (k + 127) >> 7;
    const long nw = (long)gridDim.x * 4;
    for (long st = (long)blockIdx.x * 4 + (threadIdx.x >> 6); st < steps; st += nw) {
        const long row = st / groups;
        const int g = (int)(st % groups), c = g * 512 + lane * 8;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = 0.f;
        if (c < k) {
            fp8_load8(x + row * ldx + c, v);
            if constexpr (SWIGLU) {
                float u[8];
                fp8_load8(x + row * ldx + k + c, u);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = fp8_silu_mul(v[e], u[e]);
            }
        }
        int byte;
        const uint2 w = fp8_quantize8(v, &byte);
        if (c < k) *(uint2 *)(q + row * ldq + c) = w;
        const unsigned sw = fp8_scale_word(byte, 4 * g + (lane >> 4), blocks);
        if (lane == 0) *(unsigned *)(s + row * lds + 4 * g) = sw;
    }
}

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
// Eight columns as they are stored
template <class T> struct Row8 { Vec16<T> h[8 / Vec16<T>::N]; };
template <class T> __device__ __forceinline__ Row8<T> load8(const T *p, bool there) {
    Row8<T> r = {};
    if (there) {
#pragma unroll
        for (int i = 0; i < 8 / Vec16<T>::N; ++i) r.h[i] = ldv(p + i * Vec16<T>::N);
    }
    return r;
}
template <class T> __device__ __forceinline__ void floats(const Row8<T> &r, float *v) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = to_f32(r.h[e / Vec16<T>::N].v[e % Vec16<T>::N]);
}

// RMSNorm, then the same: one wave per row, NC x 512 columns of it in registers as they are stored (wider rows are read again).  Latency bounds it
// (loads, the row's sum, the codes), so that what counts is how many waves fit: 4096 columns of bf16 in 63 registers (32768 rows 78 us, 5.2 TB/s;
// kept as floats in 90 it took 96), gains read again per row from L2 (held in registers across rows with the next row's loads, 208: 104).
template <class T, class TX, int NC>
__global__ __launch_bounds__(256) void norm_fp8_kernel(const TX *__restrict__ x, const T *__restrict__ g, uint8_t *__restrict__ q, long ldq,
                                                       uint8_t *__restrict__ s, long lds, int n, int d, float eps) {
    const int lane = threadIdx.x & 63, blocks = (d + 127) >> 7, groups = (blocks + 3) >> 2;
    const long row = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= n) return;
    const TX *xr = x + row * d;
    Row8<TX> v[NC];
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < NC; ++i) v[i] = load8(xr + i * 512 + lane * 8, i * 512 + lane * 8 < d);
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        float t[8];
        floats(v[i], t);
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = __builtin_fmaf(t[e], t[e], ss);
    }
    for (int c = NC * 512 + lane * 8; c < d; c += 512) {
        float t[8];
        fp8_load8(xr + c, t);
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = __builtin_fmaf(t[e], t[e], ss);
    }
    const float r = rsqrtf(wave_sum(ss) / d + eps);
    auto emit = [&](int i, float *t) {
        const int c = i * 512 + lane * 8;
        if (c < d) {
            float gv[8];
            fp8_load8(g + c, gv);
#pragma unroll
            for (int e = 0; e < 8; ++e) t[e] = t[e] * r * gv[e];
        }
        int byte;
        const uint2 w = fp8_quantize8(t, &byte);
        if (c < d) *(uint2 *)(q + row * ldq + c) = w;
        const unsigned sw = fp8_scale_word(byte, 4 * i + (lane >> 4), blocks);
        if (lane == 0) *(unsigned *)(s + row * lds + 4 * i) = sw;
    };
#pragma unroll
    for (int i = 0; i < NC; ++i)
        if (i < groups) {
            float t[8];
            if constexpr (sizeof(TX) == 2) {             // (unpacked again: as floats they would take twice the registers)
                u32x4 raw = __builtin_bit_cast(u32x4, v[i].h[0]);
                asm("" : "+v"(raw));
                v[i].h[0] = __builtin_bit_cast(Vec16<TX>, raw);
            }
            floats(v[i], t);
            emit(i, t);
        }
    for (int i = NC; i < groups; ++i) {
        float t[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] = 0.f;
        if (i * 512 + lane * 8 < d) fp8_load8(xr + i * 512 + lane * 8, t);
        emit(i, t);
    }
}

// 128 x 128 blocks: one workgroup each, the block in registers between its maximum and its codes, which leave non-temporally (22016 x 4096 53.1 ->
// 51.6 us, 5.2 TB/s, 4096 x 11008 30.4 -> 26.6; rows, which a product reads next, are 2 % slower so)
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
template <class T>
__global__ __launch_bounds__(256) void fp8_blocks_kernel(const T *__restrict__ x, long ldx, uint8_t *__restrict__ q, long ldq, uint8_t *__restrict__ s, long lds,
                                                         int n, int k) {
    __shared__ unsigned red[4];
    const int tid = threadIdx.x, blocks = (k + 127) >> 7, kb = blockIdx.x % blocks;
    const long rb = blockIdx.x / blocks;
    const int c = kb * 128 + (tid & 15) * 8;
    float v[8][8];
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const long row = rb * 128 + i * 16 + (tid >> 4);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
        if (row < n && c < k) fp8_load8(x + row * ldx + c, v[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) m = max(m, fp8_finite_bits(v[i][e]));
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) m = max(m, (unsigned)__shfl_xor((int)m, o, 64));
    if ((tid & 63) == 0) red[tid >> 6] = m;
    __syncthreads();
    m = max(max(red[0], red[1]), max(red[2], red[3]));
    const int byte = fp8_scale_byte(m);
    const float is = fp8_inverse_scale(byte);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const long row = rb * 128 + i * 16 + (tid >> 4);
        if (row < n && c < k)
            __builtin_nontemporal_store(u32x2{fp8_pack4(v[i][0] * is, v[i][1] * is, v[i][2] * is, v[i][3] * is),
                                              fp8_pack4(v[i][4] * is, v[i][5] * is, v[i][6] * is, v[i][7] * is)}, (u32x2 *)(q + row * ldq + c));
    }
    const int last = kb + 1 == blocks ? (blocks + 3) / 4 * 4 : kb + 1;       // the row's padding gets 127
    if (tid < last - kb) s[rb * lds + kb + tid] = (uint8_t)(tid == 0 ? byte : 127);
}

bool aligned(const void *p, int to) { return ((uintptr_t)p & (to - 1)) == 0; }

ms_status check(const char *who, int dtype, long n, long k, long es, const void *x, long ldx, const void *q, long ldq, const void *s, long lds) {
    if (dtype != MS_BF16 && dtype != MS_F32) return ms_fail(MS_ERR_INVALID_ARG, "%s: bad dtype %d", who, dtype);
    if (!x || !q || !s || n < 0 || k <= 0) return ms_fail(MS_ERR_INVALID_ARG, "%s: null pointer or bad size", who);
    if (k % 16) return ms_fail(MS_ERR_UNSUPPORTED, "%s: %ld columns, not a multiple of 16", who, k);
    if (ldx < k || ldq < k || lds < (k + 511) / 512 * 4) return ms_fail(MS_ERR_SHAPE, "%s: a row stride is less than a row", who);
    if (ldx * es % 16 || ldq % 16 || lds % 4 || !aligned(x, 16) || !aligned(q, 16) || !aligned(s, 4))
        return ms_fail(MS_ERR_UNSUPPORTED, "%s: rows and codes must be 16-byte, scales 4-byte aligned", who);
    return MS_OK;
}

}  // namespace

extern "C" ms_status ms_k_fp8_quantize(int32_t dtype, int32_t block_rows, int32_t n, int32_t k, const void *x, int64_t ldx, void *q, int64_t ldq,
                                       void *scales, int64_t lds, void *stream) {
    if (n == 0) return MS_OK;
    const int es = dtype == MS_BF16 ? 2 : 4;
    MS_TRY(check("fp8_quantize", dtype, n, k, es, x, ldx, q, ldq, scales, lds));
    if (block_rows != 1 && block_rows != 128) return ms_fail(MS_ERR_INVALID_ARG, "fp8_quantize: blocks of %d rows (1 or 128)", block_rows);
    hipStream_t s = (hipStream_t)stream;
    ProfScope ps(11, (double)n * k * (es + 1), s);
    if (block_rows == 1) {
        const int groups = ms_cdiv(k, 512);
        const long steps = (long)n * groups, wg = (steps + 3) / 4;
        const int grid = (int)(wg < (1 << 22) ? wg : (1 << 22));
        if (dtype == MS_BF16) fp8_rows_kernel<bf16_t, false><<<grid, 256, 0, s>>>((const bf16_t *)x, ldx, (uint8_t *)q, ldq, (uint8_t *)scales, lds, k, groups, steps);
        else fp8_rows_kernel<float, false><<<grid, 256, 0, s>>>((const float *)x, ldx, (uint8_t *)q, ldq, (uint8_t *)scales, lds, k, groups, steps);
    } else {
        const long wg = (long)ms_cdiv(n, 128) * ms_cdiv(k, 128);
        if (!ms_launch_fits(wg, 256)) return ms_fail(MS_ERR_UNSUPPORTED, "fp8_quantize: %d x %d has too many blocks for one launch", n, k);
        if (dtype == MS_BF16) fp8_blocks_kernel<bf16_t><<<(int)wg, 256, 0, s>>>((const bf16_t *)x, ldx, (uint8_t *)q, ldq, (uint8_t *)scales, lds, n, k);
        else fp8_blocks_kernel<float><<<(int)wg, 256, 0, s>>>((const float *)x, ldx, (uint8_t *)q, ldq, (uint8_t *)scales, lds, n, k);
    }
    MS_LAUNCH_CHECK();
    return MS_OK;
}

extern "C" ms_status ms_k_norm_fp8(int32_t dtype, int32_t x_fp32, int32_t n, int32_t d, float eps, const void *x, const void *g, void *q, int64_t ldq,
                                   void *scales, int64_t lds, void *stream) {
    if (n == 0) return MS_OK;
    const bool xf = x_fp32 || dtype == MS_F32;
    MS_TRY(check("norm_fp8", dtype, n, d, xf ? 4 : 2, x, d, q, ldq, scales, lds));
    if (!g || !(eps >= 0.f)) return ms_fail(MS_ERR_INVALID_ARG, "norm_fp8: null gain or negative eps");
    if (!aligned(g, 16)) return ms_fail(MS_ERR_UNSUPPORTED, "norm_fp8: gains must be 16-byte aligned");
    if (!ms_launch_fits(ms_cdiv(n, 4), 256)) return ms_fail(MS_ERR_UNSUPPORTED, "norm_fp8: %d rows are too many for one launch", n);
    hipStream_t s = (hipStream_t)stream;
    ProfScope ps(4, (double)n * d * ((xf ? 4 : 2) + 1), s);
    const int nc = ms_cdiv(d, 512);
#define GO_NC(T, TX, NC) norm_fp8_kernel<T, TX, NC><<<ms_cdiv(n, 4), 256, 0, s>>>((const TX *)x, (const T *)g, (uint8_t *)q, ldq, (uint8_t *)scales, lds, n, d, eps)
#define GO(T, TX)                            \
    do {                                     \
        if (nc <= 1) GO_NC(T, TX, 1);        \
        else if (nc <= 2) GO_NC(T, TX, 2);   \
        else if (nc <= 4) GO_NC(T, TX, 4);   \
        else GO_NC(T, TX, 8);                \
    } while (0)
    if (dtype == MS_F32) GO(float, float);
    else if (xf) GO(bf16_t, float);
    else GO(bf16_t, bf16_t);
#undef GO
#undef GO_NC
    MS_LAUNCH_CHECK();
    return MS_OK;
}

extern "C" ms_status ms_k_swiglu_fp8(int32_t dtype, int32_t n, int32_t f, const void *gate_up, int64_t ldgu, void *q, int64_t ldq, void *scales,
                                     int64_t lds, void *stream) {
    if (n == 0) return MS_OK;
    const int es = dtype == MS_BF16 ? 2 : 4;
    MS_TRY(check("swiglu_fp8", dtype, n, f, es, gate_up, ldgu, q, ldq, scales, lds));
    if (ldgu < 2L * f) return ms_fail(MS_ERR_SHAPE, "swiglu_fp8: rows of %ld elements, less than gate and up of %d", (long)ldgu, f);
    hipStream_t s = (hipStream_t)stream;
    ProfScope ps(6, (double)n * f * (2 * es + 1), s);
    const int groups = ms_cdiv(f, 512);
    const long steps = (long)n * groups, wg = (steps + 3) / 4;
    const int grid = (int)(wg < (1 << 22) ? wg : (1 << 22));
    if (dtype == MS_BF16) fp8_rows_kernel<bf16_t, true><<<grid, 256, 0, s>>>((const bf16_t *)gate_up, ldgu, (uint8_t *)q, ldq, (uint8_t *)scales, lds, f, groups, steps);
    else fp8_rows_kernel<float, true><<<grid, 256, 0, s>>>((const float *)gate_up, ldgu, (uint8_t *)q, ldq, (uint8_t *)scales, lds, f, groups, steps);
    MS_LAUNCH_CHECK();
    return MS_OK;
}
