// GEMM kernels of the section path.
//
// bf16: C = alpha * A(m,k) B(n,k) on the CDNA4 matrix cores, all four operand layouts.
//   * gemm_bf16_pp_kernel: workgroup tile 256 x 256 x 64, K-contiguous operands, two wave groups that take turns;
//   * gemm_bf16_fast_kernel: workgroup tile 256 x 256 x 64 (8 waves, wave tile 128 x 64, one workgroup per CU) or
//     128 x 128 x 64 (4 waves, two per CU) for grids that fill the chip, and 128 x 256, 128 x 128, 64 x 128 and 64 x 64
//     tiles with a ring of three or four LDS stages for grids that do not (launch_plan.h);
//     v_mfma_f32_16x16x32_bf16 by default (v_mfma_f32_32x32x16_bf16 selectable for the first two);
//   * every operand tile goes global -> LDS directly (buffer_load ... lds), two (or more) LDS buffers per operand, one
//     barrier per K tile; a K-contiguous operand lands as [rows][64] with the 16-byte chunk index XOR-swizzled (applied on the
//     global side of the load; the swizzle makes every fragment read pattern free of LDS bank conflicts), a K-major operand (weight gradients, input gradients) lands as a row tile and is read
//     through the transposing LDS load (ds_read_b64_tr_b16), so no layout needs a transposed copy;
//   * fragments are double-buffered in registers, LDS reads of the next k-step interleaved with the MFMAs;
//   * epilogues (bias, bf16 / fp32 residual, fp32 or bf16 output, accumulate, fused SwiGLU, fused KD statistics / dz)
//     pass the accumulators through the idle LDS buffers so that each lane stores 4 consecutive columns, with
//     non-temporal global accesses; split-K uses fp32 atomics;
//   * workgroup ids are remapped so that each XCD works on a contiguous range of tiles, ordered in groups of M-tiles
//     x all N-tiles, and shares operand panels in its L2;
//   * gemm_bf16_kernel is the register-staged, bounds-checked fallback (K not a multiple of 64 with a K-contiguous
//     operand, matrices of 4 GB and more).
// fp32: v_mfma_f32_16x16x4_f32 on 32 x 32 tiles with K split over the waves of a workgroup.
#include <stdlib.h>

#include <atomic>

#include "common.h"
#include "launch.h"
#include "launch_plan.h"
#include "gemm_bf16.h"

namespace {

template <int BM, int BN, bool TA, bool TB>
__global__ __launch_bounds__(256) void gemm_bf16_kernel(GemmParams p) {
    constexpr int WTM = BM / 2, WTN = BN / 2, MI = WTM / 32, NI = WTN / 32;
    extern __shared__ __align__(16) unsigned char smem_raw[];
    bf16_t *As = (bf16_t *)smem_raw;         // [2][BM*64]
    bf16_t *Bs = As + 2 * BM * BK;           // [2][BN*64]

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int wm = wave >> 1, wn = wave & 1;

    // XCD-aware remap of the workgroup id, then grouped (8 tile rows) ordering
    int pid;
    {
        const int nb = gridDim.x, b = blockIdx.x;
        const int per = nb >> 3, rem = nb & 7, x = b & 7, q = b >> 3;
        pid = x * per + (x < rem ? x : rem) + q;
    }
    constexpr int GM = 8;
    const int group = pid / (GM * p.tiles_n);
    const int first_m = group * GM;
    const int gsize = (p.tiles_m - first_m) < GM ? (p.tiles_m - first_m) : GM;
    const int tm = first_m + (pid % (GM * p.tiles_n)) % gsize;
    const int tn = (pid % (GM * p.tiles_n)) / gsize;
    const int m0 = tm * BM, n0 = tn * BN;

    const int kt_begin = blockIdx.y * p.k_tiles_per_split;
    int kt_end = kt_begin + p.k_tiles_per_split;
    const int kt_total = (p.K + BK - 1) / BK;
    if (kt_end > kt_total) kt_end = kt_total;
    const int nk = kt_end - kt_begin;
    if (nk <= 0) return;
    const int k_end = p.K;

    const bf16_t *A = (const bf16_t *)p.A, *B = (const bf16_t *)p.B;
    Stager<BM, TA> sa;
    Stager<BN, TB> sb;

    f32x16 acc[MI][NI];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

    sa.load(A, p.lda, m0, p.M, kt_begin * BK, k_end, tid);
    sb.load(B, p.ldb, n0, p.N, kt_begin * BK, k_end, tid);
    sa.store(As, tid);
    sb.store(Bs, tid);
    __syncthreads();

    const int frow = lane & 31, fhalf = lane >> 5;
    for (int kt = 0; kt < nk; ++kt) {
        const int cur = kt & 1;
        if (kt + 1 < nk) {
            sa.load(A, p.lda, m0, p.M, (kt_begin + kt + 1) * BK, k_end, tid);
            sb.load(B, p.ldb, n0, p.N, (kt_begin + kt + 1) * BK, k_end, tid);
        }
        // fragments of k-step kk+1 are fetched from LDS while the MFMAs of k-step kk run
        bf16x8 af[2][MI], bfr[2][NI];
        auto load_frags = [&](int kk, int slot) {
#pragma unroll
            for (int i = 0; i < MI; ++i)
                af[slot][i] = *(const bf16x8 *)(As + cur * BM * BK + lds_off(wm * WTM + i * 32 + frow, kk * 2 + fhalf));
#pragma unroll
            for (int j = 0; j < NI; ++j)
                bfr[slot][j] = *(const bf16x8 *)(Bs + cur * BN * BK + lds_off(wn * WTN + j * 32 + frow, kk * 2 + fhalf));
        };
        load_frags(0, 0);
#pragma unroll
        for (int kk = 0; kk < BK / 16; ++kk) {
            if (kk + 1 < BK / 16) load_frags(kk + 1, (kk + 1) & 1);
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NI; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(af[kk & 1][i], bfr[kk & 1][j], acc[i][j], 0, 0, 0);
        }
        if (kt + 1 < nk) {
            sa.store(As + (cur ^ 1) * BM * BK, tid);
            sb.store(Bs + (cur ^ 1) * BN * BK, tid);
        }
        __syncthreads();
    }

    // epilogue: acc[i][j][r] is C(row, col) with row = 8*(r/4) + 4*(lane/32) + r%4, col = lane%32
    const bf16_t *bias = (const bf16_t *)p.bias, *res = (const bf16_t *)p.residual;
    const float *res32 = (const float *)p.residual;
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            const int col = n0 + wn * WTN + j * 32 + frow;
            if (col >= p.N) continue;
            const float bv = bias ? (float)bias[col] : 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int row = m0 + wm * WTM + i * 32 + 8 * (r >> 2) + 4 * fhalf + (r & 3);
                if (row >= p.M) continue;
                float v = acc[i][j][r] * p.alpha + bv;
                if (res) v += p.res_fp32 ? res32[(long)row * p.ldr + col] : (float)res[(long)row * p.ldr + col];
                if (p.c_fp32) {
                    float *c = (float *)p.C + (long)row * p.ldc + col;
                    if (p.atomic) unsafeAtomicAdd(c, v);
                    else if (p.accumulate) *c += v;
                    else *c = v;
                } else {
                    ((bf16_t *)p.C)[(long)row * p.ldc + col] = (bf16_t)v;
                }
            }
        }
}

template <int BM, int BN, int WM, int WN, bool TA, bool TB, int EPI = EPI_NONE, bool M16 = false, int NST = 2>
__global__ __launch_bounds__(64 * WM * WN) __attribute__((amdgpu_waves_per_eu(fast_waves_per_simd(BM, WM * WN, EPI, NST)))) void gemm_bf16_fast_kernel(GemmParams p) {
    MS_FAST_LDS(BM, BN, NST);
    gemm_fast_body<BM, BN, WM, WN, TA, TB, EPI, M16, NST>(p, lds, blockIdx.x, gridDim.x, blockIdx.y);
}

// Both products of a linear layer's backward pass, which share dy and nothing else, in one grid: the input gradient's
// workgroups (pd: dx = dy W, K-major B) and the weight gradient's (pw: dW += dy^T x, both K-major, `splits` parts of K).
// One product of a small micro-batch leaves CUs idle (100-250 workgroups) and any product has a last round; together they
// leave one.  The product with the longer workgroups comes first (see ms_choose_pair).  One MI355X, us, backward GEMMs of a
// layer apart -> together: c2 student at 2053 tokens 176 -> 146, encoder at 1031 tokens 175 -> 130; the fp32 form (five pairs in
// the c1 step) takes the step from 271 to 242.
// EPI = EPI_SWIGLU_BWD: x is the output of a SwiGLU; the input gradient goes through its derivative in the epilogue and leaves as
// [dgate | dup].  A kernel of its own read the 2 f pre-activations too, but also da, which the product had written (c5 student
// layer at 32768 tokens 532 us, 5.5 TB/s): 13.16 -> 13.09 ms, c2 student layer at 2053 tokens 438 -> 434 us; the epilogue's
// bursts are not behind MFMAs, which eats most of the bytes saved.
template <int BM, int BN, int WM, int WN, int NST, int EPI = EPI_NONE>
__global__ __launch_bounds__(64 * WM * WN) __attribute__((amdgpu_waves_per_eu(fast_waves_per_simd(BM, WM * WN, EPI_NONE, NST)))) void gemm_bf16_pair_kernel(GemmParams pd, GemmParams pw, int nd, int nw, int wgrad_first) {
    MS_FAST_LDS(BM, BN, NST);
    const int b = blockIdx.x, total_w = gridDim.x - nd;
    if (wgrad_first ? b < total_w : b >= nd) {
        const int bw = wgrad_first ? b : b - nd;
        gemm_fast_body<BM, BN, WM, WN, true, true, EPI_NONE, true, NST>(pw, lds, bw % nw, nw, bw / nw);
    } else {
        gemm_fast_body<BM, BN, WM, WN, false, true, EPI, true, NST>(pd, lds, wgrad_first ? b - total_w : b, nd, 0);
    }
}

template <int EPI>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) void gemm_bf16_pp_kernel(GemmParams p) {
    MS_PP_LDS;
    gemm_pp_body<EPI>(p, lds, blockIdx.x, gridDim.x, blockIdx.y);
}

// A chunk's student logits with a KD epilogue (ps, EPI) and another chunk's teacher logits (pt) in one grid.  The student's
// epilogue reads the stored teacher logits, 256 KB per 256 x 256 tile; in a launch of its own all CUs come to it together
// and wait for HBM with idle matrix cores.  Here the two kinds of tiles take turns, a round of the chip each (`run`; the last rounds
// of both together), the kind with the longer workgroups first (`first`, 1: student): their
// times differ, so that one kind's epilogues come to run beside the other's main loops, and one last round is left instead of
// two (see ms_choose_two for what it gains).  The order is the one that ms_choose_two reckons with.  With runs of 256 also where a round is
// 512 workgroups, part of the longer ones waited for the shorter (64 x 128 tiles, 300 tokens, H = 4096 / 1536, chunks of 8192, loss
// only, V = 49152: 416 us, two launches 339).  In runs of 8 or 64 the two products' operand panels compete for the L2s from the start
// (256 x 256 tiles, 8192 tokens, V = 151936: 33.6 .. 34.0 ms; apart 32.98, in runs of 256 32.75).
struct TwoSlot { int student, index; };
__device__ __forceinline__ TwoSlot two_slot(int b, int nt, int ns, int run, int first) {
    const int both = (nt < ns ? nt : ns) / run * run;
    if (b < 2 * both) return {((b / run) & 1) ^ first, b / (2 * run) * run + b % run};
    const int r = b - 2 * both, more = (first ? ns : nt) - both;
    return r < more ? TwoSlot{first, both + r} : TwoSlot{first ^ 1, both + r - more};
}
template <int EPI>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) void gemm_bf16_pp_two_kernel(GemmParams pt, GemmParams ps, int nt, int ns, int run, int first) {
    MS_PP_LDS;
    const TwoSlot t = two_slot(blockIdx.x, nt, ns, run, first);
    if (t.student) gemm_pp_body<EPI>(ps, lds, t.index, ns, 0);
    else gemm_pp_body<EPI_NONE>(pt, lds, t.index, nt, 0);
}
template <int BM, int BN, int WM, int WN, int NST, int EPI>
__global__ __launch_bounds__(64 * WM * WN) __attribute__((amdgpu_waves_per_eu(fast_waves_per_simd(BM, WM * WN, EPI, NST)))) void gemm_bf16_two_kernel(GemmParams pt, GemmParams ps, int nt, int ns, int run, int first) {
    MS_FAST_LDS(BM, BN, NST);
    const TwoSlot t = two_slot(blockIdx.x, nt, ns, run, first);
    if (t.student) gemm_fast_body<BM, BN, WM, WN, false, false, EPI, true, NST>(ps, lds, t.index, ns, 0);
    else gemm_fast_body<BM, BN, WM, WN, false, false, EPI_NONE, true, NST>(pt, lds, t.index, nt, 0);
}

// ------------------------------------------------------------------ fp32
struct GemmF32Params {
    const float *A, *B;
    float *C;
    const float *bias, *residual;
    long lda, ldb, ldc, ldr;
    int M, N, K, tiles_n;
    float alpha;
    int accumulate;
    const float *sw_up;      // SwiGLU backward: pre-activations [M, 2 N]; the product is da and C = [dgate | dup]
};

// One operand's fragments for v_mfma_f32_16x16x4_f32: two 16-row blocks x 16 k.  Lane = (row lane % 16, k-group
// lane / 16); component c of a block's four values is k = k0 + 4 (lane / 16) + c, so four MFMAs (one per component)
// contract 16 k.  TRANS: the operand is stored [K][rows].  Rows and k past the end read as zero.  FAST: loads through a
// buffer descriptor whose range check returns the zeros, so that nothing but the MFMAs waits for a load.
template <bool TRANS, bool FAST> struct F32Frag {
    float v[2][4];
    __device__ __forceinline__ void load(const float *P, __amdgpu_buffer_rsrc_t rs, long ld, int row0, int rows, int k0, int K, int lane) {
        const int k = k0 + 4 * (lane >> 4);
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int r = row0 + 16 * b + (lane & 15);
            if constexpr (FAST && !TRANS) {
                const unsigned off = r < rows && k < K ? (unsigned)((long)r * ld + k) * 4u : kOob;
                const u32x4 t = __builtin_amdgcn_raw_buffer_load_b128(rs, off, 0, 0);
#pragma unroll
                for (int c = 0; c < 4; ++c) v[b][c] = __uint_as_float(t[c]);
            } else {
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const bool ok = r < rows && k + c < K;
                    const long at = TRANS ? (long)(k + c) * ld + r : (long)r * ld + k + c;
                    if constexpr (FAST) v[b][c] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rs, ok ? (unsigned)at * 4u : kOob, 0, 0));
                    else v[b][c] = ok ? P[at] : 0.f;
                }
            }
        }
    }
};

// fp32 GEMM for the small matrices of the fp32 workload (a few hundred rows): latency is what it costs, not flops.  A
// workgroup computes a 32 x 32 tile; its four waves take every fourth 16-deep slice of K each (a quarter of the serial
// chain) and add up through LDS.  Fragments come straight from global memory (the operands are a few hundred KB and
// stay in L2), three slices ahead of the MFMAs that use them; what the epilogue reads is requested before the main loop.
// The 64 x 64 FMA kernel that this replaces took 1.3 us per 16 k (10..80 workgroups, a load latency and two barriers
// each): 47 us per launch on average in the c1 step, against 6.9 us now.
// FAST needs 16-byte aligned K-contiguous rows with K % 4 == 0 and operands below 4 GB; the other form covers the rest.
// (The first slices are requested before the loop, also where K = 0 leaves it nothing to do: the range is then empty.)
template <bool TA, bool TB, bool FAST>
__device__ __forceinline__ void gemm_f32_body(const GemmF32Params &p, float (&part)[4][32][33], int b_) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int m0 = b_ / p.tiles_n * 32, n0 = b_ % p.tiles_n * 32;
    const int slices = (p.K + 15) / 16, mine = slices > wave ? (slices - wave + 3) / 4 : 0;
    const __amdgpu_buffer_rsrc_t ra = make_rsrc(p.A, FAST ? ms_matrix_extent(TA ? p.K : p.M, TA ? p.M : p.K, p.lda) * 4 : 0);
    const __amdgpu_buffer_rsrc_t rb = make_rsrc(p.B, FAST ? ms_matrix_extent(TB ? p.K : p.N, TB ? p.N : p.K, p.ldb) * 4 : 0);
    F32Frag<TA, FAST> a[4];
    F32Frag<TB, FAST> b[4];
    f32x4 acc[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto load = [&](int slot, int s) __attribute__((always_inline)) {
        const int k0 = (wave + 4 * s) * 16;
        a[slot].load(p.A, ra, p.lda, m0, p.M, k0, p.K, lane);
        b[slot].load(p.B, rb, p.ldb, n0, p.N, k0, p.K, lane);
    };
    load(0, 0);
    load(1, 1);
    load(2, 2);
    // this thread's four output elements: rows threadIdx.x / 32 + 8 e, column threadIdx.x % 32
    const int rr = threadIdx.x >> 5, cc = threadIdx.x & 31, col = n0 + cc;
    float add[4] = {0.f, 0.f, 0.f, 0.f};
    if (p.bias && col < p.N) add[0] = add[1] = add[2] = add[3] = p.bias[col];
    float res[4] = {0.f, 0.f, 0.f, 0.f}, old[4] = {0.f, 0.f, 0.f, 0.f};
    auto inside = [&](int e) { return m0 + rr + 8 * e < p.M && col < p.N; };
    if (p.residual)
#pragma unroll
        for (int e = 0; e < 4; ++e) if (inside(e)) res[e] = p.residual[(long)(m0 + rr + 8 * e) * p.ldr + col];
    if (p.accumulate)
#pragma unroll
        for (int e = 0; e < 4; ++e) if (inside(e)) old[e] = p.C[(long)(m0 + rr + 8 * e) * p.ldc + col];
    if (p.sw_up)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (inside(e)) {
                res[e] = p.sw_up[(long)(m0 + rr + 8 * e) * 2 * p.N + col];            // gate
                old[e] = p.sw_up[(long)(m0 + rr + 8 * e) * 2 * p.N + p.N + col];      // up
            }
    for (int s = 0; s < mine; s += 4) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            load((u + 3) & 3, s + u + 3);             // (slices past the end are zeros)
            __builtin_amdgcn_sched_barrier(0);        // the requests stay in front of the MFMAs
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[u].v[i][c], b[u].v[j][c], acc[i][j], 0, 0, 0);
        }
    }
    // accumulator (i, j) register r: row 16 i + 4 (lane / 16) + r, column 16 j + lane % 16
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) part[wave][16 * i + 4 * (lane >> 4) + r][16 * j + (lane & 15)] = acc[i][j][r];
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int q = rr + 8 * e;
        if (p.sw_up) {
            float dg, du;
            swiglu_derivative((part[0][q][cc] + part[1][q][cc] + part[2][q][cc] + part[3][q][cc]) * p.alpha, res[e], old[e], &dg, &du);
            if (inside(e)) {
                p.C[(long)(m0 + q) * p.ldc + col] = dg;
                p.C[(long)(m0 + q) * p.ldc + p.N + col] = du;
            }
            continue;
        }
        const float v = (part[0][q][cc] + part[1][q][cc] + part[2][q][cc] + part[3][q][cc]) * p.alpha + add[e] + res[e];
        if (inside(e)) p.C[(long)(m0 + q) * p.ldc + col] = p.accumulate ? old[e] + v : v;
    }
}
template <bool TA, bool TB, bool FAST>
__global__ __launch_bounds__(256) void gemm_f32_kernel(GemmF32Params p) {
    __shared__ float part[4][32][33];
    gemm_f32_body<TA, TB, FAST>(p, part, (int)blockIdx.x);
}
// Both products of a linear layer's backward pass in one grid (see gemm_bf16_pair_kernel), the one with the longer workgroups, whose K is
// the token count or the layer's outputs, first.  With the weight gradient always behind, a few long workgroups were
// left over at large token counts (us, two launches / weight gradient last / this order: 688 x 256 at 4000 tokens 53.8 / 62.1 / 43.7,
// at 12000 139 / 179 / 114; 512 x 512 at 12000 159 / 203 / 137; over 11 layers x 64 .. 12000 tokens never slower than two).
template <bool WGRAD_FIRST>
__global__ __launch_bounds__(256) void gemm_f32_pair_kernel(GemmF32Params pd, GemmF32Params pw, int first) {
    __shared__ float part[4][32][33];
    const int b = (int)blockIdx.x;
    if ((b < first) != WGRAD_FIRST) gemm_f32_body<false, true, true>(pd, part, WGRAD_FIRST ? b - first : b);
    else gemm_f32_body<true, true, true>(pw, part, WGRAD_FIRST ? b : b - first);
}

// Two products with K-contiguous operands in one grid; the first n0 workgroups are the first one's.  Both load in the same way: where
// only one of them can be read 16 bytes at a time, it has a launch of its own (teacher and student logits of 2000 tokens, V = 8192, H = 1024
// / 512, student states 4 bytes off: head 4.36 ms together, 3.2 apart).
template <bool FAST>
__global__ __launch_bounds__(256) void gemm_f32_two_kernel(GemmF32Params p0, GemmF32Params p1, int n0) {
    __shared__ float part[4][32][33];
    const int b = (int)blockIdx.x;
    if (b < n0) gemm_f32_body<false, false, FAST>(p0, part, b);
    else gemm_f32_body<false, false, FAST>(p1, part, b - n0);
}

// Explicit instantiations: the host pass has been seen to reference the launch stubs of some of these
// without defining them when they are only instantiated implicitly from the launcher below.
#define MS_INST(BM, WN, TA, TB)                                                                          \
    template __global__ void gemm_bf16_fast_kernel<BM, BM, 2, WN, TA, TB, EPI_NONE, false>(GemmParams); \
    template __global__ void gemm_bf16_fast_kernel<BM, BM, 2, WN, TA, TB, EPI_NONE, true>(GemmParams)
template __global__ void gemm_bf16_fast_kernel<256, 256, 2, 4, false, false, EPI_NONE, false>(GemmParams);
MS_INST(256, 4, false, true); MS_INST(256, 4, true, false); MS_INST(256, 4, true, true);
MS_INST(128, 2, false, false); MS_INST(128, 2, false, true); MS_INST(128, 2, true, false); MS_INST(128, 2, true, true);
#undef MS_INST
template __global__ void gemm_bf16_pp_kernel<EPI_NONE>(GemmParams);
template __global__ void gemm_bf16_pp_kernel<EPI_SWIGLU>(GemmParams);
template __global__ void gemm_bf16_pp_kernel<EPI_KD_DZ>(GemmParams);
template __global__ void gemm_bf16_pp_kernel<EPI_KD_STATS>(GemmParams);
#define MS_INST_RING(BM, BN, WM, WN, NST, TA, TB) \
    template __global__ void gemm_bf16_fast_kernel<BM, BN, WM, WN, TA, TB, EPI_NONE, true, NST>(GemmParams)
#define MS_INST_RINGS(BM, BN, WM, WN, NST)                                                             \
    MS_INST_RING(BM, BN, WM, WN, NST, false, false); MS_INST_RING(BM, BN, WM, WN, NST, false, true);   \
    MS_INST_RING(BM, BN, WM, WN, NST, true, false); MS_INST_RING(BM, BN, WM, WN, NST, true, true);     \
    template __global__ void gemm_bf16_fast_kernel<BM, BN, WM, WN, false, false, EPI_KD_DZ, true, NST>(GemmParams);     \
    template __global__ void gemm_bf16_fast_kernel<BM, BN, WM, WN, false, false, EPI_KD_STATS, true, NST>(GemmParams);  \
    template __global__ void gemm_bf16_fast_kernel<BM, BN, WM, WN, false, false, EPI_SWIGLU, true, NST>(GemmParams)
MS_INST_RINGS(128, 128, 4, 2, 4); MS_INST_RINGS(128, 256, 2, 4, 3); MS_INST_RINGS(64, 128, 2, 2, 3); MS_INST_RINGS(64, 64, 2, 1, 4);
#undef MS_INST_RINGS
#define MS_INST_TWO(EPI)                                                                                              \
    template __global__ void gemm_bf16_pp_two_kernel<EPI>(GemmParams, GemmParams, int, int, int, int);                          \
    template __global__ void gemm_bf16_two_kernel<128, 128, 2, 2, 2, EPI>(GemmParams, GemmParams, int, int, int, int);          \
    template __global__ void gemm_bf16_two_kernel<128, 128, 4, 2, 4, EPI>(GemmParams, GemmParams, int, int, int, int);          \
    template __global__ void gemm_bf16_two_kernel<128, 256, 2, 4, 3, EPI>(GemmParams, GemmParams, int, int, int, int);          \
    template __global__ void gemm_bf16_two_kernel<64, 128, 2, 2, 3, EPI>(GemmParams, GemmParams, int, int, int, int);           \
    template __global__ void gemm_bf16_two_kernel<64, 64, 2, 1, 4, EPI>(GemmParams, GemmParams, int, int, int, int)
MS_INST_TWO(EPI_KD_DZ); MS_INST_TWO(EPI_KD_STATS);
#undef MS_INST_TWO
#define MS_INST_PAIR(BM, BN, WM, WN, NST)                                                                                    \
    template __global__ void gemm_bf16_pair_kernel<BM, BN, WM, WN, NST, EPI_NONE>(GemmParams, GemmParams, int, int, int);   \
    template __global__ void gemm_bf16_pair_kernel<BM, BN, WM, WN, NST, EPI_SWIGLU_BWD>(GemmParams, GemmParams, int, int, int)
MS_INST_PAIR(256, 256, 2, 4, 2); MS_INST_PAIR(128, 128, 2, 2, 2); MS_INST_PAIR(128, 128, 4, 2, 4); MS_INST_PAIR(128, 256, 2, 4, 3);
MS_INST_PAIR(64, 128, 2, 2, 3); MS_INST_PAIR(64, 64, 2, 1, 4);
#undef MS_INST_PAIR
#undef MS_INST_RING
#define MS_INST_EPI(EPI)                                                                                      \
    template __global__ void gemm_bf16_fast_kernel<256, 256, 2, 4, false, false, EPI, false>(GemmParams);    \
    template __global__ void gemm_bf16_fast_kernel<128, 128, 2, 2, false, false, EPI, false>(GemmParams);    \
    template __global__ void gemm_bf16_fast_kernel<128, 128, 2, 2, false, false, EPI, true>(GemmParams)
MS_INST_EPI(EPI_KD_DZ); MS_INST_EPI(EPI_KD_STATS); MS_INST_EPI(EPI_SWIGLU);
#undef MS_INST_EPI

// Kernel selection switches, for measurements and tests only: the environment gives the process-wide setting
// (MS_GEMM_TILE = a tile code of kTiles, or 256256, forces the fast kernels' tile, -1 disables them; MS_GEMM_MFMA16 = 0
// selects v_mfma_f32_32x32x16_bf16 and the two-stage tiles), ms_k_gemm_config overrides it at run time.  The overrides are atomics, so changing them
// from one thread while another launches is defined, but which setting a concurrent launch sees is not: production
// callers leave them alone (automatic choice by shape).
constexpr int kUnset = -1000;
std::atomic<int> g_tile_override{kUnset}, g_mfma16_override{kUnset};
int forced_tile() {
    static const int env = [] { const char *e = getenv("MS_GEMM_TILE"); return e ? atoi(e) : 0; }();
    const int o = g_tile_override.load(std::memory_order_relaxed);
    return o != kUnset ? o : env;
}
bool use_mfma16() {
    static const bool env = [] { const char *e = getenv("MS_GEMM_MFMA16"); return !e || atoi(e) != 0; }();
    const int o = g_mfma16_override.load(std::memory_order_relaxed);
    return o != kUnset ? o != 0 : env;
}

// The tile for an M x N output (N = rows of B) of kt K tiles whose epilogue moves out_bytes per element (ms_choose_tile)
int choose_tile(int M, int N, int kt, double out_bytes) { return ms_choose_tile(M, N, kt, out_bytes, forced_tile(), use_mfma16()); }

template <int BM, int BN, int WM, int WN, int NST, int EPI>
void launch_fast_tile(const GemmParams &p, int ta, int tb, dim3 grid, hipStream_t s) {
    constexpr int NT = 64 * WM * WN;
#define GO(TA, TB)                                                                                                  \
    do {                                                                                                            \
        if constexpr (NST > 2) gemm_bf16_fast_kernel<BM, BN, WM, WN, TA, TB, EPI, true, NST><<<grid, NT, 0, s>>>(p); \
        else if (!use_mfma16()) gemm_bf16_fast_kernel<BM, BN, WM, WN, TA, TB, EPI, false><<<grid, NT, 0, s>>>(p);    \
        else if constexpr (BM == 256 && !TA && !TB) gemm_bf16_pp_kernel<EPI><<<grid, NT, 0, s>>>(p);                \
        else gemm_bf16_fast_kernel<BM, BN, WM, WN, TA, TB, EPI, true><<<grid, NT, 0, s>>>(p);                        \
    } while (0)
    if constexpr (EPI != EPI_NONE) GO(false, false);
    else if (!ta && !tb) GO(false, false);
    else if (!ta && tb) GO(false, true);
    else if (ta && !tb) GO(true, false);
    else GO(true, true);
#undef GO
}

// p.tiles_m / tiles_n are set here; EPI_SWIGLU tiles cover bn / 2 output columns (gate and up rows of B)
template <int EPI>
ms_status launch_bf16_fast(GemmParams &p, int tile, int ta, int tb, int splits, double flops, hipStream_t s) {
    const MsTile &t = kTiles[tile];
    p.tiles_m = ms_cdiv(p.M, t.bm);
    p.tiles_n = ms_cdiv(p.N, EPI == EPI_SWIGLU ? t.bn / 2 : t.bn);
    dim3 grid(p.tiles_m * p.tiles_n, splits);
    ProfScope ps((ta || tb) ? 1 : 0, flops, s);
    switch (tile) {
        case T256: launch_fast_tile<256, 256, 2, 4, 2, EPI>(p, ta, tb, grid, s); break;
        case R128: launch_fast_tile<128, 128, 4, 2, 4, EPI>(p, ta, tb, grid, s); break;
        case R128x256: launch_fast_tile<128, 256, 2, 4, 3, EPI>(p, ta, tb, grid, s); break;
        case R64x128: launch_fast_tile<64, 128, 2, 2, 3, EPI>(p, ta, tb, grid, s); break;
        case R64: launch_fast_tile<64, 64, 2, 1, 4, EPI>(p, ta, tb, grid, s); break;
        default: launch_fast_tile<128, 128, 2, 2, 2, EPI>(p, ta, tb, grid, s); break;
    }
    MS_LAUNCH_CHECK();
    return MS_OK;
}

template <int BM, int BN>
ms_status launch_bf16(const GemmParams &p, int ta, int tb, int splits, hipStream_t s) {
    const size_t smem = (size_t)2 * (BM + BN) * BK * sizeof(bf16_t);
    dim3 grid(p.tiles_m * p.tiles_n, splits);
    ProfScope ps((ta || tb) ? 1 : 0, 2.0 * p.M * p.N * p.K, s);
#define GO(TA, TB)                                                                                        \
    do {                                                                                                  \
        static bool attr_set = false;                                                                     \
        if (!attr_set && smem > 48 * 1024) {                                                              \
            MS_CHECK_HIP(hipFuncSetAttribute((const void *)gemm_bf16_kernel<BM, BN, TA, TB>,              \
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem));     \
            attr_set = true;                                                                              \
        }                                                                                                 \
        gemm_bf16_kernel<BM, BN, TA, TB><<<grid, 256, smem, s>>>(p);                                      \
    } while (0)
    if (!ta && !tb) GO(false, false);
    else if (!ta && tb) GO(false, true);
    else if (ta && !tb) GO(true, false);
    else GO(true, true);
#undef GO
    MS_LAUNCH_CHECK();
    return MS_OK;
}

// fp32: whether an operand (rows x K as the product sees it) can be read through a descriptor, 16 bytes at a time where it is
// K-contiguous
bool f32_fast(const void *q, long ld, bool trans, long rows, long K) {
    return (trans || (((uintptr_t)q & 15) == 0 && ld % 4 == 0 && K % 4 == 0)) && ms_buffer_range_ok(trans ? K : rows, trans ? rows : K, ld, 4);
}

// Checked arguments of a bf16 product, all but the split of K
struct Bf16Gemm {
    GemmParams p;
    bool fast;          // the direct-to-LDS kernels take it
    int kt;             // K tiles
    double out_bytes;   // what the epilogue moves per output element
};
ms_status prepare_bf16(int trans_a, int trans_b, int M, int N, int K, float alpha, const void *A, long lda, const void *B, long ldb,
                       void *C, long ldc, int c_fp32, int accumulate, const void *bias, const void *residual, long ldr,
                       int residual_fp32, Bf16Gemm *g) {
    auto al = [](const void *q) { return ((uintptr_t)q & 15) == 0; };
    if (!al(A) || !al(B) || lda % 8 || ldb % 8 || (trans_a ? M % 8 : K % 8) || (trans_b ? N % 8 : K % 8))
        return ms_fail(MS_ERR_UNSUPPORTED,
                       "gemm(bf16): contiguous dimension of each operand must be a multiple of 8 and 16-byte aligned "
                       "(M=%d N=%d K=%d ta=%d tb=%d lda=%ld ldb=%ld)", M, N, K, trans_a, trans_b, (long)lda, (long)ldb);
    GemmParams &p = g->p;
    p = {};
    p.A = A; p.B = B; p.C = C; p.bias = bias; p.residual = residual;
    p.lda = lda; p.ldb = ldb; p.ldc = ldc; p.ldr = ldr; p.M = M; p.N = N; p.K = K; p.alpha = alpha;
    p.c_fp32 = c_fp32; p.accumulate = accumulate; p.res_fp32 = residual_fp32;
    // fast path (direct-to-LDS loads, descriptor-addressed epilogue) needs full K tiles for a K-contiguous
    // operand and 32-bit byte offsets
    const long lim = (1L << 32) - (1L << 20);
    const long rows_a = trans_a ? K : M, rows_b = trans_b ? K : N;
    g->fast = forced_tile() >= 0 && ((trans_a && trans_b) || K % BK == 0) && (rows_a + 256) * lda * 2 < lim &&
              (rows_b + 256) * ldb * 2 < lim && ((long)M + 256) * ldc * 4 < lim &&
              (!residual || ((long)M + 256) * ldr * 4 < lim);
    g->kt = ms_cdiv(K, BK) < 1 ? 1 : ms_cdiv(K, BK);
    g->out_bytes = (c_fp32 ? 4 : 2) + (residual ? (residual_fp32 ? 4 : 2) : 0) + (accumulate ? 4 : 0);
    return MS_OK;
}
// The last arguments, which depend on the number of K splits; returns how many there really are
int set_splits(Bf16Gemm &g, int splits) {
    GemmParams &p = g.p;
    auto al = [](const void *q) { return ((uintptr_t)q & 15) == 0; };
    if (splits > g.kt) splits = g.kt;
    p.k_tiles_per_split = ms_cdiv(g.kt, splits);
    splits = ms_cdiv(g.kt, p.k_tiles_per_split);
    p.atomic = splits > 1;
    p.vec_epilogue = !p.atomic && p.N % 4 == 0 && p.ldc % 4 == 0 && al(p.C) && (!p.residual || (p.ldr % 4 == 0 && al(p.residual))) &&
                     (!p.bias || ((uintptr_t)p.bias & 7) == 0);
    return splits;
}

}  // namespace

int gemm_forced_tile() { return forced_tile(); }

extern "C" ms_status ms_k_gemm_config(int32_t tile, int32_t mfma16) {
    bool known = tile == -1 || tile == 0 || tile == kPingPong;
    for (const MsTile &t : kTiles) known = known || tile == t.code;
    if (!known || mfma16 < -1 || mfma16 > 1)
        return ms_fail(MS_ERR_INVALID_ARG, "gemm_config: tile must be -1, 0, 128, 256, 256256, 128128, 128256, 64128 or 64064 and mfma16 -1, 0 or 1");
    g_tile_override = tile == 0 ? kUnset : tile;
    g_mfma16_override = mfma16 < 0 ? kUnset : mfma16;
    return MS_OK;
}

extern "C" ms_status ms_k_gemm(int32_t dtype, int32_t trans_a, int32_t trans_b, int32_t M, int32_t N, int32_t K,
                               float alpha, const void *A, int64_t lda, const void *B, int64_t ldb, void *C,
                               int64_t ldc, int32_t c_fp32, int32_t accumulate, const void *bias,
                               const void *residual, int64_t ldr, int32_t residual_fp32, int32_t split_k,
                               void *stream) {
    if (M == 0 || N == 0) return MS_OK;
    if (!A || !B || !C || M < 0 || N < 0 || K < 0) return ms_fail(MS_ERR_INVALID_ARG, "gemm: null pointer or negative size");
    if (accumulate && !c_fp32 && dtype == MS_BF16) return ms_fail(MS_ERR_INVALID_ARG, "gemm: accumulate needs an fp32 C");
    hipStream_t s = (hipStream_t)stream;
    if (dtype == MS_F32) {
        GemmF32Params p = {};
        p.A = (const float *)A; p.B = (const float *)B; p.C = (float *)C;
        p.bias = (const float *)bias; p.residual = (const float *)residual;
        p.lda = lda; p.ldb = ldb; p.ldc = ldc; p.ldr = ldr; p.M = M; p.N = N; p.K = K; p.alpha = alpha; p.accumulate = accumulate;
        p.tiles_n = ms_cdiv(N, 32);
        const long tiles = (long)ms_cdiv(M, 32) * p.tiles_n;
        if (!ms_launch_fits(tiles, 256)) {   // more tiles than one launch takes: the two halves of C along its longer side
            const bool rows = ms_cdiv(M, 32) >= p.tiles_n;
            const int cut = (int)(((rows ? M : N) / 2L + 31) / 32 * 32);
            const long a = rows ? (trans_a ? cut : cut * lda) : 0, b = rows ? 0 : (trans_b ? cut : cut * ldb), c = rows ? cut * ldc : cut;
            const long r = rows ? cut * ldr : cut;
            MS_TRY(ms_k_gemm(dtype, trans_a, trans_b, rows ? cut : M, rows ? N : cut, K, alpha, A, lda, B, ldb, C, ldc, c_fp32, accumulate, bias,
                             residual, ldr, residual_fp32, split_k, stream));
            return ms_k_gemm(dtype, trans_a, trans_b, rows ? M - cut : M, rows ? N : N - cut, K, alpha, p.A + a, lda, p.B + b, ldb, p.C + c,
                             ldc, c_fp32, accumulate, bias && !rows ? p.bias + cut : bias, residual ? p.residual + r : nullptr, ldr,
                             residual_fp32, split_k, stream);
        }
        const unsigned grid = (unsigned)tiles;
#define GO(TA, TB)                                                                                     \
    do {                                                                                               \
        if (f32_fast(A, lda, TA, M, K) && f32_fast(B, ldb, TB, N, K)) gemm_f32_kernel<TA, TB, true><<<grid, 256, 0, s>>>(p);  \
        else gemm_f32_kernel<TA, TB, false><<<grid, 256, 0, s>>>(p);                                   \
    } while (0)
        if (!trans_a && !trans_b) GO(false, false);
        else if (!trans_a && trans_b) GO(false, true);
        else if (trans_a && !trans_b) GO(true, false);
        else GO(true, true);
#undef GO
        MS_LAUNCH_CHECK();
        return MS_OK;
    }
    Bf16Gemm g;
    MS_TRY(prepare_bf16(trans_a, trans_b, M, N, K, alpha, A, lda, B, ldb, C, ldc, c_fp32, accumulate, bias, residual, ldr, residual_fp32, &g));
    int tile = g.fast ? choose_tile(M, N, g.kt, g.out_bytes) : T128;
    int splits = split_k;
    if (splits <= 0) {  // automatic: only when accumulating into fp32 (weight gradients: small M x N, long K)
        splits = 1;
        if (accumulate && c_fp32 && g.fast) {
            const MsSplit c = ms_choose_split(M, N, g.kt, forced_tile(), use_mfma16());
            tile = c.tile;
            splits = c.splits;
        } else if (accumulate && c_fp32) {
            const int tiles = ms_cdiv(M, 128) * ms_cdiv(N, 128);
            while (tiles * splits < 512 && g.kt / (splits * 2) >= 8) splits *= 2;
        }
    }
    if (splits > 1 && !(accumulate && c_fp32)) return ms_fail(MS_ERR_INVALID_ARG, "gemm: split_k needs accumulate into fp32");
    splits = set_splits(g, splits);
    if (g.fast) return launch_bf16_fast<EPI_NONE>(g.p, tile, trans_a, trans_b, splits, 2.0 * M * N * K, s);
    g.p.tiles_m = ms_cdiv(M, 128); g.p.tiles_n = ms_cdiv(N, 128);
    return launch_bf16<128, 128>(g.p, trans_a, trans_b, splits, s);
}

// ------------------------------------------------------------------ backward pass of a linear layer
namespace {
// Input gradient d and weight gradient w of one layer in one grid, if that is estimated faster (done = false: it is not)
template <int EPI>
ms_status launch_pair(Bf16Gemm &d, Bf16Gemm &w, bool *done, hipStream_t s) {
    const int n = d.p.M, in = d.p.N, out = d.p.K;
    if (!d.fast || !w.fast || !use_mfma16()) return MS_OK;
    const MsPair c = ms_choose_pair(n, out, in, d.out_bytes, forced_tile());
    if (c.tile < 0) return MS_OK;
    set_splits(d, 1);
    const int splits = set_splits(w, c.splits);
    const MsTile &t = kTiles[c.tile];
    d.p.tiles_m = ms_cdiv(n, t.bm); w.p.tiles_m = ms_cdiv(out, t.bm);
    d.p.tiles_n = w.p.tiles_n = ms_cdiv(in, t.bn);
    const long nd = (long)d.p.tiles_m * d.p.tiles_n, nw = (long)w.p.tiles_m * w.p.tiles_n;
    if (!ms_launch_fits(nd + nw * splits, 512)) return MS_OK;
    *done = true;
    ProfScope ps(1, 4.0 * n * out * in, s);
    const unsigned grid = (unsigned)(nd + nw * splits);
#define GO(BM, BN, WM, WN, NST) gemm_bf16_pair_kernel<BM, BN, WM, WN, NST, EPI><<<grid, 64 * WM * WN, 0, s>>>(d.p, w.p, (int)nd, (int)nw, c.wgrad_first)
    switch (c.tile) {
        case T256: GO(256, 256, 2, 4, 2); break;
        case R128: GO(128, 128, 4, 2, 4); break;
        case R128x256: GO(128, 256, 2, 4, 3); break;
        case R64x128: GO(64, 128, 2, 2, 3); break;
        case R64: GO(64, 64, 2, 1, 4); break;
        default: GO(128, 128, 2, 2, 2); break;
    }
#undef GO
    MS_LAUNCH_CHECK();
    return MS_OK;
}
ms_status launch_pair_f32(int n, int out, int in, const float *dy, long ldy, const float *W, const float *x, float *dx, long ldx, int accumulate,
                          float *dW, const float *sw_up, bool *done, hipStream_t s) {
    const long nd = (long)ms_cdiv(n, 32) * ms_cdiv(in, 32), nw = (long)ms_cdiv(out, 32) * ms_cdiv(in, 32);
    // (dy rows that cannot be read 16 bytes at a time slow dx = dy W down, but not the weight gradient, which keeps its own launch then)
    if (!ms_launch_fits(nd + nw, 256) || !f32_fast(dy, ldy, false, n, out) || !f32_fast(W, in, true, in, out) || !f32_fast(dy, ldy, true, out, n) ||
        !f32_fast(x, in, true, in, n))
        return MS_OK;
    *done = true;
    GemmF32Params pd = {}, pw = {};
    pd.A = pw.A = dy; pd.lda = pw.lda = ldy;
    pd.B = W; pw.B = x; pd.ldb = pw.ldb = in;
    pd.C = dx; pd.ldc = ldx; pw.C = dW; pw.ldc = in;
    pd.M = n; pd.N = in; pd.K = out; pw.M = out; pw.N = in; pw.K = n;
    pd.tiles_n = pw.tiles_n = ms_cdiv(in, 32);
    pd.alpha = pw.alpha = 1.f; pd.accumulate = accumulate; pw.accumulate = 1;
    pd.sw_up = sw_up;
    if (n > out) gemm_f32_pair_kernel<true><<<(unsigned)(nd + nw), 256, 0, s>>>(pd, pw, (int)nw);
    else gemm_f32_pair_kernel<false><<<(unsigned)(nd + nw), 256, 0, s>>>(pd, pw, (int)nd);
    MS_LAUNCH_CHECK();
    return MS_OK;
}
}  // namespace

extern "C" ms_status ms_k_linear_backward(int32_t dtype, int32_t n, int32_t out, int32_t in, const void *dy, int64_t ldy, const void *W,
                                          const void *x, void *dx, int32_t dx_fp32, int32_t dx_accumulate, void *dW, void *stream) {
    auto one_by_one = [&]() {
        MS_TRY(ms_k_gemm(dtype, 0, 1, n, in, out, 1.f, dy, ldy, W, in, dx, in, dx_fp32, dx_accumulate, nullptr, nullptr, 0, 0, 1, stream));
        return ms_k_gemm(dtype, 1, 1, out, in, n, 1.f, dy, ldy, x, in, dW, in, 1, 1, nullptr, nullptr, 0, 0, 0, stream);
    };
    if (n <= 0 || out <= 0 || in <= 0 || !dy || !W || !x || !dx || !dW) return one_by_one();      // (which has the checks)
    hipStream_t s = (hipStream_t)stream;
    if (dtype == MS_F32) {
        bool done = false;
        MS_TRY(launch_pair_f32(n, out, in, (const float *)dy, ldy, (const float *)W, (const float *)x, (float *)dx, in, dx_accumulate, (float *)dW,
                               nullptr, &done, s));
        return done ? MS_OK : one_by_one();
    }
    if (dx_accumulate && !dx_fp32) return one_by_one();
    Bf16Gemm d, w;
    MS_TRY(prepare_bf16(0, 1, n, in, out, 1.f, dy, ldy, W, in, dx, in, dx_fp32, dx_accumulate, nullptr, nullptr, 0, 0, &d));
    MS_TRY(prepare_bf16(1, 1, out, in, n, 1.f, dy, ldy, x, in, dW, in, 1, 1, nullptr, nullptr, 0, 0, &w));
    bool done = false;
    MS_TRY(launch_pair<EPI_NONE>(d, w, &done, s));
    return done ? MS_OK : one_by_one();
}

// The down projection of a SwiGLU block backwards: dW += dy^T act and [dgate | dup] from da = dy W, which is not stored where the
// two products share a grid.
extern "C" ms_status ms_k_swiglu_linear_backward(int32_t dtype, int32_t n, int32_t out, int32_t f, const void *dy, const void *W, const void *act,
                                                 const void *gate_up, void *da, void *d_gate_up, void *dW, void *stream) {
    hipStream_t s = (hipStream_t)stream;
    auto al = [](const void *q) { return ((uintptr_t)q & 15) == 0; };
    if (dtype == MS_BF16 && n > 0 && out > 0 && f > 0 && f % 4 == 0 && dy && W && act && gate_up && d_gate_up && dW && al(gate_up) && al(d_gate_up) && ((long)n + 256) * 2 * f * 2 < (1L << 32) - (1L << 20)) {
        Bf16Gemm d, w;
        MS_TRY(prepare_bf16(0, 1, n, f, out, 1.f, dy, out, W, f, d_gate_up, 2L * f, 0, 0, nullptr, nullptr, 0, 0, &d));
        MS_TRY(prepare_bf16(1, 1, out, f, n, 1.f, dy, out, act, f, dW, f, 1, 1, nullptr, nullptr, 0, 0, &w));
        d.p.sg_f = f;
        d.p.sg_gu = const_cast<void *>(gate_up);
        d.p.sg_ldgu = 2L * f;
        d.out_bytes = 8;
        bool done = false;
        MS_TRY(launch_pair<EPI_SWIGLU_BWD>(d, w, &done, s));
        if (done) return MS_OK;
    }
    if (dtype == MS_F32 && n > 0 && out > 0 && f > 0 && dy && W && act && gate_up && d_gate_up && dW) {
        bool done = false;
        MS_TRY(launch_pair_f32(n, out, f, (const float *)dy, out, (const float *)W, (const float *)act, (float *)d_gate_up, 2L * f, 0, (float *)dW,
                               (const float *)gate_up, &done, s));
        if (done) return MS_OK;
    }
    MS_TRY(ms_k_linear_backward(dtype, n, out, f, dy, out, W, act, da, 0, 0, dW, s));
    return ms_k_act_backward(0, dtype, n, f, da, gate_up, d_gate_up, s);
}

ms_status gemm_f32_two(int M, int N, const float *A0, const float *B0, float *C0, int K0, const float *A1, const float *B1, float *C1, int K1,
                       long ldc, hipStream_t s) {
    const long tiles = (long)ms_cdiv(M, 32) * ms_cdiv(N, 32);
    const bool fast = f32_fast(A0, K0, false, M, K0) && f32_fast(B0, K0, false, N, K0);
    if (!ms_launch_fits(2 * tiles, 256) || fast != (f32_fast(A1, K1, false, M, K1) && f32_fast(B1, K1, false, N, K1))) {
        MS_TRY(ms_k_gemm(MS_F32, 0, 0, M, N, K0, 1.f, A0, K0, B0, K0, C0, ldc, 1, 0, nullptr, nullptr, 0, 0, 1, s));
        return ms_k_gemm(MS_F32, 0, 0, M, N, K1, 1.f, A1, K1, B1, K1, C1, ldc, 1, 0, nullptr, nullptr, 0, 0, 1, s);
    }
    GemmF32Params p0 = {}, p1 = {};
    p0.A = A0; p0.B = B0; p0.C = C0; p0.lda = p0.ldb = p0.K = K0;
    p1.A = A1; p1.B = B1; p1.C = C1; p1.lda = p1.ldb = p1.K = K1;
    p0.ldc = p1.ldc = ldc; p0.M = p1.M = M; p0.N = p1.N = N; p0.tiles_n = p1.tiles_n = ms_cdiv(N, 32); p0.alpha = p1.alpha = 1.f;
    if (fast) gemm_f32_two_kernel<true><<<(unsigned)(2 * tiles), 256, 0, s>>>(p0, p1, (int)tiles);
    else gemm_f32_two_kernel<false><<<(unsigned)(2 * tiles), 256, 0, s>>>(p0, p1, (int)tiles);
    MS_LAUNCH_CHECK();
    return MS_OK;
}

// ------------------------------------------------------------------ student-logits GEMM with KD epilogues
// zs = A[M,K] B[N,K]^T is never stored: mode EPI_KD_STATS folds it (with the teacher logits zt of the same
// chunk) into per-strip partial statistics, mode EPI_KD_DZ turns it into dz.  bf16 fast path only.
bool gemm_kd_epilogue_supported(int M, int N, int K, const void *A, long lda, const void *B, long ldb, const float *zt,
                                long ldz, const void *dz, long lddz, int dz_fp32) {
    auto al = [](const void *q) { return ((uintptr_t)q & 15) == 0; };
    const long lim = (1L << 32) - (1L << 20);
    const int forced = forced_tile();
    return forced >= 0 && M > 0 && N > 0 && K > 0 && K % BK == 0 && N % 4 == 0 && al(A) && al(B) && al(zt) && lda % 8 == 0 &&
           ldb % 8 == 0 && ldz % 4 == 0 && ((long)M + 256) * lda * 2 < lim && ((long)N + 256) * ldb * 2 < lim &&
           ((long)M + 256) * ldz * 4 < lim && (!dz || (al(dz) && lddz % 4 == 0 && ((long)M + 256) * lddz * (dz_fp32 ? 4 : 2) < lim));
}

static ms_status prepare_kd(int mode, int M, int N, int K, const void *A, long lda, const void *B, long ldb, const float *zt,
                            long ldz, float *stats, float *part, int nparts, float inv_t, float coef, void *dz, long lddz,
                            int dz_fp32, GemmParams *out) {
    if (!gemm_kd_epilogue_supported(M, N, K, A, lda, B, ldb, zt, ldz, mode == EPI_KD_DZ ? dz : nullptr, lddz, dz_fp32))
        return ms_fail(MS_ERR_UNSUPPORTED, "gemm_kd_epilogue: shape or alignment outside the fast path");
    if ((mode == EPI_KD_DZ && (!dz || !stats)) || (mode == EPI_KD_STATS && (!part || nparts < ms_cdiv(N, 64))) ||
        (mode != EPI_KD_DZ && mode != EPI_KD_STATS))
        return ms_fail(MS_ERR_INVALID_ARG, "gemm_kd_epilogue: bad mode or null buffer");
    GemmParams &p = *out;
    p = {};
    p.A = A; p.B = B; p.C = dz; p.lda = lda; p.ldb = ldb; p.ldc = lddz; p.M = M; p.N = N; p.K = K; p.alpha = 1.f;
    p.c_fp32 = dz_fp32;
    p.kd_zt = zt; p.kd_ldz = ldz; p.kd_stats = stats; p.kd_part = part; p.kd_nparts = nparts; p.kd_inv_t = inv_t; p.kd_coef = coef;
    p.k_tiles_per_split = ms_cdiv(K, BK);
    return MS_OK;
}

ms_status gemm_kd_epilogue(int mode, int M, int N, int K, const void *A, long lda, const void *B, long ldb, const float *zt,
                           long ldz, float *stats, float *part, int nparts, float inv_t, float coef, void *dz, long lddz,
                           int dz_fp32, hipStream_t s) {
    GemmParams p;
    MS_TRY(prepare_kd(mode, M, N, K, A, lda, B, ldb, zt, ldz, stats, part, nparts, inv_t, coef, dz, lddz, dz_fp32, &p));
    const int tile = choose_tile(M, N, p.k_tiles_per_split, kKdEpilogueBytes);
    if (mode == EPI_KD_DZ) return launch_bf16_fast<EPI_KD_DZ>(p, tile, 0, 0, 1, 2.0 * M * N * K, s);
    return launch_bf16_fast<EPI_KD_STATS>(p, tile, 0, 0, 1, 2.0 * M * N * K, s);
}

template <int EPI> static void launch_two(int tile, int first, GemmParams &pt, GemmParams &ps, hipStream_t s) {
    const MsTile &t = kTiles[tile];
    pt.tiles_m = ps.tiles_m = ms_cdiv(ps.M, t.bm);
    pt.tiles_n = ms_cdiv(pt.N, t.bn);
    ps.tiles_n = ms_cdiv(ps.N, t.bn);
    const int nt = pt.tiles_m * pt.tiles_n, ns = ps.tiles_m * ps.tiles_n, run = 256 * t.per_cu;
    if (tile == T256) {
        gemm_bf16_pp_two_kernel<EPI><<<nt + ns, 512, 0, s>>>(pt, ps, nt, ns, run, first);
        return;
    }
#define GO(BM, BN, WM, WN, NST) gemm_bf16_two_kernel<BM, BN, WM, WN, NST, EPI><<<nt + ns, 64 * WM * WN, 0, s>>>(pt, ps, nt, ns, run, first)
    switch (tile) {
        case R128: GO(128, 128, 4, 2, 4); break;
        case R128x256: GO(128, 256, 2, 4, 3); break;
        case R64x128: GO(64, 128, 2, 2, 3); break;
        case R64: GO(64, 64, 2, 1, 4); break;
        default: GO(128, 128, 2, 2, 2); break;
    }
#undef GO
}

ms_status gemm_kd_and_teacher(int mode, int M, int N, int K, const void *A, const void *B, const float *zt, float *stats, float *part, int nparts,
                              float inv_t, float coef, void *dz, long ld, int Nt, int Kt, const void *At, const void *Bt, float *next_zt, hipStream_t s) {
    GemmParams ps;
    MS_TRY(prepare_kd(mode, M, N, K, A, K, B, K, zt, ld, stats, part, nparts, inv_t, coef, dz, ld, 0, &ps));
    Bf16Gemm t;
    MS_TRY(prepare_bf16(0, 0, M, Nt, Kt, 1.f, At, Kt, Bt, Kt, next_zt, ld, 1, 0, nullptr, nullptr, 0, 0, &t));
    int first = 0;
    const int tile = t.fast && use_mfma16() ? ms_choose_two(M, N, ps.k_tiles_per_split, Nt, t.kt, forced_tile(), &first) : -1;
    if (tile >= 0 && ms_launch_fits(ms_tiles(kTiles[tile], M, N) + ms_tiles(kTiles[tile], M, Nt), 512)) {
        set_splits(t, 1);
        ProfScope prof(0, 2.0 * M * ((double)N * K + (double)Nt * Kt), s);
        if (mode == EPI_KD_DZ) launch_two<EPI_KD_DZ>(tile, first, t.p, ps, s);
        else launch_two<EPI_KD_STATS>(tile, first, t.p, ps, s);
        MS_LAUNCH_CHECK();
        return MS_OK;
    }
    MS_TRY(gemm_kd_epilogue(mode, M, N, K, A, K, B, K, zt, ld, stats, part, nparts, inv_t, coef, dz, ld, 0, s));
    return ms_k_gemm(MS_BF16, 0, 0, M, Nt, Kt, 1.f, At, Kt, Bt, Kt, next_zt, ld, 1, 0, nullptr, nullptr, 0, 0, 1, s);
}

// ------------------------------------------------------------------ fused gate/up GEMM + SwiGLU
// act[M, F] = silu(A W_gate^T) * (A W_up^T) with W = [gate rows | up rows] ([2F, K]); gate_up (optional,
// [M, 2F]) also receives the rounded pre-activations for the backward pass.  bf16 fast path only.
bool gemm_swiglu_supported(int M, int F, int K, const void *A, long lda, const void *W, long ldw, const void *act, long ldact,
                           const void *gate_up, long ldgu) {
    auto al = [](const void *q) { return ((uintptr_t)q & 15) == 0; };
    const long lim = (1L << 32) - (1L << 20);
    const int forced = forced_tile();
    return forced >= 0 && M > 0 && F > 0 && K > 0 && K % BK == 0 && F % 4 == 0 && al(A) && al(W) && al(act) && lda % 8 == 0 &&
           ldw % 8 == 0 && ldact % 4 == 0 && ((long)M + 256) * lda * 2 < lim && (2L * F + 256) * ldw * 2 < lim &&
           ((long)M + 256) * ldact * 2 < lim && (!gate_up || (al(gate_up) && ldgu % 4 == 0 && ((long)M + 256) * ldgu * 2 < lim));
}

ms_status gemm_swiglu(int M, int F, int K, const void *A, long lda, const void *W, long ldw, void *act, long ldact,
                      void *gate_up, long ldgu, hipStream_t s) {
    if (!gemm_swiglu_supported(M, F, K, A, lda, W, ldw, act, ldact, gate_up, ldgu))
        return ms_fail(MS_ERR_UNSUPPORTED, "gemm_swiglu: shape or alignment outside the fast path");
    GemmParams p = {};
    p.A = A; p.B = W; p.C = act; p.lda = lda; p.ldb = ldw; p.ldc = ldact; p.M = M; p.N = F; p.K = K; p.alpha = 1.f;
    p.sg_f = F; p.sg_gu = gate_up; p.sg_ldgu = ldgu;
    p.k_tiles_per_split = ms_cdiv(K, BK);
    return launch_bf16_fast<EPI_SWIGLU>(p, choose_tile(M, 2 * F, p.k_tiles_per_split, gate_up ? 3 : 1), 0, 0, 1, 4.0 * M * F * K, s);
}

extern "C" ms_status ms_k_gemm_swiglu(int32_t M, int32_t F, int32_t K, const void *A, int64_t lda, const void *W, int64_t ldw,
                                      void *act, int64_t ldact, void *gate_up, int64_t ldgu, void *stream) {
    if (!A || !W || !act) return ms_fail(MS_ERR_INVALID_ARG, "gemm_swiglu: null pointer");
    return gemm_swiglu(M, F, K, A, lda, W, ldw, act, ldact, gate_up, ldgu, (hipStream_t)stream);
}
