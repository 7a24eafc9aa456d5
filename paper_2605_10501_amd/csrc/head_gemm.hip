// bf16 matrix products of the losses at the end of a section: the tiles and main loops of gemm_bf16.h under kernels that take the number of rows
// from device memory.  Only tokens that count have a row, and how many do is not known to the host: a grid is made for all of a block's tokens, and the
// workgroups past the rows that there are end at once (16384 tokens, three quarters of them scored, V = 151936: the products take three quarters of the time).
#include "common.h"
#include "gemm_bf16.h"
#include "head_gemm.h"
#include "launch.h"
#include "launch_plan.h"

namespace {

__device__ __forceinline__ int rows_in_use(int rows, const int *count) { return count ? (*count < rows ? *count : rows) : rows; }

template <int EPI>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) void head_pp_kernel(GemmParams p, const int *count) {
    MS_PP_LDS;
    PpLds all = lds;
    if constexpr (EPI == EPI_EXP) {
        MS_HEAD_LDS(256, 256);
        all.head = {head_rows, head_marks, head_first};
    }
    p.M = rows_in_use(p.M, count);
    p.tiles_m = (p.M + 255) / 256;
    const int nb = p.tiles_m * p.tiles_n;
    if ((int)blockIdx.x >= nb) return;
    gemm_pp_body<EPI>(p, all, blockIdx.x, nb, 0);
}
template <int BM, int BN, int WM, int WN, int NST, int EPI>
__global__ __launch_bounds__(64 * WM * WN) __attribute__((amdgpu_waves_per_eu(fast_waves_per_simd(BM, WM * WN, EPI, NST)))) void head_tile_kernel(GemmParams p, const int *count) {
    MS_FAST_LDS(BM, BN, NST);
    FastLds<BM, BN, NST> all = lds;
    if constexpr (EPI == EPI_EXP) {
        MS_HEAD_LDS(BM, BN);
        all.head = {head_rows, head_marks, head_first};
    }
    p.M = rows_in_use(p.M, count);
    p.tiles_m = (p.M + BM - 1) / BM;
    const int nb = p.tiles_m * p.tiles_n;
    if ((int)blockIdx.x >= nb) return;
    gemm_fast_body<BM, BN, WM, WN, false, false, EPI, true, NST>(p, all, blockIdx.x, nb, 0);
}

// Input gradient (pd: rows = M, in `parts` parts of K, each with a result of its own, part_ld elements apart) and weight gradient (pw: rows = K) in one grid, as
// gemm_bf16_pair_kernel; nw workgroups of the latter (0: none), pd.M = 0: none of the former
template <int BM, int BN, int WM, int WN, int NST>
__global__ __launch_bounds__(64 * WM * WN) __attribute__((amdgpu_waves_per_eu(fast_waves_per_simd(BM, WM * WN, EPI_NONE, NST)))) void head_pair_kernel(GemmParams pd, GemmParams pw, int parts, long part_ld,
                                                                                                                                                      int nw, int wgrad_first, const int *count) {
    MS_FAST_LDS(BM, BN, NST);
    pd.M = rows_in_use(pd.M, count);
    pw.K = rows_in_use(pw.K, count);
    pd.tiles_m = (pd.M + BM - 1) / BM;
    const int b = blockIdx.x, tiles = pd.tiles_m * pd.tiles_n, nd = tiles * parts;
    if (b >= nd + nw) return;
    if (wgrad_first ? b < nw : b >= nd) {
        gemm_fast_body<BM, BN, WM, WN, true, true, EPI_NONE, true, NST>(pw, lds, wgrad_first ? b : b - nd, nw, 0);
    } else {
        const int bd = wgrad_first ? b - nw : b, part = bd / tiles;
        pd.C = (float *)pd.C + part * part_ld;
        gemm_fast_body<BM, BN, WM, WN, false, true, EPI_NONE, true, NST>(pd, lds, bd - part * tiles, tiles, part);
    }
}

GemmParams product(int M, int N, int K, const void *A, long lda, const void *B, long ldb, void *C, long ldc, int c_fp32, int accumulate) {
    GemmParams p = {};
    p.A = A; p.B = B; p.C = C; p.lda = lda; p.ldb = ldb; p.ldc = ldc; p.M = M; p.N = N; p.K = K;
    p.alpha = 1.f; p.c_fp32 = c_fp32; p.accumulate = accumulate;
    p.k_tiles_per_split = ms_cdiv(K, BK) < 1 ? 1 : ms_cdiv(K, BK);
    p.vec_epilogue = 1;
    return p;
}

// Whether `rows` rows of ld numbers lie within reach of 32-bit offsets, as the plan sees to (head_plan)
bool in_reach(long rows, long ld, int bytes) { return (rows + 256) * ld * bytes <= kHeadReach; }

template <int EPI> ms_status launch_rows(GemmParams &p, double out_bytes, const int *count, hipStream_t s) {
    if (!in_reach(p.M, p.lda, 2) || !in_reach(p.N, p.ldb, 2) || (p.C && !in_reach(p.M, p.ldc, p.c_fp32 ? 4 : 2)))
        return ms_fail(MS_ERR_UNSUPPORTED, "head: operands or logits of %d x %d x %d beyond 4 GB", p.M, p.N, p.K);
    const int tile = count ? head_logits_tile(p.M, p.N, p.k_tiles_per_split, out_bytes, gemm_forced_tile()) : ms_choose_tile(p.M, p.N, p.k_tiles_per_split, out_bytes, gemm_forced_tile(), true);
    const MsTile &t = kTiles[tile];
    p.tiles_m = ms_cdiv(p.M, t.bm);
    p.tiles_n = ms_cdiv(p.N, t.bn);
    if (!ms_launch_fits((long)p.tiles_m * p.tiles_n, 512)) return ms_fail(MS_ERR_UNSUPPORTED, "head: %d x %d logits in one launch", p.M, p.N);
    const dim3 grid(p.tiles_m * p.tiles_n);
    ProfScope ps(0, 2.0 * p.M * p.N * p.K, s);
#define GO(BM, BN, WM, WN, NST) head_tile_kernel<BM, BN, WM, WN, NST, EPI><<<grid, 64 * WM * WN, 0, s>>>(p, count)
    switch (tile) {
        case T256: head_pp_kernel<EPI><<<grid, 512, 0, s>>>(p, count); break;
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

}  // namespace

ms_status head_gemm_exp(int rows, int cw, int d, const void *h, const void *w, const float2 *ref, int v0, float *z_label, const HeadMarks &marks, float it2, void *c, long ldc, float2 *part, long ld,
                        const int *count, hipStream_t s) {
    GemmParams p = product(rows, cw, d, h, d, w, d, c, ldc, 0, 0);
    p.kd_stats = (float *)const_cast<float2 *>(ref); p.kd_part = (float *)part; p.kd_ldz = ld; p.kd_inv_t = it2; p.sg_f = v0; p.sg_gu = z_label;
    if (marks.word) p.residual = marks.word, p.bias = marks.first, p.sg_gu = marks.z, p.ldr = marks.k;
    return launch_rows<EPI_EXP>(p, c ? 4 : 2, count, s);
}

ms_status head_gemm_logits(int rows, int cw, int d, const void *h, const void *w, float it2, float *c, long ldc, float2 *part, long ld, hipStream_t s) {
    GemmParams p = product(rows, cw, d, h, d, w, d, c, ldc, 1, 0);
    p.kd_part = (float *)part; p.kd_ldz = ld; p.kd_inv_t = it2;
    return launch_rows<EPI_LOGITS>(p, 6, nullptr, s);
}

ms_status head_gemm_backward(const HeadChoice &c, int rows, int cw, int d, const void *e, long ld, const void *w, const void *x, float *d_h, int add, float *d_w,
                             const int *count, hipStream_t s) {
    GemmParams pd = product(d_h ? rows : 0, d, cw, e, ld, w, d, d_h, d, 1, add), pw = product(cw, d, rows, e, ld, x, d, d_w, d, 1, 1);
    const MsTile &t = kTiles[c.tile];
    if (!in_reach(rows, ld, 2) || !in_reach(cw, d, d_w ? 4 : 2) || !in_reach(rows, d, d_h ? 4 : 2)) return ms_fail(MS_ERR_UNSUPPORTED, "head: gradients of %d x %d x %d beyond 4 GB", rows, cw, d);
    pd.k_tiles_per_split = ms_cdiv(pd.k_tiles_per_split, c.parts);
    const int parts = ms_cdiv(ms_cdiv(cw, BK), pd.k_tiles_per_split);
    if (d_h && !add && parts != c.parts) return ms_fail(MS_ERR_INVALID_ARG, "head: %d parts of %d columns", c.parts, cw);   // (later slabs may add to fewer)
    pd.tiles_n = ms_cdiv(pd.N, t.bn);
    pw.tiles_m = ms_cdiv(pw.M, t.bm);
    pw.tiles_n = ms_cdiv(pw.N, t.bn);
    const long nd = (long)ms_cdiv(pd.M, t.bm) * pd.tiles_n * parts, nw = d_w ? (long)pw.tiles_m * pw.tiles_n : 0;
    if (!ms_launch_fits(nd + nw, 512)) return ms_fail(MS_ERR_UNSUPPORTED, "head: gradients of %d x %d in one launch", rows, cw);
    const unsigned grid = (unsigned)(nd + nw);
    ProfScope ps(1, 2.0 * rows * d * (double)cw * ((d_h ? 1 : 0) + (d_w ? 1 : 0)), s);
#define GO(BM, BN, WM, WN, NST) head_pair_kernel<BM, BN, WM, WN, NST><<<grid, 64 * WM * WN, 0, s>>>(pd, pw, parts, (long)rows * d, (int)nw, c.wgrad_first, count)
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
