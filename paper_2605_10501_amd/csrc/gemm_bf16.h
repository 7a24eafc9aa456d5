// The parts that bf16 matrix-product kernels are made of (gemm.hip says what each tile is for): how operand tiles get into LDS and registers, the
// main loops of a workgroup, and their epilogues.  The kernels around them are in gemm.hip and head_gemm.hip.
#pragma once
#include <type_traits>
#include <utility>

#include "common.h"
#include "mfma_tiles.h"

namespace {

// gcc-style vectors: the return types of the buffer load builtins
typedef unsigned int u32x4 __attribute__((vector_size(16)));
typedef unsigned int u32x2 __attribute__((vector_size(8)));

struct GemmParams {
    const void *A, *B;
    void *C;
    const void *bias, *residual;
    long lda, ldb, ldc, ldr;
    int M, N, K;
    int tiles_m, tiles_n;
    int k_tiles_per_split;  // in units of 64
    float alpha;
    int c_fp32, accumulate, atomic, res_fp32, vec_epilogue;
    // KD epilogues (EPI != 0): the tile holds student logits zs; zt = teacher logits of the same chunk
    const float *kd_zt;      // [M, kd_ldz] fp32
    long kd_ldz;
    float *kd_stats;         // EPI_KD_DZ: [M][8] per-token statistics (lse_t at 6, lse_s at 7), read
    float *kd_part;          // EPI_KD_STATS: [M][kd_nparts][8] partial statistics per 64-column strip, written
    int kd_nparts;
    float kd_inv_t, kd_coef;
    // EPI_SWIGLU: B = [gate rows (sg_f) | up rows (sg_f)], N = sg_f output columns; C = silu(gate) * up
    // [M, ldc]; sg_gu (optional) also receives the rounded gate | up pre-activations [M, sg_ldgu]
    int sg_f;
    void *sg_gu;
    long sg_ldgu;
};

// EPI_SWIGLU_BWD: the tile holds da = dL/d(silu(gate) * up); sg_gu = the pre-activations [M, sg_ldgu], read; C = [dgate | dup] [M, ldc]
// EPI_EXP, EPI_LOGITS: the tile holds logits z (head_gemm.hip).  EXP: kd_stats = (reference, label as an int) of each row [M]; C (may be null) = 2^(x - reference) with
// x = z kd_inv_t, bf16, zeros in the columns N .. N + 63 / 64 * 64; sg_gu (fp32) = z of a row's label [M], if that is one of the columns sg_f .. sg_f + N - 1 of the vocabulary,
// or, with marks, of a row's selected ids [M][ldr]: residual = which columns of a strip those are (a 64-bit word for each strip and row, [strip][kd_ldz]), bias = the place of the
// first (a byte each); LOGITS: C = z, fp32.  kd_part = (offset, sum) of every 64-column strip and row, [strip][kd_ldz].
enum { EPI_NONE = 0, EPI_KD_DZ = 1, EPI_KD_STATS = 2, EPI_SWIGLU = 3, EPI_SWIGLU_BWD = 4, EPI_EXP = 5, EPI_LOGITS = 6 };

// Reductions over the four 16-lane groups of a wave, on the vector ALU (no LDS crossbar): lane l gets the result over lanes
// l % 16, l % 16 + 16, + 32 and + 48.  v_permlane16_swap of a register with itself leaves the even groups' values in one
// result and the odd groups' in the other, v_permlane32_swap the lower and the upper half's.
template <class F> __device__ __forceinline__ float across_groups(float v, F f) {
    const unsigned a = __builtin_bit_cast(unsigned, v);
    const auto q = __builtin_amdgcn_permlane16_swap(a, a, false, false);
    const unsigned b = __builtin_bit_cast(unsigned, f(__builtin_bit_cast(float, (unsigned)q[0]), __builtin_bit_cast(float, (unsigned)q[1])));
    const auto h = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    return f(__builtin_bit_cast(float, (unsigned)h[0]), __builtin_bit_cast(float, (unsigned)h[1]));
}
// What EPI_EXP reads of a tile's rows, (reference, label) and the marks of their strips, comes to LDS by direct loads that a workgroup issues before all others: read in the
// epilogue, each of its 32-row blocks waited for memory (marks, 32768 x 50688 x 1536: 4.22 ms without any, 4.41 read there, 4.37 so).  At least 128 rows, the 1 KB of a wave's load.
struct HeadRowsLds {
    float2 *rows;                            // [128 or 256]
    unsigned long long *marks;               // [tile's strips][128 or 256]
    unsigned char *first;                    // the same
};
#define MS_HEAD_LDS(BM, BN)                                                                                            \
    constexpr int kHeadRows = BM > 128 ? BM : 128;                                                                     \
    __shared__ __align__(16) float2 head_rows[kHeadRows];                                                              \
    __shared__ __align__(16) unsigned long long head_marks[BN / 64 * kHeadRows];                                       \
    __shared__ __align__(16) unsigned char head_first[BN / 64 * kHeadRows]
template <int BM, int BN, int WAVES>
__device__ __forceinline__ void head_rows_fetch(const GemmParams &p, const HeadRowsLds &lds, int m0, int n0, int wave, int lane) {
    constexpr int kRows = BM > 128 ? BM : 128, kPieces = kRows / 128;
    const __amdgpu_buffer_rsrc_t rr = make_rsrc(p.kd_stats, (long)((p.M + 1) / 2) * 16);
#pragma unroll
    for (int i = wave; i < kPieces; i += WAVES)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rr, (lds_void *)(lds.rows + i * 128), 16, (unsigned)(m0 + i * 128) * 8 + lane * 16, 0, 0, 0);
    if (!p.residual) return;
    // (rows past the last one read the next strip's words, which nobody looks at; the last strip's end is the descriptor's)
    const int strips = (p.N + 63) >> 6, first = n0 >> 6;
#pragma unroll
    for (int i = wave; i < BN / 64 * kPieces; i += WAVES) {
        const int strip = i / kPieces, piece = i % kPieces;
        const long at = (long)(first + strip) * p.kd_ldz + m0 + piece * 128, left = (long)strips * p.kd_ldz - at;
        const __amdgpu_buffer_rsrc_t rm = make_rsrc((const unsigned long long *)p.residual + (left > 0 ? at : 0), left > 0 ? (left < 128 ? left : 128) * 8 : 0);      // (kd_ldz is a multiple of 16)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rm, (lds_void *)(lds.marks + i * 128), 16, lane * 16, 0, 0, 0);
        const __amdgpu_buffer_rsrc_t rf = make_rsrc((const unsigned char *)p.bias + (left > 0 ? at : 0), left > 0 ? (left < 128 ? left : 128) : 0);
        if (lane < 8) __builtin_amdgcn_raw_ptr_buffer_load_lds(rf, (lds_void *)(lds.first + i * 128), 16, lane * 16, 0, 0, 0);
    }
}

// Reductions over each 16 lanes that hold a row's 64 columns four by four; every lane gets the result
template <class F> __device__ __forceinline__ float across_row(float v, F f) {
    auto turned = [](float a, auto by) { return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, a), 0x120 + decltype(by)::value, 0xf, 0xf, true)); };
    v = f(v, turned(v, std::integral_constant<int, 8>{}));
    v = f(v, turned(v, std::integral_constant<int, 4>{}));
    v = f(v, turned(v, std::integral_constant<int, 2>{}));
    return f(v, turned(v, std::integral_constant<int, 1>{}));
}
// fmaxf of three values that no instruction has produced yet (loads) costs three more to quiet signalling NaNs; v_max3 does so itself
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// Cache policy of the vector epilogues' global accesses (auxiliary operand of the buffer instructions): non-temporal.
// The output tile, the residual and the teacher logits stream through once, and the 4 MB L2 of an XCD is what
// keeps the operand panels that its 32 CUs share; left at the default policy the epilogue traffic evicts them
// (measured: fp32-output and fp32-residual GEMMs 7-8 % slower, the c2 step 2.5 %).  The operand loads keep the
// default: made non-temporal they lose that sharing (15 % slower).
constexpr int kStream = 2;

// ------------------------------------------------------------------ fast path
// Same tiling and MFMA loop, but
//   * an operand stored K-contiguous goes global -> LDS directly (buffer_load ... lds, 16 bytes per
//     lane, one instruction fills 8 tile rows = 1 KB): lane l of the instruction that fills rows
//     8G .. 8G+7 lands at row 8G + l/8, chunk position l%8, so it fetches the chunk that the LDS
//     swizzle assigns to that position.  No staging registers, no LDS store instructions; rows
//     past the end of the matrix read as zero through the buffer descriptor's range check;
//   * the epilogue addresses C (and the residual) through buffer descriptors as well, so rows
//     past M are dropped by the range check and columns past N by one select per column:
//     no per-element branches.
// Needs K % 64 == 0 when an operand is K-contiguous and every matrix below 4 GB.
// The same for an operand stored K-major: the tile is 64 k-rows x COLS columns, kept as COLS/64 sub-tiles
// [64][64]; instruction idx fills 8-row group idx % 8 of sub-tile idx / 8.  Rows past K fall outside the
// descriptor (zeros), so K needs no padding; columns past the matrix edge read the next row (never stored).
template <int COLS, int NWAVES>
struct RowTileStager {
    static constexpr int NI = COLS / 8 / NWAVES;
    unsigned base[NI];                     // byte offset of this lane's 16 bytes at k0 = 0, per instruction
    unsigned ldb;                          // bytes per k-row
    __device__ __forceinline__ void init(long ld, int col0, int wave, int lane) {
        ldb = (unsigned)(ld * 2);
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int idx = wave * NI + i, sub = idx >> 3, g = idx & 7;
            const int r = g * 8 + (lane >> 3);
            const int c = (lane & 7) ^ swz_row(r);
            base[i] = (unsigned)r * ldb + (unsigned)(col0 + sub * 64 + c * 8) * 2;
        }
    }
    __device__ __forceinline__ void issue(__amdgpu_buffer_rsrc_t rs, bf16_t *tile, int k0, int wave, unsigned inv) const {
        const unsigned koff = (unsigned)k0 * ldb;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int idx = wave * NI + i;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void *)(tile + (idx >> 3) * 4096 + (idx & 7) * 512), 16,
                                                     (base[i] + koff) | inv, 0, 0, 0);
        }
    }
};

// B tile of the fused gate/up + SwiGLU GEMM: tile row R = 64 * w + 32 * u + l holds weight row
// u * F + col0 + 32 * w + l (u = 0 gate, 1 up), so that the two 32-column blocks of wave column w are
// the gate and the up pre-activation of the same 32 output columns (same lane, same register).
template <int ROWS, int NWAVES>
struct GateUpStager {
    static constexpr int NI = ROWS / 8 / NWAVES;
    unsigned lanepart;                     // (lane >> 3) rows + swizzle-free part, in bytes
    unsigned ldb;                          // bytes per row
    int x, col0, f;
    __device__ __forceinline__ void init(long ld, int col0_, int f_, int lane) {
        ldb = (unsigned)(ld * 2);
        lanepart = (unsigned)(lane >> 3) * ldb;
        x = (lane & 7) ^ swz_row(lane >> 3);
        col0 = col0_;
        f = f_;
    }
    __device__ __forceinline__ void issue(__amdgpu_buffer_rsrc_t rs, bf16_t *tile, int k0, int wave, unsigned inv) const {
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int g = wave * NI + i;                                   // 8-row group of the tile (scalar)
            const int wrow = ((g >> 2) & 1) * f + col0 + (g >> 3) * 32 + (g & 3) * 8;
            const unsigned voff = ((unsigned)wrow * ldb + lanepart + ((x ^ swz_row(8 * g)) << 4)) | inv;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void *)(tile + g * 8 * BK), 16, voff, k0 * 2, 0, 0);
        }
    }
};

template <int ROWS, int NWAVES>
struct DmaStager {
    static constexpr int NI = ROWS / 8 / NWAVES;   // instructions per wave per tile
    unsigned rowoff;                       // byte offset of this lane's row within an 8-row group
    unsigned ld8;                          // bytes between 8-row groups
    int x;                                 // (lane & 7) ^ swz_row(lane >> 3): chunk swizzle without the group term swz_row(8 g)
    __device__ __forceinline__ void init(long ld, int row0, int lane) {
        rowoff = (unsigned)(((long)(row0 + (lane >> 3)) * ld) * 2);
        ld8 = (unsigned)(ld * 16);
        x = (lane & 7) ^ swz_row(lane >> 3);
    }
    // wave (scalar) fills 8-row groups wave*NI .. wave*NI + NI-1 of the tile
    // inv = 0, or kOob to fill the tile with zeros (OR-ing it in puts every lane out of range without a branch)
    __device__ __forceinline__ void issue(__amdgpu_buffer_rsrc_t rs, bf16_t *tile, int k0, int wave, unsigned inv) const {
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int g = wave * NI + i;
            const unsigned voff = (rowoff + g * ld8 + ((x ^ swz_row(8 * g)) << 4)) | inv;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void *)(tile + g * 8 * BK), 16, voff, k0 * 2, 0, 0);
        }
    }
};

// Scheduling pattern of one k-step: spread R LDS reads over the first MFMAs (R/M each, at least one),
// then the remaining MFMAs back to back.
template <int N>
__device__ __forceinline__ void sched_reads_then_mfma() {
    __builtin_amdgcn_sched_group_barrier(0x100, N, 0);   // N LDS reads
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);   // one MFMA
}
template <int R, int PER, int... I>
__device__ __forceinline__ void sched_pairs(std::integer_sequence<int, I...>) {
    (sched_reads_then_mfma<((I + 1) * PER <= R ? PER : R - I * PER)>(), ...);
}
// Scheduling pattern of one k-step with 16-row fragments: per row block, its NB MFMAs and then the reads that
// refill its A fragment (RA reads) and the next BPB of the NB B fragments (RB reads each).
// VM = number of direct-to-LDS loads issued in this k-step (0, or one tile's worth): spread evenly over the row blocks.
template <int NB, int RA, int RB, int VM, int... I>
__device__ __forceinline__ void sched_mfma_then_reads(std::integer_sequence<int, I...>) {
    constexpr int MB = sizeof...(I), PB = (VM + MB - 1) / MB;      // loads per row block
    constexpr int BPB = (NB + MB - 1) / MB;                        // B fragments per row block
    ((__builtin_amdgcn_sched_group_barrier(0x008, NB, 0),
      __builtin_amdgcn_sched_group_barrier(0x100, RA + RB * (I * BPB >= NB ? 0 : (NB - I * BPB < BPB ? NB - I * BPB : BPB)), 0),
      (I * PB < VM ? __builtin_amdgcn_sched_group_barrier(0x020, (VM - I * PB < PB ? VM - I * PB : PB), 0) : (void)0)), ...);
}
template <int R, int M>
__device__ __forceinline__ void interleave_reads_with_mfma() {
    constexpr int PER = R >= M ? (R + M - 1) / M : 1;     // reads in front of each of the first MFMAs
    constexpr int PAIRS = (R + PER - 1) / PER;
    static_assert(PAIRS <= M, "more read groups than MFMAs");
    sched_pairs<R, PER>(std::make_integer_sequence<int, PAIRS>{});
    if constexpr (M > PAIRS) __builtin_amdgcn_sched_group_barrier(0x008, M - PAIRS, 0);
}

// Addresses of the transposing reads of a K-major operand for v_mfma_f32_16x16x32_bf16: the 16 lanes of group g
// (= lane / 16) read k rows 8g .. 8g+7 of the k-step (two reads of four rows) for the 16 columns of a block.
// The LDS swizzle of those rows does not depend on the k-step, and the two 16-column halves of a 32-column
// block differ by one flipped chunk bit: four registers per operand, everything else is a constant offset.
struct TrFragAddr16 {
    int base[2][2];   // [16-column half of the 32-column block][first / second read], element offset within the tile
    __device__ __forceinline__ void init(int w32, int lane) {
        const int g = lane >> 4, r = lane & 15, q = r >> 2;
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            const int m = w32 * 32 + 16 * hf + 4 * (r & 3);
            const int sub = m >> 6, chunk = (m & 63) >> 3;
#pragma unroll
            for (int rd = 0; rd < 2; ++rd) {
                const int rl = 8 * g + q + 4 * rd;                       // row within the 32-row k-step
                const int sw = swz_row(rl);
                base[hf][rd] = sub * 4096 + rl * 64 + ((chunk ^ sw) << 3) + (m & 7);
            }
        }
    }
    // block16 = index of the wave's 16-column block; off = element offset of its 32-column block's sub-tile pair
    __device__ __forceinline__ bf16x8 frag(const bf16_t *tile, int kk, int block16, int off) const {
        return tr_frag(tile + base[block16 & 1][0] + kk * 2048 + off, tile + base[block16 & 1][1] + kk * 2048 + off);
    }
};

// Addresses of the 16-byte fragment reads of a K-contiguous operand for v_mfma_f32_16x16x32_bf16: lane = (row
// lane % 16 of the 16-row block, k-group lane / 16).  The LDS swizzle makes the chunk position depend on the
// parity of the block and on the k-step; four registers per operand cover all blocks with constant offsets.
struct KFragAddr16 {
    int base[2][2];   // [block parity][k-step], element offset within the tile of block 0 / 1
    __device__ __forceinline__ void init(int row0, int lane) {      // row0 = first tile row of the wave (multiple of 32)
        const int r = lane & 15, g = lane >> 4;
#pragma unroll
        for (int par = 0; par < 2; ++par)
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) base[par][kk] = lds_off(row0 + par * 16 + r, kk * 4 + g) - par * 16 * BK;
    }
    __device__ __forceinline__ bf16x8 frag(const bf16_t *tile, int kk, int block16) const {
        return *(const bf16x8 *)(tile + base[block16 & 1][kk] + block16 * 16 * BK);
    }
};

// Epilogue of the fast kernels.  acc[i][j]: the wave's MI x NI accumulator blocks (16 x 16 with M16, else 32 x 32) of 64
// columns in all; the wave's 32-row block i starts at tile row row_base(i), its 32-column block j at tile column
// col_base(j); stg: 8 KB of LDS that belong to the wave (the operand buffers are idle by now).
template <int EPI, bool M16, bool TA, bool TB, int MI, int NI, class ACC, class RB, class CB>
__device__ __forceinline__ void gemm_epilogue(const GemmParams &p, ACC (&acc)[MI][NI], float *stg, int m0, int n0, int wn, int lane,
                                              RB row_base, CB col_base, const HeadRowsLds &head, int head_ld) {
    constexpr int FR = M16 ? 16 : 32, ACC_N = M16 ? 4 : 16, MI32 = MI * FR / 32, WTN = 64;
    static_assert(NI * FR == WTN, "staging assumes 64-column wave tiles");
    const int frow = lane & (FR - 1), fhalf = lane / FR;
    // ---- epilogue staging: the accumulators of the wave's 32-row block i go to LDS as [32 rows][64 columns]
    // fp32 (v = value transform), from where each lane reads 4 consecutive columns of a row.  The 16-column
    // group index (32x32 MFMA: column bit 5 only) is XOR-ed with row bits so that the lanes of one store
    // instruction, which hold the same columns of rows 4 apart, use different banks.
    auto stg_swz = [](int row) { return M16 ? ((row >> 2) & 3) << 4 : ((row >> 2) & 1) << 5; };
    // The lanes of a wave exchange data through the staging area, and the LDS executes a wave's accesses in
    // program order; what has to be kept is the program order itself: to the compiler a lane's reads and another
    // lane's writes are unrelated addresses that it may reorder.  wave_sync() is a compiler-level fence between the
    // two phases (no instruction).
    auto wave_sync = []() __attribute__((always_inline)) {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    };
    auto stage_block = [&](int i, auto v) __attribute__((always_inline)) {
        wave_sync();     // the reads of the previous block come first
        if constexpr (M16) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < NI; ++j)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int row = h * 16 + 4 * fhalf + r;
                        stg[row * 64 + ((j * 16 + frow) ^ stg_swz(row))] = v(acc[2 * i + h][j][r]);
                    }
        } else {
#pragma unroll
            for (int j = 0; j < NI; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int row = 8 * (r >> 2) + 4 * fhalf + (r & 3);
                    stg[row * 64 + ((j * 32 + frow) ^ stg_swz(row))] = v(acc[i][j][r]);
                }
        }
        wave_sync();     // every lane's values are in LDS before any lane reads
    };
    // ---- epilogue (EPI_EXP, which has other things in p.residual, p.bias and p.ldr, comes back before anything of rr is read).  C and the residual are addressed through buffer descriptors: rows past M are
    // dropped (stores) or read as zero by the range check, columns past N by one select.
    // Byte offset of row r of the wave's block i: the lane's part (its row within the pass and its column) once, the rest, which is
    // the same in all lanes, on the scalar unit.  A product per row and lane on the vector ALU is a quarter-rate instruction; with the
    // packed conversions below it was 46 instead of 35 vector instructions for four rows of the dz epilogue, 42 instead of 32 for
    // SwiGLU's (distillation head of 8192 tokens, V = 151936 31.01 -> 30.84 ms, 1024 tokens, V = 32000 638 -> 635 us, others even).
    auto row_bytes = [&](int i, int r, long ld, int es) { return (unsigned)(m0 + row_base(i) + r) * (unsigned)ld * (unsigned)es; };
    // four values in the storage type, two conversions of two
    auto pack4 = [](const float *v) {
        typedef bf16_t pair_t __attribute__((ext_vector_type(2)));
        u32x2 w;
        w[0] = __builtin_bit_cast(unsigned, pair_t{(bf16_t)v[0], (bf16_t)v[1]});
        w[1] = __builtin_bit_cast(unsigned, pair_t{(bf16_t)v[2], (bf16_t)v[3]});
        return w;
    };
    const int esz = p.c_fp32 ? 4 : 2;
    const __amdgpu_buffer_rsrc_t rc = make_rsrc(p.C, (long)p.M * p.ldc * esz);
    const int rsz = p.res_fp32 ? 4 : 2;
    const __amdgpu_buffer_rsrc_t rr = make_rsrc(p.residual ? p.residual : p.C, p.residual ? (long)p.M * p.ldr * rsz : 0);
    const bf16_t *bias = (const bf16_t *)p.bias;
    if constexpr (EPI == EPI_SWIGLU) {
        // acc[i][0] = gate, acc[i][1] = up of output columns n0/2 + wn*32 + (0..31).  Both are rounded to
        // the storage type first (they are the values a separate activation kernel would read back), staged
        // through LDS as [32 rows][gate 32 | up 32], and each lane then owns 4 consecutive output columns.
        static_assert(!TA && !TB, "SwiGLU epilogue is built for the K-contiguous layout");
        const int prow = lane >> 3, pcol = (lane & 7) * 4;
        const int colg = n0 / 2 + wn * 32 + pcol;
        const bool cok = colg < p.N;
        const unsigned lane_c = (unsigned)((prow * p.ldc + colg) * 2), lane_g = (unsigned)((prow * p.sg_ldgu + colg) * 2);
        const __amdgpu_buffer_rsrc_t rg = make_rsrc(p.sg_gu ? p.sg_gu : p.C, p.sg_gu ? (long)p.M * p.sg_ldgu * 2 : 0);
#pragma unroll
        for (int i = 0; i < MI32; ++i) {
            stage_block(i, [&](float a) { return (float)(bf16_t)(a * p.alpha); });
#pragma unroll
            for (int ps = 0; ps < 4; ++ps) {
                const int row = ps * 8 + prow;
                const int flip = stg_swz(row);
                const float4 g4 = *(const float4 *)(stg + row * 64 + (pcol ^ flip));
                const float4 u4 = *(const float4 *)(stg + row * 64 + ((32 + pcol) ^ flip));
                const float gv[4] = {g4.x, g4.y, g4.z, g4.w}, uv[4] = {u4.x, u4.y, u4.z, u4.w};
                float a[4];
#pragma unroll
                for (int e = 0; e < 4; ++e)   // silu(g) u = g u / (1 + e^-g); hardware reciprocal (1 ulp) instead of the division sequence
                    a[e] = gv[e] * uv[e] * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * gv[e]));
                __builtin_amdgcn_raw_buffer_store_b64(pack4(a), rc, cok ? lane_c + row_bytes(i, ps * 8, p.ldc, 2) : kOob, 0, kStream);
                if (p.sg_gu) {
                    const unsigned go = cok ? lane_g + row_bytes(i, ps * 8, p.sg_ldgu, 2) : kOob;
                    __builtin_amdgcn_raw_buffer_store_b64(pack4(gv), rg, go, 0, kStream);
                    __builtin_amdgcn_raw_buffer_store_b64(pack4(uv), rg, cok ? go + (unsigned)p.sg_f * 2 : kOob, 0, kStream);
                }
            }
        }
        return;
    }
    if constexpr (EPI == EPI_EXP || EPI == EPI_LOGITS) {
        // A lane has four consecutive columns of eight rows of each 32-row block, 16 lanes a row.  EXP: exponentials at the row's reference, which is a
        // logit of the row itself, so that their sum needs no maximum; a strip whose sum passes 2^64 (a column is 58 above the reference and more)
        // takes an offset of its own, which head.hip evens out.  LOGITS: the strip's maximum and the sum of 2^(x - maximum).
        static_assert(!TA && !TB && M16, "head epilogues are built for K-contiguous operands and 16-row fragments");
        const int prow = lane >> 4, pcol = (lane & 15) * 4, idx = lane & 15;
        const int colg = n0 + col_base(pcol >> 5) + (pcol & 31), strip = n0 + col_base(0);
        const bool cok = colg < p.N, stored = colg < (p.N + 63) / 64 * 64, full = strip + 64 <= p.N;     // (full: wave-uniform)
        const float it2 = p.kd_inv_t;
        const unsigned lane_c = (unsigned)((prow * p.ldc + colg) * (EPI == EPI_EXP ? 2 : 4));
        const __amdgpu_buffer_rsrc_t rz = make_rsrc(p.C ? p.C : p.kd_part, p.C ? (long)p.M * p.ldc * (EPI == EPI_EXP ? 2 : 4) : 0);
        auto sum = [](float a, float b) { return a + b; };
        auto larger = [](float a, float b) { return fmaxf(a, b); };
#pragma unroll
        for (int i = 0; i < MI32; ++i) {
            float ref[8], s[8], off[8];
            u32x2 w[8];
            int label = -1;                                                              // of the row that this lane stores for (idx < 8)
            if constexpr (EPI == EPI_EXP) {
#pragma unroll
                for (int ps = 0; ps < 8; ++ps) ref[ps] = head.rows[row_base(i) + ps * 4 + prow].x;
                label = __float_as_int(head.rows[row_base(i) + (idx & 7) * 4 + prow].y);
            }
            stage_block(i, [](float a) { return a; });
            auto row_of = [&](int ps, float (&z)[4]) __attribute__((always_inline)) {
                const int row = ps * 4 + prow;
                const float4 t = *(const float4 *)(stg + row * 64 + (pcol ^ stg_swz(row)));
                z[0] = t.x; z[1] = t.y; z[2] = t.z; z[3] = t.w;
            };
#pragma unroll
            for (int ps = 0; ps < 8; ++ps) {
                float z[4], e[4];
                row_of(ps, z);
                if constexpr (EPI == EPI_EXP) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) e[k] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[k], it2, -ref[ps]));
                    if (!full) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) e[k] = cok ? e[k] : 0.f;
                    }
                    w[ps] = pack4(e);
                    off[ps] = 0.f;
                } else {
                    float m = cok ? fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])) : -INFINITY;
                    m = across_row(m, larger);
                    const float u = m == -INFINITY ? 0.f : m;
#pragma unroll
                    for (int k = 0; k < 4; ++k) e[k] = cok ? __builtin_amdgcn_exp2f((z[k] - u) * it2) : 0.f;
                    off[ps] = m;
                    u32x4 v;
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[k] = __builtin_bit_cast(unsigned, z[k]);
                    __builtin_amdgcn_raw_buffer_store_b128(v, rz, cok ? lane_c + row_bytes(i, ps * 4, p.ldc, 4) : kOob, 0, kStream);
                }
                s[ps] = across_row((e[0] + e[1]) + (e[2] + e[3]), sum);
            }
            if constexpr (EPI == EPI_EXP) {
                const int row_here = idx * 4 + prow, at = label - p.sg_f - strip;
                const bool mine = idx < 8 && (unsigned)at < 64 && at < p.N - strip && m0 + row_base(i) + row_here < p.M;
                if (__any(mine) && mine) ((float *)p.sg_gu)[m0 + row_base(i) + row_here] = stg[row_here * 64 + (at ^ stg_swz(row_here))];
                if (p.residual) {
                    unsigned long long marks = idx < 8 && strip < p.N && m0 + row_base(i) + row_here < p.M ? head.marks[((strip - n0) >> 6) * head_ld + row_base(i) + row_here] : 0;
                    if (__any(marks != 0)) {
                        float *o = (float *)p.sg_gu + (m0 + row_base(i) + row_here) * p.ldr;
                        if (marks) o += head.first[((strip - n0) >> 6) * head_ld + row_base(i) + row_here];
                        for (; marks; marks &= marks - 1) *o++ = stg[row_here * 64 + ((__ffsll((long long)marks) - 1) ^ stg_swz(row_here))];
                    }
                }
                bool far = false;
#pragma unroll
                for (int ps = 0; ps < 8; ++ps) far |= !(s[ps] < 0x1p64f);
                if (__any(far)) {
#pragma unroll
                    for (int ps = 0; ps < 8; ++ps) {
                        float z[4], x[4], e[4];
                        row_of(ps, z);
#pragma unroll
                        for (int k = 0; k < 4; ++k) x[k] = cok ? __builtin_fmaf(z[k], it2, -ref[ps]) : -INFINITY;
                        const float m = across_row(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), larger);
                        const bool this_row = !(s[ps] < 0x1p64f);                        // the same in the row's 16 lanes
                        off[ps] = this_row ? rintf(m) : 0.f;
#pragma unroll
                        for (int k = 0; k < 4; ++k) e[k] = cok ? __builtin_amdgcn_exp2f(x[k] - off[ps]) : 0.f;
                        const float t = across_row((e[0] + e[1]) + (e[2] + e[3]), sum);
                        if (this_row) s[ps] = t, w[ps] = pack4(e);
                    }
                }
                if (p.C) {
#pragma unroll
                    for (int ps = 0; ps < 8; ++ps) __builtin_amdgcn_raw_buffer_store_b64(w[ps], rz, stored ? lane_c + row_bytes(i, ps * 4, p.ldc, 2) : kOob, 0, kStream);
                }
            }
            // lane idx of a row group takes row 4 idx + prow of the block: 32 rows in one store
            float so = s[0], oo = off[0];
#pragma unroll
            for (int ps = 1; ps < 8; ++ps) {
                so = idx == ps ? s[ps] : so;
                oo = idx == ps ? off[ps] : oo;
            }
            const int row = m0 + row_base(i) + idx * 4 + prow;
            if (idx < 8 && row < p.M && strip < p.N) *(float2 *)(p.kd_part + ((long)(strip >> 6) * p.kd_ldz + row) * 2) = make_float2(oo, so);
        }
        return;
    }
    // ---- vector epilogues.  Each wave passes its accumulators through LDS, 32 rows at a time, to turn the
    // MFMA layout (a lane owns one column) into rows: a lane then handles 4 consecutive columns of a row, so
    // global reads and writes are 8..16 bytes per lane and 128..256 contiguous bytes per row.  What the
    // epilogue reads from memory for a 32-row block (fp32/bf16 residual, C when accumulating, teacher logits)
    // is fetched one block ahead into registers: the loads of block i+1 are issued before the stores of
    // block i, so no pass waits for a store or for its own load's full latency.
    if (EPI != EPI_NONE || p.vec_epilogue) {
        const int prow = lane >> 4, pcol = (lane & 15) * 4;
        const int colg = n0 + col_base(pcol >> 5) + (pcol & 31);
        const bool cok = colg < p.N;
        // the prefetched stream: KD -> teacher logits (fp32); else residual (fp32 or bf16); else C (accumulate)
        // (SwiGLU backward -> gate and up, 4 bf16 each)
        const bool aux_res = EPI == EPI_NONE && p.residual != nullptr;
        const bool aux_c = EPI == EPI_NONE && !aux_res && p.accumulate && p.c_fp32;
        const bool has_aux = EPI != EPI_NONE || aux_res || aux_c;
        const bool aux4 = EPI != EPI_NONE || aux_c || p.res_fp32;                  // 4-byte elements
        const long aux_ld = EPI != EPI_NONE ? p.kd_ldz : (aux_res ? p.ldr : p.ldc);
        const __amdgpu_buffer_rsrc_t ra_ = EPI == EPI_SWIGLU_BWD ? make_rsrc(p.sg_gu, (long)p.M * p.sg_ldgu * 2)
                                           : EPI != EPI_NONE     ? make_rsrc(p.kd_zt, (long)p.M * p.kd_ldz * 4) : (aux_res ? rr : rc);
        const __amdgpu_buffer_rsrc_t rl = make_rsrc(EPI == EPI_KD_DZ ? (const void *)p.kd_stats : p.C, EPI == EPI_KD_DZ ? (long)p.M * 32 : 0);
        u32x4 aux[2][8];
        float2 lsev[2][8];                                                         // EPI_KD_DZ: (lse_t, lse_s) of the row
        const unsigned lane_c = (unsigned)((prow * p.ldc + colg) * esz), lane_aux = (unsigned)((prow * aux_ld + colg) * (aux4 ? 4 : 2));
        const unsigned lane_g = (unsigned)((prow * p.sg_ldgu + colg) * 2);
        auto prefetch = [&](int i, u32x4 *dst, float2 *ldst) {
#pragma unroll
            for (int ps = 0; ps < 8; ++ps) {
                if constexpr (EPI == EPI_SWIGLU_BWD) {
                    const unsigned go = cok ? lane_g + row_bytes(i, ps * 4, p.sg_ldgu, 2) : kOob;
                    const u32x2 g = __builtin_amdgcn_raw_buffer_load_b64(ra_, go, 0, kStream);
                    const u32x2 u = __builtin_amdgcn_raw_buffer_load_b64(ra_, cok ? go + (unsigned)p.sg_f * 2 : kOob, 0, kStream);
                    dst[ps][0] = g[0]; dst[ps][1] = g[1]; dst[ps][2] = u[0]; dst[ps][3] = u[1];
                    continue;
                }
                const unsigned off = cok ? lane_aux + row_bytes(i, ps * 4, aux_ld, aux4 ? 4 : 2) : kOob;
                if (aux4) dst[ps] = __builtin_amdgcn_raw_buffer_load_b128(ra_, off, 0, kStream);
                else {
                    const u32x2 q = __builtin_amdgcn_raw_buffer_load_b64(ra_, off, 0, kStream);
                    dst[ps][0] = q[0]; dst[ps][1] = q[1];
                }
                if constexpr (EPI == EPI_KD_DZ) ldst[ps] = __builtin_bit_cast(float2, __builtin_amdgcn_raw_buffer_load_b64(rl, prow * 32 + 24 + row_bytes(i, ps * 4, 8, 4), 0, 0));
            }
        };
        float bv[4] = {0.f, 0.f, 0.f, 0.f};
        if (EPI == EPI_NONE && bias && cok) {
            const uint2 b2 = *(const uint2 *)(bias + colg);
            bv[0] = (float)__builtin_bit_cast(bf16_t, (unsigned short)(b2.x & 0xffff));
            bv[1] = (float)__builtin_bit_cast(bf16_t, (unsigned short)(b2.x >> 16));
            bv[2] = (float)__builtin_bit_cast(bf16_t, (unsigned short)(b2.y & 0xffff));
            bv[3] = (float)__builtin_bit_cast(bf16_t, (unsigned short)(b2.y >> 16));
        }
        auto store4 = [&](const float *v, unsigned co) {
            if (p.c_fp32) {
                u32x4 w;
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = __builtin_bit_cast(unsigned, v[e]);
                __builtin_amdgcn_raw_buffer_store_b128(w, rc, co, 0, kStream);
            } else {
                __builtin_amdgcn_raw_buffer_store_b64(pack4(v), rc, co, 0, kStream);
            }
        };
        const float it = p.kd_inv_t;
        const float it2 = it * 1.4426950408889634f;      // e^{z/T - m} = 2^{z it2 - m log2(e)}: one fused multiply-add feeds exp2
        // Statistics of the wave's 32-row block i: per row, over the wave's 64 columns, max and sum of exponentials of zt/T and
        // zs/T and the cross term sum e^{zt/T - m_t} (zt - zs)/T -> kd_part.  16 rows at a time both tiles go through LDS ([16][64]
        // fp32 each, 16-byte chunk c of row r at c ^ r: no bank conflicts on either side), from where lane l takes chunks l / 16 +
        // 4 k of row l % 16: a row is then 16 values in a lane and four lanes, and each of the five reductions costs two steps per
        // 16 rows.  With a row's four columns per lane as in the other epilogues it is four steps for every four rows, and their
        // moves, address arithmetic and branches were two thirds of this epilogue, which the vector ALU bounds.
        auto kd_statistics = [&](int i, const u32x4 *q) __attribute__((always_inline)) {
            const int r16 = lane & 15, grp = lane >> 4;
            const bool full = n0 + wn * WTN + WTN <= p.N;                          // wave-uniform
            float *stz = stg + 1024;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                wave_sync();
                if constexpr (M16) {
#pragma unroll
                    for (int j = 0; j < NI; ++j)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const int row = 4 * fhalf + r;
                            stg[row * 64 + ((j * 16 + frow) ^ (row << 2))] = acc[2 * i + h][j][r];
                        }
                } else {
#pragma unroll
                    for (int j = 0; j < NI; ++j)
#pragma unroll
                        for (int r = 0; r < 8; ++r) {
                            const int row = 8 * (r >> 2) + 4 * fhalf + (r & 3);
                            stg[row * 64 + ((j * 32 + frow) ^ (row << 2))] = acc[i][j][8 * h + r];
                        }
                }
#pragma unroll
                for (int ps = 0; ps < 4; ++ps) {
                    const int row = ps * 4 + prow;
                    *(u32x4 *)(stz + row * 64 + (pcol ^ (row << 2))) = q[h * 4 + ps];
                }
                wave_sync();
                float zs[16], zt[16], d[16];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int at = r16 * 64 + (((4 * k + grp) ^ r16) << 2);
                    const float4 a = *(const float4 *)(stg + at), b = *(const float4 *)(stz + at);
                    zs[4 * k] = a.x; zs[4 * k + 1] = a.y; zs[4 * k + 2] = a.z; zs[4 * k + 3] = a.w;
                    zt[4 * k] = b.x; zt[4 * k + 1] = b.y; zt[4 * k + 2] = b.z; zt[4 * k + 3] = b.w;
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) d[e] = zt[e] - zs[e];
                if (!full) {                                                       // columns past N take no part
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int c = (e & ~3) + grp;
                        const bool ok = n0 + col_base(c >> 3) + (c & 7) * 4 < p.N;
                        zs[e] = ok ? zs[e] : -INFINITY;
                        zt[e] = ok ? zt[e] : -INFINITY;
                        d[e] = ok ? d[e] : 0.f;
                    }
                }
                float mt = max3(zt[0], zt[1], zt[2]), ms = max3(zs[0], zs[1], zs[2]);
#pragma unroll
                for (int e = 3; e < 15; e += 2) {
                    mt = max3(mt, zt[e], zt[e + 1]);
                    ms = max3(ms, zs[e], zs[e + 1]);
                }
                auto larger = [](float a, float b) { return max3(a, b, b); };
                mt = across_groups(larger(mt, zt[15]), larger) * it;               // T > 0
                ms = across_groups(larger(ms, zs[15]), larger) * it;
                const float mt2 = mt == -INFINITY ? 0.f : mt * 1.4426950408889634f;
                const float ms2 = ms == -INFINITY ? 0.f : ms * 1.4426950408889634f;
                float st = 0.f, ss = 0.f, ac = 0.f;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float et = __builtin_amdgcn_exp2f(__builtin_fmaf(zt[e], it2, -mt2));
                    st += et;
                    ac = __builtin_fmaf(et, d[e], ac);
                    ss += __builtin_amdgcn_exp2f(__builtin_fmaf(zs[e], it2, -ms2));
                }
                auto sum = [](float a, float b) { return a + b; };
                st = across_groups(st, sum);
                ss = across_groups(ss, sum);
                ac = across_groups(ac * it, sum);
                const long rowg = m0 + row_base(i) + h * 16 + r16;
                if (grp == 0 && rowg < p.M && n0 + wn * WTN < p.N) {
                    float *o = p.kd_part + (rowg * p.kd_nparts + (n0 + wn * WTN) / 64) * 8;
                    *(float4 *)o = make_float4(mt, st, ms, ss);
                    o[4] = ac;
                }
            }
        };
        if (has_aux) prefetch(0, aux[0], lsev[0]);
#pragma unroll
        for (int i = 0; i < MI32; ++i) {
            if (has_aux && i + 1 < MI32) prefetch(i + 1, aux[(i + 1) & 1], lsev[(i + 1) & 1]);
            if constexpr (EPI == EPI_KD_STATS) {
                kd_statistics(i, aux[i & 1]);
                continue;
            }
            stage_block(i, [&](float a) { return EPI == EPI_KD_DZ ? a : a * p.alpha; });     // (the KD epilogues have alpha = 1)
#pragma unroll
            for (int ps = 0; ps < 8; ++ps) {
                const int row = ps * 4 + prow;
                const float4 t = *(const float4 *)(stg + row * 64 + (pcol ^ stg_swz(row)));
                const u32x4 q = aux[i & 1][ps];
                const unsigned co = cok ? lane_c + row_bytes(i, ps * 4, p.ldc, esz) : kOob;
                if constexpr (EPI == EPI_NONE) {
                    float v[4] = {t.x + bv[0], t.y + bv[1], t.z + bv[2], t.w + bv[3]};
                    if (aux_res || aux_c) {
                        if (aux4) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) v[e] += __uint_as_float(q[e]);
                        } else {
                            v[0] += (float)__builtin_bit_cast(bf16_t, (unsigned short)(q[0] & 0xffff));
                            v[1] += (float)__builtin_bit_cast(bf16_t, (unsigned short)(q[0] >> 16));
                            v[2] += (float)__builtin_bit_cast(bf16_t, (unsigned short)(q[1] & 0xffff));
                            v[3] += (float)__builtin_bit_cast(bf16_t, (unsigned short)(q[1] >> 16));
                        }
                    }
                    if (aux_res && p.accumulate && p.c_fp32) {        // both a residual and += : C is read in place
                        const u32x4 c4 = __builtin_amdgcn_raw_buffer_load_b128(rc, co, 0, 0);
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[e] += __uint_as_float(c4[e]);
                    }
                    store4(v, co);
                } else if constexpr (EPI == EPI_SWIGLU_BWD) {
                    // da is rounded to the storage type first (it is what a separate activation kernel would read back)
                    const float da[4] = {(float)(bf16_t)t.x, (float)(bf16_t)t.y, (float)(bf16_t)t.z, (float)(bf16_t)t.w};
                    float dg[4], du[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float gg = (float)__builtin_bit_cast(bf16_t, (unsigned short)(q[e >> 1] >> (16 * (e & 1))));
                        const float uu = (float)__builtin_bit_cast(bf16_t, (unsigned short)(q[2 + (e >> 1)] >> (16 * (e & 1))));
                        swiglu_derivative(da[e], gg, uu, &dg[e], &du[e]);
                    }
                    store4(dg, co);
                    store4(du, cok ? co + (unsigned)p.sg_f * 2 : kOob);
                } else {
                    // the tile holds student logits zs; q = teacher logits zt of the same elements
                    const float zs[4] = {t.x, t.y, t.z, t.w};
                    float zt[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) zt[e] = __uint_as_float(q[e]);
                    // dz = coef * (exp(zs/T - lse_s) - exp(zt/T - lse_t)) -> C (storage dtype)
                    const float lt2 = lsev[i & 1][ps].x * 1.4426950408889634f, ls2 = lsev[i & 1][ps].y * 1.4426950408889634f;
                    float v[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        v[e] = p.kd_coef * (__builtin_amdgcn_exp2f(__builtin_fmaf(zs[e], it2, -ls2)) -
                                            __builtin_amdgcn_exp2f(__builtin_fmaf(zt[e], it2, -lt2)));
                    store4(v, co);
                }
            }
        }
        return;
    }
    // scalar epilogue: split-K atomics and shapes whose rows are not 4-element aligned
#pragma unroll
    for (int j = 0; j < NI; ++j) {
        const int col = n0 + (M16 ? col_base(j >> 1) + (j & 1) * 16 : col_base(j)) + frow;
        const bool cok = col < p.N;
        const float bv = (bias && cok) ? (float)bias[col] : 0.f;
#pragma unroll
        for (int i = 0; i < MI; ++i) {
#pragma unroll
            for (int r = 0; r < ACC_N; ++r) {
                const int row = m0 + (M16 ? row_base(i >> 1) + (i & 1) * 16 : row_base(i)) + (M16 ? 4 * fhalf + r : 8 * (r >> 2) + 4 * fhalf + (r & 3));
                float v = acc[i][j][r] * p.alpha + bv;
                if (p.residual) {
                    const unsigned ro = cok ? (unsigned)(((long)row * p.ldr + col) * rsz) : kOob;
                    if (p.res_fp32) v += __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rr, ro, 0, 0));
                    else v += (float)__builtin_bit_cast(bf16_t, __builtin_amdgcn_raw_buffer_load_b16(rr, ro, 0, 0));
                }
                const unsigned co = cok ? (unsigned)(((long)row * p.ldc + col) * esz) : kOob;
                if (p.c_fp32) {
                    if (p.atomic) {
                        if (cok && row < p.M) unsafeAtomicAdd((float *)p.C + (long)row * p.ldc + col, v);
                    } else {
                        if (p.accumulate) v += __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rc, co, 0, 0));
                        __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, v), rc, co, 0, 0);
                    }
                } else {
                    __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(unsigned short, (bf16_t)v), rc, co, 0, 0);
                }
            }
            // keep the scheduler from pulling every accumulator out of the AGPRs at once
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

// M16 selects v_mfma_f32_16x16x32_bf16 (16-row fragments, two k-steps of 32 per K tile) instead of
// v_mfma_f32_32x32x16_bf16 (32-row fragments, four k-steps of 16): the same LDS traffic and the same number of
// accumulator registers, but on operands with realistic bit activity the chip sustains a higher clock on it.
// NST = LDS stages: two (a K tile is requested one tile time before its first use, which is what the big tile's LDS
// allows) or a deeper ring for grids that leave CUs with one workgroup, where a tile time is shorter than the latency
// of a load (see kTiles).
// The attribute only adds to what the launch bounds say for the two-stage 128 x 128 kernel with the dz epilogue: left to
// itself the compiler gives it 276 registers, which leave a CU with one workgroup, instead of 173 (dz at
// 3629 x 4480 x 1536: 70.9 us; 74.2 on v_mfma_f32_32x32x16, which needs fewer).
constexpr int fast_waves_per_simd(int bm, int waves, int epi, int nst) { return waves == 8 || (bm == 128 && nst == 2 && epi == EPI_KD_DZ) ? 2 : 1; }
template <int BM, int BN, int NST> struct FastLds {
    bf16_t *a[4], *b[4];
    HeadRowsLds head;
};
// The kernel's LDS: separate objects (not one carved array), because the compiler orders LDS reads against in-flight
// direct-to-LDS loads by alias analysis, and can only tell the buffer being filled from the buffer being read when
// they are distinct objects
#define MS_FAST_LDS(BM, BN, NST)                                                                                       \
    static_assert(NST >= 2 && NST <= 4, "ring of 2..4 stages");                                                        \
    __shared__ __align__(16) bf16_t As0[BM * BK], As1[BM * BK], As2[NST > 2 ? BM * BK : 8], As3[NST > 3 ? BM * BK : 8]; \
    __shared__ __align__(16) bf16_t Bs0[BN * BK], Bs1[BN * BK], Bs2[NST > 2 ? BN * BK : 8], Bs3[NST > 3 ? BN * BK : 8]; \
    const FastLds<BM, BN, NST> lds = {{As0, As1, As2, As3}, {Bs0, Bs1, Bs2, Bs3}}

// Workgroup b of the nb that compute one product (of one K split)
template <int BM, int BN, int WM, int WN, bool TA, bool TB, int EPI, bool M16, int NST>
__device__ __forceinline__ void gemm_fast_body(const GemmParams &p, const FastLds<BM, BN, NST> &lds, int b, int nb, int split) {
    constexpr int FR = M16 ? 16 : 32;                         // rows of an MFMA fragment / accumulator block
    constexpr int KSTEP = M16 ? 32 : 16, KS = BK / KSTEP;     // contraction depth of an MFMA, k-steps per K tile
    constexpr int WTM = BM / WM, WTN = BN / WN, MI = WTM / FR, NI = WTN / FR;
    constexpr int MI32 = WTM / 32, NI32 = WTN / 32;           // the epilogues work on 32-row blocks
    using acc_t = std::conditional_t<M16, f32x4, f32x16>;
    constexpr int ACC_N = M16 ? 4 : 16;
    bf16_t *const As0 = lds.a[0], *const As1 = lds.a[1], *const Bs0 = lds.b[0], *const Bs1 = lds.b[1];
    bf16_t *const Ast[4] = {lds.a[0], lds.a[1], lds.a[2], lds.a[3]}, *const Bst[4] = {lds.b[0], lds.b[1], lds.b[2], lds.b[3]};

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);   // wave-uniform: keep it in a scalar register
    const int wm = wave / WN, wn = wave % WN;
    int pid;
    {
        const int per = nb >> 3, rem = nb & 7, x = b & 7, q = b >> 3;
        pid = x * per + (x < rem ? x : rem) + q;
    }
    constexpr int GM = BM >= 256 ? 4 : 8;
    const int group = pid / (GM * p.tiles_n);
    const int first_m = group * GM;
    const int gsize = (p.tiles_m - first_m) < GM ? (p.tiles_m - first_m) : GM;
    const int tm = first_m + (pid % (GM * p.tiles_n)) % gsize;
    const int tn = (pid % (GM * p.tiles_n)) / gsize;
    const int m0 = tm * BM, n0 = tn * BN;

    const int kt_begin = split * p.k_tiles_per_split;
    int kt_end = kt_begin + p.k_tiles_per_split;
    const int kt_total = (p.K + BK - 1) / BK;
    if (kt_end > kt_total) kt_end = kt_total;
    const int nk = kt_end - kt_begin;
    if (nk <= 0) return;

    if constexpr (EPI == EPI_EXP) head_rows_fetch<BM, BN, WM * WN>(p, lds.head, m0, n0, wave, lane);
    const bf16_t *A = (const bf16_t *)p.A, *B = (const bf16_t *)p.B;
    std::conditional_t<TA, RowTileStager<BM, WM * WN>, DmaStager<BM, WM * WN>> da;
    std::conditional_t<EPI == EPI_SWIGLU, GateUpStager<BN, WM * WN>,
                       std::conditional_t<TB, RowTileStager<BN, WM * WN>, DmaStager<BN, WM * WN>>> db;
    // descriptor ranges: rows x leading dimension of the matrix as stored ([M or N][K], or [K][M or N])
    const __amdgpu_buffer_rsrc_t ra = make_rsrc(A, TA ? ((long)(p.K - 1) * p.lda + p.M) * 2 : ((long)(p.M - 1) * p.lda + p.K) * 2);
    const __amdgpu_buffer_rsrc_t rb = make_rsrc(B, TB ? ((long)(p.K - 1) * p.ldb + p.N) * 2
                                                      : ((long)((EPI == EPI_SWIGLU ? 2 * p.sg_f : p.N) - 1) * p.ldb + p.K) * 2);
    if constexpr (TA) da.init(p.lda, m0, wave, lane); else da.init(p.lda, m0, lane);
    if constexpr (EPI == EPI_SWIGLU) db.init(p.ldb, n0 / 2, p.sg_f, lane);   // tile tn covers output columns tn * BN/2 ..
    else if constexpr (TB) db.init(p.ldb, n0, wave, lane);
    else db.init(p.ldb, n0, lane);

    acc_t acc[MI][NI];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int r = 0; r < ACC_N; ++r) acc[i][j][r] = 0.f;

    // Start moving K tile kt towards LDS; a tile past the end of this workgroup's K range arrives as zeros.
    // An operand stored K-major ([K][M]) is loaded as a "row tile" (64 k-rows x BM columns) and read back
    // through the transposing LDS load, so every layout goes global -> LDS without staging registers.
    auto fetch = [&](int kt, bf16_t *as, bf16_t *bs) {
        const bool valid = kt < nk;
        const unsigned inv = valid ? 0u : kOob;
        const int k0 = (kt_begin + kt) * BK;
        da.issue(ra, as, k0, wave, inv);
        db.issue(rb, bs, k0, wave, inv);
    };
    // lane -> (fragment row, k-group of 8 consecutive k): 32 rows x 2 groups, or 16 rows x 4 groups
    const int frow = lane & (FR - 1), fhalf = lane / FR;
    // 32-row block i (32-column block j) of this wave within the tile.  For a K-major operand the blocks
    // of a wave are spread one per 64-wide LDS sub-tile pair so that all of them share one LDS address
    // register (constant offsets); for a K-contiguous operand they are adjacent for the same reason.
    auto row_base = [&](int i) { return TA ? i * (32 * WM) + wm * 32 : wm * WTM + i * 32; };
    auto col_base = [&](int j) { return TB ? j * (32 * WN) + wn * 32 : wn * WTN + j * 32; };
    // the same for fragment blocks (16-row blocks are the halves of the 32-row blocks)
    auto frow_base = [&](int i) { return M16 ? row_base(i >> 1) + (i & 1) * 16 : row_base(i); };
    auto fcol_base = [&](int j) { return M16 ? col_base(j >> 1) + (j & 1) * 16 : col_base(j); };
    // Operand fragments are double-buffered in registers: the LDS reads of k-step kk+1 are issued between
    // the MFMAs of k-step kk.
    bf16x8 af[2][MI], bfr[2][NI];
    std::conditional_t<M16, TrFragAddr16, TrFragAddr> tra, trb, trb1;
    static_assert((WM == 2 || (WM == 4 && BM == 128 && M16)) && (WN >= 2 || M16), "K-major blocks are spread over sub-tile pairs");
    if constexpr (TA) tra.init(wm, lane);     // block i of the wave: columns i * 32 * WM + wm * 32 of the row tile
    if constexpr (TB) trb.init(wn, lane);
    if constexpr (TB && WN == 1) trb1.init(1, lane);   // one wave column: its two 32-column blocks are the halves of a sub-tile
    KFragAddr16 ka, kb;
    if constexpr (M16 && !TA) ka.init(wm * WTM, lane);
    if constexpr (M16 && !TB) kb.init(wn * WTN, lane);
    auto load_a = [&](const bf16_t *as, int kk, int slot, int i) {
        if constexpr (TA && M16) af[slot][i] = tra.frag(as, kk, i, (i >> 1) * (32 * WM / 64) * 4096);
        else if constexpr (TA) af[slot][i] = tra.frag(as, kk, i * (32 * WM / 64) * 4096);
        else if constexpr (M16) af[slot][i] = ka.frag(as, kk, i);
        else af[slot][i] = *(const bf16x8 *)(as + lds_off(frow_base(i) + frow, kk * (KSTEP / 8) + fhalf));
    };
    auto load_b = [&](const bf16_t *bs, int kk, int slot, int j) {
        if constexpr (TB && WN == 1) bfr[slot][j] = (j >> 1 ? trb1 : trb).frag(bs, kk, j, 0);
        else if constexpr (TB && M16) bfr[slot][j] = trb.frag(bs, kk, j, (j >> 1) * (32 * WN / 64) * 4096);
        else if constexpr (TB) bfr[slot][j] = trb.frag(bs, kk, j * (32 * WN / 64) * 4096);
        else if constexpr (M16) bfr[slot][j] = kb.frag(bs, kk, j);
        else bfr[slot][j] = *(const bf16x8 *)(bs + lds_off(fcol_base(j) + frow, kk * (KSTEP / 8) + fhalf));
    };
    auto load_frags = [&](const bf16_t *as, const bf16_t *bs, int kk, int slot) {
#pragma unroll
        for (int i = 0; i < MI; ++i) load_a(as, kk, slot, i);
#pragma unroll
        for (int j = 0; j < NI; ++j) load_b(bs, kk, slot, j);
    };
    auto mfma_step = [&](int slot) {
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                if constexpr (M16) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(af[slot][i], bfr[slot][j], acc[i][j], 0, 0, 0);
                else acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(af[slot][i], bfr[slot][j], acc[i][j], 0, 0, 0);
            }
    };
    constexpr int LDS_READS = (TA ? 2 : 1) * MI + (TB ? 2 : 1) * NI, MFMAS = MI * NI;
    // One k-step: the MFMAs on fragment slot `cur`, with the reads of the next k-step's fragments (tile la / lb,
    // k-step lkk) between them.  With 32-row fragments all reads go in front (one per MFMA).  With 16-row
    // fragments there are twice as many fragment registers per k-step, so the A fragment of row block i is
    // read right after the MFMAs of row block i, into the registers those MFMAs have just released; only the
    // B fragments are held twice.
    auto step = [&](auto cur_c, auto fetch_c, const bf16_t *la, const bf16_t *lb, int lkk) __attribute__((always_inline)) {
        constexpr int cur = decltype(cur_c)::value;          // compile-time: the fragment arrays must stay registers
        constexpr int VM = decltype(fetch_c)::value ? (BM + BN) / 8 / (WM * WN) : 0;   // loads of a fetch issued just before
        if constexpr (M16) {
            constexpr int BPB = (NI + MI - 1) / MI;          // B fragments read behind each row block
            // (columns alternate in direction, so that neighbouring MFMAs differ in one operand: 0.3-0.5 % at the same power)
#pragma unroll
            for (int i = 0; i < MI; ++i) {
#pragma unroll
                for (int jj = 0; jj < NI; ++jj) {
                    const int j = (i & 1) ? NI - 1 - jj : jj;
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(af[cur][i], bfr[cur][j], acc[i][j], 0, 0, 0);
                }
                load_a(la, lkk, cur ^ 1, i);
#pragma unroll
                for (int j = i * BPB; j < NI && j < (i + 1) * BPB; ++j) load_b(lb, lkk, cur ^ 1, j);
            }
            sched_mfma_then_reads<NI, (TA ? 2 : 1), (TB ? 2 : 1), VM>(std::make_integer_sequence<int, MI>{});
        } else {
            load_frags(la, lb, lkk, cur ^ 1);
            mfma_step(cur);
            interleave_reads_with_mfma<LDS_READS, MFMAS>();
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // One K tile: steps 0..2 read the next step's fragments from the same tile; before the last step the
    // next tile has landed (own loads: vmcnt(0); the other waves': barrier) and everybody is done reading
    // this one, so its buffers are handed to the tile after next and the last step reads the first
    // fragments of the next tile.  One barrier per tile.
    auto tile = [&](const bf16_t *ca, const bf16_t *cb, const bf16_t *na, const bf16_t *nb, bf16_t *fa, bf16_t *fb,
                    int kt_fetch) __attribute__((always_inline)) {
        using S0 = std::integral_constant<int, 0>;
        using S1 = std::integral_constant<int, 1>;
        static_assert(KS == 2 || KS == 4, "k-steps per K tile");
        step(S0{}, S0{}, ca, cb, 1);
        if constexpr (KS == 4) {
            step(S1{}, S0{}, ca, cb, 2);
            step(S0{}, S0{}, ca, cb, 3);
        }
        if constexpr (NST == 2) {
            dma_publish_barrier();
        } else {
            // own loads of the next tile have landed; the NST - 2 younger tiles' loads stay in flight
            wait_vmcnt_lgkm0<(NST - 2) * ((BM + BN) / 8 / (WM * WN))>();
            lds_barrier();
        }
        fetch(kt_fetch, fa, fb);
        step(S1{}, S1{}, na, nb, 0);
    };

    if constexpr (NST == 2) {
        fetch(0, As0, Bs0);
        dma_publish_barrier();
        fetch(1, As1, Bs1);
    } else {
#pragma unroll
        for (int k = 0; k < NST; ++k) fetch(k, Ast[k], Bst[k]);
        wait_vmcnt_lgkm0<(NST - 1) * ((BM + BN) / 8 / (WM * WN))>();
        lds_barrier();
    }
    load_frags(As0, Bs0, 0, 0);
    // NST K tiles per trip so that each part names its LDS buffers statically; the tile count is
    // rounded up with tiles of zeros (a single loop exit keeps the accumulators in place)
    for (int kt = 0; kt < nk; kt += NST) {
#pragma unroll
        for (int k = 0; k < NST; ++k)
            tile(Ast[k], Bst[k], Ast[(k + 1) % NST], Bst[(k + 1) % NST], Ast[k], Bst[k], kt + k + NST);
    }
    dma_publish_barrier();   // the (all-zero) tiles still in flight must land before the epilogue reuses LDS

    // waves share the idle operand buffers, 8 KB each: WPA of them fit into one A buffer
    constexpr int WPA = BM / 64;
    const int sq = wave / WPA;
    float *stg = (float *)(sq == 0 ? As0 : sq == 1 ? As1 : sq == 2 ? Bs0 : Bs1) + (wave % WPA) * 2048;
    gemm_epilogue<EPI, M16, TA, TB>(p, acc, stg, m0, n0, wn, lane, row_base, col_base, lds.head, BM > 128 ? BM : 128);
}

// The 256 x 256 tile with two wave groups that take turns on the matrix cores; K-contiguous operands only.
//   * Waves 0..3 and 4..7 (one of each per SIMD) run the same program half a phase apart: while one group issues the 16
//     MFMAs of a quarter of its wave tile (64 x 32, both k-steps), the other reads its next operand fragments from LDS
//     and requests the next half tile.  Two barriers per phase keep them in step; the one extra barrier that group 1
//     takes before the loop and group 0 after it is the offset.
//   * An operand tile is two halves of 128 rows with an LDS slot each and two stages: eight 16 KB slots.  Per K tile the
//     phases read A0 -> Bs -> A1 -> Bf of the next tile, where Bf / Bs are the B half used first / second; they swap roles
//     every tile, so that the quarters (A0 Bf)(A0 Bs)(A1 Bs)(A1 Bf) change one operand at a time.  Two of the eight
//     fragments of an A half are read in the phase before its own, so that every phase has six reads.  A phase requests
//     the half of tile t + 2 that goes into the slot whose last read was in the phase before: every half is requested at
//     least six phases (1.5 K tiles) before it is read, instead of one K tile in gemm_bf16_fast_kernel, and the wait
//     is for all but the 10 youngest loads of a wave, never for all of them.
//   * Same tile order, MFMA and order of K as the other tiles: bit-identical results.
// It is the 256 x 256 tile of K-contiguous operands for every shape and epilogue.  Against gemm_bf16_fast_kernel<256, 256> with
// operands that have left the caches, as they have when a step comes round to them again, it was faster on 108 of 110 shapes
// (M = 1500 .. 32768, 22 outputs; the other two within 0.6 %), us: 8192 x 8192 x 4096 with fp32 output 437 -> 391,
// 8192 x 1280 x 5120 135 -> 114, 4096 x 3072 x 2048 51.5 -> 44.5, 32768 x 4096 x 11008 2199 -> 2010, 32768 x 1536 x 1536
// 174 -> 170; the distillation head at 8192 tokens, V = 151936, H = 4096 / 2048 35.4 -> 32.8 ms.  On operands that stay in
// the 256 MB Infinity Cache the two are equal (8192^3 704 / 707) up to 4 % on a short K (32768 x 2048 x 1536 154 / 160).
// For K-major operands (twice the LDS reads) it was built too: 6-12 % slower warm, 2-8 % slower cold wherever the grid fills
// the chip (32768 x 8960 x 1536 736 -> 788), and in smaller grids behind the other tiles.
// B half g holds the rows 64 w + 32 g .. + 31 of every wave column w (a wave's 64 columns stay adjacent); for SwiGLU
// g = 0 gate rows, g = 1 up rows.
struct HalfStager {
    unsigned rowoff, ld2;
    int x;
    __device__ __forceinline__ void init(long ld, int row0, int lane) {
        rowoff = (unsigned)(((long)(row0 + (lane >> 3)) * ld) * 2);
        ld2 = (unsigned)(ld * 2);
        x = (lane & 7) ^ swz_row(lane >> 3);
    }
    // eight matrix rows from row0 + row into 8-row group lg of the half's slot (both wave-uniform)
    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t rs, bf16_t *slot, int row, int lg, int k0, unsigned inv) const {
        const unsigned voff = (rowoff + (unsigned)row * ld2 + ((x ^ swz_row(8 * lg)) << 4)) | inv;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void *)(slot + lg * 8 * BK), 16, voff, k0 * 2, 0, 0);
    }
};
struct PpLds {
    bf16_t *a[2][2], *b[2][2];                          // [stage][half]
    HeadRowsLds head;
};
#define MS_PP_LDS                                                                                                     \
    constexpr int HS = 128 * BK; /* elements of a half tile */                                                        \
    __shared__ __align__(16) bf16_t A00[HS], A01[HS], A10[HS], A11[HS], B00[HS], B01[HS], B10[HS], B11[HS];           \
    const PpLds lds = {{{A00, A01}, {A10, A11}}, {{B00, B01}, {B10, B11}}}
// Workgroup b of the nb that compute one product (of one K split)
template <int EPI>
__device__ __forceinline__ void gemm_pp_body(const GemmParams &p, const PpLds &lds, int b, int nb, int split) {
    bf16_t *const A00 = lds.a[0][0], *const A01 = lds.a[0][1], *const A10 = lds.a[1][0], *const A11 = lds.a[1][1];
    bf16_t *const B00 = lds.b[0][0], *const B01 = lds.b[0][1], *const B10 = lds.b[1][0], *const B11 = lds.b[1][1];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave >> 2, wn = wave & 3;            // wm = wave group
    int pid;
    {
        const int per = nb >> 3, rem = nb & 7, x = b & 7, q = b >> 3;
        pid = x * per + (x < rem ? x : rem) + q;
    }
    constexpr int GM = 4;
    const int group = pid / (GM * p.tiles_n);
    const int first_m = group * GM;
    const int gsize = (p.tiles_m - first_m) < GM ? (p.tiles_m - first_m) : GM;
    const int tm = first_m + (pid % (GM * p.tiles_n)) % gsize;
    const int tn = (pid % (GM * p.tiles_n)) / gsize;
    const int m0 = tm * 256, n0 = tn * 256;

    const int kt_begin = split * p.k_tiles_per_split;
    int kt_end = kt_begin + p.k_tiles_per_split;
    const int kt_total = (p.K + BK - 1) / BK;
    if (kt_end > kt_total) kt_end = kt_total;
    const int nk = kt_end - kt_begin;
    if (nk <= 0) return;

    const __amdgpu_buffer_rsrc_t ra = make_rsrc(p.A, ((long)(p.M - 1) * p.lda + p.K) * 2);
    const __amdgpu_buffer_rsrc_t rb = make_rsrc(p.B, ((long)((EPI == EPI_SWIGLU ? 2 * p.sg_f : p.N) - 1) * p.ldb + p.K) * 2);
    HalfStager da, db;
    da.init(p.lda, m0, lane);
    db.init(p.ldb, EPI == EPI_SWIGLU ? n0 / 2 : n0, lane);
    // request half h of K tile kt (two loads per wave; a tile past the end arrives as zeros)
    auto fetch_a = [&](int kt, int h, bf16_t *slot) __attribute__((always_inline)) {
        const unsigned inv = kt < nk ? 0u : kOob;
        const int k0 = (kt_begin + kt) * BK;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int g = wave * 2 + i;
            da.load(ra, slot, h * 128 + g * 8, g, k0, inv);
        }
    };
    auto fetch_b = [&](int kt, int h, bf16_t *slot) __attribute__((always_inline)) {
        const unsigned inv = kt < nk ? 0u : kOob;
        const int k0 = (kt_begin + kt) * BK;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int g = wave * 2 + i;
            if constexpr (EPI == EPI_SWIGLU) db.load(rb, slot, h * p.sg_f + g * 8, g, k0, inv);
            else db.load(rb, slot, (g >> 2) * 64 + h * 32 + (g & 3) * 8, g, k0, inv);
        }
    };

    f32x4 acc[8][4];                                    // [16-row block: 4 h + b][16-column block: 2 g + c]
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    // A: [block][k-step] of the current half, its first two fragments apart (ax[half]); B: [half][block][k-step]
    bf16x8 af[4][2], ax[2][2], bfr[2][2][2];
    KFragAddr16 ka, kb;
    ka.init(wm * 64, lane);
    kb.init(wn * 32, lane);
    auto read_a_first = [&](auto half, const bf16_t *slot) __attribute__((always_inline)) {
        constexpr int h = decltype(half)::value;
        ax[h][0] = ka.frag(slot, 0, 0);
        ax[h][1] = ka.frag(slot, 0, 1);
    };
    auto read_a_rest = [&](const bf16_t *slot) __attribute__((always_inline)) {
        af[2][0] = ka.frag(slot, 0, 2);
        af[3][0] = ka.frag(slot, 0, 3);
#pragma unroll
        for (int b = 0; b < 4; ++b) af[b][1] = ka.frag(slot, 1, b);
    };
    auto read_b = [&](auto half, const bf16_t *slot) __attribute__((always_inline)) {
        constexpr int g = decltype(half)::value;
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
            for (int c = 0; c < 2; ++c) bfr[g][c][kk] = kb.frag(slot, kk, c);
    };
    // End of a phase's first half: the half tile that the next phase reads has landed (own loads), this phase's reads are
    // done; then the quarter's MFMAs between two barriers.
    auto turn = [&](auto ah, auto bh) __attribute__((always_inline)) {
        constexpr int h = decltype(ah)::value, g = decltype(bh)::value;
        __builtin_amdgcn_sched_barrier(0);
        wait_vmcnt_lgkm0<10>();
        lds_barrier();
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
            for (int b = 0; b < 4; ++b)
#pragma unroll
                for (int c = 0; c < 2; ++c)
                    acc[4 * h + b][2 * g + c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kk == 0 && b < 2 ? ax[h][b] : af[b][kk], bfr[g][c][kk], acc[4 * h + b][2 * g + c], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
        lds_barrier();
        __builtin_amdgcn_sched_barrier(0);
    };
    using I0 = std::integral_constant<int, 0>;
    using I1 = std::integral_constant<int, 1>;
    // K tile kt in stage slots (a0, a1, f = its first B half F, s = its second B half); nb: the slot of the next tile's first
    // B half, which is half 1 - F
    auto tile = [&](int kt, auto F, bf16_t *a0, bf16_t *a1, bf16_t *f, bf16_t *s, const bf16_t *nb, const bf16_t *na) __attribute__((always_inline)) {
        constexpr int fh = decltype(F)::value;
        using FH = std::integral_constant<int, fh>;
        using SH = std::integral_constant<int, 1 - fh>;
        read_a_rest(a0);
        fetch_b(kt + 2, fh, f);
        turn(I0{}, FH{});
        read_b(SH{}, s);
        read_a_first(I1{}, a1);
        fetch_a(kt + 2, 0, a0);
        turn(I0{}, SH{});
        read_a_rest(a1);
        fetch_b(kt + 2, 1 - fh, s);
        turn(I1{}, SH{});
        // fragments of half F are still needed by this quarter; the next tile's first half goes to the other set
        read_b(SH{}, nb);
        read_a_first(I0{}, na);
        fetch_a(kt + 2, 1, a1);
        turn(I1{}, FH{});
    };
    if constexpr (EPI == EPI_EXP) head_rows_fetch<256, 256, 8>(p, lds.head, m0, n0, wave, lane);
    // in the order in which the loop would have requested them
    fetch_b(0, 0, B00); fetch_a(0, 0, A00); fetch_b(0, 1, B01); fetch_a(0, 1, A01);
    fetch_b(1, 1, B11); fetch_a(1, 0, A10); fetch_b(1, 0, B10); fetch_a(1, 1, A11);
    wait_vmcnt_lgkm0<12>();
    lds_barrier();
    read_b(I0{}, B00);
    read_a_first(I0{}, A00);
    wait_vmcnt_lgkm0<10>();
    lds_barrier();
    if (wm == 1) lds_barrier();
    for (int kt = 0; kt < nk; kt += 2) {                // an odd count is rounded up with a tile of zeros
        tile(kt, I0{}, A00, A01, B00, B01, B11, A10);
        tile(kt + 1, I1{}, A10, A11, B11, B10, B00, A00);
    }
    if (wm == 0) lds_barrier();
    dma_publish_barrier();   // the (all-zero) half tiles still in flight must land before the epilogue reuses LDS
    auto row_base = [&](int i) { return (i >> 1) * 128 + wm * 64 + (i & 1) * 32; };
    auto col_base = [&](int j) { return wn * 64 + j * 32; };
    const int sq = wave >> 1;
    float *stg = (float *)(sq == 0 ? A00 : sq == 1 ? A01 : sq == 2 ? A10 : A11) + (wave & 1) * 2048;
    gemm_epilogue<EPI, true, false, false>(p, acc, stg, m0, n0, wn, lane, row_base, col_base, lds.head, 256);
}

}  // namespace
