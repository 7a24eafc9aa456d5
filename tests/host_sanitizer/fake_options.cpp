// Stand-ins for the kernels of sections with options (section_options.hip calls them through its table), in the manner of fake_backend.cpp:
// inputs are read and outputs filled over their full documented extent, and what a call writes may not overlap what it reads.
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <map>
#include <string>

#include "launch.h"

extern std::map<std::string, long> g_calls;
extern volatile unsigned g_sink;

namespace {
size_t es_of(int dtype) { return dtype == MS_BF16 ? 2 : 4; }
size_t up256(size_t x) { return (x + 255) / 256 * 256; }
size_t mat(long rows, long cols, long ld, size_t es) { return rows > 0 ? ((size_t)(rows - 1) * ld + cols) * es : 0; }
size_t words(long k) { return (size_t)(k + 511) / 512 * 4; }
struct Span { const void *p; size_t bytes; };
void rd(Span s) {
    unsigned acc = 0;
    for (size_t i = 0; s.p && i < s.bytes; ++i) acc += ((const unsigned char *)s.p)[i];
    g_sink = g_sink + acc;
}
void wr(void *p, size_t bytes) { if (p && bytes) memset(p, 0x5a, bytes); }
void wr_rows(void *p, long rows, size_t row, size_t stride) { for (long r = 0; r < rows; ++r) wr((char *)p + r * stride, row); }
void need(bool ok, const char *what) { if (!ok) { fprintf(stderr, "FAILED: %s\n", what); exit(1); } }
template <size_t N> void apart(const char *who, Span out, const Span (&in)[N]) {
    for (const Span &s : in)
        need(!s.p || !s.bytes || (const char *)out.p + out.bytes <= (const char *)s.p || (const char *)s.p + s.bytes <= (const char *)out.p, who);
}
}  // namespace

extern "C" {

ms_status ms_k_embedding_scaled_forward(int32_t dtype, int32_t out_fp32, int32_t n, int32_t d, int32_t vocab, float, const int32_t *ids, const void *table,
                                        void *x, void *) {
    ++g_calls["embedding_scaled"];
    rd({ids, (size_t)n * 4}); rd({table, (size_t)vocab * d * es_of(dtype)});
    wr(x, (size_t)n * d * (out_fp32 ? 4 : es_of(dtype)));
    return MS_OK;
}
size_t ms_k_embedding_sorted_backward_scratch_bytes(int32_t n, int32_t d, int32_t vocab) {
    return n <= 0 || n > 1 << 24 ? 0 : up256((size_t)n * 20 + (size_t)d * 8 + (size_t)vocab % 7);
}
ms_status ms_k_embedding_sorted_backward(int32_t dtype, int32_t n, int32_t d, int32_t vocab, float, const int32_t *ids, const void *dx, float *d_table,
                                         void *scratch, size_t scratch_bytes, void *) {
    ++g_calls["embedding_sorted"];
    need(scratch_bytes >= ms_k_embedding_sorted_backward_scratch_bytes(n, d, vocab), "embedding scratch");
    const Span in[] = {{ids, (size_t)n * 4}, {dx, (size_t)n * d * es_of(dtype)}, {d_table, (size_t)vocab * d * 4}};
    for (const Span &s : in) rd(s);
    apart("embedding scratch overlaps", {scratch, scratch_bytes}, in);
    wr(scratch, scratch_bytes); wr(d_table, (size_t)vocab * d * 4);
    return MS_OK;
}

ms_status ms_k_qk_norm_rope_forward(int32_t dtype, int32_t n, int32_t nq, int32_t nkv, int32_t hd, float, const void *x, int64_t xs, const void *g_q,
                                    const void *g_k, const int32_t *pos, const float *table, int32_t max_pos, void *y, int64_t ys, void *) {
    ++g_calls[x == y ? "qk_forward_in_place" : "qk_forward"];
    const size_t es = es_of(dtype), all = (size_t)(nq + 2 * nkv) * hd, written = x == y ? (size_t)(nq + nkv) * hd : all;
    const Span in[] = {{g_q, hd * es}, {g_k, hd * es}, {pos, (size_t)n * 4}, {table, (size_t)max_pos * hd * 4}, {x == y ? nullptr : x, mat(n, all, xs, es)}};
    for (const Span &s : in) rd(s);
    rd({x, mat(n, written, xs, es)});
    apart("qk output overlaps", {y, mat(n, written, ys, es)}, in);
    wr_rows(y, n, written * es, ys * es);
    return MS_OK;
}
size_t ms_k_qk_norm_rope_backward_scratch_bytes(int32_t hd) { return up256((size_t)768 * hd * 4); }
ms_status ms_k_qk_norm_rope_backward(int32_t dtype, int32_t n, int32_t nq, int32_t nkv, int32_t hd, float, const void *dy, int64_t dys, const void *x,
                                     int64_t xs, const void *g_q, const void *g_k, const int32_t *pos, const float *table, int32_t max_pos, void *dx,
                                     int64_t dxs, float *dg_q, float *dg_k, void *scratch, void *) {
    ++g_calls["qk_backward"];
    const size_t es = es_of(dtype), qk = (size_t)(nq + nkv) * hd, all = qk + (size_t)nkv * hd, written = dx == dy ? qk : all;
    const Span in[] = {{x, mat(n, qk, xs, es)}, {g_q, hd * es}, {g_k, hd * es}, {pos, (size_t)n * 4}, {table, (size_t)max_pos * hd * 4},
                       {dg_q, (size_t)hd * 4}, {dg_k, (size_t)hd * 4}};
    for (const Span &s : in) rd(s);
    rd({dy, mat(n, written, dys, es)});
    apart("dx overlaps", {dx, mat(n, written, dxs, es)}, in);
    apart("qk scratch overlaps", {scratch, ms_k_qk_norm_rope_backward_scratch_bytes(hd)}, in);
    const Span rows[] = {{dx, mat(n, written, dxs, es)}};
    apart("qk scratch overlaps dx", {scratch, ms_k_qk_norm_rope_backward_scratch_bytes(hd)}, rows);
    wr_rows(dx, n, written * es, dxs * es);
    wr(dg_q, (size_t)hd * 4); wr(dg_k, (size_t)hd * 4); wr(scratch, ms_k_qk_norm_rope_backward_scratch_bytes(hd));
    return MS_OK;
}

static ms_status codes_of(const char *name, int32_t n, long k, Span x, void *q, int64_t ldq, void *s, int64_t lds) {
    ++g_calls[name];
    const Span in[] = {x};
    rd(x);
    apart("codes overlap their input", {q, mat(n, k, ldq, 1)}, in);
    apart("scales overlap their input", {s, mat(n, words(k), lds, 1)}, in);
    const Span codes[] = {{q, mat(n, k, ldq, 1)}};
    apart("scales overlap codes", {s, mat(n, words(k), lds, 1)}, codes);
    wr_rows(q, n, k, ldq); wr_rows(s, n, words(k), lds);
    return MS_OK;
}
ms_status ms_k_norm_fp8(int32_t dtype, int32_t x_fp32, int32_t n, int32_t d, float, const void *x, const void *g, void *q, int64_t ldq, void *s, int64_t lds,
                        void *) {
    rd({g, d * es_of(dtype)});
    return codes_of("norm_fp8", n, d, {x, (size_t)n * d * (x_fp32 ? 4 : es_of(dtype))}, q, ldq, s, lds);
}
ms_status ms_k_fp8_quantize(int32_t dtype, int32_t block_rows, int32_t n, int32_t k, const void *x, int64_t ldx, void *q, int64_t ldq, void *s, int64_t lds, void *) {
    need(block_rows == 1, "rows of activations");
    return codes_of("quantize", n, k, {x, mat(n, k, ldx, es_of(dtype))}, q, ldq, s, lds);
}
ms_status ms_k_swiglu_fp8(int32_t dtype, int32_t n, int32_t f, const void *gate_up, int64_t ld, void *q, int64_t ldq, void *s, int64_t lds, void *) {
    return codes_of("swiglu_pass", n, f, {gate_up, mat(n, 2L * f, ld, es_of(dtype))}, q, ldq, s, lds);
}
ms_status ms_k_gemm_fp8(int32_t M, int32_t N, int32_t K, const void *A, int64_t lda, const void *sA, int64_t ldsa, const void *W, int64_t ldw, const void *sW,
                        int64_t ldsw, void *C, int64_t ldc, int32_t c_fp32, const void *R, int64_t ldr, int32_t r_fp32, void *) {
    ++g_calls["gemm_fp8"]; ++g_calls["gemm_fp8 kind " + std::to_string(c_fp32)];
    const size_t ec = c_fp32 == 1 || c_fp32 == 2 ? 4 : 2;
    const Span in[] = {{A, mat(M, K, lda, 1)}, {sA, mat(M, words(K), ldsa, 1)}, {W, mat(N, K, ldw, 1)}, {sW, mat((N + 127) / 128, words(K), ldsw, 1)},
                       {R == C ? nullptr : R, mat(M, N, ldr, r_fp32 ? 4 : 2)}};
    for (const Span &s : in) rd(s);
    apart("C overlaps", {C, mat(M, N, ldc, ec)}, in);
    wr_rows(C, M, N * ec, ldc * ec);
    return MS_OK;
}
size_t ms_k_gemm_fp8_swiglu_scratch_bytes(int32_t M, int32_t F, int32_t) { return up256((size_t)(M > 64 && F % 128 == 0 ? 64 : M) * 2 * F * 4); }
ms_status ms_k_gemm_fp8_swiglu(int32_t M, int32_t F, int32_t K, const void *A, int64_t lda, const void *sA, int64_t ldsa, const void *W, int64_t ldw,
                               const void *sW, int64_t ldsw, void *q, int64_t ldq, void *s, int64_t lds, void *scratch, size_t scratch_bytes, void *) {
    const size_t need_bytes = ms_k_gemm_fp8_swiglu_scratch_bytes(M, F, K);
    need(scratch_bytes >= need_bytes, "swiglu scratch");
    const Span in[] = {{A, mat(M, K, lda, 1)}, {sA, mat(M, words(K), ldsa, 1)}, {W, mat(2L * F, K, ldw, 1)}, {sW, mat((2L * F + 127) / 128, words(K), ldsw, 1)},
                       {q, mat(M, F, ldq, 1)}, {s, mat(M, words(F), lds, 1)}};
    for (const Span &i : in) rd(i);
    apart("swiglu scratch overlaps", {scratch, need_bytes}, in);
    wr(scratch, need_bytes);
    const Span ops[] = {in[0], in[1], in[2], in[3]};
    apart("swiglu codes overlap", in[4], ops);
    return codes_of("swiglu_gemm", M, F, {nullptr, 0}, q, ldq, s, lds);
}

}  // extern "C"
