// Sections with options on exact-size buffers, with the kernels replaced by the stand-ins of fake_backend.cpp and fake_options.cpp: the workspace
// plan (unnormed qkv, codes, scales, scratch of the sorted gradient and of the gains' gradient) and the order of the calls.
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>
#include <map>
#include <memory>
#include <string>
#include <vector>

#include "launch.h"

extern std::map<std::string, long> g_calls;
struct PartialRows { const float *p; int np, c; };
extern std::vector<PartialRows> g_pending;
static int g_checks = 0;
#define CHECK(cond)                                                                              \
    do {                                                                                         \
        ++g_checks;                                                                              \
        if (!(cond)) { fprintf(stderr, "FAILED %s:%d: %s  [%s]\n", __FILE__, __LINE__, #cond, ms_last_error()); exit(1); } \
    } while (0)

struct Buf {
    void *p;
    size_t n;
    explicit Buf(size_t bytes) : p(bytes ? malloc(bytes) : nullptr), n(bytes) { if (p) memset(p, 1, bytes); }
    ~Buf() { free(p); }
    Buf(const Buf &) = delete;
};

static size_t words(long k) { return (size_t)(k + 511) / 512 * 4; }

static void run(ms_section_config c, std::vector<int32_t> cu, float scale, bool qk, int fp8) {
    const size_t es = c.dtype == MS_BF16 ? 2 : 4, em = fp8 ? 1 : es;
    const int n = cu.back(), n_seqs = (int)cu.size() - 1, d = c.d_model, f = c.d_ffn;
    const int dqkv = (c.n_q_heads + 2 * c.n_kv_heads) * c.head_dim, dattn = c.n_q_heads * c.head_dim;
    int longest = 0;
    for (int i = 0; i < n_seqs; ++i) longest = std::max(longest, cu[i + 1] - cu[i]);
    std::vector<std::unique_ptr<Buf>> keep;
    auto blk = [&](size_t bytes) { keep.emplace_back(new Buf(bytes)); return keep.back()->p; };
    std::vector<ms_layer_ptrs> wl(c.n_layers), gl(c.n_layers);
    std::vector<ms_layer_options> lo(c.n_layers), go(c.n_layers);
    for (int i = 0; i < c.n_layers; ++i) {
        wl[i] = {blk(d * es), nullptr, blk((size_t)dqkv * d * em), nullptr, blk((size_t)d * dattn * em), nullptr,
                 blk(d * es), nullptr, blk((size_t)2 * f * d * em), nullptr, blk((size_t)d * f * em), nullptr};
        gl[i] = {blk(d * 4), nullptr, blk((size_t)dqkv * d * 4), nullptr, blk((size_t)d * dattn * 4), nullptr,
                 blk(d * 4), nullptr, blk((size_t)2 * f * d * 4), nullptr, blk((size_t)d * f * 4), nullptr};
        lo[i] = {}; go[i] = {};
        if (qk) { lo[i].q_norm_g = blk(c.head_dim * es); lo[i].k_norm_g = blk(c.head_dim * es); go[i].q_norm_g = blk(c.head_dim * 4); go[i].k_norm_g = blk(c.head_dim * 4); }
        if (fp8) {
            auto sc = [&](long rows, long k) { return blk((rows + 127) / 128 * words(k)); };
            lo[i].s_qkv = sc(dqkv, d); lo[i].s_o = sc(d, dattn); lo[i].s_up = sc(2L * f, d); lo[i].s_down = sc(d, f);
        }
    }
    const ms_section_ptrs w = {c.vocab ? blk((size_t)c.vocab * d * es) : nullptr, wl.data(), blk(d * es), nullptr};
    const ms_section_ptrs g = {c.vocab ? blk((size_t)c.vocab * d * 4) : nullptr, gl.data(), blk(d * 4), nullptr};
    const ms_section_options o = {scale, qk, fp8, qk || fp8 ? lo.data() : nullptr};
    Buf cu_dev(cu.size() * 4), x_in(c.vocab ? (size_t)n * 4 : (size_t)n * d * es), h_out((size_t)n * d * es), d_h((size_t)n * d * es);
    memcpy(cu_dev.p, cu.data(), cu.size() * 4);
    const ms_batch b = {n, n_seqs, (const int32_t *)cu_dev.p, cu.data()};
    auto calls = [](const char *k) { return g_calls[k]; };
    const long L = c.n_layers;
    {
        g_calls.clear();
        const size_t need = ms_section_workspace_bytes_with(&c, &o, n, longest, 0);
        CHECK(need > 0);
        Buf ws(need);
        CHECK(ms_section_forward_with(&c, &o, &w, &b, x_in.p, h_out.p, ws.p, need - 1, nullptr) == MS_ERR_WORKSPACE && g_calls.empty());
        CHECK(ms_section_forward_with(&c, &o, &w, &b, x_in.p, h_out.p, ws.p, need, nullptr) == MS_OK);
        CHECK(calls("embedding_scaled") == (c.vocab && scale != 1.f) && calls("embedding_forward") == (c.vocab && scale == 1.f));
        CHECK(calls("qk_forward_in_place") == (qk ? L : 0) && calls("qk_forward") == 0);
        CHECK(calls("norm_fp8") == (fp8 ? 2 * L : 0) && calls("quantize") == (fp8 ? L : 0));
        CHECK(calls("gemm_fp8") == (fp8 == 2 ? 4 * L : fp8 ? 3 * L : 0) && calls("swiglu_gemm") == (fp8 && fp8 != 2 ? L : 0) && calls("swiglu_pass") == (fp8 == 2 ? L : 0));
        CHECK(calls("gemm_fp8 kind 0") == (fp8 && fp8 != 2 ? L : 0) && calls("gemm_fp8 kind 2") == (fp8 && fp8 != 2 ? 2 * L : 0));
        CHECK(calls("gemm_fp8 kind 3") == (fp8 == 2 ? L : 0) && calls("gemm_fp8 kind 1") == (fp8 == 2 ? 3 * L : 0));
        if (fp8) CHECK(calls("gemm") == 0 && calls("gemm_swiglu") == 0);
    }
    g_calls.clear();
    const size_t need = ms_section_workspace_bytes_with(&c, &o, n, longest, 1);
    if (fp8) {
        CHECK(need == 0);
        CHECK(ms_section_forward_backward_with(&c, &o, go.data(), &w, &g, &b, x_in.p, h_out.p, d_h.p, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr,
                                               x_in.p, 1 << 20, nullptr) == MS_ERR_UNSUPPORTED && g_calls.empty());
        return;
    }
    Buf ws(need), d_x(c.vocab ? 0 : (size_t)n * d * es);
    auto backward = [&](size_t bytes) {
        return ms_section_forward_backward_with(&c, &o, qk ? go.data() : nullptr, &w, &g, &b, x_in.p, h_out.p, d_h.p, nullptr, nullptr, nullptr, nullptr, nullptr,
                                                d_x.p, ws.p, bytes, nullptr);
    };
    CHECK(backward(need - 1) == MS_ERR_WORKSPACE && g_calls.empty());
    CHECK(backward(need) == MS_OK && g_pending.empty());
    CHECK(calls("qk_forward") == (qk ? L : 0) && calls("qk_backward") == (qk ? L : 0) && calls("qk_forward_in_place") == 0);
    CHECK(calls("embedding_sorted") == (c.vocab ? 1 : 0) && calls("embedding_backward") == 0);
    // the calls without options need less or as much, and none of these kernels
    g_calls.clear();
    const size_t plain = ms_section_workspace_bytes(&c, n, longest, 1);
    CHECK(plain == ms_section_workspace_bytes_with(&c, nullptr, n, longest, 1) && plain <= need);
    Buf wp(plain);
    CHECK(ms_section_forward_backward_with(&c, nullptr, nullptr, &w, &g, &b, x_in.p, h_out.p, d_h.p, nullptr, nullptr, nullptr, nullptr, nullptr, d_x.p, wp.p,
                                           plain, nullptr) == MS_OK);
    CHECK(calls("qk_forward") + calls("qk_backward") + calls("embedding_sorted") + calls("embedding_scaled") == 0);
}

int main() {
    const ms_section_config bf16 = {MS_DECODER, MS_BF16, 2, 128, 4, 2, 64, 192, 96, 1e-6f, 1e4f};
    const ms_section_config wide = {MS_DECODER, MS_BF16, 1, 80, 2, 1, 128, 640, 40, 1e-6f, 1e4f};      // attention wider than the model
    const ms_section_config narrow = {MS_DECODER, MS_BF16, 3, 528, 1, 1, 64, 176, 0, 1e-6f, 1e4f};     // the model wider than attention, embeddings in
    const ms_section_config f32 = {MS_DECODER, MS_F32, 2, 64, 2, 2, 64, 88, 40, 1e-6f, 1e4f};
    const std::vector<std::vector<int32_t>> batches = {{0, 1}, {0, 5, 5, 21, 30}, {0, 70}, {0, 130, 131}};
    for (const auto &cu : batches) {
        for (int qk = 0; qk < 2; ++qk) {
            for (int fp8 = 0; fp8 < 3; ++fp8) {
                run(bf16, cu, 3.f, qk, fp8);
                run(wide, cu, 1.f, qk, fp8);
                run(narrow, cu, 1.f, qk, fp8);
            }
            run(f32, cu, 2.f, qk, 0);
        }
    }
    printf("host sanitizer driver: OK (%d checks)\n", g_checks);
    return 0;
}
