// Plans of the losses at the end of a section (csrc/head_host.cpp) whose gradients are 32-bit numbers: the bf16 products reach what they read and what they write by 32-bit byte offsets, up to 256
// rows past the last one, so every slab of the lm_head and its fp32 gradient, every block of hidden states and its fp32 gradient, and every slab of what is kept between the halves of a pass
// have to lie below 4 GB, at sizes on both sides of it; and memory for more tokens serves fewer there too.
#include <stdio.h>

#include <algorithm>
#include <vector>

#include "head.h"

static int failures;
#define CHECK(x) do { if (!(x) && ++failures < 20) printf("line %d: %s (vocab %d hidden %d block %d n %d use %d pairs %d: slabs %d cols %d rows %d)\n", __LINE__, #x, c.vocab, c.hidden, c.token_block, n, use, pairs, p.slabs, p.cols, p.rows); } while (0)

int gemm_forced_tile() { return 0; }
extern "C" size_t ms_k_embedding_sorted_backward_scratch_bytes(int32_t n, int32_t d, int32_t vocab) { return n > 0 && d > 0 && vocab > 0 ? (size_t)n * 24 : 0; }

int main() {
    const struct { int vocab, hidden; } heads[] = {{152064, 8192}, {151936, 7040}, {151936, 7104}, {262144, 5376}, {262208, 5376}, {262144, 4096}, {262136, 4096}, {128256, 16384}, {256000, 12288},
                                                   {1 << 24, 64}, {1 << 21, 128}, {1 << 24, 65536}, {32768, 32768}, {16384, 65536}, {1024, 4096}, {32000, 4096}, {8, 65536}, {151936, 1536}, {151936, 7112}, {1024, 4104}, {1024, 65528}};
    const int tokens[] = {1, 64, 100, 4096, 15000, 33000, 65536, 131072, 262144, 265000, 300000, 530000, 3000000};
    const long reach = 1L << 32;
    long plans = 0;
    for (int dtype : {(int)MS_BF16, MS_BF16 | MS_HEAD_FP32_DZ})
    for (auto [v, d] : heads)
        for (int b : {0, 4096, 300000, 1 << 24})
            for (HeadUse use : {HEAD_TOP, HEAD_FORWARD, HEAD_BACKWARD})
                for (int whole = 0; whole < 2; ++whole) {
                    ms_head_config c = {};
                    c.vocab = v; c.hidden = d; c.dtype = dtype; c.token_block = b; c.temperature = 1.f; c.loss_scale = 1.f; c.w_dev = (const void *)4096;
                    size_t before = 0;
                    std::vector<long> counts(std::begin(tokens), std::end(tokens));
                    for (long bytes : {2, 4})                                   // the longest blocks there are, and a token more and less
                        for (long more : {-1, 0, 1}) counts.push_back(std::min(((1L << 32) - (1L << 20)) / (bytes * d) - 512 + more, 1L << 24));
                    std::sort(counts.begin(), counts.end());
                    for (long count : counts) {
                        const int n = (int)count;
                        const int k = use == HEAD_TOP ? 8 : 0, pairs = whole ? n / 2 : -1;
                        if (whole && use == HEAD_TOP) continue;
                        const size_t bytes = use == HEAD_TOP ? ms_top_logits_workspace_bytes(&c, n, k) : whole ? ms_preference_workspace_bytes(&c, n, pairs, use == HEAD_BACKWARD)
                                                                                                               : ms_head_workspace_bytes(&c, n, k, use == HEAD_BACKWARD);
                        if (whole && bytes == 0) continue;                     // (more tokens than one block takes: refused)
                        const HeadPlan p = head_plan(&c, n, k, use, pairs, nullptr);
                        const long r = p.rows + 256L, w = p.cols + 256L;
                        CHECK(validate_head(&c, n, k, "plan") == MS_OK && p.fast == (d % 64 == 0 && (use == HEAD_TOP || dtype == MS_BF16)) && p.bytes == bytes && bytes >= before);
                        before = bytes;
                        CHECK(r * d * 2 < reach && w * d * 2 < reach);
                        if (use == HEAD_BACKWARD && p.tiles) CHECK(r * d * 4 < reach && w * d * 4 < reach);
                        if (use == HEAD_BACKWARD) CHECK(p.tiles || (whole && !p.fast));       // (one block that is too long for them has products that take 64-bit offsets)
                        if (use != HEAD_FORWARD || !p.fast) CHECK(r * p.cols * (use == HEAD_TOP || !p.fast ? 4 : 2) < reach);
                        // a forward pass keeps nothing of the logits: what bounds it is the largest launch, and its strips' sums
                        if (p.fast && use == HEAD_FORWARD) CHECK(ms_launch_fits((long)ms_cdiv(p.rows, 64) * ms_cdiv(v < p.cols ? v : p.cols, 64), 512));
                        if (p.fast && use == HEAD_FORWARD && b == 0 && !whole) CHECK(p.bytes < 40ul << 30);
                        if (p.fast && use != HEAD_TOP && b == 0 && !whole) CHECK(p.block <= 65536);       // (one workgroup finds its rows)
                        if (p.dz_rest || (use == HEAD_BACKWARD && dtype != MS_BF16)) {
                            char *const base = (char *)(1ul << 45);            // (never followed)
                            const HeadPlan q = head_plan(&c, n, k, use, pairs, base);
                            const long slab = (long)p.rows * p.cols;
                            CHECK(q.dz && (char *)q.dz + slab * 2 <= (char *)q.dz_rest && (char *)q.dz_rest + slab * 2 <= (char *)q.z && (char *)q.z + slab * 4 * p.slabs <= base + bytes);
                        }
                        ++plans;
                    }
                }
    if (failures) { printf("%d failures\n", failures); return 1; }
    printf("head reach: OK (%ld)\n", plans);
    return 0;
}
