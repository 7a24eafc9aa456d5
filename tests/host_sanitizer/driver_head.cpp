// Plans of the losses at the end of a section (csrc/head_host.cpp) over many sizes: every piece lies inside the workspace and behind the one before it, slabs cover
// the vocabulary within reach of 32-bit offsets, blocks cover the tokens, and the parts of d_h are those that its product is cut into.
#include <stdio.h>
#include <stdlib.h>

#include <vector>

#include "head.h"

static int failures;
#define CHECK(x) do { if (!(x) && ++failures < 20) printf("line %d: %s (vocab %d hidden %d dtype %d block %d n %d k %d use %d pairs %d)\n", __LINE__, #x, c.vocab, c.hidden, c.dtype, c.token_block, n, k, use, pairs); } while (0)

static int forced;
int gemm_forced_tile() { return forced; }
extern "C" size_t ms_k_embedding_sorted_backward_scratch_bytes(int32_t n, int32_t d, int32_t vocab) { return n > 0 && d > 0 && vocab > 0 ? (size_t)n * 24 : 0; }

static void check(const ms_head_config &c, int n, int k, HeadUse use, int pairs) {
    if (pairs >= 0 && n > head_most_rows(&c)) return;
    const HeadPlan size = head_plan(&c, n, k, use, pairs, nullptr);
    char *const base = (char *)(1ul << 45);                        // (never followed)
    const HeadPlan p = head_plan(&c, n, k, use, pairs, base);
    CHECK(size.bytes == p.bytes && size.rows == p.rows && size.cols == p.cols && size.parts == p.parts);
    const long V = c.vocab, d = c.hidden, r = p.rows, es = c.dtype == MS_BF16 ? 2 : 4, kk = k ? k : 1, reach = (1L << 32) - (1L << 20);
    if (n == 0) return;
    CHECK(r % 16 == 0 && r >= p.block && r < p.block + 16 && p.block >= 1 && p.block <= n && (pairs < 0 || p.block == n));
    CHECK(c.token_block == 0 || pairs >= 0 || p.block <= c.token_block);
    CHECK((long)p.slabs * p.cols >= V && (long)(p.slabs - 1) * p.cols < V && (long)p.strips * 64 >= V && (long)(p.strips - 1) * 64 < V);
    CHECK(p.slabs == 1 || p.cols % 256 == 0);
    CHECK(p.fast == (c.dtype == MS_BF16 && d % 64 == 0 && forced >= 0));
    CHECK(!p.fast || p.cols % 64 == 0);
    const bool keeps = use != HEAD_FORWARD || !p.fast;
    const long ez = p.fast && use != HEAD_TOP ? 2 : 4;
    CHECK((p.cols + 256L) * d * 2 < reach && (r + 256) * d * 2 < reach);
    if (keeps) CHECK((r + 256) * p.cols * ez <= reach + 256 * 256 * ez);
    struct Piece { const void *at; size_t bytes; };
    std::vector<Piece> all = {{p.slot, (size_t)r * 4}, {p.token, (size_t)r * 4}, {p.count, 4}, {p.h, (size_t)(r * d * es)}, {p.ref, (size_t)r * 8}, {p.stat, (size_t)r * 8}};
    if (p.fast || use == HEAD_TOP) all.push_back({p.part, (size_t)r * p.strips * 8});
    if (use != HEAD_TOP) {
        all.push_back({p.z_sel, (size_t)(r * kk * 4)});
        all.push_back({p.z_label, (size_t)r * 4});
        all.push_back({p.logp, (size_t)r * 4});
        if (k) {
            all.push_back({p.log_p, (size_t)(r * k * 4)});
            all.push_back({p.mass, (size_t)r * 4});
            all.push_back({p.ids, (size_t)(r * k * 4)});
            all.push_back({p.key, (size_t)r * 4});
            all.push_back({p.best, (size_t)r * 4});
            CHECK((p.marks != nullptr) == (p.fast && head_use_marks(k, d, p.strips)));
            if (p.marks) {
                all.push_back({p.marks, (size_t)r * p.strips * 8});
                all.push_back({p.marks_first, (size_t)r * p.strips});
            }
        }
        all.push_back({p.per_token, (size_t)(pairs >= 0 ? pairs : n) * 4});
        if (pairs >= 0) all.push_back({p.margin, (size_t)pairs * 4});
    }
    if (use == HEAD_BACKWARD) {
        all.push_back({p.rho, (size_t)(r * kk * 4)});
        all.push_back({p.scale, (size_t)r * 4});
        all.push_back({p.factor, (size_t)r * 4});
        if (p.fast) {
            CHECK(p.fixes >= 1 && p.fixes <= kHeadFixes && p.fixes <= kk);
            const size_t f = (size_t)r * p.fixes;
            all.push_back({p.fix_id, f * 4});
            all.push_back({p.fix_rest, f * 4});
            all.push_back({p.fix, f * d * 2});
            if (f > (size_t)kHeadScan) {
                CHECK(p.fix_scratch_bytes >= f * 24);
                all.push_back({p.fix_scratch, p.fix_scratch_bytes});
            }
            const int cw = V < p.cols ? (int)V : p.cols, kt = (cw + 63) / 64, per = (kt + p.parts - 1) / p.parts;
            CHECK(p.parts == p.choice.parts && p.parts >= 1 && (kt + per - 1) / per == p.parts && p.choice.tile >= 0 && p.choice.tile < kNumTiles);
        }
        if (c.dtype == MS_BF16) all.push_back({p.d_h, (size_t)(r * d * 4) * p.parts});
        if (c.dtype == MS_BF16 && !p.fast) all.push_back({p.dz, (size_t)(r * p.cols * 2)});
    }
    if (keeps) all.push_back({p.z, (size_t)(r * p.cols * ez) * p.slabs});
    const char *end = base;
    for (const Piece &q : all) {
        CHECK((const char *)q.at >= end && ((size_t)q.at & 255) == 0);
        end = (const char *)q.at + q.bytes;
    }
    CHECK((size_t)(end - base) <= p.bytes);
}

int main() {
    const int vocabs[] = {8, 64, 72, 1024, 32000, 151936, 270336, 1 << 24}, hiddens[] = {8, 64, 72, 128, 1536, 4096, 65536}, tokens[] = {0, 1, 2, 45, 293, 4096, 4097, 32768, 200001, 3000000};
    const int blocks[] = {0, 8, 4096}, ks[] = {0, 1, 3, 64, 128};
    long plans = 0;
    for (int tile : {0, -1, 64064, 256})
    for (int dtype : {(int)MS_F32, (int)MS_BF16})
        for (int v : vocabs)
            for (int d : hiddens)
                for (int b : blocks) {
                    ms_head_config c = {};
                    c.vocab = v; c.hidden = d; c.dtype = dtype; c.token_block = b; c.temperature = 1.f; c.loss_scale = 1.f; c.w_dev = (const void *)4096;
                    forced = tile;
                    for (int n : tokens)
                        for (int k : ks) {
                            if (k > v) continue;
                            for (HeadUse use : {HEAD_TOP, HEAD_FORWARD, HEAD_BACKWARD}) {
                                if (use == HEAD_TOP && !k) continue;
                                if (n && validate_head(&c, n, k, "plan") != MS_OK) { printf("%s\n", ms_last_error()); ++failures; }
                                check(c, n, k, use, -1);
                                if (use != HEAD_TOP && !k) check(c, n, 0, use, n / 7);
                                ++plans;
                            }
                        }
                }
    if (failures) { printf("%d failures\n", failures); return 1; }
    printf("head plans: OK (%ld)\n", plans);
    return 0;
}
