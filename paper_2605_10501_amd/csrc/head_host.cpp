// Host-side plan and validation of the losses at the end of a section (see head.h); kernels and their sequencing are in head.hip.
#include "head.h"
#include "launch.h"
#include <math.h>

namespace {
constexpr long kReach = kHeadReach;
constexpr long kBlockBytes = 16L << 30;                 // a block's exponentials or logits, if the caller does not say (288 GB per GPU)
constexpr long kLaunchLogits = 1L << 34;                // logits of one launch: 2^22 of the smallest tiles, of the 2^23 workgroups of 512 threads that fit one
constexpr long kTopBlockBytes = 4L << 30;               // the same for logits that are only looked through
// Tokens of a block of the fast products, whose rows one workgroup finds (head_rows_kernel): 300000 tokens of V = 8192, d = 256 forward and backward in one block 10.36 ms, so 6.97; 2 million of V = 1024, d = 128
// 20.3 and 17.8; 131072 of V = 32000, d = 1024 21.4 with both, in blocks of 32768 21.7
constexpr long kBlockRows = 65536;
long least(long a, long b) { return a < b ? a : b; }
long round_up(long x, long a) { return (x + a - 1) / a * a; }
}  // namespace

static bool bf16_tiles(const ms_head_config *c) { return head_dtype(c) == MS_BF16 && gemm_forced_tile() >= 0; }
static bool fast_products(const ms_head_config *c, HeadUse use) { return bf16_tiles(c) && c->hidden % 64 == 0 && (use == HEAD_TOP || !head_fp32_dz(c)); }
// Rows of the hidden size, of numbers of so many bytes, that the products of head_gemm.hip reach; their gradients come out in fp32.  (The products of the other path look at their operands themselves
// and take 64-bit offsets where they have to.)
static long reached_rows(const ms_head_config *c, int bytes) { return kReach / (bytes * (long)c->hidden) - 512; }
long head_most_rows(const ms_head_config *c, HeadUse use) { return least(reached_rows(c, use == HEAD_BACKWARD && fast_products(c, use) ? 4 : 2), kReach / (4 * 256) - 512); }

HeadPlan head_plan(const ms_head_config *c, int n, int k, HeadUse use, int pairs, void *ws) {
    HeadPlan p = {};
    const bool whole = pairs >= 0;
    const long V = c->vocab, d = c->hidden;
    const size_t es = ms_dtype_size(head_dtype(c));
    const bool gradients = use == HEAD_BACKWARD && head_dtype(c) == MS_BF16;
    p.fast = fast_products(c, use);
    const bool keeps = use != HEAD_FORWARD || !p.fast;                       // something of every (row, vocabulary entry)
    const size_t ez = p.fast && use != HEAD_TOP ? 2 : 4;
    // tokens of a block: the caller's choice, or what the memory above holds, in blocks of about equal size
    long most = head_most_rows(c, use);
    if (gradients && !whole) most = least(most, reached_rows(c, 4));
    if (!whole && c->token_block > 0) most = least(most, c->token_block);
    else if (!whole) {
        if (p.fast && use != HEAD_TOP) most = least(most, kBlockRows);
        if (!keeps) most = least(most, round_up(kBlockBytes / (8 * ((V + kStrip - 1) / kStrip)) + 1, 256));
        else most = least(most, round_up((use == HEAD_TOP ? kTopBlockBytes : kBlockBytes) / (long)(ez * V) + 1, 256));
    }
    const long blocks = whole || n <= most ? 1 : (n + most - 1) / most;
    p.block = (int)(blocks == 1 ? n : least(most, round_up((n + blocks - 1) / blocks, 8)));
    p.rows = (int)round_up(p.block, 16);                                       // (a strip's words and bytes start at 16 bytes)
    p.tiles = gradients && bf16_tiles(c) && p.block <= reached_rows(c, 4);
    auto slabs_of = [&](long rows) {
        long widest = reached_rows(c, gradients ? 4 : 2);
        if (keeps) widest = least(widest, kReach / (long)(ez * (rows + 256L)));
        else widest = least(widest, kLaunchLogits / (rows + 256L));
        widest = widest / 256 * 256;
        return (V + widest - 1) / widest;
    };
    p.slabs = (int)slabs_of(p.rows);
    p.cols = p.slabs == 1 ? (int)V : (int)round_up((V + p.slabs - 1) / p.slabs, 256);
    if (p.fast || p.tiles) p.cols = (int)round_up(p.cols, 64);               // (d_h's product reads whole K tiles)
    p.strips = (int)((V + kStrip - 1) / kStrip);
    // What is taken is for the largest block of calls up to this one, so that memory for n tokens serves fewer (97 tokens in blocks of at most 80 are two of 56)
    const size_t r = (size_t)round_up(least(n, most), 16);
    Arena a(ws);
    p.slot = a.take<int>(r * 4);
    p.token = a.take<int>(r * 4);
    p.count = a.take<int>(4);
    p.h = a.take<void>(r * d * es);
    p.ref = a.take<float2>(r * 8);
    p.stat = a.take<float2>(r * 8);
    if (p.fast || use == HEAD_TOP) p.part = a.take<float2>(r * p.strips * 8);
    if (use != HEAD_TOP) {
        p.z_sel = a.take<float>(r * (k ? k : 1) * 4);
        p.z_label = a.take<float>(r * 4);
        p.logp = a.take<float>(r * 4);
        if (k) {
            p.log_p = a.take<float>(r * k * 4);
            p.mass = a.take<float>(r * 4);
            p.ids = a.take<int>(r * k * 4);
            p.key = a.take<int>(r * 4);
            p.best = a.take<int>(r * 4);
            if (p.fast && head_use_marks(k, d, p.strips)) {
                p.marks = a.take<unsigned long long>(r * p.strips * 8);
                p.marks_first = a.take<unsigned char>(r * p.strips);
            }
        }
        p.per_token = a.take<float>((size_t)(whole ? pairs : n) * 4);
        if (whole) p.margin = a.take<float>((size_t)pairs * 4);
    }
    if (use == HEAD_BACKWARD) {
        p.rho = a.take<float>(r * (k ? k : 1) * 4);
        p.scale = a.take<float>(r * 4);
        p.factor = a.take<float>(r * 4);
        p.parts = 1;
        if (p.tiles) {
            p.choice = head_choose(p.block, V < p.cols ? V : p.cols, d, gemm_forced_tile());
            p.parts = p.choice.parts;
        }
        if (p.fast) {
            p.fixes = k < 1 ? 1 : k < kHeadFixes ? k : kHeadFixes;
            const size_t f = r * p.fixes;
            p.fix_id = a.take<int>(f * 4);
            p.fix_rest = a.take<float>(f * 4);
            p.fix = a.take<void>(f * d * 2);
            if (f > (size_t)kHeadScan) {
                p.fix_scratch_bytes = ms_k_embedding_sorted_backward_scratch_bytes((int)f, (int)d, (int)V);
                p.fix_scratch = a.take<void>(p.fix_scratch_bytes);
            }
        }
        const long sums = (long)r * d, in_parts = least(kHeadMostParts * sums, kHeadPartsRoom);
        if (head_dtype(c) == MS_BF16) p.d_h = a.take<float>((p.tiles && in_parts > sums ? in_parts : sums) * 4);
        if (!p.fast && head_dtype(c) == MS_BF16) {
            const size_t most_dz = least((long)r * (V + 256), kReach / 4) * 2;
            p.dz = a.take<void>(most_dz);
            if (head_fp32_dz(c)) p.dz_rest = a.take<void>(most_dz);
        }
    }
    if (keeps) p.z = a.take<void>(r * (V + 257 * slabs_of((long)r)) * ez);
    p.bytes = a.off;
    return p;
}

ms_status validate_head(const ms_head_config *c, int n, int k, const char *what) {
    if (!c) return ms_fail(MS_ERR_INVALID_ARG, "%s: null config", what);
    if (n < 0) return ms_fail(MS_ERR_INVALID_ARG, "%s: negative token count", what);
    if (head_dtype(c) != MS_BF16 && c->dtype != MS_F32) return ms_fail(MS_ERR_INVALID_ARG, "%s: bad dtype", what);
    if (c->vocab <= 0 || c->hidden <= 0) return ms_fail(MS_ERR_SHAPE, "%s: vocab and hidden size must be positive", what);
    if (c->vocab % 8 || c->hidden % 8) return ms_fail(MS_ERR_UNSUPPORTED, "%s: vocab and hidden size must be multiples of 8", what);
    if ((long)c->hidden > 65536 || c->vocab > (1 << 24)) return ms_fail(MS_ERR_UNSUPPORTED, "%s: hidden size over 65536 or vocab over 2^24", what);
    if (!(c->temperature > 0.f) || !isfinite(c->temperature) || !isfinite(1.f / c->temperature))
        return ms_fail(MS_ERR_INVALID_ARG, "%s: temperature must be positive", what);
    if (!isfinite(c->loss_scale)) return ms_fail(MS_ERR_INVALID_ARG, "%s: loss_scale must be finite", what);
    if (c->token_block < 0 || c->token_block % 8) return ms_fail(MS_ERR_INVALID_ARG, "%s: token_block must be 0 or a positive multiple of 8", what);
    if (k < 0 || k > kHeadMaxTop || k > c->vocab) return ms_fail(MS_ERR_UNSUPPORTED, "%s: k must be 1 .. %d and at most the vocabulary", what, kHeadMaxTop);
    if (!c->w_dev) return ms_fail(MS_ERR_INVALID_ARG, "%s: null lm_head pointer", what);
    return MS_OK;
}

static size_t bytes_of(const ms_head_config *c, int n, int k, HeadUse use, int pairs) {
    if (!c || n < 0 || c->vocab <= 0 || c->hidden <= 0 || c->hidden > 65536 || c->vocab > (1 << 24) || c->token_block < 0 || k < 0 || k > kHeadMaxTop) return 0;
    if (pairs >= 0 && n > head_most_rows(c, use)) return 0;
    return head_plan(c, n, k, use, pairs, nullptr).bytes;
}
extern "C" size_t ms_top_logits_workspace_bytes(const ms_head_config *c, int32_t max_tokens, int32_t k) { return k < 1 ? 0 : bytes_of(c, max_tokens, k, HEAD_TOP, -1); }
extern "C" size_t ms_head_workspace_bytes(const ms_head_config *c, int32_t max_tokens, int32_t k, int32_t need_backward) {
    return bytes_of(c, max_tokens, k, need_backward ? HEAD_BACKWARD : HEAD_FORWARD, -1);
}
extern "C" size_t ms_preference_workspace_bytes(const ms_head_config *c, int32_t max_tokens, int32_t max_pairs, int32_t need_backward) {
    return max_pairs < 0 ? 0 : bytes_of(c, max_tokens, 0, need_backward ? HEAD_BACKWARD : HEAD_FORWARD, max_pairs);
}
