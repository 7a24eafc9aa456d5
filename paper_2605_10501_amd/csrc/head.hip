// Losses, log-probabilities and top logits at the end of a decoder section (maestro_section.h).
//
// With x = z log2(e), z = h w^T / T the logits of a row (a token that counts), everything goes by sums of 2^(x - reference) over strips of 64 columns:
//   lse = ln 2 (reference + log2 sum),   q_v = 2^(x_v - reference) / sum,   dz_v = scale_row q_v but at the few selected ids of the row
// (its label, or the teacher's entries), where rho = dz / scale_row is q - 1 or q - p / sum p.  The logits there are dot products of their own.
#include <initializer_list>

#include "common.h"
#include "head.h"
#include "head_f32.h"
#include "head_gemm.h"
#include "launch.h"

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr double kLog2e64 = 1.4426950408889634, kLn264 = 0.6931471805599453;

// Logits [slab][rows][cols] (or what is kept in their place)
struct Slabs {
    int rows, cols, vocab;
    __device__ __forceinline__ long at(int row, int v) const {
        const int s = v / cols;
        return ((long)s * rows + row) * cols + (v - s * cols);
    }
};

__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// ------------------------------------------------------------------ which tokens count
// The teacher's entries of a token, one wave each: those that count, in the order of their ids (-1 behind them), ln p of each, the sum of p, and the id of the largest (the lowest of equal ones:
// it is the reference of the row's exponentials, whose roundings go by it).
struct Teacher {
    int k, vocab;
    float inv_t;
    const int *top_ids;                                                            // [n][k]; null: no entries
    const float *top, *lse;
    int *ids, *best, *key;
    float *log_p, *mass;
};
// Sum of p below which a token is left out: its terms are as small, and the entries' shares p / sum p, by which the gradient goes, would need 1 / sum p beyond fp32
constexpr float kLeastMass = 0x1p-100f;
// Token t for this wave (not below n: none), of four in the workgroup, all of which come here; returns whether the token counts
__device__ __forceinline__ bool teacher_entries(const Teacher &a, int n, long t, int (&seen)[kHeadMaxTop]) {
    const int lane = threadIdx.x & 63, k = a.k;
    if (t < n)
        for (int j = lane; j < k; j += 64) seen[j] = a.top_ids[t * k + j];
    __syncthreads();
    float y[2] = {-INFINITY, -INFINITY}, m = -INFINITY;
    int id[2] = {-1, -1};
    if (t < n) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int j = lane + 64 * e;
            id[e] = j < k ? seen[j] : -1;
            if (id[e] >= a.vocab) id[e] = -1;
            if (id[e] >= 0)
                for (int i = 0; i < j; ++i)
                    if (seen[i] == id[e]) id[e] = -1;
            y[e] = id[e] >= 0 ? a.top[t * k + j] * a.inv_t : -INFINITY;
            m = fmaxf(m, y[e]);                                                     // (passes over NaN, which the sum has)
        }
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 2; ++e)
        if (lane + 64 * e < k) seen[lane + 64 * e] = id[e];
    __syncthreads();
    if (t >= n) return false;
    m = wave_max(m);
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 2; ++e)
        if (id[e] >= 0 && !(y[e] == -INFINITY)) s += expf(y[e] - (m == -INFINITY ? 0.f : m));
    s = wave_sum(s);
    const bool some = !(s == 0.f);                                              // an entry above -inf, or a NaN
    const float L = a.lse ? (some ? a.lse[t] : 0.f) : m + logf(s);
    float total = 0.f;
    int valid = 0, best = 0x7fffffff;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const bool in = some && id[e] >= 0;
        valid += __popcll(__ballot(in));
        if (!in) continue;
        const float lp = y[e] - L;
        int at = 0;
        for (int i = 0; i < k; ++i) at += seen[i] >= 0 && seen[i] < id[e];
        a.ids[t * k + at] = id[e];
        a.log_p[t * k + at] = lp;
        total += expf(lp);
        if (y[e] == m) best = id[e] < best ? id[e] : best;
    }
    for (int j = valid + lane; j < k; j += 64) a.ids[t * k + j] = -1;
    total = wave_sum(total);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const int other = __shfl_xor(best, o, 64);
        best = other < best ? other : best;
    }
    const bool counts = some && !(total < kLeastMass);
    if (lane == 0) {
        a.mass[t] = counts ? total : 0.f;
        a.key[t] = counts ? 0 : -1;
        a.best[t] = m == -INFINITY ? (valid ? 0 : -1) : some ? best : -1;       // (-infinity: only NaN among them)
    }
    return counts;
}
// 32768 tokens of 64 entries: 30 us, and the marks' 622 MB cleared beside them 115 (HBM).  clear: n_clear 16-byte words (the marks, see MarkWords) that are zero afterwards
__global__ __launch_bounds__(256) void head_entries_kernel(int n, Teacher a, float4 *__restrict__ clear, long n_clear) {
    __shared__ int seen[4][kHeadMaxTop];
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < n_clear; i += 256L * gridDim.x) clear[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    teacher_entries(a, n, (long)blockIdx.x * 4 + (threadIdx.x >> 6), seen[threadIdx.x >> 6]);
}

// Rows of a block: the tokens that count (key in [0, limit)) in their order, without gaps; out0, out1 of the others are 0.  One workgroup: a block has at most
// 65536 tokens, of which it reads four bytes (if the caller does not ask for longer ones; a preference loss, whose tokens are one block, up to some million, 1024 at a time).
__global__ __launch_bounds__(1024) void head_rows_kernel(int n, const int *__restrict__ key, int limit, int *__restrict__ slot, int *__restrict__ token, int *__restrict__ count,
                                                         float *__restrict__ out0, float *__restrict__ out1) {
    __shared__ int sm[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int base = 0;
    for (int t0 = 0; t0 < n; t0 += 1024) {
        const int t = t0 + threadIdx.x;
        const bool in = t < n && key[t] >= 0 && key[t] < limit;
        if (t < n && !in) {
            if (out0) out0[t] = 0.f;
            if (out1) out1[t] = 0.f;
        }
        const unsigned long long mask = __ballot(in);
        if (lane == 0) sm[wave] = __popcll(mask);
        __syncthreads();
        int before = base, all = 0;
        for (int i = 0; i < 16; ++i) {
            if (i < wave) before += sm[i];
            all += sm[i];
        }
        before += __popcll(mask & ((1ull << lane) - 1));
        if (t < n) slot[t] = in ? before : -1;
        if (in) token[before] = t;
        base += all;
        __syncthreads();
    }
    if (threadIdx.x == 0) *count = base;
}

// ------------------------------------------------------------------ rows and their selected logits
// Copies the hidden states of the rows together, and takes the logits of each row's k selected ids (h rows . w rows, fp32); the reference of the
// row's exponentials is the largest of them, as a whole power of two, so that 2^(x - reference) of a row sum to one or more.  For several ids; one id, and the
// teacher's best of many whose logits come out of the matrix product, are head_pick_one_kernel's.  W waves a row, four ids at a time.
template <int W>
__global__ __launch_bounds__(64 * W) void head_pick_kernel(int d, int k, const bf16_t *__restrict__ h, const bf16_t *__restrict__ w, const int *__restrict__ token,
                                                           const int *__restrict__ count, const int *__restrict__ sel, float it2, bf16_t *__restrict__ out,
                                                           float *__restrict__ z_sel, float2 *__restrict__ ref) {
    __shared__ float sm[W];
    const int row = blockIdx.x;
    if (row >= *count) return;
    const int t = token[row], lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const bf16_t *hr = h + (long)t * d;
    for (int i = threadIdx.x * 8; i < d; i += 64 * W * 8) stv(out + (long)row * d + i, ldv(hr + i));
    float best = -INFINITY;
    for (int j0 = wave * 4; j0 < k; j0 += 4 * W) {
        const bf16_t *wr[4];
        int id[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            id[j] = j0 + j < k ? sel[(long)t * k + j0 + j] : -1;
            wr[j] = w + (long)(id[j] < 0 ? 0 : id[j]) * d;
        }
        float acc[4] = {0.f, 0.f, 0.f, 0.f};
        for (int i = lane * 8; i < d; i += 64 * 8) {
            const Vec16<bf16_t> a = ldv(hr + i);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (id[j] < 0) continue;
                const Vec16<bf16_t> b = ldv(wr[j] + i);
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[j] = __builtin_fmaf((float)a.v[e], (float)b.v[e], acc[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            acc[j] = wave_sum(acc[j]);
            if (id[j] < 0) continue;
            best = fmaxf(best, acc[j]);
            if (lane == 0) z_sel[(long)row * k + j0 + j] = acc[j];
        }
    }
    if (lane == 0) sm[wave] = best;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < W; ++i) best = fmaxf(best, sm[i]);
        ref[row] = make_float2(rintf(best * it2), __int_as_float(-1));
    }
}

// Marks of a row's entries (ids of its token in their order), whose logits the matrix product then leaves in z_sel; the words are zero before
struct MarkWords {
    int k, ld;
    const int *ids;
    unsigned long long *word;                                                      // [strips][ld]; null: no marks
    unsigned char *first;
};
__device__ __forceinline__ void mark_entries(const MarkWords &a, int t, int row) {  // by a wave
    const int *r = a.ids + (long)t * a.k;
    for (int j = threadIdx.x & 63; j < a.k; j += 64) {
        const int id = r[j], strip = id >> 6;
        if (id < 0 || (j > 0 && r[j - 1] >> 6 == strip)) continue;              // the first of its strip writes the word
        unsigned long long word = 0;
        for (int i = j; i < a.k && r[i] >= 0 && r[i] >> 6 == strip; ++i) word |= 1ull << (r[i] & 63);
        a.word[(long)strip * a.ld + row] = word;
        a.first[(long)strip * a.ld + row] = (unsigned char)j;
    }
}

// The same with one id a row, a label's (z_sel given) or the teacher's best, one wave per row, which marks its entries too.  FIND: the rows are found here too, instead of by head_rows_kernel (a launch
// less): wave j is token j, and its workgroup counts the tokens before it that have rows.  For n <= kHeadFind, which is then a load of 16 keys by every thread.
// HBM: 32768 rows of 1536, 302 MB, 59 us; with 64 entries to mark, whose words lie in as many cache lines, 169.
constexpr int kHeadFind = 4096;
template <bool FIND>
__global__ __launch_bounds__(256) void head_pick_one_kernel(int n, int d, const bf16_t *__restrict__ h, const bf16_t *__restrict__ w, const int *__restrict__ key, int limit, int *slot, int *token,
                                                            int *count, float *__restrict__ out0, float *__restrict__ out1, const int *__restrict__ sel, float it2, bf16_t *__restrict__ out,
                                                            float *__restrict__ z_sel, float2 *__restrict__ ref, MarkWords marks) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int row = blockIdx.x * 4 + wave, t;
    if constexpr (FIND) {
        __shared__ int sm[4];
        const int first = blockIdx.x * 4;
        auto counts = [&](int j) { return key[j] >= 0 && key[j] < limit; };
        int before = 0;
#pragma unroll
        for (int u = 0; u < kHeadFind / 256; ++u) {
            const int j = u * 256 + threadIdx.x;
            before += __popcll(__ballot(j < first && counts(j)));
        }
        if (lane == 0) sm[wave] = before;
        __syncthreads();
        t = row;
        row = sm[0] + sm[1] + sm[2] + sm[3];
        if (t >= n) return;
        for (int j = first; j < t; ++j) row += counts(j);
        const bool in = counts(t);
        if (lane == 0) {
            slot[t] = in ? row : -1;
            if (in) token[row] = t;
            else {
                if (out0) out0[t] = 0.f;
                if (out1) out1[t] = 0.f;
            }
            if (t == n - 1) *count = row + in;
        }
        if (!in) return;
    } else {
        if (row >= *count) return;
        t = token[row];
    }
    const int id = sel[t];
    const bf16_t *hr = h + (long)t * d, *wr = w + (long)(id < 0 ? 0 : id) * d;
    float acc = 0.f;
    for (int i = lane * 8; i < d; i += 64 * 8) {
        const Vec16<bf16_t> a = ldv(hr + i), b = ldv(wr + i);
        stv(out + (long)row * d + i, a);
#pragma unroll
        for (int e = 0; e < 8; ++e) acc = __builtin_fmaf((float)a.v[e], (float)b.v[e], acc);
    }
    acc = wave_sum(acc);
    if (marks.word) mark_entries(marks, t, row);
    if (lane != 0) return;
    if (z_sel) z_sel[row] = acc;
    ref[row] = make_float2(rintf(acc * it2), __int_as_float(z_sel ? id : -1));
}

// ------------------------------------------------------------------ sums over the vocabulary
// Stored fp32 logits: largest logit of a strip of 64 columns and sum of 2^(x - largest x).  One wave per strip, four per workgroup.
__global__ __launch_bounds__(256) void head_strips_kernel(Slabs sl, int rows, int strips, const float *__restrict__ z, float it2, float2 *__restrict__ part) {
    const int lane = threadIdx.x & 63, strip = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (strip >= strips) return;
    for (int row = blockIdx.y; row < rows; row += gridDim.y) {
        const int v = strip * kStrip + lane;
        const bool in = v < sl.vocab;
        const float a = in ? z[sl.at(row, v)] : -INFINITY;
        const float m = wave_max(a), u = m == -INFINITY ? 0.f : m;                  // (differences first: exact near the largest, whatever its size)
        const float s = wave_sum(in ? __builtin_amdgcn_exp2f((a - u) * it2) : 0.f);
        if (lane == 0) part[(long)strip * sl.rows + row] = make_float2(m, s);
    }
}

// ------------------------------------------------------------------ what a token's gradient is
// Labels: dz = g / T (1_label - q), g = d loss / d logp, so scale = -g / T and rho = q - 1.
struct LabelRows {
    const int *slot;
    float *scale, *rho, minus_inv_t;                                            // scale null: forward only
    __device__ __forceinline__ void set(int row, float g, float logp) const {
        if (!scale) return;
        scale[row] = minus_inv_t * g;
        rho[row] = expm1f(logp);
    }
};

struct PolicyArgs {
    const float *old_logp, *ref_logp, *adv, *weights;
    float *loss_tok;
    float low, high, kl, loss_scale;
};
__device__ __forceinline__ float policy_term(const PolicyArgs &a, int t, float l) {                // writes the loss, returns d loss / d logp
    const float adv = a.adv[t], wt = a.weights ? a.weights[t] : 1.f;
    const float r = expf(l - a.old_logp[t]);
    const bool inside = adv > 0.f ? r <= 1.f + a.high : r >= 1.f - a.low;          // (a NaN ratio is not; it is in `gain` all the same)
    const float gain = adv == 0.f ? 0.f : adv * (inside || !(r == r) ? r : adv > 0.f ? 1.f + a.high : 1.f - a.low);
    float loss = -gain, g = inside || !(r == r) ? -gain : 0.f;
    if (a.ref_logp) {
        const float u = a.ref_logp[t] - l, away = expm1f(u);
        loss += a.kl * (away - u);
        g -= a.kl * away;
    }
    a.loss_tok[t] = wt * loss;
    return a.loss_scale * wt * g;
}
// What follows for a row with a label once its sum is there
enum { AFTER_NOTHING = 0, AFTER_LOGP = 1, AFTER_GIVEN = 2, AFTER_POLICY = 3 };
struct After {
    int what;
    double inv_t;
    const float *z_label;
    float *logp;                                                                   // by token
    const float *d_logp;                                                           // given
    LabelRows rows;
    PolicyArgs policy;
};

// A row's log-probability and what follows.  x = (x of the label) - (reference of the sum s), in_sum = what the sum has for the label.
// The label's logit is a dot product of its own (64 partial sums), nearer than the matrix product's, whose error would be there in full where the label is unlikely; in the
// sum it takes the place of the matrix product's, so that they go together where it is likely.  In 64 bits: logarithms of 15 summed over a sequence, and their differences.
__device__ __forceinline__ double x_label(const After &a, float z) { return (double)z * a.inv_t * kLog2e64; }
__device__ __forceinline__ float label_after(const After &a, int t, int row, double x, float s, float in_sum) {
    const double others = (double)s - (double)in_sum, v = kLn264 * x - log((others < 0.0 ? 0.0 : others) + exp2(x));       // (comparisons that a NaN passes, as fmax and fmin do not let it)
    const float l = (float)(v > 0.0 ? 0.0 : v);
    a.logp[t] = l;
    if (a.what == AFTER_POLICY) a.rows.set(row, policy_term(a.policy, t, l), l);
    else if (a.what == AFTER_GIVEN) a.rows.set(row, a.d_logp[t], l);
    return l;
}

// What follows for a row with the teacher's entries (one wave): KL of the token, scale = loss_scale / T sum p, rho = q - p / sum p
struct EntryRows {
    int k;
    const int *ids;                                                                // by token, as log_p, mass and kl
    const float *log_p, *mass, *z_sel;
    float it2, coef;
    float *kl, *scale, *rho;                                                       // kl null: no entries; scale, rho null: forward only
};
__device__ __forceinline__ void entries_after(const EntryRows &a, int t, int row, float base, float sum) {       // sum of 2^(x - base)
    const int lane = threadIdx.x & 63;
    const float l2 = __log2f(sum), mass = a.mass[t], inv_mass = 1.f / mass;
    float kl = 0.f;
    for (int j = lane; j < a.k; j += 64) {
        if (a.ids[(long)t * a.k + j] < 0) continue;
        const float lp = a.log_p[(long)t * a.k + j], p = expf(lp);
        const float zj = a.z_sel[(long)row * a.k + j], lq = kLn2 * (__builtin_fmaf(zj, a.it2, -base) - l2);
        if (!(p == 0.f)) kl += p * (lp - lq);
        if (a.rho) a.rho[(long)row * a.k + j] = expf(lq) - p * inv_mass;
    }
    kl = wave_sum(kl);
    if (lane == 0) {
        a.kl[t] = kl;
        if (a.scale) a.scale[row] = a.coef * mass;
    }
}

// ------------------------------------------------------------------ sums over the vocabulary, joined
// Behind the vocabulary: sum of the strips' sums at a common reference.  part holds (offset, sum) of each strip [strips][ld]: stored logits' offsets are logits
// (`unit` of x each), those of exponentials (`ref` given) count in x on top of the row's reference.  A row's strips are shared by 64 threads whatever the number
// of rows, so that a token's sum does not depend on its batch; a workgroup takes `rows_per` rows, up to 16 (128 bytes of neighbouring rows per strip).
// stat[row] = (sum, offset) and lse, by row, where asked for; then what follows.  HBM: 32768 rows x 2374 strips, 622 MB, 127 us (4.9 TB/s); 1000 rows x 500 5, of latency.
__global__ __launch_bounds__(1024) void head_combine_kernel(int ld, int rows, int rows_per, int strips, const float2 *__restrict__ part, float unit, const float2 *__restrict__ ref,
                                                            const int *__restrict__ token, const int *__restrict__ count, const float *__restrict__ z_sel, float it2,
                                                            float2 *__restrict__ stat, float *__restrict__ lse, After after, EntryRows en) {
    __shared__ float2 sm[1024];
    const int r = threadIdx.x & (rows_per - 1), g = threadIdx.x / rows_per;
    const int row = blockIdx.x * rows_per + r, n = count ? *count : rows;
    float m = -INFINITY, s = 0.f;
    auto merge = [&](float mi, float si) {
        const float to = fmaxf(m, mi), u = to == -INFINITY ? 0.f : to;
        s = s * __builtin_amdgcn_exp2f((m - u) * unit) + si * __builtin_amdgcn_exp2f((mi - u) * unit);
        m = to;
    };
    if (row < n) {
        const float2 *p = part + row;
        for (int i = g; i < strips; i += 64 * 8) {
            float2 q[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) q[e] = i + 64 * e < strips ? p[(long)(i + 64 * e) * ld] : make_float2(-INFINITY, 0.f);
#pragma unroll
            for (int e = 0; e < 8; ++e) merge(q[e].x, q[e].y);
        }
    }
    sm[threadIdx.x] = make_float2(m, s);
    for (int half = 32; half > 0; half >>= 1) {
        __syncthreads();
        if (g < half) {
            const float2 q = sm[threadIdx.x + half * rows_per];
            merge(q.x, q.y);
            sm[threadIdx.x] = make_float2(m, s);
        }
    }
    if (g == 0 && row < n) {
        if (stat) stat[row] = make_float2(s, m);
        if (lse) lse[row] = kLn2 * (m * unit + __log2f(s));
        if (after.what != AFTER_NOTHING)
            label_after(after, token[row], row, x_label(after, z_sel[row]) - (ref ? (double)ref[row].x + m : (double)m * after.inv_t * kLog2e64), s,
                        __builtin_amdgcn_exp2f(ref ? __builtin_fmaf(after.z_label[row], it2, -ref[row].x) - m : (after.z_label[row] - m) * it2));
    }
    if (!en.kl) return;
    __syncthreads();
    const int wave = threadIdx.x >> 6, mine = blockIdx.x * rows_per + wave;          // as many waves as rows
    if (mine < n) entries_after(en, token[mine], mine, ref[mine].x + sm[wave].x, sm[wave].y);
}

// One workgroup per pair: margin, loss, and the gradient of every token of its two sequences.  Sums in 64 bits: differences of
// some thousand logarithms each.
__global__ __launch_bounds__(256) void head_pairs_kernel(const int *__restrict__ cu, LabelRows rows, const float *__restrict__ ref_logp, float beta, float smoothing,
                                                         float loss_scale, const float *__restrict__ logp, float *__restrict__ margin, float *__restrict__ loss) {
    __shared__ double sm[4];
    __shared__ int any[4];
    const int pair = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int a = cu[2 * pair], b = cu[2 * pair + 1], c = cu[2 * pair + 2];
    double sum = 0.0;
    int seen = 0;
    for (int t = a + threadIdx.x; t < c; t += 256) {
        if (rows.slot[t] < 0) continue;
        const double diff = (double)logp[t] - (ref_logp ? (double)ref_logp[t] : 0.0);
        sum += t < b ? diff : -diff;
        seen = 1;
    }
    sum = wave_sum_f64(sum);
    const bool some = __any(seen);
    if (lane == 0) {
        sm[wave] = sum;
        any[wave] = some;
    }
    __syncthreads();
    const float m = (float)(sm[0] + sm[1] + sm[2] + sm[3]);
    const bool counts = any[0] | any[1] | any[2] | any[3];
    const float x = beta * m;
    // -ln s(x) = max(-x, 0) + ln(1 + e^-|x|)
    const float tail = log1pf(expf(-fabsf(x)));
    const float lose = fmaxf(-x, 0.f) + tail, win = fmaxf(x, 0.f) + tail;
    // s(x) - (1 - smoothing) = smoothing s(x) - (1 - smoothing) s(-x), each without cancellation
    const float e = expf(-fabsf(x)), big = 1.f / (1.f + e), small = e / (1.f + e);
    const float sp = x >= 0.f ? big : small, sn = x >= 0.f ? small : big;
    const float g = x == x ? loss_scale * beta * (smoothing * sp - (1.f - smoothing) * sn) : x;
    if (threadIdx.x == 0) {
        margin[pair] = counts ? m : 0.f;
        loss[pair] = !counts ? 0.f : x == x ? (1.f - smoothing) * lose + (smoothing > 0.f ? smoothing * win : 0.f) : x;
    }
    if (rows.scale)
        for (int t = a + threadIdx.x; t < c; t += 256) {
            const int row = rows.slot[t];
            if (row >= 0) rows.set(row, t < b ? g : -g, logp[t]);
        }
}

// One workgroup of 256: the loss from its terms, in an order that only their number fixes
struct LossTerms {
    const float *terms;
    int n;
    float scale;
    float *loss;                                                                   // null: not here
};
__device__ __forceinline__ void sum_loss(const LossTerms &a) {                      // by the first 256 threads; all of the workgroup come here
    __shared__ float sm[4];
    float acc = 0.f;
    if (threadIdx.x < 256)
        for (int i = threadIdx.x; i < a.n; i += 256 * 8) {
            float v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = i + u * 256 < a.n ? a.terms[i + u * 256] : 0.f;
#pragma unroll
            for (int u = 0; u < 8; ++u) acc += v[u];
        }
    acc = wave_sum(acc);
    if (threadIdx.x < 256 && (threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = acc;
    __syncthreads();
    if (threadIdx.x == 0) *a.loss = a.scale * (sm[0] + sm[1] + sm[2] + sm[3]);
}
__global__ __launch_bounds__(256) void head_loss_kernel(LossTerms a) { sum_loss(a); }
// fp32, whose d_h the product has written, zeros of dz times the lm_head for a token that is left out: NaN where the lm_head has NaN or an infinity, so those rows are set here, 16 to a workgroup.  Then the loss,
// if it is asked for (the last workgroup).  A launch of latency: 3.1 us at 293 tokens, as long as the loss by itself; calls of 293 .. 20000 tokens take as long as without it.
__global__ __launch_bounds__(256) void head_end_f32_kernel(const int *__restrict__ slot, int n, int d, float *__restrict__ d_h, LossTerms loss) {
    if (loss.loss && blockIdx.x == gridDim.x - 1) {
        sum_loss(loss);
        return;
    }
    const int row = blockIdx.x * 16 + (threadIdx.x >> 4);
    if (row >= n || slot[row] >= 0) return;
    for (int i = (threadIdx.x & 15) * 4; i < d; i += 64) *(float4 *)(d_h + (long)row * d + i) = make_float4(0.f, 0.f, 0.f, 0.f);
}

// ------------------------------------------------------------------ rows of stored logits
struct Entries {
    const float *log_p, *mass;
    float *kl, coef;                                                               // kl by token; dz = coef (q sum p - p)
};
// Where logits are stored, row t is token t, and a token that is left out has a row too: its hidden states may hold anything, and its logits are not looked at.
struct RowInputs {
    int d, limit;
    const int *labels;                                                             // null: the teacher's entries
    const void *h, *w;
    void *h_out;                                                                   // hidden states for d_w, zeros for a token that is left out; null: forward only
    int *slot, *token;
    float *out0, *out1;                                                            // zeroed for a token that is left out
};
// Everything of a row once its logits are stored: its teacher's entries in their order, a label's logit as a dot product of its own, the hidden states for d_w, the sum of exponentials, the
// log-probabilities of the selected ids, the loss's term, and, with `dz`, the gradient of the logits in their place (fp32).  G threads a row: a wave where a row is a few KB, a workgroup
// above.  Two or three passes over logits that the caches hold: 30000 rows of 1024 33 us (sums only, 123 MB), 20000 rows with entries and gradient 48 (164 MB read and written).  Hidden states and
// entries in a launch of their own before the product took 5.8 us of 293 tokens' 31 and 18 of 20000's 285; here they add 3 and 9.
template <int G, class T>
__global__ __launch_bounds__(256) void head_row_kernel(Slabs sl, int n, int k, float it2, RowInputs in, Teacher teacher, const int *sel, float *z, After after, Entries en, float2 *stat, float *scale,
                                                       float *rho, int dz) {
    __shared__ float sm[4], sh_scale;
    const int g = threadIdx.x & (G - 1), row = G == 64 ? blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x;
    bool counts;
    if (teacher.top_ids) {                                                          // (the first wave's work where a workgroup has one row)
        __shared__ int seen[4][kHeadMaxTop], sh_counts;
        const int wave = threadIdx.x >> 6;
        counts = teacher_entries(teacher, n, G == 64 || wave == 0 ? row : n, seen[wave]);
        if constexpr (G > 64) {
            if (threadIdx.x == 0) sh_counts = counts;
            __syncthreads();
            counts = sh_counts;
        } else {
            __threadfence_block();                                                  // entries go from lane to lane through memory
        }
    } else {
        const int at = row < n ? in.labels[row] : -1;
        counts = at >= 0 && at < in.limit;
    }
    if (row >= n) return;
    if (g == 0) {
        in.slot[row] = in.token[row] = counts ? row : -1;
        if (in.out0 && !counts) in.out0[row] = 0.f;
        if (in.out1 && !counts) in.out1[row] = 0.f;
    }
    auto join = [&](float v, auto f, auto across) __attribute__((always_inline)) {
        v = across(v);
        if constexpr (G > 64) {
            if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = v;
            __syncthreads();
            v = f(f(sm[0], sm[1]), f(sm[2], sm[3]));
            __syncthreads();
        }
        return v;
    };
    auto sum_of = [&](float v) { return join(v, [](float a, float b) { return a + b; }, [](float a) { return wave_sum(a); }); };
    auto max_of = [&](float v) { return join(v, [](float a, float b) { return fmaxf(a, b); }, [](float a) { return wave_max(a); }); };
    auto each = [&](auto f) __attribute__((always_inline)) {                        // the row, four columns at a time, the same ones whatever the slabs
        if (sl.cols >= sl.vocab) {
            float4 *zr = (float4 *)(z + (long)row * sl.cols);
            for (int i = g; i < sl.vocab >> 2; i += G) f(zr[i]);
        } else {
            for (int i = g; i < sl.vocab >> 2; i += G) f(*(float4 *)(z + sl.at(row, i * 4)));
        }
    };
    constexpr int N = Vec16<T>::N;
    const T *hr = (const T *)in.h + (long)row * in.d;
    float z_label = 0.f;
    if (in.h_out || (in.labels && counts)) {
        const T *wr = in.labels && counts ? (const T *)in.w + (long)in.labels[row] * in.d : nullptr;
        for (int i = g * N; i < in.d; i += G * N) {
            Vec16<T> a;
#pragma unroll
            for (int e = 0; e < N; ++e) a.v[e] = from_f32<T>(0.f);
            if (counts) a = ldv(hr + i);
            if (in.h_out) stv((T *)in.h_out + (long)row * in.d + i, a);
            if (wr) {
                const Vec16<T> b = ldv(wr + i);
#pragma unroll
                for (int e = 0; e < N; ++e) z_label = __builtin_fmaf(to_f32(a.v[e]), to_f32(b.v[e]), z_label);
            }
        }
        if (wr) z_label = sum_of(z_label);
    }
    const int t = row;
    if (!counts) {
        if (dz) each([](float4 &a) { a = make_float4(0.f, 0.f, 0.f, 0.f); });
        if (en.kl && g == 0) en.kl[row] = 0.f;
        return;
    }
    float m = -INFINITY, s = 0.f;
    each([&](float4 &a) { m = fmaxf(fmaxf(m, fmaxf(a.x, a.y)), fmaxf(a.z, a.w)); });
    m = max_of(m);
    const float u = m == -INFINITY ? 0.f : m;
    each([&](float4 &a) {
        s += __builtin_amdgcn_exp2f((a.x - u) * it2) + __builtin_amdgcn_exp2f((a.y - u) * it2) + __builtin_amdgcn_exp2f((a.z - u) * it2) + __builtin_amdgcn_exp2f((a.w - u) * it2);
    });
    s = sum_of(s);
    if (stat && g == 0) stat[row] = make_float2(s, m);
    float c = 0.f, r[2] = {0.f, 0.f};                                              // dz = c q, c r[] at the selected ids j = g, g + 64 (k <= 128)
    int id[2] = {-1, -1};
    if (after.what != AFTER_NOTHING) {
        if (g == 0) {
            id[0] = sel[t];
            const float l = label_after(after, t, row, x_label(after, z_label) - (double)m * after.inv_t * kLog2e64, s, __builtin_amdgcn_exp2f((z[sl.at(row, id[0])] - u) * it2));
            r[0] = expm1f(l);
            if (dz) c = after.rows.scale[row];
        }
        if (dz) {
            if constexpr (G == 64) c = __shfl(c, 0, 64);
            else {
                if (g == 0) sh_scale = c;
                __syncthreads();
                c = sh_scale;
            }
        }
    } else {
        const float l2 = __log2f(s), mass = en.mass[t], inv_mass = 1.f / mass;
        c = en.coef * mass;
        float kl = 0.f;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int j = g + 64 * x;
            if (g >= 64 || j >= k) continue;
            id[x] = sel[(long)t * k + j];
            if (id[x] < 0) continue;
            const float lp = en.log_p[(long)t * k + j], p = expf(lp), lq = kLn2 * ((z[sl.at(row, id[x])] - u) * it2 - l2);
            if (!(p == 0.f)) kl += p * (lp - lq);
            r[x] = expf(lq) - p * inv_mass;
            if (rho) rho[(long)row * k + j] = r[x];
        }
        kl = sum_of(kl);
        if (g == 0) {
            en.kl[t] = kl;
            if (scale) scale[row] = c;
        }
    }
    if (!dz) return;
    const float f = c == 0.f ? 0.f : c / s;
    if (c == 0.f) each([](float4 &a) { a = make_float4(0.f, 0.f, 0.f, 0.f); });
    else each([&](float4 &a) {
        a = make_float4(f * __builtin_amdgcn_exp2f((a.x - u) * it2), f * __builtin_amdgcn_exp2f((a.y - u) * it2), f * __builtin_amdgcn_exp2f((a.z - u) * it2), f * __builtin_amdgcn_exp2f((a.w - u) * it2));
    });
    if constexpr (G == 64) __threadfence_block(); else __syncthreads();             // the row's stores come before those at the selected ids
    if (c == 0.f) return;
#pragma unroll
    for (int x = 0; x < 2; ++x)
        if (id[x] >= 0) z[sl.at(row, id[x])] = c * r[x];
}

// ------------------------------------------------------------------ gradients
// Stored fp32 logits of a slab -> their gradient (in place for fp32), zeros in the columns cw .. cw_zero.  One workgroup per row.  A row without a token, or with scale 0, is zeros.
// bf16: the gradient rounded once, or, with `rest`, as the sum of two bf16 numbers (2^-16 of it is lost), each with a pair of products of its own.  1031 tokens of 33 entries, V = 32000, d = 1024: error of
// d_w 1.3e-3 from stored exponentials, 2.5e-6 so, 291 -> 589 us; 32768 tokens of 64 entries, V = 151936, d = 1536 37.8 -> 79.6 ms.
template <class T>
__global__ __launch_bounds__(256) void head_dz_kernel(int d_cols, int cw, int cw_zero, int v0, int k, const int *__restrict__ token, const int *__restrict__ sel, const float *z, float it2,
                                                      const float2 *__restrict__ stat, const float *__restrict__ scale, const float *__restrict__ rho, T *dz, T *rest) {
    const int row = blockIdx.x, t = token[row];
    const float *zr = z + (long)row * d_cols;
    T *o = dz + (long)row * d_cols, *more = rest ? rest + (long)row * d_cols : nullptr;
    auto put = [&](int i, float v) __attribute__((always_inline)) {
        o[i] = from_f32<T>(v);
        if (more) more[i] = from_f32<T>(v - to_f32(from_f32<T>(v)));
    };
    const float c = t < 0 ? 0.f : scale[row];                                   // (a row without a token has none)
    for (int i = (c == 0.f ? 0 : cw) + threadIdx.x; i < cw_zero; i += 256) put(i, 0.f);
    if (c == 0.f) return;
    const float2 st = stat[row];
    const float f = c / st.x;
    for (int i = threadIdx.x; i < cw; i += 256) put(i, f * __builtin_amdgcn_exp2f((zr[i] - st.y) * it2));
    __syncthreads();
    for (int j = threadIdx.x; j < k; j += 256) {
        const int v = sel[(long)t * k + j] - v0;
        if (v >= 0 && v < cw) put(v, c * rho[(long)row * k + j]);
    }
}

// Exponentials -> gradient of the logits over the row's factor c = scale / sum: the selected ids get theirs, c goes onto the hidden states (for d_w) and is kept (for d_h).  One
// workgroup per row.  Strips that are far above the row's reference (its label is 2^64 times less likely than another id) have offsets, which are evened out first.
//
// The exponentials are rounded to the storage type where they are stored, and c h here.  The selected ids with the largest gradients are most of the gradient's norm (a label's is the sum
// of all others'), so what those two roundings take from them is put back: rest = dz - c (stored e), which d_h adds times its row of w, and dz h - (stored e) (stored c h),
// a row that head_fix_kernel or the sorted sums of embedding_sorted.hip add to the id's row of d_w.  Error of d_w, rounded to bf16 by itself, against 64 bits: 2.9e-3 without, with
// 1.8e-3; the rounding alone is 1.7e-3.  (A caller who wants less of it asks for fp32's precision instead: MS_HEAD_FP32_DZ, head_dz_kernel.)  HBM: 32768 rows of 1536 with four rows to complete each, 0.6 GB, 140 us.
__global__ __launch_bounds__(256) void head_apply_kernel(Slabs sl, int d, int k, int strips, const float2 *__restrict__ part, const int *__restrict__ token, const int *__restrict__ count,
                                                         const int *__restrict__ sel, const float2 *__restrict__ stat, const float *__restrict__ scale, const float *__restrict__ rho,
                                                         bf16_t *__restrict__ e, bf16_t *__restrict__ h, float *__restrict__ factor, int fixes, int *__restrict__ fix_id,
                                                         float *__restrict__ fix_rest, bf16_t *__restrict__ fix) {
    __shared__ float s_dz[kHeadFixes], s_e[kHeadFixes];
    __shared__ int s_id[kHeadFixes];
    const int row = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (row >= *count) {
        if ((int)threadIdx.x < fixes) fix_id[(long)row * fixes + threadIdx.x] = -1;
        return;
    }
    const int t = token[row];
    const float2 st = stat[row];
    if (st.y != 0.f) {
        for (int i = wave; i < strips; i += 4) {
            const float off = part[(long)i * sl.rows + row].x;
            const int v = i * kStrip + lane;
            if (off == st.y || v >= sl.vocab) continue;
            bf16_t *at = e + sl.at(row, v);
            *at = (bf16_t)((float)*at * __builtin_amdgcn_exp2f(off - st.y));
        }
        __syncthreads();
    }
    const float sc = scale[row], c = sc == 0.f ? 0.f : sc / st.x;
    if (threadIdx.x == 0) factor[row] = c;
    if (wave == 0) {
        float r[2];
        int id[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int j = lane + 64 * x;
            id[x] = j < k ? sel[(long)t * k + j] : -1;
            r[x] = id[x] >= 0 ? rho[(long)row * k + j] : 0.f;
            if (id[x] >= 0) e[sl.at(row, id[x])] = (bf16_t)(r[x] * st.x);
        }
        float least = 0.f;                                                      // an eighth of the largest: the others are left as they are
        for (int f = 0; f < fixes; ++f) {
            float a0 = id[0] >= 0 ? fabsf(r[0]) : -1.f, a1 = id[1] >= 0 ? fabsf(r[1]) : -1.f;
            const float mine = fmaxf(a0, a1), best = wave_max(mine);
            if (f == 0) least = 0.125f * best;
            const unsigned long long who = __ballot(mine == best);
            const bool there = sc != 0.f && best > 0.f && best >= least && who;
            if (who && lane == __ffsll((long long)who) - 1) {
                const int x = a0 >= a1 ? 0 : 1;
                const float rx = x ? r[1] : r[0], held = (float)(bf16_t)(rx * st.x);
                const int at = there ? (x ? id[1] : id[0]) : -1;
                s_id[f] = at;
                s_dz[f] = sc * rx;
                s_e[f] = held;
                fix_id[(long)row * fixes + f] = at;
                fix_rest[(long)row * fixes + f] = __builtin_fmaf(-c, held, sc * rx);
                if (x) id[1] = -1; else id[0] = -1;
            } else if (!who && lane == 0) {
                s_id[f] = -1;
                fix_id[(long)row * fixes + f] = -1;
            }
        }
    }
    __syncthreads();
    for (int i = threadIdx.x * 8; i < d; i += 256 * 8) {
        const Vec16<bf16_t> a = ldv(h + (long)row * d + i);
        Vec16<bf16_t> b;
#pragma unroll
        for (int x = 0; x < 8; ++x) b.v[x] = (bf16_t)(c == 0.f ? 0.f : c * (float)a.v[x]);
        stv(h + (long)row * d + i, b);
        for (int f = 0; f < fixes; ++f) {
            if (s_id[f] < 0) continue;
            Vec16<bf16_t> o;
#pragma unroll
            for (int x = 0; x < 8; ++x) o.v[x] = (bf16_t)__builtin_fmaf(s_dz[f], (float)a.v[x], -s_e[f] * (float)b.v[x]);
            stv(fix + ((long)row * fixes + f) * d + i, o);
        }
    }
}

// d_w[id] += the rows of `fix` with that id, in their order; n <= kHeadScan of them.  A workgroup takes eight rows and 512 columns: each of its waves looks for the others of one
// row's id in a copy of the ids in LDS, and the first row of an id sums them all, by itself or, where there are many, with all eight waves (an eighth of the rows each).
// (A workgroup per row that reads the ids itself: 18 us for 2053 rows of 1024, 41 for 4124; waves by themselves 38 and 26; now 14 and 22.)
constexpr int kFixWaves = 8, kFixMany = 8, kFixList = 256;
struct FixLds {
    __align__(16) int ids[kHeadScan];
    unsigned short found[kFixWaves][kFixList];
    float join[(kFixWaves - 1) * 512];
    int many[kFixWaves];
};
__device__ __forceinline__ void fix_rows(FixLds &lds, int block, int block_col, int n, int d, const int *__restrict__ id, const bf16_t *__restrict__ fix, float *__restrict__ d_w) {
    constexpr int kMany = kFixMany, kList = kFixList;
    auto &ids = lds.ids;
    auto &found = lds.found;
    auto &join = lds.join;
    auto &many = lds.many;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, chunks = (n + 255) >> 8;
    for (int j0 = tid; j0 < chunks * 256; j0 += 8 * 64 * kFixWaves) {
        int q[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) q[u] = j0 + u * 64 * kFixWaves < n ? id[j0 + u * 64 * kFixWaves] : -1;
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (j0 + u * 64 * kFixWaves < chunks * 256) ids[j0 + u * 64 * kFixWaves] = q[u];
    }
    __syncthreads();
    auto wave_sync = []() __attribute__((always_inline)) {                       // the lanes of a wave exchange places through `found`
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    };
    const int i = block * kFixWaves + wave, mine = i < n ? ids[i] : -1, col = block_col * 512 + lane * 8;
    float acc[8] = {};
    auto sum = [&](const unsigned short *list, int from, int to) __attribute__((always_inline)) {
        if (col < d)
            for (int j = from; j < to; j += 8) {
                Vec16<bf16_t> a[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) a[u] = ldv(fix + (long)list[j + u < to ? j + u : to - 1] * d + col);
#pragma unroll
                for (int u = 0; u < 8; ++u)
                    if (j + u < to)
#pragma unroll
                        for (int x = 0; x < 8; ++x) acc[x] += (float)a[u].v[x];
            }
    };
    auto put = [&](int row) __attribute__((always_inline)) {
        if (col >= d) return;
        float4 *o = (float4 *)(d_w + (long)row * d + col), x = o[0], y = o[1];
        o[0] = make_float4(x.x + acc[0], x.y + acc[1], x.z + acc[2], x.w + acc[3]);
        o[1] = make_float4(y.x + acc[4], y.y + acc[5], y.z + acc[6], y.w + acc[7]);
    };
    // the lanes' four ids of a chunk that are this row's
    auto same = [&](int c) __attribute__((always_inline)) {
        const int4 q = *(const int4 *)(ids + c * 256 + lane * 4);
        return (unsigned)(q.x == mine) | (unsigned)(q.y == mine) << 1 | (unsigned)(q.z == mine) << 2 | (unsigned)(q.w == mine) << 3;
    };
    bool first = mine >= 0;
    int total = 0;
    if (first) {
        int before = 0;
        for (int c = 0; c < chunks; ++c) {
            const unsigned m = same(c);
            const int j = c * 256 + lane * 4;
            total += __popc(m);
            if (j < i) before |= j + 4 <= i ? m : m & ((1u << (i - j)) - 1);
        }
        first = !__any(before);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) total += __shfl_xor(total, o, 64);
    }
    const bool shared = first && total > kMany && total <= kList;
    if (lane == 0) many[wave] = shared ? total : 0;
    if (first) {
        int have = 0;
        for (int c = i >> 8; c < chunks; ++c) {
            const unsigned m = same(c);
            if (!__any(m)) continue;
            int upto = __popc(m);
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int v = __shfl_up(upto, o, 64);
                if (lane >= o) upto += v;
            }
            int at = have + upto - __popc(m);
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (m >> u & 1) found[wave][at++] = (unsigned short)(c * 256 + lane * 4 + u);
            have += __shfl(upto, 63, 64);
            if (!shared && have >= kList - 256) {                                // (more than the list holds: it is emptied in between)
                wave_sync();
                sum(found[wave], 0, have);
                wave_sync();
                have = 0;
            }
        }
        if (!shared) {
            wave_sync();
            sum(found[wave], 0, have);
            put(mine);
        }
    }
    __syncthreads();
    for (int e = 0; e < kFixWaves; ++e) {
        const int rows = many[e];
        if (!rows) continue;                                                     // (the same in all waves)
        const int per = (rows + kFixWaves - 1) / kFixWaves, from = wave * per, to = from + per < rows ? from + per : rows;
#pragma unroll
        for (int x = 0; x < 8; ++x) acc[x] = 0.f;
        sum(found[e], from, to);
        if (wave)
#pragma unroll
            for (int x = 0; x < 8; ++x) join[(wave - 1) * 512 + x * 64 + lane] = acc[x];
        __syncthreads();
        if (wave == 0) {
#pragma unroll
            for (int x = 0; x < 8; ++x)
                for (int w = 0; w < kFixWaves - 1; ++w) acc[x] += join[w * 512 + x * 64 + lane];
            put(ids[block * kFixWaves + e]);
        }
        __syncthreads();
    }
}

// d_h of the block's tokens: a row's sums (in `parts` parts) times its factor, and what the selected ids' lack; zeros for tokens that were left out
struct RowSums {
    const float *sums, *factor;                                                    // [parts][part_ld], [rows] (null: 1)
    int parts;
    long part_ld;
    int fixes;
    const int *fix_id;
    const float *fix_rest;
    const bf16_t *w;
    const int *slot;
};
__device__ __forceinline__ void row_gradient(const RowSums &a, long i, int d, bf16_t *d_h) {       // four columns from i on
    const int t = (int)(i / d), c = (int)(i - (long)t * d), row = a.slot[t];
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    const float f = row < 0 ? 0.f : a.factor ? a.factor[row] : 1.f;
    if (row >= 0 && f != 0.f) {
        for (int q0 = 0; q0 < a.parts; q0 += 8) {
            float4 x[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) x[q] = q0 + q < a.parts ? *(const float4 *)(a.sums + (q0 + q) * a.part_ld + (long)row * d + c) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int q = 0; q < 8; ++q) { v.x += x[q].x; v.y += x[q].y; v.z += x[q].z; v.w += x[q].w; }
        }
        v.x *= f; v.y *= f; v.z *= f; v.w *= f;
        for (int q = 0; q < a.fixes; ++q) {
            const int id = a.fix_id[(long)row * a.fixes + q];
            if (id < 0) continue;
            const float rest = a.fix_rest[(long)row * a.fixes + q];
            const bf16_t *x = a.w + (long)id * d + c;
            v.x = __builtin_fmaf(rest, (float)x[0], v.x);
            v.y = __builtin_fmaf(rest, (float)x[1], v.y);
            v.z = __builtin_fmaf(rest, (float)x[2], v.z);
            v.w = __builtin_fmaf(rest, (float)x[3], v.w);
        }
    }
    bf16_t *o = d_h + i;
    o[0] = (bf16_t)v.x; o[1] = (bf16_t)v.y; o[2] = (bf16_t)v.z; o[3] = (bf16_t)v.w;
}

// What is left behind the gradients' products, in one launch: rows of d_w to complete (fix_blocks workgroups, fix_cols of them for each eight rows; FIX: there are some), d_h, and the
// loss (the last workgroup).  Apart they took 15, 12 and 5 us at 2053 tokens of 1024, each of them latency; now 17.  d_h of 32768 tokens of 1536 with four rows of w for each: 0.7 GB, 215 us.
template <bool FIX>
__global__ __launch_bounds__(64 * kFixWaves) void head_end_kernel(int fix_blocks, int fix_cols, int n_fix, const int *__restrict__ fix_id, const bf16_t *__restrict__ fix, float *__restrict__ d_w, RowSums rows,
                                                                  long total, int d, bf16_t *d_h, LossTerms loss) {
    int b = blockIdx.x;
    if constexpr (FIX) {
        __shared__ FixLds lds;
        if (b < fix_blocks) {
            fix_rows(lds, b / fix_cols, b % fix_cols, n_fix, d, fix_id, fix, d_w);
            return;
        }
        b -= fix_blocks;
    }
    if (loss.loss && blockIdx.x == gridDim.x - 1) {
        sum_loss(loss);
        return;
    }
    const long i = ((long)b * 64 * kFixWaves + threadIdx.x) * 4;
    if (i < total) row_gradient(rows, i, d, d_h);
}

// ------------------------------------------------------------------ top logits
// Order of values: larger first, equal ones by their place.  A NaN counts as larger than all.
__device__ __forceinline__ unsigned ordered(float v) {
    const unsigned u = __float_as_uint(v == v ? v + 0.f : INFINITY);                 // (+ 0: one zero)
    return v == v ? (u & 0x80000000u ? ~u : u | 0x80000000u) : 0xffffffffu;
}
__device__ __forceinline__ float entry_value(unsigned long long key) {
    const unsigned u = (unsigned)(key >> 32);
    return u == 0xffffffffu ? NAN : __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}

// sorts n (a power of two) keys in LDS, largest first
__device__ __forceinline__ void sort_keys(unsigned long long *key, int n) {
    for (int size = 2; size <= n; size <<= 1)
        for (int step = size >> 1; step > 0; step >>= 1) {
            __syncthreads();
            for (int i = threadIdx.x; i < n >> 1; i += blockDim.x) {
                const int lo = 2 * i - (i & (step - 1)), hi = lo + step;
                const unsigned long long a = key[lo], b = key[hi];
                if (((lo & size) == 0) == (a < b)) {
                    key[lo] = b;
                    key[hi] = a;
                }
            }
        }
    __syncthreads();
}

// The k largest logits of a row, one workgroup each.  They lie in the k strips with the largest maxima (equal ones by their place): an entry of another
// strip has k maxima before it.  So: those strips, by the bits of the k-th largest maximum (four passes over a histogram of eight bits each); their entries
// that are not below that maximum, which are few more than k; those sorted.  One row of 151936, 64 entries: 21 us, a chain of some 30 barriers; 4096 rows 164, the same chain with four rows
// a CU (78 MB of maxima and 70 MB of strips are read).
constexpr int kTopKeys = 2048;                      // candidates that are sorted in LDS
constexpr int kTopThreads = 512, kTopHeld = 8;      // strips of a thread whose maxima it keeps in registers (V up to 262144); more are read again in each pass
__global__ __launch_bounds__(kTopThreads) void head_top_kernel(Slabs sl, int rows, int strips, int k, const float *__restrict__ z, const float2 *__restrict__ part, float it2,
                                                               float *__restrict__ lse, float *__restrict__ values, int *__restrict__ ids) {
    __shared__ unsigned hist[kTopThreads / 64][256], sh_prefix;                     // one for each wave: maxima share their leading bits
    __shared__ int sh_want, n_strips, n_keys, wsum[kTopThreads / 64];
    __shared__ int list[kHeadMaxTop];
    __shared__ unsigned long long keys[kTopKeys];
    // neighbouring rows, whose maxima share cache lines, go to one XCD (workgroups go to the eight in turn)
    const int each = (rows + 7) >> 3, row = (blockIdx.x & 7) * each + (blockIdx.x >> 3);
    if (row >= rows) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // of n values ordered(value(i)): the `want`-th largest (its bits) and how many of those equal to it belong to the `want` largest
    auto nth = [&](int n, int want, auto value, unsigned *bits, int *equal) __attribute__((always_inline)) {
        unsigned prefix = 0;
        int left = want;
        for (int shift = 24; shift >= 0; shift -= 8) {
            for (int i = tid; i < (kTopThreads / 64) * 256; i += kTopThreads) (&hist[0][0])[i] = 0;
            __syncthreads();
            for (int i = tid; i < n; i += kTopThreads) {
                const unsigned o = value(i);
                if (shift == 24 || (o >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[wave][(o >> shift) & 255], 1u);
            }
            __syncthreads();
            if (wave == 0) {                                                         // from the top bin down: where the count passes `left`
                unsigned h[4], mine = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    h[e] = 0;
                    for (int w = 0; w < kTopThreads / 64; ++w) h[e] += hist[w][255 - (lane * 4 + e)];
                    mine += h[e];
                }
                unsigned upto = mine;
#pragma unroll
                for (int o = 1; o < 64; o <<= 1) {
                    const unsigned v = __shfl_up(upto, o, 64);
                    if (lane >= o) upto += v;
                }
                unsigned before = upto - mine;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (before < (unsigned)left && before + h[e] >= (unsigned)left) {
                        sh_prefix = prefix | (unsigned)(255 - (lane * 4 + e)) << shift;
                        sh_want = left - (int)before;
                    }
                    before += h[e];
                }
            }
            __syncthreads();
            prefix = sh_prefix;
            left = sh_want;
        }
        *bits = prefix;
        *equal = left;
        __syncthreads();
    };
    if (tid == 0) n_strips = n_keys = 0;
    __syncthreads();
    unsigned floor_ = 0;
    const bool all = !part || k >= strips;
    if (!part) {                                                                    // a small vocabulary: the sum too
        __shared__ float sm[kTopThreads / 64];
        float m = -INFINITY, s = 0.f;
        for (int v = tid; v < sl.vocab; v += kTopThreads) m = fmaxf(m, z[sl.at(row, v)]);
        m = wave_max(m);
        if (lane == 0) sm[wave] = m;
        __syncthreads();
        for (int w = 0; w < kTopThreads / 64; ++w) m = fmaxf(m, sm[w]);
        __syncthreads();
        const float u = m == -INFINITY ? 0.f : m;
        for (int v = tid; v < sl.vocab; v += kTopThreads) s += __builtin_amdgcn_exp2f((z[sl.at(row, v)] - u) * it2);
        s = wave_sum(s);
        if (lane == 0) sm[wave] = s;
        __syncthreads();
        s = 0.f;
        for (int w = 0; w < kTopThreads / 64; ++w) s += sm[w];
        if (tid == 0) lse[row] = kLn2 * (m * it2 + __log2f(s));
    }
    if (!all) {
        // strips above the k-th largest maximum, and the first of those equal to it
        int left;
        const bool held = strips <= kTopThreads * kTopHeld;
        unsigned mine[kTopHeld];
#pragma unroll
        for (int u = 0; u < kTopHeld; ++u) {
            const int i = tid + u * kTopThreads;
            mine[u] = held && i < strips ? ordered(part[(long)i * sl.rows + row].x) : 0;
        }
        auto maximum = [&](int i) {
            if (!held) return ordered(part[(long)i * sl.rows + row].x);
            const int at = i / kTopThreads;
            unsigned o = mine[0];
#pragma unroll
            for (int u = 1; u < kTopHeld; ++u) o = at == u ? mine[u] : o;
            return o;
        };
        nth(strips, k, maximum, &floor_, &left);
        int equal = 0;
        for (int i0 = 0; i0 < strips; i0 += kTopThreads) {
            const int i = i0 + tid;
            const unsigned o = i < strips ? maximum(i) : 0;
            const bool is = i < strips && o == floor_;
            const unsigned long long mask = __ballot(is);
            if (lane == 0) wsum[wave] = __popcll(mask);
            __syncthreads();
            int place = equal + __popcll(mask & ((1ull << lane) - 1));
            for (int w = 0; w < kTopThreads / 64; ++w) {
                if (w < wave) place += wsum[w];
                equal += wsum[w];
            }
            if (i < strips && (o > floor_ || (is && place < left))) {
                const int at = atomicAdd(&n_strips, 1);
                if (at < kHeadMaxTop) list[at] = i;
            }
            __syncthreads();
        }
    }
    // their entries
    const int strips_here = all ? strips : n_strips < k ? n_strips : k;
    auto entry = [&](int i, int *v) {                                                // i: place among the strips' columns; 0: outside the vocabulary
        *v = (all ? i >> 6 : list[i >> 6]) * kStrip + (i & 63);
        return *v < sl.vocab ? ordered(z[sl.at(row, *v)]) : 0u;
    };
    auto collect = [&](auto wanted) __attribute__((always_inline)) {
        for (int i0 = tid; i0 < strips_here * kStrip; i0 += 8 * kTopThreads) {
            unsigned o[8];
            int v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                v[u] = sl.vocab;
                o[u] = i0 + u * kTopThreads < strips_here * kStrip ? entry(i0 + u * kTopThreads, &v[u]) : 0u;
            }
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const bool in = v[u] < sl.vocab && wanted(o[u], v[u]);
                const unsigned long long mask = __ballot(in);
                if (!mask) continue;
                int base = 0;
                if (lane == 0) base = atomicAdd(&n_keys, __popcll(mask));
                base = __shfl(base, 0, 64) + __popcll(mask & ((1ull << lane) - 1));
                if (in && base < kTopKeys) keys[base] = (unsigned long long)o[u] << 32 | (0xffffffffu - (unsigned)v[u]);
            }
        }
        __syncthreads();
    };
    collect([&](unsigned o, int) { return o >= floor_; });
    int have = n_keys;
    if (have > kTopKeys) {                                                           // equal or nearly equal values: the k-th largest itself, and of those equal to it the first
        unsigned bits, place;
        int equal, last;
        auto value = [&](int i) { int v; return entry(i, &v); };
        __syncthreads();
        nth(strips_here * kStrip, k, value, &bits, &equal);
        nth(strips_here * kStrip, equal, [&](int i) { int v; const unsigned o = entry(i, &v); return o == bits && v < sl.vocab ? 0xffffffffu - (unsigned)v : 0u; }, &place, &last);
        if (tid == 0) n_keys = 0;
        __syncthreads();
        collect([&](unsigned o, int v) { return o > bits || (o == bits && 0xffffffffu - (unsigned)v >= place); });
        have = n_keys < kTopKeys ? n_keys : kTopKeys;
    }
    // many more than k (a small vocabulary): those above the k-th largest value, and those equal to it, to the front
    if (have > 4 * k && have > 128) {
        unsigned bits;
        int equal;
        nth(have, k, [&](int i) { return (unsigned)(keys[i] >> 32); }, &bits, &equal);
        if (tid == 0) n_keys = 0;
        for (int i0 = 0; i0 < have; i0 += kTopThreads) {                             // (what moves goes to a place that has been read)
            const unsigned long long key = i0 + tid < have ? keys[i0 + tid] : 0;
            __syncthreads();
            if (i0 + tid < have && (unsigned)(key >> 32) >= bits) keys[atomicAdd(&n_keys, 1)] = key;
            __syncthreads();
        }
        have = n_keys;
    }
    __syncthreads();
    auto put = [&](int i, unsigned long long key) {
        values[(long)row * k + i] = entry_value(key);
        ids[(long)row * k + i] = (int)(0xffffffffu - (unsigned)key);
    };
    if (have <= kTopThreads) {                                                       // each key to its rank (they all differ): no barriers (sorted step by step, 128 keys: 7 us more)
        if (tid < have) {
            const unsigned long long key = keys[tid];
            int rank = 0;
            for (int i = 0; i < have; ++i) rank += keys[i] > key;
            if (rank < k) put(rank, key);
        }
    } else {
        int n = 2;
        while (n < have) n <<= 1;
        for (int i = have + tid; i < n; i += kTopThreads) keys[i] = 0;
        sort_keys(keys, n);
        for (int i = tid; i < k; i += kTopThreads) put(i, keys[i]);                   // (have > k)
    }
    for (int i = have + tid; i < k; i += kTopThreads) {
        values[(long)row * k + i] = -INFINITY;
        ids[(long)row * k + i] = -1;
    }
}

// ------------------------------------------------------------------ sequencing
// Logits of `rows` rows h: stored (fp32), or their exponentials at p.ref (fast losses; not stored in a forward pass); the fast products leave the sums of their strips too
HeadMarks marks_of(const HeadPlan &p, int v0, int k) {
    if (!p.marks) return {};
    const size_t at = (size_t)(v0 / kStrip) * p.rows;
    return {p.marks + at, p.marks_first + at, p.z_sel, k};
}
ms_status logits(const ms_head_config *c, const HeadPlan &p, HeadUse use, int k, int rows, const void *h, hipStream_t s) {
    const int V = c->vocab, d = c->hidden;
    const size_t es = ms_dtype_size(head_dtype(c));
    const float it2 = kLog2e / c->temperature;
    for (int i = 0; i < p.slabs; ++i) {
        const int v0 = i * p.cols, cw = V - v0 < p.cols ? V - v0 : p.cols;
        const char *w = (const char *)c->w_dev + (size_t)v0 * d * es;
        const size_t slab = (size_t)i * p.rows * p.cols;
        float2 *part = p.part + (size_t)(v0 / kStrip) * p.rows;
        if (head_dtype(c) == MS_F32 && head_f32_logits_tiled(rows, V)) MS_TRY(head_f32_logits(rows, cw, d, (const float *)h, (const float *)w, (float *)p.z + slab, p.cols, s));
        else if (!p.fast) MS_TRY(ms_k_gemm(head_dtype(c), 0, 0, rows, cw, d, 1.f, h, d, w, d, (float *)p.z + slab, p.cols, 1, 0, nullptr, nullptr, 0, 0, 1, s));
        else if (use == HEAD_TOP) MS_TRY(head_gemm_logits(rows, cw, d, h, w, it2, (float *)p.z + slab, p.cols, part, p.rows, s));
        else MS_TRY(head_gemm_exp(rows, cw, d, h, w, p.ref, v0, p.z_label, marks_of(p, v0, k), it2, use == HEAD_BACKWARD ? (bf16_t *)p.z + slab : nullptr, p.cols, part, p.rows, p.count, s));
    }
    return MS_OK;
}

ms_status combine(const HeadPlan &p, int rows, float unit, const float2 *ref, float it2, float2 *stat, float *lse, const After &after, const EntryRows &en, const int *count, hipStream_t s) {
    int per = 1;
    while (per < 16 && per < rows) per <<= 1;
    ProfScope ps(9, 8.0 * rows * p.strips, s);
    head_combine_kernel<<<ms_cdiv(rows, per), per * 64, 0, s>>>(p.rows, rows, per, p.strips, p.part, unit, ref, p.token, count, p.z_sel, it2, stat, lse, after, en);
    MS_LAUNCH_CHECK();
    return MS_OK;
}

// What the losses have in common, for the tokens t0 .. t0 + n of a call
struct HeadCall {
    const ms_head_config *c;
    HeadPlan p;
    HeadUse use;
    int k;                               // selected ids of a row
    const void *h;
    void *d_h, *d_w;
    hipStream_t s;
};

// Rows, their logits, sums over the vocabulary, and what follows.  key / sel: per token of the block (labels, or the entries' keys and ids); out0, out1: zeroed for the
// tokens that are left out.  Labels: after; the teacher's entries: teacher, en.  *dz_done: the gradient of stored logits is in their place already.
ms_status rows_forward(const HeadCall &a, int t0, int n, const int *key, int limit, const int *sel, float *out0, float *out1, const After &after, const Teacher &teacher, const Entries &en, bool dz_here,
                       bool *dz_done) {
    const ms_head_config *c = a.c;
    const HeadPlan &p = a.p;
    const int d = c->hidden, V = c->vocab;
    const float it2 = kLog2e / c->temperature;
    const char *h = (const char *)a.h + (size_t)t0 * d * ms_dtype_size(head_dtype(c));
    const bool labels = after.what != AFTER_NOTHING;
    if (!p.fast) {
        MS_TRY(logits(c, p, a.use, a.k, n, h, a.s));
        *dz_done = dz_here && head_dtype(c) == MS_F32 && a.use == HEAD_BACKWARD;
        const Slabs sl = {p.rows, p.cols, V};
        float *scale = a.use == HEAD_BACKWARD ? p.scale : nullptr, *rho = a.use == HEAD_BACKWARD ? p.rho : nullptr;
        ProfScope ps(9, 4.0 * n * V * (*dz_done ? 2 : 1), a.s);
        const RowInputs in = {d, limit, labels ? sel : nullptr, h, c->w_dev, a.use == HEAD_BACKWARD ? p.h : nullptr, p.slot, p.token, out0, out1};
#define GO(G, T, rows) head_row_kernel<G, T><<<rows, 256, 0, a.s>>>(sl, n, a.k, it2, in, teacher, sel, (float *)p.z, after, en, p.stat, scale, rho, *dz_done)
        if (head_dtype(c) == MS_F32) {
            if (V <= 4096) GO(64, float, ms_cdiv(n, 4)); else GO(256, float, n);
        } else {
            if (V <= 4096) GO(64, bf16_t, ms_cdiv(n, 4)); else GO(256, bf16_t, n);
        }
#undef GO
        MS_LAUNCH_CHECK();
        return MS_OK;
    }
    if (teacher.top_ids) {
        const long clear = p.marks ? (long)p.rows * p.strips / 2 : 0, most = clear / 1024 < 2048 ? clear / 1024 : 2048;      // (rows are a multiple of 16)
        head_entries_kernel<<<(unsigned)(most > ms_cdiv(n, 4) ? most : ms_cdiv(n, 4)), 256, 0, a.s>>>(n, teacher, (float4 *)p.marks, clear);
        MS_LAUNCH_CHECK();
    }
    const bool one = p.marks || a.k == 1, find = one && n <= kHeadFind;
    if (!find) {
        ProfScope ps(11, 0, a.s);
        head_rows_kernel<<<1, 1024, 0, a.s>>>(n, key, limit, p.slot, p.token, p.count, out0, out1);
        MS_LAUNCH_CHECK();
    }
    {
        ProfScope ps(9, 0, a.s);
        const bf16_t *hb = (const bf16_t *)h, *wb = (const bf16_t *)c->w_dev;
        const int *id = p.marks ? p.best : sel;
        float *z = p.marks ? nullptr : p.z_sel;
        const MarkWords marks = {a.k, p.rows, p.ids, p.marks, p.marks_first};
        if (find) head_pick_one_kernel<true><<<ms_cdiv(n, 4), 256, 0, a.s>>>(n, d, hb, wb, key, limit, p.slot, p.token, p.count, out0, out1, id, it2, (bf16_t *)p.h, z, p.ref, marks);
        else if (one) head_pick_one_kernel<false><<<ms_cdiv(n, 4), 256, 0, a.s>>>(n, d, hb, wb, key, limit, p.slot, p.token, p.count, out0, out1, id, it2, (bf16_t *)p.h, z, p.ref, marks);
        else if (a.k > 4) head_pick_kernel<4><<<n, 256, 0, a.s>>>(d, a.k, hb, wb, p.token, p.count, sel, it2, (bf16_t *)p.h, p.z_sel, p.ref);
        else head_pick_kernel<1><<<n, 64, 0, a.s>>>(d, a.k, hb, wb, p.token, p.count, sel, it2, (bf16_t *)p.h, p.z_sel, p.ref);
    }
    MS_LAUNCH_CHECK();
    MS_TRY(logits(c, p, a.use, a.k, n, p.h, a.s));
    const bool back = a.use == HEAD_BACKWARD;
    const EntryRows entries = {a.k, p.ids, p.log_p, p.mass, p.z_sel, it2, en.coef, en.kl, back ? p.scale : nullptr, back ? p.rho : nullptr};
    return combine(p, n, 1.f, p.ref, it2, p.stat, nullptr, after, labels ? EntryRows{} : entries, p.count, a.s);
}

ms_status total_loss(const LossTerms &a, hipStream_t s) {
    head_loss_kernel<<<1, 256, 0, s>>>(a);
    MS_LAUNCH_CHECK();
    return MS_OK;
}

// scale and rho are there: gradients of the block's hidden states and of the lm_head; then the loss, if it is asked for here
ms_status rows_backward(const HeadCall &a, int t0, int n, const int *sel, bool dz_done, const LossTerms &loss) {
    const ms_head_config *c = a.c;
    const HeadPlan &p = a.p;
    const int d = c->hidden, V = c->vocab, dt = head_dtype(c);
    const size_t es = ms_dtype_size(dt);
    const float it2 = kLog2e / c->temperature;
    if (p.fast) {
        const Slabs sl = {p.rows, p.cols, V};
        ProfScope ps(10, 4.0 * n * d, a.s);
        head_apply_kernel<<<n, 256, 0, a.s>>>(sl, d, a.k, p.strips, p.part, p.token, p.count, sel, p.stat, p.scale, p.rho, (bf16_t *)p.z, (bf16_t *)p.h, p.factor, p.fixes, p.fix_id, p.fix_rest,
                                              (bf16_t *)p.fix);
    }
    MS_LAUNCH_CHECK();
    for (int i = 0; i < p.slabs; ++i) {
        const int v0 = i * p.cols, cw = V - v0 < p.cols ? V - v0 : p.cols;
        const char *w = (const char *)c->w_dev + (size_t)v0 * d * es;
        if (p.fast) {
            MS_TRY(head_gemm_backward(p.choice, n, cw, d, (const bf16_t *)p.z + (size_t)i * p.rows * p.cols, p.cols, w, p.h, a.d_h ? p.d_h : nullptr, i > 0,
                                      a.d_w ? (float *)a.d_w + (size_t)v0 * d : nullptr, p.count, a.s));
            continue;
        }
        float *z = (float *)p.z + (size_t)i * p.rows * p.cols, *d_w = a.d_w ? (float *)a.d_w + (size_t)v0 * d : nullptr;
        void *dz = dt == MS_F32 ? (void *)z : p.dz;
        if (!dz_done) {
            ProfScope ps(10, (4.0 + es) * n * cw, a.s);
            if (dt == MS_F32) head_dz_kernel<float><<<n, 256, 0, a.s>>>(p.cols, cw, cw, v0, a.k, p.token, sel, z, it2, p.stat, p.scale, p.rho, (float *)dz, (float *)nullptr);
            else head_dz_kernel<bf16_t><<<n, 256, 0, a.s>>>(p.cols, cw, p.tiles ? (cw + 63) / 64 * 64 : cw, v0, a.k, p.token, sel, z, it2, p.stat, p.scale, p.rho, (bf16_t *)dz, (bf16_t *)p.dz_rest);
        }
        MS_LAUNCH_CHECK();
        // (in fp32 the sums are the result: zeros for the tokens that are left out, whose rows of dz are)
        float *sums = dt == MS_F32 ? (float *)a.d_h + (size_t)t0 * d : p.d_h;
        if (p.tiles) {
            MS_TRY(head_gemm_backward(p.choice, n, cw, d, dz, p.cols, w, p.h, a.d_h ? p.d_h : nullptr, i > 0, d_w, nullptr, a.s));
            if (p.dz_rest) MS_TRY(head_gemm_backward(p.choice, n, cw, d, p.dz_rest, p.cols, w, p.h, a.d_h ? p.d_h : nullptr, 1, d_w, nullptr, a.s));
            continue;
        }
        if (dt == MS_F32 && a.d_h && a.d_w) {
            MS_TRY(ms_k_linear_backward(dt, n, cw, d, dz, p.cols, w, p.h, sums, 1, i > 0, d_w, a.s));
            continue;
        }
        // (K in one piece: bf16 pieces would be added up by atomics, in any order)
        for (const void *e : {(const void *)dz, (const void *)p.dz_rest}) {
            if (!e) continue;
            if (a.d_h) MS_TRY(ms_k_gemm(dt, 0, 1, n, d, cw, 1.f, e, p.cols, w, d, sums, d, 1, i > 0 || e != dz, nullptr, nullptr, 0, 0, 1, a.s));
            if (a.d_w) MS_TRY(ms_k_gemm(dt, 1, 1, cw, d, n, 1.f, e, p.cols, p.h, d, d_w, d, 1, 1, nullptr, nullptr, 0, 0, 1, a.s));
        }
    }
    if (dt == MS_F32) {
        if (!a.d_h) return loss.loss ? total_loss(loss, a.s) : MS_OK;
        head_end_f32_kernel<<<ms_cdiv(n, 16) + (loss.loss != nullptr), 256, 0, a.s>>>(p.slot, n, d, (float *)a.d_h + (size_t)t0 * d, loss);
        MS_LAUNCH_CHECK();
        return MS_OK;
    }
    const int n_fix = p.fast && a.d_w ? n * p.fixes : 0;
    if (n_fix > kHeadScan) MS_TRY(ms_k_embedding_sorted_backward(dt, n_fix, d, V, 1.f, p.fix_id, p.fix, (float *)a.d_w, p.fix_scratch, p.fix_scratch_bytes, a.s));
    const bool fix_here = n_fix > 0 && n_fix <= kHeadScan;
    const int fix_cols = ms_cdiv(d, 512), fix_blocks = fix_here ? ms_cdiv(n_fix, kFixWaves) * fix_cols : 0;
    const long total = a.d_h ? (long)n * d : 0, blocks = fix_blocks + ms_cdiv(total, 256 * kFixWaves) + (loss.loss != nullptr);
    if (blocks == 0) return MS_OK;
    const RowSums rows = {p.d_h, p.fast ? p.factor : nullptr, p.parts, (long)n * d, p.fast ? p.fixes : 0, p.fix_id, p.fix_rest, (const bf16_t *)c->w_dev, p.slot};
    bf16_t *out = a.d_h ? (bf16_t *)a.d_h + (size_t)t0 * d : nullptr;
    ProfScope ps(11, (4.0 + es) * total, a.s);
#define GO(FIX) head_end_kernel<FIX><<<(unsigned)blocks, 64 * kFixWaves, 0, a.s>>>(fix_blocks, fix_cols, n_fix, p.fix_id, (const bf16_t *)p.fix, (float *)a.d_w, rows, total, d, out, loss)
    if (fix_here) GO(true); else GO(false);
#undef GO
    MS_LAUNCH_CHECK();
    return MS_OK;
}

bool aligned(const void *q, int by) { return ((uintptr_t)q & (by - 1)) == 0; }

// What a call reads and writes beside the hidden states, the lm_head, their gradients and the workspace
struct Span {
    const void *at;                                                                // null: not given
    size_t bytes;
};
Span span(const void *at, long numbers) { return {at, (size_t)numbers * 4}; }
bool apart(const Span &x, const Span &y) { return !x.at || !y.at || (const char *)x.at + x.bytes <= (const char *)y.at || (const char *)y.at + y.bytes <= (const char *)x.at; }

// Arguments that all calls have
ms_status begin(HeadCall *a, const char *what, const ms_head_config *c, int n, int k, HeadUse use, int pairs, const void *h, void *d_h, void *d_w, std::initializer_list<Span> reads,
                std::initializer_list<Span> writes, void *ws, size_t ws_bytes, void *stream) {
    if (n && (!h || !ws)) return ms_fail(MS_ERR_INVALID_ARG, "%s: null pointer", what);
    if (!aligned(h, 16) || !aligned(c->w_dev, 16) || !aligned(d_h, 16) || !aligned(d_w, 16) || !aligned(ws, 16))
        return ms_fail(MS_ERR_UNSUPPORTED, "%s: hidden states, lm_head, their gradients and the workspace must be 16-byte aligned", what);
    const size_t hb = (size_t)n * c->hidden * ms_dtype_size(head_dtype(c)), wb = (size_t)c->vocab * c->hidden * ms_dtype_size(head_dtype(c));
    const Span states = {h, hb}, lm_head = {c->w_dev, wb}, d_states = {d_h, hb}, d_lm_head = span(d_w, (long)c->vocab * c->hidden);
    if ((d_h != h && !apart(d_states, states)) || !apart(d_states, lm_head) || !apart(d_states, d_lm_head) || !apart(d_lm_head, states) || !apart(d_lm_head, lm_head))
        return ms_fail(MS_ERR_INVALID_ARG, "%s: d_h may be h, else the gradients must not overlap the hidden states, the lm_head or each other", what);
    a->c = c;
    a->use = use;
    a->k = k ? k : 1;
    a->h = h; a->d_h = d_h; a->d_w = d_w;
    a->s = (hipStream_t)stream;
    a->p = head_plan(c, n, k, use, pairs, ws);
    if (n && ws_bytes < a->p.bytes) return ms_fail(MS_ERR_WORKSPACE, "%s: workspace %zu < %zu bytes", what, ws_bytes, a->p.bytes);
    // the workspace and the other outputs: apart from everything else
    const Span space = {ws, a->p.bytes}, large[] = {states, lm_head, d_states, d_lm_head};
    bool clear = true;
    for (const Span &x : large) clear = clear && apart(space, x);
    for (const Span &x : reads) clear = clear && apart(space, x) && apart(d_states, x) && apart(d_lm_head, x);
    for (const Span *x = writes.begin(); x != writes.end(); ++x) {
        clear = clear && apart(*x, space);
        for (const Span &y : large) clear = clear && apart(*x, y);
        for (const Span &y : reads) clear = clear && apart(*x, y);
        for (const Span *y = writes.begin(); y != x; ++y) clear = clear && apart(*x, *y);
    }
    return clear ? MS_OK : ms_fail(MS_ERR_INVALID_ARG, "%s: outputs and workspace must not overlap each other or what the call reads", what);
}
HeadUse use_of(const void *d_h, const void *d_w) { return d_h || d_w ? HEAD_BACKWARD : HEAD_FORWARD; }

LabelRows label_rows(const HeadCall &a) { return LabelRows{a.p.slot, a.p.scale, a.p.rho, -1.f / a.c->temperature}; }
After after_label(const HeadCall &a, int what, float *logp, const float *d_logp, const PolicyArgs &policy) {
    return After{what, 1.0 / a.c->temperature, a.p.z_label, logp, d_logp, label_rows(a), policy};
}
// Behind rows t0 .. t0 + nb of n: their gradients, and the loss behind the last ones
ms_status end_of_block(const HeadCall &a, int t0, int nb, int n, const int *sel, bool dz_done, const LossTerms &all) {
    const LossTerms here = t0 + nb == n ? all : LossTerms{};
    if (a.d_h || a.d_w) return rows_backward(a, t0, nb, sel, dz_done, here);
    return here.loss ? total_loss(here, a.s) : MS_OK;
}

}  // namespace

extern "C" ms_status ms_top_logits(const ms_head_config *c, int32_t n, const void *h, int32_t k, float *values, int32_t *ids, float *lse, void *ws,
                                   size_t ws_bytes, void *stream) {
    MS_TRY(validate_head(c, n, k, "top_logits"));
    if (k < 1) return ms_fail(MS_ERR_UNSUPPORTED, "top_logits: k must be 1 .. %d and at most the vocabulary", kHeadMaxTop);
    if (n == 0) return MS_OK;
    if (!values || !ids || !lse) return ms_fail(MS_ERR_INVALID_ARG, "top_logits: null pointer");
    HeadCall a;
    MS_TRY(begin(&a, "top_logits", c, n, k, HEAD_TOP, -1, h, nullptr, nullptr, {}, {span(values, (long)n * k), span(ids, (long)n * k), span(lse, n)}, ws, ws_bytes, stream));
    const HeadPlan &p = a.p;
    const float it2 = kLog2e / c->temperature;
    const bool whole = !p.fast && c->vocab <= kTopKeys;                            // a row is looked through at once, without sums of strips
    for (int t0 = 0; t0 < n; t0 += p.block) {
        const int nb = n - t0 < p.block ? n - t0 : p.block;
        const Slabs sl = {p.rows, p.cols, c->vocab};
        MS_TRY(logits(c, p, HEAD_TOP, k, nb, (const char *)h + (size_t)t0 * c->hidden * ms_dtype_size(head_dtype(c)), a.s));
        if (!p.fast && !whole) {
            head_strips_kernel<<<dim3(ms_cdiv(p.strips, 4), nb < 32768 ? nb : 32768), 256, 0, a.s>>>(sl, nb, p.strips, (const float *)p.z, it2, p.part);
            MS_LAUNCH_CHECK();
        }
        if (!whole) MS_TRY(combine(p, nb, it2, nullptr, it2, nullptr, lse + t0, After{}, EntryRows{}, nullptr, a.s));
        head_top_kernel<<<ms_cdiv(nb, 8) * 8, kTopThreads, 0, a.s>>>(sl, nb, p.strips, k, (const float *)p.z, whole ? nullptr : p.part, it2, lse + t0, values + (long)t0 * k, ids + (long)t0 * k);
        MS_LAUNCH_CHECK();
    }
    return MS_OK;
}

extern "C" ms_status ms_topk_kd_loss_forward_backward(const ms_head_config *c, int32_t n, const void *h, int32_t k, const int32_t *top_ids, const float *top_logits,
                                                      const float *lse_teacher, float *loss, float *kl_tok, void *d_h, void *d_w, void *ws, size_t ws_bytes, void *stream) {
    MS_TRY(validate_head(c, n, k, "topk_kd"));
    if (k < 1) return ms_fail(MS_ERR_UNSUPPORTED, "topk_kd: k must be 1 .. %d and at most the vocabulary", kHeadMaxTop);
    if (!loss) return ms_fail(MS_ERR_INVALID_ARG, "topk_kd: loss_dev is null");
    if (n == 0) return launch_fill_f32(loss, 1, 0.f, (hipStream_t)stream);
    if (!top_ids || !top_logits) return ms_fail(MS_ERR_INVALID_ARG, "topk_kd: null pointer");
    HeadCall a;
    MS_TRY(begin(&a, "topk_kd", c, n, k, use_of(d_h, d_w), -1, h, d_h, d_w, {span(top_ids, (long)n * k), span(top_logits, (long)n * k), span(lse_teacher, n)}, {span(loss, 1), span(kl_tok, n)},
                 ws, ws_bytes, stream));
    const HeadPlan &p = a.p;
    const float inv_t = 1.f / c->temperature;
    float *kl = kl_tok ? kl_tok : p.per_token;
    const LossTerms all = {kl, n, c->loss_scale, loss};
    for (int t0 = 0; t0 < n; t0 += p.block) {
        const int nb = n - t0 < p.block ? n - t0 : p.block;
        bool dz_done = false;
        const Teacher teacher = {k, c->vocab, inv_t, top_ids + (long)t0 * k, top_logits + (long)t0 * k, lse_teacher ? lse_teacher + t0 : nullptr, p.ids, p.best, p.key, p.log_p, p.mass};
        MS_TRY(rows_forward(a, t0, nb, p.key, 1, p.ids, kl + t0, nullptr, After{}, teacher, Entries{p.log_p, p.mass, kl + t0, c->loss_scale * inv_t}, true, &dz_done));
        MS_TRY(end_of_block(a, t0, nb, n, p.ids, dz_done, all));
    }
    return MS_OK;
}

static ms_status token_logprobs(const char *what, const ms_head_config *c, int n, const void *h, const int32_t *labels, const float *d_logp, float *logp, void *d_h, void *d_w,
                                void *ws, size_t ws_bytes, void *stream) {
    MS_TRY(validate_head(c, n, 0, what));
    if (n == 0) return MS_OK;
    const bool back = d_logp != nullptr;
    if (!labels) return ms_fail(MS_ERR_INVALID_ARG, "%s: null pointer", what);
    HeadCall a;
    MS_TRY(begin(&a, what, c, n, 0, back ? HEAD_BACKWARD : HEAD_FORWARD, -1, h, d_h, d_w, {span(labels, n), span(d_logp, n)}, {span(logp, n)}, ws, ws_bytes, stream));
    const HeadPlan &p = a.p;
    for (int t0 = 0; t0 < n; t0 += p.block) {
        const int nb = n - t0 < p.block ? n - t0 : p.block;
        bool dz_done = false;
        float *lp = logp ? logp + t0 : p.logp;
        MS_TRY(rows_forward(a, t0, nb, labels + t0, c->vocab, labels + t0, lp, nullptr, after_label(a, back ? AFTER_GIVEN : AFTER_LOGP, lp, back ? d_logp + t0 : nullptr, {}), {}, {}, true, &dz_done));
        MS_TRY(end_of_block(a, t0, nb, n, labels + t0, dz_done, LossTerms{}));
    }
    return MS_OK;
}
extern "C" ms_status ms_token_logprobs(const ms_head_config *c, int32_t n, const void *h, const int32_t *labels, float *logp, void *ws, size_t ws_bytes, void *stream) {
    if (n > 0 && !logp) return ms_fail(MS_ERR_INVALID_ARG, "token_logprobs: null pointer");
    return token_logprobs("token_logprobs", c, n, h, labels, nullptr, logp, nullptr, nullptr, ws, ws_bytes, stream);
}
extern "C" ms_status ms_token_logprobs_backward(const ms_head_config *c, int32_t n, const void *h, const int32_t *labels, const float *d_logp, float *logp, void *d_h, void *d_w,
                                                void *ws, size_t ws_bytes, void *stream) {
    if (n > 0 && (!d_logp || (!d_h && !d_w))) return ms_fail(MS_ERR_INVALID_ARG, "token_logprobs_backward: null pointer");
    return token_logprobs("token_logprobs_backward", c, n, h, labels, d_logp, logp, d_h, d_w, ws, ws_bytes, stream);
}

extern "C" ms_status ms_policy_loss_forward_backward(const ms_head_config *c, const ms_policy_config *pc, int32_t n, const void *h, const int32_t *labels, const float *old_logp,
                                                     const float *ref_logp, const float *advantages, const float *weights, float *loss, float *loss_tok, float *logp, void *d_h,
                                                     void *d_w, void *ws, size_t ws_bytes, void *stream) {
    MS_TRY(validate_head(c, n, 0, "policy_loss"));
    if (!pc || !loss) return ms_fail(MS_ERR_INVALID_ARG, "policy_loss: null config or loss_dev");
    if (!(pc->clip_low >= 0.f && pc->clip_low <= 1.f) || !(pc->clip_high >= 0.f && pc->clip_high < INFINITY) || !(pc->kl_coef >= 0.f && pc->kl_coef < INFINITY))
        return ms_fail(MS_ERR_INVALID_ARG, "policy_loss: clip_low must be in [0, 1], clip_high and kl_coef not negative");
    if (pc->kl_coef > 0.f && n > 0 && !ref_logp) return ms_fail(MS_ERR_INVALID_ARG, "policy_loss: kl_coef without ref_logp");
    if (n == 0) return launch_fill_f32(loss, 1, 0.f, (hipStream_t)stream);
    if (!labels || !old_logp || !advantages) return ms_fail(MS_ERR_INVALID_ARG, "policy_loss: null pointer");
    HeadCall a;
    MS_TRY(begin(&a, "policy_loss", c, n, 0, use_of(d_h, d_w), -1, h, d_h, d_w, {span(labels, n), span(old_logp, n), span(ref_logp, n), span(advantages, n), span(weights, n)},
                 {span(loss, 1), span(loss_tok, n), span(logp, n)}, ws, ws_bytes, stream));
    const HeadPlan &p = a.p;
    float *terms = loss_tok ? loss_tok : p.per_token;
    const LossTerms all = {terms, n, c->loss_scale, loss};
    for (int t0 = 0; t0 < n; t0 += p.block) {
        const int nb = n - t0 < p.block ? n - t0 : p.block;
        bool dz_done = false;
        float *lp = logp ? logp + t0 : p.logp;
        const PolicyArgs pa = {old_logp + t0, pc->kl_coef > 0.f ? ref_logp + t0 : nullptr, advantages + t0, weights ? weights + t0 : nullptr, terms + t0, pc->clip_low, pc->clip_high,
                               pc->kl_coef, c->loss_scale};
        MS_TRY(rows_forward(a, t0, nb, labels + t0, c->vocab, labels + t0, lp, terms + t0, after_label(a, AFTER_POLICY, lp, nullptr, pa), {}, {}, true, &dz_done));
        MS_TRY(end_of_block(a, t0, nb, n, labels + t0, dz_done, all));
    }
    return MS_OK;
}

extern "C" ms_status ms_preference_loss_forward_backward(const ms_head_config *c, const ms_preference_config *pc, const ms_batch *batch, const void *h, const int32_t *labels,
                                                         const float *ref_logp, float *loss, float *margin, float *logp, void *d_h, void *d_w, void *ws, size_t ws_bytes,
                                                         void *stream) {
    if (!batch) return ms_fail(MS_ERR_INVALID_ARG, "preference_loss: null batch");
    const int n = batch->n_tokens, pairs = batch->n_seqs / 2;
    MS_TRY(validate_head(c, n, 0, "preference_loss"));
    if (!pc || !loss) return ms_fail(MS_ERR_INVALID_ARG, "preference_loss: null config or loss_dev");
    if (!(pc->beta > 0.f && pc->beta < INFINITY) || !(pc->label_smoothing >= 0.f && pc->label_smoothing < 1.f))
        return ms_fail(MS_ERR_INVALID_ARG, "preference_loss: beta must be positive and label_smoothing in [0, 1)");
    const int32_t *cu = batch->cu_seqlens_host;
    if (batch->n_seqs < 0 || batch->n_seqs % 2) return ms_fail(MS_ERR_SHAPE, "preference_loss: %d sequences are no pairs", batch->n_seqs);
    if (!cu || !batch->cu_seqlens_dev) return ms_fail(MS_ERR_INVALID_ARG, "preference_loss: null cu_seqlens");
    if (cu[0] != 0 || cu[batch->n_seqs] != n) return ms_fail(MS_ERR_SHAPE, "preference_loss: cu_seqlens must go from 0 to n_tokens");
    for (int i = 0; i < batch->n_seqs; ++i)
        if (cu[i + 1] < cu[i]) return ms_fail(MS_ERR_SHAPE, "preference_loss: cu_seqlens must not decrease");
    if (n == 0) {
        MS_TRY(launch_fill_f32(loss, 1, 0.f, (hipStream_t)stream));
        return margin && pairs ? launch_fill_f32(margin, pairs, 0.f, (hipStream_t)stream) : MS_OK;
    }
    if (!labels) return ms_fail(MS_ERR_INVALID_ARG, "preference_loss: null pointer");
    HeadCall a;
    const HeadUse use = use_of(d_h, d_w);
    if (n > head_most_rows(c, use)) return ms_fail(MS_ERR_UNSUPPORTED, "preference_loss: %d tokens in one block, at most %ld", n, head_most_rows(c, use));
    MS_TRY(begin(&a, "preference_loss", c, n, 0, use, pairs, h, d_h, d_w, {span(labels, n), span(ref_logp, n), span(batch->cu_seqlens_dev, batch->n_seqs + 1L)},
                 {span(loss, 1), span(margin, pairs), span(logp, n)}, ws, ws_bytes, stream));
    const HeadPlan &p = a.p;
    float *lp = logp ? logp : p.logp;
    bool dz_done = false;
    MS_TRY(rows_forward(a, 0, n, labels, c->vocab, labels, lp, nullptr, after_label(a, AFTER_LOGP, lp, nullptr, {}), {}, {}, false, &dz_done));
    head_pairs_kernel<<<pairs, 256, 0, a.s>>>(batch->cu_seqlens_dev, label_rows(a), ref_logp, pc->beta, pc->label_smoothing, c->loss_scale, lp, margin ? margin : p.margin, p.per_token);
    MS_LAUNCH_CHECK();
    return end_of_block(a, 0, n, n, labels, dz_done, LossTerms{p.per_token, pairs, c->loss_scale, loss});
}
