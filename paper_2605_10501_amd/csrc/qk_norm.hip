// RMSNorm of every query and key head together with the rotary embedding, forward and backward.
//
//   forward   r = (mean_hd x^2 + eps)^-1/2,  y = R(pos) (x r g)          R: half-split rotation by the table's (cos, sin)
//   backward  d = R(pos)^T dy,  dg += sum d x r,  dx = r (d g - x r mean_hd(d g x r))
//
// A lane holds one 16-byte vector of each half of a head (the pairs that the rotation mixes), G lanes hold a head, a wave 64 / G heads:
// everything between the load and the store of an element stays in registers, in fp32, and is rounded once.  (Norm and
// rotation as two kernels read and write q and k twice and round in between.)
// HBM bounds both on large batches, the vector ALU closely behind: a wave-instruction takes four cycles of a SIMD, and 5.8 TB/s leave a
// wave that handles 64 vector pairs about 180 (forward) or 280 (backward) of them.
#include "common.h"
#include "launch.h"
#include "launch_plan.h"

namespace {

constexpr int kPartRows = 768;       // workgroups of the backward kernel, one partial row of dg each: three per CU, as its registers allow (four need spills and are no faster)

// Results leave non-temporally: 20011 tokens x 16 heads forward 33.9 -> 28.8 us, 4096 x 24 12.1 -> 9.8, backward 3-8 % (repeated passes on operands that
// the caches hold in part; 32.5 us on operands from memory.  Loads by that policy too gain 2 % on the largest batches and lose up to 18 % on small ones)
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
template <class T> __device__ __forceinline__ void put(T *p, const Vec16<T> &r) { __builtin_nontemporal_store(*(const u32x4 *)&r, (u32x4 *)p); }

template <int G> __device__ __forceinline__ float group_sum(float v) {
#pragma unroll
    for (int o = G / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

struct QknArgs {
    const void *x, *dy;              // forward: x -> out; backward: (dy, x) -> out
    void *out;
    const void *g_q, *g_k;
    const int *pos;
    const float2 *table;
    long xs, dys, os;                // row strides in elements
    int n, nq, nkv, hd, max_pos;
    float eps;
};

// The (cos, sin) of a lane's V pairs; a position outside the table does not rotate (and reads nothing)
template <int V> __device__ __forceinline__ void load_angles(const QknArgs &a, int p, int i0, bool live, float *c, float *s) {
    if (live && (unsigned)p < (unsigned)a.max_pos) {
        const float4 *t = (const float4 *)(a.table + (long)p * (a.hd >> 1) + i0);
#pragma unroll
        for (int q = 0; q < V / 2; ++q) {
            const float4 v = t[q];
            c[2 * q] = v.x; s[2 * q] = v.y; c[2 * q + 1] = v.z; s[2 * q + 1] = v.w;
        }
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) { c[e] = 1.f; s[e] = 0.f; }
    }
}

// One wave per token and `spw` groups of 64 / G heads of it (blockIdx.y takes the others), so that the angles are read once per
// token.  heads: those that are written, V heads too where the output is another tensor.
template <class T, int G>
__global__ __launch_bounds__(256) void qk_norm_rope_fwd_kernel(QknArgs a, int heads, int spw) {
    constexpr int V = Vec16<T>::N, HPW = 64 / G;
    const int lane = threadIdx.x & 63, j = lane & (G - 1), hl = lane / G;
    const int half = a.hd >> 1, nqk = a.nq + a.nkv;
    const bool live = j * V < half;
    const float inv_hd = 1.f / a.hd;
    const int h0 = blockIdx.y * spw * HPW + hl, h_end = min(heads, ((int)blockIdx.y + 1) * spw * HPW);
    for (long t = (long)blockIdx.x * 4 + (threadIdx.x >> 6); t < a.n; t += (long)gridDim.x * 4) {
        const T *xr = (const T *)a.x + t * a.xs + j * V;
        T *yr = (T *)a.out + t * a.os + j * V;
        float c[V], s[V];
        load_angles<V>(a, a.pos[t], j * V, live, c, s);
        Vec16<T> lo, hi;
        if (live && h0 < h_end) { lo = ldv(xr + (long)h0 * a.hd); hi = ldv(xr + (long)h0 * a.hd + half); }
        for (int h = h0; h - hl < h_end; h += HPW) {             // (all lanes of the wave take every trip: the sums need them)
            const bool mine = live && h < h_end;
            Vec16<T> nlo, nhi, glo, ghi;
            if (live && h + HPW < h_end) { nlo = ldv(xr + (long)(h + HPW) * a.hd); nhi = ldv(xr + (long)(h + HPW) * a.hd + half); }
            if (mine) {
                const T *g = (const T *)(h < a.nq ? a.g_q : a.g_k) + j * V;
                glo = ldv(g); ghi = ldv(g + half);
            }
            float xl[V], xh[V], ss = 0.f;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                xl[e] = to_f32(lo.v[e]); xh[e] = to_f32(hi.v[e]);
                ss = __builtin_fmaf(xl[e], xl[e], ss);
                ss = __builtin_fmaf(xh[e], xh[e], ss);
            }
            const float r = rsqrtf(group_sum<G>(mine ? ss : 0.f) * inv_hd + a.eps);
            if (mine) {
                Vec16<T> ol, oh;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float p = xl[e] * r * to_f32(glo.v[e]), q = xh[e] * r * to_f32(ghi.v[e]);
                    ol.v[e] = from_f32<T>(p * c[e] - q * s[e]);
                    oh.v[e] = from_f32<T>(q * c[e] + p * s[e]);
                }
                if (h >= nqk) { ol = lo; oh = hi; }              // a V head is copied
                put(yr + (long)h * a.hd, ol);
                put(yr + (long)h * a.hd + half, oh);
            }
            lo = nlo; hi = nhi;
        }
    }
}

// Workgroups 0 .. bq-1 take the query heads, bq .. bq+bk-1 the key heads, so that a lane adds up one gain's gradient; the rest copy
// dV where dx is another tensor than dy.  The heads of a kind are numbered through all tokens and cut into one contiguous piece per
// wave: no lane idles where a token has fewer heads than a wave holds.
template <class T, int G>
__global__ __launch_bounds__(256) void qk_norm_rope_bwd_kernel(QknArgs a, float *part, int bq, int bk) {
    constexpr int V = Vec16<T>::N, HPW = 64 / G;
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, half = a.hd >> 1;
    int b = blockIdx.x;
    if (b >= bq + bk) {
        b -= bq + bk;
        const long vpr = (long)a.nkv * a.hd / V, total = a.n * vpr, stride = (long)(gridDim.x - bq - bk) * 256;
        const long col = (long)(a.nq + a.nkv) * a.hd;
        for (long i = (long)b * 256 + threadIdx.x; i < total; i += stride) {
            const long t = i / vpr, cv = i % vpr;
            put((T *)a.out + t * a.os + col + cv * V, ldv((const T *)a.dy + t * a.dys + col + cv * V));
        }
        return;
    }
    const bool key = b >= bq;
    const int nh = key ? a.nkv : a.nq, first = key ? a.nq : 0, nb = key ? bk : bq, w = (key ? b - bq : b) * 4 + wv;
    const int j = lane & (G - 1), hl = lane / G;
    const bool live = j * V < half;
    const float inv_hd = 1.f / a.hd;
    float gl[V], gh[V], dgl[V], dgh[V];
    {
        Vec16<T> l, h;
        const T *g = (const T *)(key ? a.g_k : a.g_q) + j * V;
        if (live) { l = ldv(g); h = ldv(g + half); }
#pragma unroll
        for (int e = 0; e < V; ++e) {
            gl[e] = live ? to_f32(l.v[e]) : 0.f; gh[e] = live ? to_f32(h.v[e]) : 0.f;
            dgl[e] = 0.f; dgh[e] = 0.f;
        }
    }
    const long items = (long)a.n * nh, steps = (items + HPW - 1) / HPW, per = (steps + 4 * nb - 1) / (4 * nb);
    const long s0 = w * per, s1 = s0 + per < steps ? s0 + per : steps;
    const int dt = HPW / nh, dh = HPW % nh;
    long t = (s0 * HPW + hl) / nh;
    int h = (int)((s0 * HPW + hl) % nh);
    Vec16<T> v0, v1, v2, v3;
    auto load = [&](bool ok, long t, int h) {            // zeros where there is nothing (one test for the wave instead of selects for each element)
        if (!__all(ok)) {
            const uint4 z = make_uint4(0, 0, 0, 0);
            *(uint4 *)&v0 = z; *(uint4 *)&v1 = z; *(uint4 *)&v2 = z; *(uint4 *)&v3 = z;
        }
        if (!ok) return;
        const long at = (long)(first + h) * a.hd + j * V;
        const T *xp = (const T *)a.x + t * a.xs + at, *dp = (const T *)a.dy + t * a.dys + at;
        v0 = ldv(xp); v1 = ldv(xp + half); v2 = ldv(dp); v3 = ldv(dp + half);
    };
    const bool some = s0 < s1;
    load(some && live && t < a.n, t, h);
    int p = some && t < a.n ? a.pos[t] : -1;
    for (long st = s0; st < s1; ++st) {
        const bool mine = live && t < a.n;
        float xl[V], xh[V], yl[V], yh[V], ss = 0.f;
        const long at = (long)(first + h) * a.hd + j * V, now = t;
        float c[V], s[V];
        load_angles<V>(a, p, j * V, live, c, s);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            xl[e] = to_f32(v0.v[e]); xh[e] = to_f32(v1.v[e]);
            yl[e] = to_f32(v2.v[e]); yh[e] = to_f32(v3.v[e]);
            ss = __builtin_fmaf(xl[e], xl[e], ss);
            ss = __builtin_fmaf(xh[e], xh[e], ss);
        }
        h += dh; t += dt;                                // the next heads are on their way while these are worked on
        if (h >= nh) { h -= nh; ++t; }
        const bool more = st + 1 < s1 && t < a.n;
        load(more && live, t, h);
        p = more ? a.pos[t] : -1;
        ss = group_sum<G>(ss);
        const float r = mine ? rsqrtf(ss * inv_hd + a.eps) : 0.f;
        float m = 0.f;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float dl = (yl[e] * c[e] + yh[e] * s[e]) * r, dhh = (yh[e] * c[e] - yl[e] * s[e]) * r;
            dgl[e] = __builtin_fmaf(dl, xl[e], dgl[e]);
            dgh[e] = __builtin_fmaf(dhh, xh[e], dgh[e]);
            yl[e] = dl * gl[e];
            yh[e] = dhh * gh[e];
            m = __builtin_fmaf(yl[e], xl[e], m);
            m = __builtin_fmaf(yh[e], xh[e], m);
        }
        m = group_sum<G>(m) * inv_hd * r * r;
        if (mine) {
            Vec16<T> ol, oh;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                ol.v[e] = from_f32<T>(__builtin_fmaf(-xl[e], m, yl[e]));
                oh.v[e] = from_f32<T>(__builtin_fmaf(-xh[e], m, yh[e]));
            }
            T *o = (T *)a.out + now * a.os + at;
            put(o, ol);
            put(o + half, oh);
        }
    }
    // heads of the wave, then waves, in a fixed order
    __shared__ float red[4][2 * G * V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
#pragma unroll
        for (int o = G; o < 64; o <<= 1) {
            dgl[e] += __shfl_xor(dgl[e], o, 64);
            dgh[e] += __shfl_xor(dgh[e], o, 64);
        }
        if (hl == 0) { red[wv][j * V + e] = dgl[e]; red[wv][G * V + j * V + e] = dgh[e]; }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.hd; i += 256) {
        const int k = i < half ? i : G * V + i - half;
        part[(long)blockIdx.x * a.hd + i] = red[0][k] + red[1][k] + red[2][k] + red[3][k];
    }
}

ms_status check(const char *who, int dtype, const QknArgs &a, bool backward) {
    if (!a.x || !a.out || !a.g_q || !a.g_k || !a.pos || !a.table || (backward && !a.dy)) return ms_fail(MS_ERR_INVALID_ARG, "%s: null pointer", who);
    if (dtype != MS_BF16 && dtype != MS_F32) return ms_fail(MS_ERR_INVALID_ARG, "%s: bad dtype %d", who, dtype);
    if (a.n < 0 || a.nq <= 0 || a.nkv <= 0 || a.hd <= 0 || a.max_pos <= 0 || !(a.eps >= 0.f)) return ms_fail(MS_ERR_INVALID_ARG, "%s: bad size or eps", who);
    if (a.hd % 16 || a.hd > 512) return ms_fail(MS_ERR_UNSUPPORTED, "%s: head_dim=%d must be a multiple of 16 and at most 512", who, a.hd);
    const int V = dtype == MS_BF16 ? 8 : 4;
    const long qk = (long)(a.nq + a.nkv) * a.hd, all = qk + (long)a.nkv * a.hd;
    const void *in = backward ? a.dy : a.x;
    const long is = backward ? a.dys : a.xs;
    if (a.nq > 65536 || a.nkv > 65536) return ms_fail(MS_ERR_UNSUPPORTED, "%s: more than 65536 heads", who);
    if (a.xs < qk || is < (a.out == in ? qk : all) || a.os < (a.out == in ? qk : all)) return ms_fail(MS_ERR_SHAPE, "%s: a row stride is less than a row", who);
    if (a.xs % V || is % V || a.os % V || (((uintptr_t)a.x | (uintptr_t)in | (uintptr_t)a.out | (uintptr_t)a.g_q | (uintptr_t)a.g_k | (uintptr_t)a.table) & 15))
        return ms_fail(MS_ERR_UNSUPPORTED, "%s: rows, gains and table must be 16-byte aligned", who);
    const long es = ms_dtype_size(dtype);
    if (a.out == in ? a.os != is : !ms_apart(in, is * es, all * es, a.out, a.os * es, all * es, a.n))
        return ms_fail(MS_ERR_INVALID_ARG, "%s: the output is neither its input nor apart from it", who);
    // (of x the query and key heads are read; dx has the V heads too unless it is dy)
    if (backward && !ms_apart(a.x, a.xs * es, qk * es, a.out, a.os * es, (a.out == in ? qk : all) * es, a.n)) return ms_fail(MS_ERR_INVALID_ARG, "%s: dx overlaps x", who);
    return MS_OK;
}

int lanes_per_head(int dtype, int hd) {
    const int vecs = hd / 2 / (dtype == MS_BF16 ? 8 : 4);
    int g = 1;
    while (g < vecs) g *= 2;
    return g;
}

#define QKN_G(T, G, CALL) case G: { constexpr int kG = G; using kT = T; CALL; break; }
#define QKN_DISPATCH(dtype, g, CALL)                                                                                        \
    if ((dtype) == MS_BF16) switch (g) { QKN_G(bf16_t, 1, CALL) QKN_G(bf16_t, 2, CALL) QKN_G(bf16_t, 4, CALL) QKN_G(bf16_t, 8, CALL) QKN_G(bf16_t, 16, CALL) QKN_G(bf16_t, 32, CALL) } \
    else switch (g) { QKN_G(float, 2, CALL) QKN_G(float, 4, CALL) QKN_G(float, 8, CALL) QKN_G(float, 16, CALL) QKN_G(float, 32, CALL) QKN_G(float, 64, CALL) }

}  // namespace

extern "C" ms_status ms_k_qk_norm_rope_forward(int32_t dtype, int32_t n, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, float eps,
                                               const void *x, int64_t x_stride, const void *g_q, const void *g_k, const int32_t *pos,
                                               const float *table, int32_t max_pos, void *y, int64_t y_stride, void *stream) {
    if (n == 0) return MS_OK;
    const QknArgs a = {x, nullptr, y, g_q, g_k, pos, (const float2 *)table, x_stride, 0, y_stride, n, n_q_heads, n_kv_heads, head_dim, max_pos, eps};
    MS_TRY(check("qk_norm_rope_forward", dtype, a, false));
    const int g = lanes_per_head(dtype, head_dim), hpw = 64 / g;
    const int heads = n_q_heads + (y == x ? 1 : 2) * n_kv_heads, steps = ms_cdiv(heads, hpw);
    // Few tokens: a wave per group of heads, for more waves; many: a wave per token, which reads its angles once.  us, group / token, operands from memory: 32 + 8
    // heads of 128 in bf16 16 tokens 3.5 / 6.3, 1024 7.5 / 8.9, 2048 11.1 / 10.9, 4096 18.8 / 19.3, 6000 37.7 / 32.6, 32768 203 / 153; 12 + 2 heads 1024 4.7 / 5.1, 3000
    // 7.4 / 6.8, 4096 8.3 / 7.7, 32768 49 / 44; 16 + 4 heads of 64 2048 5.4 / 5.6, 4096 8.1 / 7.1; 2 + 2 heads are one group
    const int spw = n >= 4096 ? steps : 1;
    const long gx = ms_cdiv(n, 4) < (1 << 20) ? ms_cdiv(n, 4) : (1 << 20);
    const dim3 grid((unsigned)gx, (unsigned)ms_cdiv(steps, spw));
    if (grid.y > 65535) return ms_fail(MS_ERR_UNSUPPORTED, "qk_norm_rope_forward: too many heads");
    hipStream_t s = (hipStream_t)stream;
    ProfScope ps(8, 2.0 * n * heads * head_dim * ms_dtype_size(dtype), s);
    QKN_DISPATCH(dtype, g, (qk_norm_rope_fwd_kernel<kT, kG><<<grid, 256, 0, s>>>(a, heads, spw)));
    MS_LAUNCH_CHECK();
    return MS_OK;
}

extern "C" size_t ms_k_qk_norm_rope_backward_scratch_bytes(int32_t head_dim) {
    return head_dim > 0 ? ms_align_up((size_t)kPartRows * head_dim * sizeof(float)) : 0;
}

extern "C" ms_status ms_k_qk_norm_rope_backward(int32_t dtype, int32_t n, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, float eps,
                                                const void *dy, int64_t dy_stride, const void *x, int64_t x_stride, const void *g_q,
                                                const void *g_k, const int32_t *pos, const float *table, int32_t max_pos, void *dx,
                                                int64_t dx_stride, float *dg_q, float *dg_k, void *scratch, void *stream) {
    if (n == 0) return MS_OK;
    const QknArgs a = {x, dy, dx, g_q, g_k, pos, (const float2 *)table, x_stride, dy_stride, dx_stride, n, n_q_heads, n_kv_heads, head_dim, max_pos, eps};
    MS_TRY(check("qk_norm_rope_backward", dtype, a, true));
    if (!dg_q || !dg_k || !scratch) return ms_fail(MS_ERR_INVALID_ARG, "qk_norm_rope_backward: null pointer");
    const int g = lanes_per_head(dtype, head_dim), hpw = 64 / g;
    // workgroups in proportion to the heads of each kind, at most kPartRows, no more than there are groups of heads
    const long sq = ((long)n * n_q_heads + hpw - 1) / hpw, sk = ((long)n * n_kv_heads + hpw - 1) / hpw;
    const int most_k = (int)(kPartRows * (double)n_kv_heads / (n_q_heads + n_kv_heads)), mk = most_k < 1 ? 1 : most_k;
    const int bq = (int)((sq + 3) / 4 < kPartRows - mk ? (sq + 3) / 4 : kPartRows - mk), bk = (int)((sk + 3) / 4 < mk ? (sk + 3) / 4 : mk);
    const long copy = dx == dy ? 0 : ((long)n * n_kv_heads * head_dim / (dtype == MS_BF16 ? 8 : 4) + 255) / 256;
    const int bc = (int)(copy < 256 ? copy : 256);
    float *part = (float *)scratch;
    hipStream_t s = (hipStream_t)stream;
    ProfScope ps(8, (double)n * head_dim * ms_dtype_size(dtype) * (3.0 * (n_q_heads + n_kv_heads) + (bc ? 2.0 : 0.0) * n_kv_heads), s);
    QKN_DISPATCH(dtype, g, (qk_norm_rope_bwd_kernel<kT, kG><<<bq + bk + bc, 256, 0, s>>>(a, part, bq, bk)));
    MS_LAUNCH_CHECK();
    const int blocks = ms_cdiv(head_dim, 32);
    const ColReduce q = {part, dg_q, bq, head_dim}, k = {part + (long)bq * head_dim, dg_k, bk, head_dim};
    if (dg_q < dg_k + head_dim && dg_k < dg_q + head_dim) {      // into the same row (one gain for both): one after the other
        MS_TRY(launch_reduce_partials(ReduceJobs{1, {0}, {q}}, blocks, s));
        return launch_reduce_partials(ReduceJobs{1, {0}, {k}}, blocks, s);
    }
    return launch_reduce_partials(ReduceJobs{2, {0, blocks}, {q, k}}, 2 * blocks, s);
}
