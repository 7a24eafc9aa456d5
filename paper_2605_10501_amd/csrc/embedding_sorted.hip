// Embedding rows times a scale, and the table's gradient from the tokens sorted by id.
//
//   forward   x[t] = round(scale E[id_t])
//   backward  dE[v] += scale sum_{t: id_t = v} dx[t], tokens in ascending order within pieces of kTile sorted places, pieces in order
//
// The gradient needs no floating-point atomics: its sums have one order, so a run repeats bit for bit, and a row that thousands
// of tokens share (padding, frequent words) is not added to by thousands of atomics.  Steps:
//   1. stable radix sort of (id, token): per digit, a workgroup ranks its tokens and places them behind those of the workgroups
//      before it (per-workgroup digit counts; integer atomics, whose order does not matter).  Ids outside the table sort last.
//   2. every kTile sorted places x one 16-byte column vector per thread: one pass over dx.  A run of equal ids that lies within
//      the piece is added to the table; what continues from or into a neighbour goes to a row of partial sums.
//   3. the runs that span pieces: their partial rows are added up and go to the table.
// HBM bounds step 2 (dx read once, touched rows read and written), launches and latency the sort.
#include "common.h"
#include "launch.h"
#include "launch_plan.h"

namespace {

constexpr int kSortThreads = 1024, kWaves = kSortThreads / 64, kDigitBits = 9, kBins = 1 << kDigitBits;
constexpr int kTile = 32;                 // sorted places of a piece
constexpr int kMaxTokens = 1 << 24;

// ------------------------------------------------------------------ forward
template <class T, class TO, int U>
__global__ __launch_bounds__(256) void embedding_scaled_kernel(const int *__restrict__ ids, const T *__restrict__ table, TO *__restrict__ x,
                                                               float scale, int n, int vpr, int vocab) {
    constexpr int V = Vec16<T>::N;
    const long d = (long)vpr * V;
    for (long t0 = ((long)blockIdx.x * blockDim.y + threadIdx.y) * U; t0 < n; t0 += (long)gridDim.x * blockDim.y * U) {
        int id[U];
#pragma unroll
        for (int u = 0; u < U; ++u) id[u] = t0 + u < n ? ids[t0 + u] : -1;
        for (int cv = threadIdx.x; cv < vpr; cv += blockDim.x) {
            Vec16<T> v[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if ((unsigned)id[u] < (unsigned)vocab) v[u] = ldv(table + id[u] * d + (long)cv * V);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (t0 + u >= n) break;
                const bool in = (unsigned)id[u] < (unsigned)vocab;       // an id outside the table embeds as zeros
                TO *o = x + (t0 + u) * d + (long)cv * V;
                float f[V];
#pragma unroll
                for (int e = 0; e < V; ++e) f[e] = in ? scale * to_f32(v[u].v[e]) : 0.f;
#pragma unroll
                for (int q = 0; q < V; q += Vec16<TO>::N) {
                    Vec16<TO> w;
#pragma unroll
                    for (int e = 0; e < Vec16<TO>::N; ++e) w.v[e] = from_f32<TO>(f[q + e]);
                    stv(o + q, w);
                }
            }
        }
    }
}

// ------------------------------------------------------------------ sort
__device__ __forceinline__ unsigned key_of(int id, int vocab) { return (unsigned)id < (unsigned)vocab ? (unsigned)id : (unsigned)vocab; }

// Digit counts of every workgroup's tokens by the first digit; clears the counters that the passes add to
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(const int *__restrict__ ids, int n, int vocab, int per, int mask,
                                                                  int *__restrict__ counts, int *__restrict__ next, long next_len) {
    __shared__ int hist[kBins];
    const int tid = threadIdx.x;
    if (tid < kBins) hist[tid] = 0;
    __syncthreads();
    const long b0 = (long)blockIdx.x * per;
    for (int i = tid; i < per && b0 + i < n; i += kSortThreads) atomicAdd(&hist[key_of(ids[b0 + i], vocab) & mask], 1);
    __syncthreads();
    if (tid < kBins) counts[(long)blockIdx.x * kBins + tid] = hist[tid];
    for (long i = (long)blockIdx.x * kSortThreads + tid; i < next_len; i += (long)gridDim.x * kSortThreads) next[i] = 0;
}

// One stable pass by the digit (key >> shift) & mask.  ids != null: the keys are the ids and the values the token numbers.
// counts: [workgroups][kBins] of this digit (null: there is one workgroup); next: the same for the following digit in the
// new order, added to here.  A wave takes 64 IPT consecutive places, a trip 64 of them: lanes of equal digits find each other
// by ballots, the first of them moves the wave's counter on.
template <int IPT>
__global__ __launch_bounds__(kSortThreads) void sort_pass_kernel(const int *__restrict__ ids, const uint2 *__restrict__ in, int n, int vocab, int shift,
                                                                 int bits, const int *__restrict__ counts, int *__restrict__ next,
                                                                 int next_shift, uint2 *__restrict__ out) {
    __shared__ int hist[kWaves][kBins];
    __shared__ int base[kBins];
    __shared__ int wsum[kBins / 64];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, mask = (1 << bits) - 1, per = kSortThreads * IPT;
    for (int i = tid; i < kWaves * kBins; i += kSortThreads) (&hist[0][0])[i] = 0;
    __syncthreads();
    const long b0 = (long)blockIdx.x * per + wv * 64 * IPT;
    uint2 kv[IPT];
    int rank[IPT];
#pragma unroll
    for (int r = 0; r < IPT; ++r) {
        const long i = b0 + r * 64 + lane;
        const bool valid = i < n;
        kv[r] = make_uint2(0, 0);
        if (valid) kv[r] = ids ? make_uint2(key_of(ids[i], vocab), (unsigned)i) : in[i];
    }
#pragma unroll
    for (int r = 0; r < IPT; ++r) {
        const bool valid = b0 + r * 64 + lane < n;
        const int dg = (kv[r].x >> shift) & mask;
        unsigned long long same = __ballot(valid);
        for (int k = 0; k < bits; ++k) {
            const unsigned long long m = __ballot((dg >> k) & 1);
            same &= (dg >> k) & 1 ? m : ~m;
        }
        const int before = __popcll(same & ((1ull << lane) - 1)), cnt = __popcll(same);
        const int pre = hist[wv][dg];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (valid && before == 0) hist[wv][dg] = pre + cnt;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        rank[r] = pre + before;
    }
    __syncthreads();
    int total = 0, ahead = 0;
    if (tid < kBins) {
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const int c = hist[w][tid];
            hist[w][tid] = total;
            total += c;
        }
        if (counts) {                                   // all tokens of this digit, and those of the workgroups in front
            total = 0;
            for (int b = 0; b < (int)gridDim.x; ++b) {
                const int c = counts[(long)b * kBins + tid];
                total += c;
                ahead += b < (int)blockIdx.x ? c : 0;
            }
        }
        int inc = total;                                // prefix sum over the digits
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int v = __shfl_up(inc, o, 64);
            if (lane >= o) inc += v;
        }
        if (lane == 63) wsum[wv] = inc;
        base[tid] = inc - total + ahead;
    }
    __syncthreads();
    if (tid < kBins) {
        int add = 0;
        for (int w = 0; w < wv; ++w) add += wsum[w];
        base[tid] += add;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < IPT; ++r) {
        if (b0 + r * 64 + lane < n) {
            const int dg = (kv[r].x >> shift) & mask;
            const int at = base[dg] + hist[wv][dg] + rank[r];
            out[at] = kv[r];
            if (next) atomicAdd(next + (long)(at / per) * kBins + ((kv[r].x >> next_shift) & mask), 1);
        }
    }
}

// ------------------------------------------------------------------ sums
// part: [pieces][2][d]: row 0 the end of a run that began in an earlier piece, row 1 the part of a run that goes on in the next
template <class T>
__global__ __launch_bounds__(256) void embedding_sum_kernel(const uint2 *__restrict__ sorted, const T *__restrict__ dx, float scale, int n, int vpr,
                                                            int vocab, float *__restrict__ d_table, float *__restrict__ part, long total) {
    constexpr int V = Vec16<T>::N, U = 8;
    const long i = (long)blockIdx.x * 256 + threadIdx.x;
    if (i >= total) return;
    const long tile = i / vpr, d = (long)vpr * V;
    const long cv = (i % vpr) * V;
    const int p0 = (int)(tile * kTile), p1 = p0 + kTile < n ? p0 + kTile : n;
    const unsigned before = p0 > 0 ? sorted[p0 - 1].x : 0xffffffffu, after = p1 < n ? sorted[p1].x : 0xffffffffu;
    float acc[V];
#pragma unroll
    for (int e = 0; e < V; ++e) acc[e] = 0.f;
    unsigned run = sorted[p0].x;
    bool first = true;                                   // the run that the piece begins with
    auto store = [&](float *o) {
#pragma unroll
        for (int q = 0; q < V; q += 4) *(float4 *)(o + q) = make_float4(acc[q], acc[q + 1], acc[q + 2], acc[q + 3]);
    };
    auto flush = [&]() {                                 // the run ends within the piece
        if (run < (unsigned)vocab) {
            if (first && run == before) {
                store(part + tile * 2 * d + cv);
            } else {
                float *o = d_table + (long)run * d + cv;
#pragma unroll
                for (int q = 0; q < V; q += 4) {
                    float4 v = *(float4 *)(o + q);
                    v.x = __builtin_fmaf(scale, acc[q], v.x); v.y = __builtin_fmaf(scale, acc[q + 1], v.y);
                    v.z = __builtin_fmaf(scale, acc[q + 2], v.z); v.w = __builtin_fmaf(scale, acc[q + 3], v.w);
                    *(float4 *)(o + q) = v;
                }
            }
        }
        first = false;
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] = 0.f;
    };
    for (int p = p0; p < p1; p += U) {
        uint2 kv[U];
        Vec16<T> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) kv[u] = sorted[p + u < p1 ? p + u : p1 - 1];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (p + u < p1 && kv[u].x < (unsigned)vocab) v[u] = ldv(dx + (long)kv[u].y * d + cv);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (p + u >= p1) break;
            if (kv[u].x != run) { flush(); run = kv[u].x; }
            if (run < (unsigned)vocab)
#pragma unroll
                for (int e = 0; e < V; ++e) acc[e] += to_f32(v[u].v[e]);
        }
    }
    if (run == after) {
        if (run < (unsigned)vocab) store(part + (tile * 2 + 1) * d + cv);
    } else {
        flush();
    }
}

// A workgroup per piece and 128 columns: where a run begins in the piece and goes on behind it, the partial rows of that run, every
// eighth by the same 32 threads, then the eight sums in order
__global__ __launch_bounds__(256) void embedding_join_kernel(const uint2 *__restrict__ sorted, const float *__restrict__ part, float scale, int n, long d,
                                                             int tiles, int vocab, float *__restrict__ d_table) {
    __shared__ float4 sm[8][32];
    const int tile = blockIdx.x, p0 = tile * kTile, p1 = p0 + kTile;
    if (p1 >= n) return;
    const unsigned run = sorted[p1 - 1].x;
    if (run != sorted[p1].x || run >= (unsigned)vocab || (p0 > 0 && sorted[p0].x == run && sorted[p0 - 1].x == run)) return;
    const int cl = threadIdx.x & 31, pl = threadIdx.x >> 5;
    for (long c0 = (long)blockIdx.y * 128; c0 < d; c0 += (long)gridDim.y * 128) {
        const long col = c0 + 4 * cl;
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int q = tile + pl; q < tiles; q += 8) {
            if (sorted[(long)q * kTile + (q == tile ? kTile - 1 : 0)].x != run) break;
            const bool more = (long)(q + 1) * kTile < n && sorted[(long)(q + 1) * kTile].x == run;
            if (col < d) {
                const float4 v = *(const float4 *)(part + ((long)q * 2 + more) * d + col);
                s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
            }
        }
        sm[pl][cl] = s;
        __syncthreads();
        if (pl == 0 && col < d) {
#pragma unroll
            for (int k = 1; k < 8; ++k) {
                const float4 v = sm[k][cl];
                s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
            }
            float4 *o = (float4 *)(d_table + (long)run * d + col), v = *o;
            v.x = __builtin_fmaf(scale, s.x, v.x); v.y = __builtin_fmaf(scale, s.y, v.y);
            v.z = __builtin_fmaf(scale, s.z, v.z); v.w = __builtin_fmaf(scale, s.w, v.w);
            *o = v;
        }
        __syncthreads();
    }
}

struct SortPlan { int bits, passes, ipt, blocks; };
SortPlan sort_plan(int n, int vocab) {
    SortPlan p;
    int bits = 1;
    while (bits < 31 && (vocab >> bits) > 0) ++bits;                 // keys 0 .. vocab
    p.passes = (bits + kDigitBits - 1) / kDigitBits;
    p.bits = (bits + p.passes - 1) / p.passes;
    p.ipt = n <= 128 * kSortThreads ? 1 : n <= 512 * kSortThreads ? 4 : 16;
    p.blocks = ms_cdiv(n, (long)p.ipt * kSortThreads);
    return p;
}
struct SortScratch { uint2 *a, *b; int *counts; float *part; size_t bytes; };
SortScratch carve(void *ws, int n, int d, int vocab) {
    const SortPlan p = sort_plan(n, vocab);
    Arena a(ws);
    SortScratch s;
    s.a = a.take<uint2>((size_t)n * 8);
    s.b = a.take<uint2>((size_t)n * 8);
    s.counts = a.take<int>((size_t)p.passes * p.blocks * kBins * 4);
    s.part = a.take<float>((size_t)ms_cdiv(n, kTile) * 2 * d * 4);
    s.bytes = a.off;
    return s;
}
bool aligned(const void *p) { return ((uintptr_t)p & 15) == 0; }

ms_status check(const char *who, int dtype, int n, int d, int vocab) {
    if (dtype != MS_BF16 && dtype != MS_F32) return ms_fail(MS_ERR_INVALID_ARG, "%s: bad dtype %d", who, dtype);
    if (n < 0 || d <= 0 || vocab <= 0 || vocab == 0x7fffffff) return ms_fail(MS_ERR_INVALID_ARG, "%s: bad size", who);
    const int V = dtype == MS_BF16 ? 8 : 4;
    if (d % V) return ms_fail(MS_ERR_UNSUPPORTED, "%s: d=%d must be a multiple of %d", who, d, V);
    return MS_OK;
}

}  // namespace

extern "C" ms_status ms_k_embedding_scaled_forward(int32_t dtype, int32_t out_fp32, int32_t n, int32_t d, int32_t vocab, float scale,
                                                   const int32_t *ids, const void *table, void *x, void *stream) {
    if (n == 0) return MS_OK;
    MS_TRY(check("embedding_scaled_forward", dtype, n, d, vocab));
    if (!ids || !table || !x) return ms_fail(MS_ERR_INVALID_ARG, "embedding_scaled_forward: null pointer");
    if (!aligned(table) || !aligned(x)) return ms_fail(MS_ERR_UNSUPPORTED, "embedding_scaled_forward: table and x must be 16-byte aligned");
    const int vpr = d / (dtype == MS_BF16 ? 8 : 4);
    int bx = 16;
    while (bx < vpr && bx < 256) bx *= 2;
    const int by = 256 / bx;
    hipStream_t s = (hipStream_t)stream;
    ProfScope ps(11, (double)n * d * (ms_dtype_size(dtype) + (out_fp32 ? 4 : ms_dtype_size(dtype))), s);
#define GO(T, TO, U)                                                                                                                        \
    do {                                                                                                                                    \
        const int g = ms_cdiv(n, (long)by * U);                                                                                             \
        embedding_scaled_kernel<T, TO, U><<<g < (1 << 20) ? g : (1 << 20), dim3(bx, by), 0, s>>>(ids, (const T *)table, (TO *)x, scale, n, vpr, vocab); \
    } while (0)
    if (dtype == MS_F32) GO(float, float, 2);
    else if (out_fp32) GO(bf16_t, float, 2);
    else GO(bf16_t, bf16_t, 2);
#undef GO
    MS_LAUNCH_CHECK();
    return MS_OK;
}

extern "C" size_t ms_k_embedding_sorted_backward_scratch_bytes(int32_t n, int32_t d, int32_t vocab) {
    if (n <= 0 || n > kMaxTokens || d <= 0 || vocab <= 0 || vocab == 0x7fffffff) return 0;
    return carve(nullptr, n, d, vocab).bytes;
}

extern "C" ms_status ms_k_embedding_sorted_backward(int32_t dtype, int32_t n, int32_t d, int32_t vocab, float scale, const int32_t *ids,
                                                    const void *dx, float *d_table, void *scratch, size_t scratch_bytes, void *stream) {
    if (n == 0) return MS_OK;
    MS_TRY(check("embedding_sorted_backward", dtype, n, d, vocab));
    if (!ids || !dx || !d_table || !scratch) return ms_fail(MS_ERR_INVALID_ARG, "embedding_sorted_backward: null pointer");
    if (n > kMaxTokens) return ms_fail(MS_ERR_UNSUPPORTED, "embedding_sorted_backward: %d tokens, at most %d", n, kMaxTokens);
    if (!aligned(dx) || !aligned(d_table) || !aligned(scratch)) return ms_fail(MS_ERR_UNSUPPORTED, "embedding_sorted_backward: dx, d_table and scratch must be 16-byte aligned");
    const SortScratch sc = carve(scratch, n, d, vocab);
    if (scratch_bytes < sc.bytes) return ms_fail(MS_ERR_WORKSPACE, "embedding_sorted_backward: scratch %zu < %zu bytes", scratch_bytes, sc.bytes);
    const int vpr = d / (dtype == MS_BF16 ? 8 : 4), tiles = ms_cdiv(n, kTile);
    const long total = (long)tiles * vpr;
    if (!ms_launch_fits((total + 255) / 256, 256)) return ms_fail(MS_ERR_UNSUPPORTED, "embedding_sorted_backward: %d tokens of %d columns are too many for one launch", n, d);
    const SortPlan p = sort_plan(n, vocab);
    hipStream_t s = (hipStream_t)stream;
    ProfScope ps(11, (double)n * d * (ms_dtype_size(dtype) + 8.0), s);
    const long cb = (long)p.blocks * kBins;
    const bool many = p.blocks > 1;
    if (many) {
        sort_count_kernel<<<p.blocks, kSortThreads, 0, s>>>(ids, n, vocab, p.ipt * kSortThreads, (1 << p.bits) - 1, sc.counts, sc.counts + cb, (p.passes - 1) * cb);
        MS_LAUNCH_CHECK();
    }
    const uint2 *in = nullptr;
    for (int k = 0; k < p.passes; ++k) {
        uint2 *out = (k & 1) ? sc.b : sc.a;
        const int *counts = many ? sc.counts + k * cb : nullptr;
        int *next = many && k + 1 < p.passes ? sc.counts + (k + 1) * cb : nullptr;
#define GO(I) sort_pass_kernel<I><<<p.blocks, kSortThreads, 0, s>>>(k ? nullptr : ids, in, n, vocab, k * p.bits, p.bits, counts, next, (k + 1) * p.bits, out)
        if (p.ipt == 1) GO(1); else if (p.ipt == 4) GO(4); else GO(16);
#undef GO
        MS_LAUNCH_CHECK();
        in = out;
    }
    const int blocks = (int)((total + 255) / 256);
    if (dtype == MS_BF16) embedding_sum_kernel<bf16_t><<<blocks, 256, 0, s>>>(in, (const bf16_t *)dx, scale, n, vpr, vocab, d_table, sc.part, total);
    else embedding_sum_kernel<float><<<blocks, 256, 0, s>>>(in, (const float *)dx, scale, n, vpr, vocab, d_table, sc.part, total);
    MS_LAUNCH_CHECK();
    if (tiles > 1) {
        const int gy = ms_cdiv(d, 128);
        embedding_join_kernel<<<dim3(tiles, gy < 65535 ? gy : 65535), 256, 0, s>>>(in, sc.part, scale, n, d, tiles, vocab, d_table);
        MS_LAUNCH_CHECK();
    }
    return MS_OK;
}
