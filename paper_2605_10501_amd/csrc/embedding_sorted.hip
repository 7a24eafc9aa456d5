// Embedding rows times a scale, and the table's gradient from the tokens sorted by id.
//
//   forward   x[t] = round(scale E[id_t])
//   backward  dE[v] += scale sum_{t: id_t = v} dx[t]: tokens in ascending order within pieces of 8 or 32 sorted places; of a run that spans pieces,
//             every fourth piece in ascending order, then those four sums
//
// The gradient needs no floating-point atomics: its sums have one order, so a run repeats bit for bit, and a row that thousands
// of tokens share (padding, frequent words) is not added to by thousands of atomics.  Steps:
//   1. stable radix sort of (id, token): per digit, a workgroup ranks its tokens and places them behind those of the workgroups
//      before it (per-workgroup digit counts; integer atomics in LDS, whose order does not matter).  Up to kSmall tokens one workgroup
//      does all digits in LDS.  Ids outside the table sort last.
//   2. pieces of 8 or 32 sorted places x one 16-byte column vector per thread: one pass over dx.  A run of equal ids that lies within
//      the piece is added to the table; what continues from or into a neighbour goes to a row of partial sums.
//   3. the runs that span pieces (step 2 lists them): their partial rows are added up, in four interleaved groups whose sums follow in order, and go to
//      the table.
// HBM bounds step 2 (dx read once, touched rows read and written), launches and latency the sort.
#include "common.h"
#include "embedding_plan.h"
#include "launch.h"
#include "launch_plan.h"

namespace {

constexpr int kWaves = kSortThreads / 64, kBins = 1 << kDigitBits;
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------------ forward
// Rows leave non-temporally, table rows stay: 32768 tokens x 1536 25.1 -> 23.1 us, x 4096 78 -> 63, 4096 x 1024 3.9 -> 3.3 (repeated passes, which find the
// batch's 12200 table rows in the caches; 35.9 us, 3.8 TB/s, for the first where they come from memory)
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
                    __builtin_nontemporal_store(*(const u32x4 *)&w, (u32x4 *)(o + q));
                }
            }
        }
    }
}

// ------------------------------------------------------------------ sort
__device__ __forceinline__ unsigned key_of(int id, int vocab) { return (unsigned)id < (unsigned)vocab ? (unsigned)id : (unsigned)vocab; }

// Digit counts of every workgroup's tokens.  (A pass that adds up the next one's counts with global atomics while it scatters saves this launch, but
// frequent ids share their upper digit: 16384 tokens of a vocabulary of 32000 15 us a pass instead of 4 and 3 for the counts.)
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(const int *__restrict__ ids, const uint2 *__restrict__ in, int n, int vocab, int per, int shift,
                                                                  int mask, int *__restrict__ counts, int *__restrict__ runs) {
    __shared__ int hist[kBins];
    const int tid = threadIdx.x;
    if (blockIdx.x == 0 && tid == 0) *runs = 0;
    if (tid < kBins) hist[tid] = 0;
    __syncthreads();
    const long b0 = (long)blockIdx.x * per;
    for (int i = tid; i < per && b0 + i < n; i += kSortThreads) atomicAdd(&hist[((ids ? key_of(ids[b0 + i], vocab) : in[b0 + i].x) >> shift) & mask], 1);
    __syncthreads();
    if (tid < kBins) counts[(long)blockIdx.x * kBins + tid] = hist[tid];
}

// Ranks of a workgroup's tokens by a digit: lanes of equal digits find each other by ballots, the first of them moves the wave's
// counter on.  A wave has 64 IPT consecutive places, 64 of them per trip; hist[w][digit] ends up as the wave's count.
template <int IPT>
__device__ __forceinline__ void rank_digit(const unsigned (&key)[IPT], const bool (&valid)[IPT], int shift, int bits, int *hist, int (&rank)[IPT]) {
    const int lane = threadIdx.x & 63, mask = (1 << bits) - 1;
#pragma unroll
    for (int r = 0; r < IPT; ++r) {
        const int dg = (key[r] >> shift) & mask;
        unsigned long long same = __ballot(valid[r]);
        for (int k = 0; k < bits; ++k) {
            const unsigned long long m = __ballot((dg >> k) & 1);
            same &= (dg >> k) & 1 ? m : ~m;
        }
        const int before = __popcll(same & ((1ull << lane) - 1)), cnt = __popcll(same);
        const int pre = hist[dg];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (valid[r] && before == 0) hist[dg] = pre + cnt;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        rank[r] = pre + before;
    }
}
// Prefix sum of the first kBins threads' values over the workgroup's digits (all threads call it)
__device__ __forceinline__ int scan_bins(int v, int *wsum) {
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    int inc = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(inc, o, 64);
        if (lane >= o) inc += u;
    }
    if (lane == 63 && wv < kBins / 64) wsum[wv] = inc;
    __syncthreads();
    int add = 0;
#pragma unroll
    for (int w = 0; w < kBins / 64; ++w) add += w < wv ? wsum[w] : 0;
    return inc - v + add;
}

// One stable pass by the digit (key >> shift) & mask.  ids != null: the keys are the ids and the values the token numbers.
// counts: [workgroups][kBins] of this digit.
template <int IPT>
__global__ __launch_bounds__(kSortThreads) void sort_pass_kernel(const int *__restrict__ ids, const uint2 *__restrict__ in, int n, int vocab, int shift,
                                                                 int bits, const int *__restrict__ counts, uint2 *__restrict__ out) {
    __shared__ int hist[kWaves][kBins];
    __shared__ int base[kBins];
    __shared__ int wsum[kBins / 64];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, mask = (1 << bits) - 1, per = kSortThreads * IPT;
    const long b0 = (long)blockIdx.x * per + wv * 64 * IPT;
    uint2 kv[IPT];
    unsigned key[IPT];
    bool valid[IPT];
    int rank[IPT];
#pragma unroll
    for (int r = 0; r < IPT; ++r) {
        const long i = b0 + r * 64 + lane;
        valid[r] = i < n;
        kv[r] = make_uint2(0, 0);
        if (valid[r]) kv[r] = ids ? make_uint2(key_of(ids[i], vocab), (unsigned)i) : in[i];
        key[r] = kv[r].x;
    }
    // all tokens of a digit, and those of the workgroups in front: two threads per digit, eight rows requested at a time
    int total = 0, ahead = 0;
    {
        const int d = tid & (kBins - 1), nb = gridDim.x, mine = blockIdx.x;
        for (int b = tid >> kDigitBits; b < nb; b += 16) {
            int c[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) c[u] = b + 2 * u < nb ? counts[(long)(b + 2 * u) * kBins + d] : 0;
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                total += c[u];
                ahead += b + 2 * u < mine ? c[u] : 0;
            }
        }
    }
    for (int i = tid; i < kWaves * kBins; i += kSortThreads) (&hist[0][0])[i] = 0;
    __syncthreads();
    rank_digit<IPT>(key, valid, shift, bits, hist[wv], rank);
    int *half = base;                                    // the upper half's sums on their way to the lower
    if (tid >= kBins) half[tid - kBins] = total;
    __syncthreads();
    if (tid < kBins) total += half[tid];
    __syncthreads();
    if (tid >= kBins) half[tid - kBins] = ahead;
    __syncthreads();
    if (tid < kBins) {
        ahead += half[tid];
        int before = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const int c = hist[w][tid];
            hist[w][tid] = before;
            before += c;
        }
    }
    const int first = scan_bins(tid < kBins ? total : 0, wsum);
    if (tid < kBins) base[tid] = first + ahead;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < IPT; ++r) {
        if (valid[r]) {
            const int dg = (key[r] >> shift) & mask;
            out[base[dg] + hist[wv][dg] + rank[r]] = kv[r];
        }
    }
}

// All digits of up to kSmall tokens in one workgroup
template <int IPT>
__global__ __launch_bounds__(kSortThreads) void sort_small_kernel(const int *__restrict__ ids, int n, int vocab, int bits, int passes, uint2 *__restrict__ out,
                                                                  int *__restrict__ runs) {
    __shared__ int hist[kWaves][kBins];
    __shared__ int base[kBins];
    __shared__ int wsum[kBins / 64];
    __shared__ uint2 item[kSortThreads * IPT];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, mask = (1 << bits) - 1, b0 = wv * 64 * IPT;
    if (tid == 0) *runs = 0;
    uint2 kv[IPT];
    unsigned key[IPT];
    bool valid[IPT];
    int rank[IPT];
#pragma unroll
    for (int r = 0; r < IPT; ++r) {
        const int i = b0 + r * 64 + lane;
        valid[r] = i < n;
        kv[r] = valid[r] ? make_uint2(key_of(ids[i], vocab), (unsigned)i) : make_uint2(0, 0);
    }
    for (int p = 0; p < passes; ++p) {
        const int shift = p * bits;
#pragma unroll
        for (int r = 0; r < IPT; ++r) {
            if (p && valid[r]) kv[r] = item[b0 + r * 64 + lane];
            key[r] = kv[r].x;
        }
        for (int i = tid; i < kWaves * kBins; i += kSortThreads) (&hist[0][0])[i] = 0;
        __syncthreads();
        rank_digit<IPT>(key, valid, shift, bits, hist[wv], rank);
        __syncthreads();
        int total = 0;
        if (tid < kBins) {
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const int c = hist[w][tid];
                hist[w][tid] = total;
                total += c;
            }
        }
        const int first = scan_bins(total, wsum);
        if (tid < kBins) base[tid] = first;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < IPT; ++r) {
            if (!valid[r]) continue;
            const int dg = (key[r] >> shift) & mask, at = base[dg] + hist[wv][dg] + rank[r];
            if (p + 1 == passes) out[at] = kv[r];
            else item[at] = kv[r];
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------ sums
// part: [pieces][2][d]: row 0 the end of a run that began in an earlier piece, row 1 the part of a run that goes on in the next.
// runs[0] counts, runs[1 ..] list the pieces in which a run begins that goes on (in any order: each is added up by itself).
// U places at a time: their rows of dx and the table rows of the runs that end there are requested together.  STREAM: dx by the non-temporal policy,
// above 80 MB (us of the whole gradient, without / with, x 1536 in bf16: 34 MB 49 / 50, 50 MB 60 / 56, 67 MB 66 / 62, 101 MB 80 / 76, 202 MB 148 / 135; x 768 in fp32: 34
// MB 38 / 40, 50 MB 42 / 44, 67 MB 48 / 48, 101 MB 62 / 58, 202 MB 101 / 91).
template <class T, int TILE, int U, bool STREAM>
__global__ __launch_bounds__(256) void embedding_sum_kernel(const uint2 *__restrict__ sorted, const T *__restrict__ dx, float scale, int n, int vpr,
                                                            int vocab, float *__restrict__ d_table, float *__restrict__ part, int *__restrict__ runs,
                                                            long total) {
    constexpr int V = Vec16<T>::N;
    const long i = (long)blockIdx.x * 256 + threadIdx.x;
    if (i >= total) return;
    const int tile = (int)(total < 0x7fffffff ? (unsigned)i / (unsigned)vpr : i / vpr);
    const long d = (long)vpr * V, cv = (i - (long)tile * vpr) * V;
    const int p0 = tile * TILE, p1 = p0 + TILE < n ? p0 + TILE : n;
    const unsigned before = p0 > 0 ? sorted[p0 - 1].x : 0xffffffffu, after = p1 < n ? sorted[p1].x : 0xffffffffu;
    float acc[V];
#pragma unroll
    for (int e = 0; e < V; ++e) acc[e] = 0.f;
    auto store = [&](float *o) {
#pragma unroll
        for (int q = 0; q < V; q += 4) *(float4 *)(o + q) = make_float4(acc[q], acc[q + 1], acc[q + 2], acc[q + 3]);
    };
    bool from_before = before != 0xffffffffu && sorted[p0].x == before;      // the present run began in an earlier piece
    bool open = false;                                                       // a run goes on in the next piece, and began here
    for (int p = p0; p < p1; p += U) {
        uint2 kv[U + 1];
        Vec16<T> v[U];
        float4 old[U][V / 4];
        bool end[U];
#pragma unroll
        for (int u = 0; u < U; ++u) kv[u] = sorted[p + u < p1 ? p + u : p1 - 1];
        kv[U].x = p + U < p1 ? sorted[p + U].x : after;
        const bool fb = from_before;
        bool seen = false;                                                   // a run has ended among these places
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const unsigned nextk = p + u + 1 < p1 ? kv[u + 1].x : after;
            end[u] = p + u < p1 && kv[u].x != nextk;
            if (p + u < p1 && kv[u].x < (unsigned)vocab) {
                if constexpr (STREAM) *(u32x4 *)&v[u] = __builtin_nontemporal_load((const u32x4 *)(dx + (long)kv[u].y * d + cv));
                else v[u] = ldv(dx + (long)kv[u].y * d + cv);
                if (end[u] && (seen || !fb)) {
                    const float *o = d_table + (long)kv[u].x * d + cv;
#pragma unroll
                    for (int q = 0; q < V / 4; ++q) old[u][q] = *(const float4 *)(o + 4 * q);
                }
            }
            seen |= end[u];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (p + u >= p1) break;
            const bool in = kv[u].x < (unsigned)vocab;
            if (in)
#pragma unroll
                for (int e = 0; e < V; ++e) acc[e] += to_f32(v[u].v[e]);
            if (end[u]) {
                if (in && from_before) {
                    store(part + (long)tile * 2 * d + cv);
                } else if (in) {
                    float *o = d_table + (long)kv[u].x * d + cv;
#pragma unroll
                    for (int q = 0; q < V / 4; ++q) {
                        const float4 t = old[u][q];
                        *(float4 *)(o + 4 * q) = make_float4(__builtin_fmaf(scale, acc[4 * q], t.x), __builtin_fmaf(scale, acc[4 * q + 1], t.y),
                                                             __builtin_fmaf(scale, acc[4 * q + 2], t.z), __builtin_fmaf(scale, acc[4 * q + 3], t.w));
                    }
                }
                from_before = false;
#pragma unroll
                for (int e = 0; e < V; ++e) acc[e] = 0.f;
            } else if (p + u + 1 == p1 && in) {
                store(part + ((long)tile * 2 + 1) * d + cv);
                open = !from_before;
            }
        }
    }
    if (open && cv == 0) runs[1 + atomicAdd(runs, 1)] = tile;
}

// The runs that span pieces.  A task is one of them and 256 columns: four row groups of 64 threads take every fourth partial row, eight
// requested at a time; their sums are added in order.
template <int TILE>
__global__ __launch_bounds__(256) void embedding_join_kernel(const uint2 *__restrict__ sorted, const float *__restrict__ part, float scale, int n, long d,
                                                             float *__restrict__ d_table, const int *__restrict__ runs) {
    __shared__ float4 sm[4][64];
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, strips = (int)((d + 255) / 256), tiles = (n + TILE - 1) / TILE;
    const long tasks = (long)runs[0] * strips;
    for (long k = blockIdx.x; k < tasks; k += gridDim.x) {
        const int tile = runs[1 + k / strips];
        const long col = (k % strips) * 256 + 4 * lane;
        const unsigned run = sorted[(long)(tile + 1) * TILE].x;
        int last = tile + 1;                             // the piece in which the run ends: 64 pieces are looked at together
        for (;; last += 64) {
            const int q = last + 1 + lane;
            const unsigned long long on = __ballot(q < tiles && sorted[(long)(q < tiles ? q : 0) * TILE].x == run);
            if (~on) { last += __ffsll(~on) - 1; break; }
        }
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
        if (col < d) {
            for (int q = tile + wv; q <= last; q += 32) {
                float4 v[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const int t = q + 4 * u;
                    v[u] = t <= last ? *(const float4 *)(part + ((long)t * 2 + (t < last)) * d + col) : make_float4(0.f, 0.f, 0.f, 0.f);
                }
#pragma unroll
                for (int u = 0; u < 8; ++u) { s.x += v[u].x; s.y += v[u].y; s.z += v[u].z; s.w += v[u].w; }
            }
        }
        sm[wv][lane] = s;
        __syncthreads();
        if (wv == 0 && col < d) {
#pragma unroll
            for (int w = 1; w < 4; ++w) {
                const float4 v = sm[w][lane];
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

struct SortScratch { uint2 *a, *b; int *counts, *runs; float *part; size_t bytes; };
SortScratch carve(void *ws, const SortPlan &p, int n, int d) {
    const size_t tiles = (size_t)ms_cdiv(n, p.tile);
    Arena a(ws);
    SortScratch s;
    s.a = a.take<uint2>((size_t)n * 8);
    s.b = a.take<uint2>((size_t)n * 8);
    s.counts = a.take<int>((size_t)p.blocks * kBins * 4);
    s.runs = a.take<int>((tiles + 1) * 4);
    s.part = a.take<float>(tiles * 2 * d * 4);
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
    // never less than for fewer tokens: where pieces or sorting workgroups grow, the count before that may need more (pieces are as small for
    // either type as for the one with fewer vectors per row)
    const int at[] = {n, kSmall, 128 * kSortThreads, 512 * kSortThreads, d / 8 > 0 ? (int)((kSmallPieces - 1) / (d / 8)) : n};
    size_t most = 0;
    for (int m : at) {
        if (m > n || m <= 0) continue;
        const size_t b = carve(nullptr, sort_plan(m, vocab, d / 8), m, d).bytes;
        most = b > most ? b : most;
    }
    return most;
}

extern "C" ms_status ms_k_embedding_sorted_backward(int32_t dtype, int32_t n, int32_t d, int32_t vocab, float scale, const int32_t *ids,
                                                    const void *dx, float *d_table, void *scratch, size_t scratch_bytes, void *stream) {
    if (n == 0) return MS_OK;
    MS_TRY(check("embedding_sorted_backward", dtype, n, d, vocab));
    if (!ids || !dx || !d_table || !scratch) return ms_fail(MS_ERR_INVALID_ARG, "embedding_sorted_backward: null pointer");
    if (n > kMaxTokens) return ms_fail(MS_ERR_UNSUPPORTED, "embedding_sorted_backward: %d tokens, at most %d", n, kMaxTokens);
    if (!aligned(dx) || !aligned(d_table) || !aligned(scratch)) return ms_fail(MS_ERR_UNSUPPORTED, "embedding_sorted_backward: dx, d_table and scratch must be 16-byte aligned");
    const int vpr = d / (dtype == MS_BF16 ? 8 : 4);
    const SortPlan p = sort_plan(n, vocab, vpr);
    const SortScratch sc = carve(scratch, p, n, d);
    const size_t need = ms_k_embedding_sorted_backward_scratch_bytes(n, d, vocab);
    if (scratch_bytes < need) return ms_fail(MS_ERR_WORKSPACE, "embedding_sorted_backward: scratch %zu < %zu bytes", scratch_bytes, need);
    const int tiles = ms_cdiv(n, p.tile);
    const long total = (long)tiles * vpr;
    if (!ms_launch_fits((total + 255) / 256, 256)) return ms_fail(MS_ERR_UNSUPPORTED, "embedding_sorted_backward: %d tokens of %d columns are too many for one launch", n, d);
    hipStream_t s = (hipStream_t)stream;
    ProfScope ps(11, (double)n * d * (ms_dtype_size(dtype) + 8.0), s);
    const uint2 *in = nullptr;
    if (p.blocks == 1) {
        if (n <= kSortThreads) sort_small_kernel<1><<<1, kSortThreads, 0, s>>>(ids, n, vocab, p.bits, p.passes, sc.a, sc.runs);
        else sort_small_kernel<4><<<1, kSortThreads, 0, s>>>(ids, n, vocab, p.bits, p.passes, sc.a, sc.runs);
        MS_LAUNCH_CHECK();
        in = sc.a;
    } else {
        for (int k = 0; k < p.passes; ++k) {
            uint2 *out = (k & 1) ? sc.b : sc.a;
            const int *first = k ? nullptr : ids;
            sort_count_kernel<<<p.blocks, kSortThreads, 0, s>>>(first, in, n, vocab, p.ipt * kSortThreads, k * p.bits, (1 << p.bits) - 1, sc.counts, sc.runs);
            MS_LAUNCH_CHECK();
#define GO(I) sort_pass_kernel<I><<<p.blocks, kSortThreads, 0, s>>>(first, in, n, vocab, k * p.bits, p.bits, sc.counts, out)
            if (p.ipt == 1) GO(1); else if (p.ipt == 4) GO(4); else GO(16);
#undef GO
            MS_LAUNCH_CHECK();
            in = out;
        }
    }
    const int blocks = (int)((total + 255) / 256), strips = ms_cdiv(d, 256);
    const long tasks = (long)(tiles - 1) * strips;       // at most
    const bool stream_dx = embedding_streams_dx(n, vpr);
#define GO(T, TILE, U, ST) embedding_sum_kernel<T, TILE, U, ST><<<blocks, 256, 0, s>>>(in, (const T *)dx, scale, n, vpr, vocab, d_table, sc.part, sc.runs, total)
    if (dtype == MS_BF16) { if (p.tile == 8) GO(bf16_t, 8, 8, false); else if (stream_dx) GO(bf16_t, 32, 4, true); else GO(bf16_t, 32, 4, false); }
    else { if (p.tile == 8) GO(float, 8, 8, false); else if (stream_dx) GO(float, 32, 8, true); else GO(float, 32, 8, false); }
#undef GO
    MS_LAUNCH_CHECK();
    if (tasks > 0) {
        const int grid = (int)(tasks < 2048 ? tasks : 2048);
        if (p.tile == 8) embedding_join_kernel<8><<<grid, 256, 0, s>>>(in, sc.part, scale, n, d, d_table, sc.runs);
        else embedding_join_kernel<32><<<grid, 256, 0, s>>>(in, sc.part, scale, n, d, d_table, sc.runs);
        MS_LAUNCH_CHECK();
    }
    return MS_OK;
}
