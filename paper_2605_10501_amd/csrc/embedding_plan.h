// Host-side rules of the sorted embedding gradient.  Plain C++ without HIP, so that they can be compiled and checked without a GPU.
#pragma once

constexpr int kSortThreads = 1024, kDigitBits = 9;
constexpr int kSmall = 4 * kSortThreads;  // tokens that one workgroup sorts in LDS
constexpr int kMaxTokens = 1 << 24;

constexpr long kSmallPieces = 16384L * 256;      // vectors of dx below which pieces have 8 places
// bits per digit, digits, tokens per thread and workgroups of the sort; places of a piece of the sums
struct SortPlan { int bits, passes, ipt, blocks, tile; };
inline SortPlan sort_plan(int n, int vocab, int vpr) {
    SortPlan p;
    int bits = 1;
    while (bits < 31 && (vocab >> bits) > 0) ++bits;                 // keys 0 .. vocab
    p.passes = (bits + kDigitBits - 1) / kDigitBits;
    p.bits = (bits + p.passes - 1) / p.passes;
    p.ipt = n <= 128 * kSortThreads ? 1 : n <= 512 * kSortThreads ? 4 : 16;
    p.blocks = n <= kSmall ? 1 : (int)((n + (long)p.ipt * kSortThreads - 1) / ((long)p.ipt * kSortThreads));
    // pieces of 8 places where 32 would leave the chip without work
    p.tile = (long)n * vpr < kSmallPieces ? 8 : 32;
    return p;
}
// dx by the non-temporal policy: n rows of vpr 16-byte vectors, more than 80 MB (pieces of 32 places then)
inline bool embedding_streams_dx(int n, int vpr) { return 16.0 * n * vpr > 80e6; }
