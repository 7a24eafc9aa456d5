// Host-side rules of the sorted embedding gradient.  Plain C++ without HIP, so that they can be compiled and checked without a GPU.
#pragma once

constexpr int kSortThreads = 1024, kDigitBits = 9;
constexpr int kSmall = 4 * kSortThreads;  // tokens that one workgroup sorts in LDS (us of the gradient, 8 columns: 1500 tokens 22.5, several workgroups 26.2; 4096 24.9 / 27.6)
constexpr int kMaxTokens = 1 << 24;

// Vectors of dx below which pieces have 8 places: 32 would leave the chip without work.  us of the gradient, 8 / 32 places: bf16 x 1536 1.0 M vectors 32 / 44, 2.1 M
// 45 / 46, 3.1 M 58 / 58, 4.2 M 77 / 67, 6.3 M 104 / 76; x 4096 1.0 M 28 / 40, 3.1 M 54 / 56, 4.2 M 73 / 64; fp32 x 768 1.0 M 30 / 35, 3.1 M 43 / 40, 4.2 M 51 / 48; narrow rows
// (bf16 x 256), whose sort weighs more, 1.0 M 44 / 47, 2.1 M 66 / 54.
constexpr long kSmallPieces = 16384L * 256;
// bits per digit, digits, tokens per thread and workgroups of the sort; places of a piece of the sums
struct SortPlan { int bits, passes, ipt, blocks, tile; };
inline SortPlan sort_plan(int n, int vocab, int vpr) {
    SortPlan p;
    int bits = 1;
    while (bits < 31 && (vocab >> bits) > 0) ++bits;                 // keys 0 .. vocab
    p.passes = (bits + kDigitBits - 1) / kDigitBits;
    p.bits = (bits + p.passes - 1) / p.passes;
    // more tokens per thread where every workgroup would read the counts of very many: us of the gradient, 8 columns, 1 / 4 / 16 tokens: 32768 tokens 38 / 45 / 81,
    // 131072 75 / 77 / 114, 200000 105 / 101 / 138, 524288 247 / 206 / 237, 1 M 553 / 360 / 412, 2 M 1512 / 715 / 733 (16 keep the counts of 16 M within 2 MB)
    p.ipt = n <= 128 * kSortThreads ? 1 : n <= 512 * kSortThreads ? 4 : 16;
    p.blocks = n <= kSmall ? 1 : (int)((n + (long)p.ipt * kSortThreads - 1) / ((long)p.ipt * kSortThreads));
    p.tile = (long)n * vpr < kSmallPieces ? 8 : 32;
    return p;
}
// dx by the non-temporal policy: n rows of vpr 16-byte vectors, more than 80 MB (pieces of 32 places then)
inline bool embedding_streams_dx(int n, int vpr) { return 16.0 * n * vpr > 80e6; }
