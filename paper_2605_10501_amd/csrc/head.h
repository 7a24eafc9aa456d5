// Losses and log-probabilities at the end of a decoder section (head.hip): what a call needs of the workspace, and which calls are
// accepted.  No device code: this part also builds for the host alone.
#pragma once
#include "common.h"
#include "head_choice.h"

constexpr int kHeadMaxTop = 128;             // entries of a token that the kernels hold
constexpr int kHeadFixes = 4;                // of a token's entries whose gradients are completed in fp32
constexpr int kHeadScan = 8192;              // rows of such, up to which each looks for the others of its id by itself
constexpr int kStrip = 64;                   // columns that share one partial sum

// Rows of hidden states meet the vocabulary a block of tokens at a time.  What a block keeps of every (row, vocabulary entry) lies in
// slabs of `cols` columns, [slab][rows][cols], because a matrix product's operand has to be within reach of 32-bit offsets.
struct HeadPlan {
    int block, rows, cols, slabs, strips;    // tokens of a block, rows that there is room for; strips over all slabs, cols / kStrip in each but the last
    bool fast;                               // bf16 products whose epilogue meets the logits (head_gemm.hip)
    bool tiles;                              // the gradients are products of head_gemm.hip too (bf16)
    int *slot, *token, *count;               // [rows] row of a token, [rows] token of a row (-1: none), [1] rows in use
    void *h;                                 // [rows, hidden] hidden states of the rows, later times the row's factor
    float2 *ref;                             // [rows] reference of a row's exponentials (in x) and its label as an int (-1: it has entries)
    float *scale, *factor;                   // [rows] dz = scale q of a row; the factor of what is stored of it
    float2 *stat;                            // [rows] sum of exponentials and its reference
    float *z_label;                          // [rows] a label's logit as the matrix product has it
    float *z_sel, *rho;                      // [rows, k] logits at the selected ids, and what a row has there in its gradient
    float *log_p, *mass;                     // [rows, k], [rows] of the teacher's entries
    int *ids;                                // [rows, k] the entries that count (-1: ignored)
    int *best;                               // [rows] the entry that the teacher thinks most of
    unsigned long long *marks;               // [strips, rows] which columns of a strip are among a row's entries, and how many entries are before them; null: the entries'
    unsigned char *marks_first;              // logits are dot products of their own
    int *key;                                // [rows] < 0: the token is left out
    float *logp;                             // [rows] by token of the block
    float2 *part;                            // [strips, rows]
    int fixes;                               // selected ids of a row whose part of the gradients is completed in fp32 (fast)
    int *fix_id;                             // [rows, fixes], -1: none
    float *fix_rest;                         // [rows, fixes] what the stored gradient of the logit lacks
    void *fix, *fix_scratch;                 // [rows fixes, hidden] what d_w's row lacks; for the sum over the rows of an id
    size_t fix_scratch_bytes;
    HeadChoice choice;                       // of the gradients' products (tiles)
    int parts;                               // of d_h
    float *d_h;                              // [parts, rows, hidden]
    void *z;                                 // slabs: logits (fp32), or their exponentials (bf16)
    void *dz, *dz_rest;                      // [rows, cols] gradient of a slab's logits where it does not take the logits' place, and what it lacks of fp32 (null: not taken along)
    float *per_token, *margin;               // [n] terms of the loss, or [pairs] both
    size_t bytes;
};

enum HeadUse { HEAD_TOP = 0, HEAD_FORWARD = 1, HEAD_BACKWARD = 2 };

// Whether the logits of a row's k entries come out of the matrix product by marks, or are dot products of their own.  A dot product of d numbers takes 0.26 d ps (its row of w comes from
// behind the L2s); marks take 8 ps for every strip and row, to clear, set and look at (32768 tokens, V = 151936, d = 1536, 64 entries: 0.85 and 0.7 ms; 32000 tokens, V = 32000,
// d = 1024, 100 entries: 0.95 and 0.25).
constexpr bool head_use_marks(long k, long d, long strips) { return k > 1 && k * d > 31 * strips; }

// The storage type, and whether a bf16 head keeps the gradient of its logits in two bf16 numbers
inline int head_dtype(const ms_head_config *c) { return c->dtype & ~MS_HEAD_FP32_DZ; }
inline bool head_fp32_dz(const ms_head_config *c) { return (c->dtype & MS_HEAD_FP32_DZ) != 0; }

// pairs >= 0: a preference loss of that many pairs, all n tokens in one block
HeadPlan head_plan(const ms_head_config *c, int n, int k, HeadUse use, int pairs, void *ws);
long head_most_rows(const ms_head_config *c, HeadUse use = HEAD_BACKWARD);   // of a block
ms_status validate_head(const ms_head_config *c, int n, int k, const char *what);
