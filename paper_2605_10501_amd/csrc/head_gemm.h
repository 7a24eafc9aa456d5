// Matrix products of the losses at the end of a section (head_gemm.hip); bf16, operands 16-byte aligned.
#pragma once
#include "common.h"
#include "head_choice.h"

// z = h w^T for `rows` rows (or *count of them, if that is given and less) and cw of the vocabulary's columns, d % 64 == 0; part [strips][ld] as the epilogues
// EPI_EXP and EPI_LOGITS (gemm_bf16.h) write it.  exp: ref = (reference, label) of each row,
// c = 2^(it2 z - reference), bf16, zeros up to the next multiple of 64 columns (c null: sums only), z_label the rows' logits of their labels (columns from v0 on), or, with marks, marks.z [rows, k] those of their selected ids;
// logits: c = z, fp32.
struct HeadMarks {
    const unsigned long long *word;          // [strips][ld] the selected columns of a strip and row (null: labels)
    const unsigned char *first;              // [strips][ld] how many selected ids of the row are in strips before it
    float *z;
    int k;
};
ms_status head_gemm_exp(int rows, int cw, int d, const void *h, const void *w, const float2 *ref, int v0, float *z_label, const HeadMarks &marks, float it2, void *c, long ldc, float2 *part, long ld,
                        const int *count, hipStream_t s);
ms_status head_gemm_logits(int rows, int cw, int d, const void *h, const void *w, float it2, float *c, long ldc, float2 *part, long ld, hipStream_t s);

// d_h (fp32) = e w and d_w [cw, d] (fp32) += e^T x, e [rows, cw] with rows ld apart and zeros up to the next multiple of 64 columns; either may be null.  d_h comes in
// c.parts parts [rows, d] (the vocabulary cut into as many, `rows` rows apart), += with `add`.  One accumulator per element, no atomics: the results do not
// depend on how a launch is scheduled.
ms_status head_gemm_backward(const HeadChoice &c, int rows, int cw, int d, const void *e, long ld, const void *w, const void *x, float *d_h, int add, float *d_w,
                             const int *count, hipStream_t s);
