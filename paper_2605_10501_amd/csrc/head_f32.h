// fp32 logits of many rows (head_f32.hip)
#pragma once
#include "common.h"

// Whether a block of that many rows takes them from here
bool head_f32_logits_tiled(long rows, long vocab);
// z [rows, cw] (rows ldz apart) = h w^T; operands 16-byte aligned, d a multiple of eight
ms_status head_f32_logits(int rows, int cw, int d, const float *h, const float *w, float *z, long ldz, hipStream_t s);
