// What the kernels that write 8-bit operands share: e4m3 codes with one power-of-two scale for each block of 128.
#pragma once
#include "common.h"

// Scale byte (2^(byte - 127)) of a block whose largest finite magnitude has the given bits: the least power of two that brings it to
// 448 = 1.75 * 2^8, the largest e4m3 number, or below; 1 for a block of zeros.  A power of two, because then scaling
// rounds nothing, the codes keep their relative step whatever the scale, and the matrix cores take the exponents as operands.
__device__ __forceinline__ int fp8_scale_byte(unsigned amax_bits) {
    const int b = (int)(amax_bits >> 23) - 8 + ((amax_bits & 0x7fffffu) > 0x600000u);
    return amax_bits == 0 ? 127 : b < 0 ? 0 : b;
}
__device__ __forceinline__ float fp8_inverse_scale(int byte) { return __uint_as_float((unsigned)(254 - byte) << 23); }

// Bits of |v| if v is finite, else 0: infinities and NaN do not set their block's scale (their codes are NaN, e4m3 has no infinity)
__device__ __forceinline__ unsigned fp8_finite_bits(float v) {
    const unsigned b = __float_as_uint(v) & 0x7fffffffu;
    return b < 0x7f800000u ? b : 0u;
}

// silu(g) u, with the reciprocal instruction (1 ulp) instead of a division: the result is rounded to four bits.  One function, because whether an
// epilogue or a pass of its own takes it depends on the sizes, and the codes must not.
__device__ __forceinline__ float fp8_silu_mul(float g, float u) {
#pragma clang fp contract(off)
    return g * __builtin_amdgcn_rcpf(1.f + __expf(-g)) * u;
}

__device__ __forceinline__ unsigned fp8_pack4(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// Maximum over 16 lanes, which are a row of the wave: by the vector ALU's lane permutations (pairs, quads, halves, mirror image), without a trip
// through LDS
__device__ __forceinline__ unsigned fp8_max16(unsigned m) {
    m = max(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xf, 0xf, true));        // quad_perm 1 0 3 2
    m = max(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xf, 0xf, true));        // quad_perm 2 3 0 1
    m = max(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0x141, 0xf, 0xf, true));       // row_half_mirror
    return max(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0x140, 0xf, 0xf, true));    // row_mirror
}

// Eight consecutive columns per lane, 16 lanes per block: codes and scale byte of the block
__device__ __forceinline__ uint2 fp8_quantize8(const float *v, int *byte) {
    unsigned m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(v[e]) & 0x7fffffffu);
    if (__builtin_expect(__any(m >= 0x7f800000u), 0)) {
        m = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) m = max(m, fp8_finite_bits(v[e]));
    }
    m = fp8_max16(m);
    *byte = fp8_scale_byte(m);
    const float s = fp8_inverse_scale(*byte);
    return make_uint2(fp8_pack4(v[0] * s, v[1] * s, v[2] * s, v[3] * s), fp8_pack4(v[4] * s, v[5] * s, v[6] * s, v[7] * s));
}
// The four blocks of a wave, as the word of their scales: blocks past the last one get 127
__device__ __forceinline__ unsigned fp8_scale_word(int byte, int block, int blocks) {
    const unsigned v = block < blocks ? (unsigned)byte : 127u;
    return (unsigned)__builtin_amdgcn_readlane((int)v, 0) | (unsigned)__builtin_amdgcn_readlane((int)v, 16) << 8 |
           (unsigned)__builtin_amdgcn_readlane((int)v, 32) << 16 | (unsigned)__builtin_amdgcn_readlane((int)v, 48) << 24;
}

template <class T> __device__ __forceinline__ void fp8_load8(const T *p, float *v) {
    if constexpr (sizeof(T) == 2) {
        const Vec16<T> t = ldv(p);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = to_f32(t.v[e]);
    } else {
        const float4 a = *(const float4 *)p, b = *(const float4 *)(p + 4);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
}
