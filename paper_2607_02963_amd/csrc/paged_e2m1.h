// 4-bit cache rows: e2m1 values (0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign), two to a
// byte, the even element in the low half, with one power of two per 32 elements of a
// row, 2^(byte - 127); a byte of 255 makes its elements NaN.
//
// A head's tokens lie one after another in a page, [num_pages, H_kv, page_size, D / 2],
// and so do their scales, [num_pages, H_kv, page_size, D / 32]: 16 keys of a head, the
// least that is always on one page, are 1 KB at D = 128, one DMA instruction and whole
// cache lines (token-major, a head's row would be half a line).
#pragma once

#include "kernel_mfma.h"
#include "paged_common.h"

namespace pdec {

constexpr int kE2m1Block = 32;  // elements to a scale

// A head's row of a page, counted in rows.
__device__ inline long e2m1_row(long page, int head, int H_kv, int page_shift, int slot)
{
    return ((page * H_kv + head) << page_shift) + slot;
}

// 2^(byte - 127) as v_cvt_scalef32_* take it: they read the exponent's bits, 0 as 2^-127
// and 255 as NaN.
__device__ inline float e2m1_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// Eight values of one scale as bf16: exact, but for the least scales' subnormals.
__device__ inline u32x4_t e2m1_bf16(uint32_t w, float scale)
{
    u32x4_t r;
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
    return r;
}

// The same as float32: exact.
__device__ inline void e2m1_f32(uint32_t w, float scale, float (&v)[8])
{
    const f32x2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1);
    const f32x2_t c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3);
    v[0] = a.x, v[1] = a.y, v[2] = b.x, v[3] = b.y, v[4] = c.x, v[5] = c.y, v[6] = d.x, v[7] = d.y;
}

// Eight elements of a row as e2m1, four lanes to a scale: its byte in `byte`, the same in
// the four.  |x| 2^-k is at most 6, but for magnitudes beyond 6 * 2^125, which become that
// (a larger power of two would let a rounded-up value pass float32's range when read back).
// To nearest even: a rounding is off by at most 2^-2 of the value, or 2^(k-2).  An infinity
// or NaN makes its 32 elements NaN, stored as zeros with a byte of 255: zeros because the
// attention multiplies a key's probability by the scale, and only 0 times that infinity is NaN.
__device__ inline uint32_t quantise4(const float (&x)[8], int& byte)
{
    uint32_t top = 0;  // |x| as its bits, which order as the values do
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
    top = max(top, (uint32_t)__shfl_xor((int)top, 1));
    top = max(top, (uint32_t)__shfl_xor((int)top, 2));
    if (top >= 0x7f800000u) {
        byte = 255;
        return 0;
    }
    // top = m 2^e, 1 <= m < 2, and 6 = 1.5 * 2^2: k = e - 2, one more where m > 1.5
    int k = (int)(top >> 23) - 127 - 2 + ((top & 0x7fffffu) > 0x400000u ? 1 : 0);
    k = top ? min(max(k, -126), 125) : 0;
    byte = k + 127;
    const float inv = __uint_as_float((uint32_t)(127 - k) << 23);  // 2^-k: exact
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0] * inv, x[1] * inv, 1.f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2] * inv, x[3] * inv, 1.f, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4] * inv, x[5] * inv, 1.f, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6] * inv, x[7] * inv, 1.f, 3);
    return w;
}

}  // namespace pdec
