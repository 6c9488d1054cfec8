// moe_mx_device.h -- microscaled 4-bit floats, as the kernels that make and read them share them.
//
// A row's elements lie two a byte, the lower half first; 32 neighbours (16 bytes of codes) have a scale byte b: element =
// code * 2^(b - 127), codes 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives (sign, two bits of exponent, one of mantissa).
// b = 255 is no number.
#pragma once
#include "moe_device.h"

namespace hccl {
namespace {

constexpr uint32_t kMxBlock = 32;

typedef _Float16 h2 __attribute__((ext_vector_type(2)));

// The scale of a block whose greatest magnitude has these bits: the least s >= -127 with m < 7 * 2^s, so that no code
// has to stand for a value further away than its neighbours are apart: b = s + 127 is m's exponent less 2, one more from a
// mantissa of 1.75 on. With an infinity or NaN it is no number.
__device__ __forceinline__ uint32_t mx_scale(uint32_t top) {
    const uint32_t e = (top + 0x00200000u) >> 23;
    return top >= 0x7f800000u ? 255u : e < 2 ? 0u : e - 2;
}
// 2^(b - 127) as the conversions take it: they read the exponent, and of an exponent of 0 that it is -127.
__device__ __forceinline__ float mx_power(uint32_t b) { return __uint_as_float(max(b << 23, 0x00400000u)); }

// Eight values to codes, nearest, ties to the even code.
__device__ __forceinline__ uint32_t mx_encode(const float (&x)[8], float power) {
    uint32_t r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0, x[0], x[1], power, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2], x[3], power, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4], x[5], power, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6], x[7], power, 3);
}
// The values of eight codes. (The byte is an operand of the instruction.)
__device__ __forceinline__ void mx_decode(uint32_t c, float power, float (&x)[8]) {
    const f2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, power, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, power, 1);
    const f2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, power, 2), e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, power, 3);
    x[0] = a[0], x[1] = a[1], x[2] = b[0], x[3] = b[1], x[4] = d[0], x[5] = d[1], x[6] = e[0], x[7] = e[1];
}

// silu(g) * u in 32 bits, with the hardware's 2^x and reciprocal.
__device__ __forceinline__ float mx_gate(float g, float u) {
    return g * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -1.44269504088896340736f)) * u;
}

// 16 bytes at byte k, a multiple of 16, of a row of `bytes`; those behind the last are zero (the row's last 16 bytes are
// moved down). LONG: the row has at least 16.
template <bool LONG>
__device__ __forceinline__ v4u load_bytes(const uint8_t* row, uint32_t k, uint32_t bytes) {
    if (k + 16 <= bytes) return load16<1>(row + k);
    v4u r = {0, 0, 0, 0};
    if (k >= bytes) return r;
    if (LONG || bytes >= 16) return shift_down(load16<1>(row + bytes - 16), 8 * (k + 16 - bytes));
#pragma unroll 1
    for (uint32_t i = bytes; i > 0; --i) {  // (k is 0) from the last byte on, each moves the others up
        r[3] = __builtin_amdgcn_alignbit(r[3], r[2], 24);
        r[2] = __builtin_amdgcn_alignbit(r[2], r[1], 24);
        r[1] = __builtin_amdgcn_alignbit(r[1], r[0], 24);
        r[0] = r[0] << 8 | *gptr<uint8_t>(row + i - 1);
    }
    return r;
}
// The codes of a row of `inner` elements at byte k; those behind the last are zero. ODD: the upper half of an odd row's
// last byte too (of one operand of a product; the other's is multiplied by that).
template <bool LONG, bool ODD>
__device__ __forceinline__ v4u load_codes(const uint8_t* row, uint32_t k, uint32_t inner) {
    const uint32_t bytes = (inner + 1) / 2;
    v4u v = load_bytes<LONG>(row, k, bytes);
    if (ODD && (inner & 1) && bytes <= k + 16) {
        const uint32_t at = (bytes - 1 - k) * 8;  // (great where the row ends before k)
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) v[i] &= at / 32 == i ? ~(0xf0u << (at & 31)) : ~0u;
    }
    return v;
}

}  // namespace
}  // namespace hccl
