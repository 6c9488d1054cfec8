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

typedef __attribute__((address_space(3))) void* lds_ptr;
__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(lds_ptr)p; }

// Two blocks of codes of a weight row and their scales.
struct Codes {
    v4u c[2];
    uint32_t scale;
};
template <bool INSIDE>
__device__ __forceinline__ Codes load_pair(const uint8_t* row, const uint8_t* scales, uint32_t k, uint32_t cols) {
    typedef uint16_t loose __attribute__((aligned(1)));
    const uint32_t b = k / 16, blocks = (cols + kMxBlock - 1) / kMxBlock;
    Codes r;
#pragma unroll
    for (int h = 0; h < 2; ++h) r.c[h] = INSIDE ? load16<1>(row + k + 16 * h) : load_codes<false, true>(row, k + 16 * h, cols);
    r.scale = INSIDE || b + 2 <= blocks ? *gptr<loose>(scales + b) : b < blocks ? *gptr<uint8_t>(scales + b) : 0u;
    return r;
}

// How weights reach a wave that takes SIDES times 16 rows of them by itself, in steps of 128 bytes (256 elements). 16 lanes hold
// 16 rows, so a load by each lane of its own would be 64 accesses of 16 bytes. Where rows are 16-byte aligned (and their
// scales 4-byte), loads go to LDS directly, 8 lanes to a row's 128 bytes of a step, and each lane reads its row's there:
// chunk c of 16 bytes of row r lies in slot c ^ (r / 2 & 7), on other banks than those of the rows read with it. A step's buffer
// is SIDES * 16 rows of 128 bytes, and then their 8 scale bytes each (of one side twice: all lanes load, as a branch would
// hide from the compiler how many loads there are); a wave has as many as steps on their way, of its own, and needs no
// barrier for them.
template <int SIDES>
constexpr uint32_t kSlot = SIDES * 16 * 128 + (SIDES + 1) / 2 * 256;
template <int SIDES>
constexpr int kSlotLoads = SIDES * 2 + (SIDES + 1) / 2;

template <int SIDES>
struct Source {  // where a lane's part of the loads comes from
    const uint8_t* code[SIDES * 2];
    const uint8_t* scale[(SIDES + 1) / 2];
};
// row(side, r): the number of row r of a side
template <int SIDES, typename F>
__device__ __forceinline__ Source<SIDES> source_of(const uint8_t* codes, uint64_t ld, const uint8_t* scales, uint64_t ld_scale, F row) {
    const uint32_t lane = threadIdx.x & 63;
    Source<SIDES> src;
#pragma unroll
    for (int n = 0; n < SIDES * 2; ++n) {
        const uint32_t r = (n & 1) * 8 + (lane >> 3);
        src.code[n] = codes + row(n / 2, r) * ld + ((lane & 7) ^ (r >> 1 & 7)) * 16;
    }
#pragma unroll
    for (int n = 0; n < (SIDES + 1) / 2; ++n) src.scale[n] = scales + row(SIDES == 1 ? 0 : n * 2 + (lane >> 5), lane >> 1 & 15) * ld_scale + (lane & 1) * 4;
    return src;
}
// where a lane finds its own in a buffer: two chunks of codes, the second at the first ^ 16, and two scale bytes
__device__ __forceinline__ uint32_t code_place(uint32_t lane) { return (lane & 15) * 128 + ((2 * (lane >> 4)) ^ (lane >> 1 & 7)) * 16; }
__device__ __forceinline__ uint32_t scale_place(int sides, uint32_t lane) { return sides * 2048 + (lane & 15) * 8 + (lane >> 4) * 2; }
template <int SIDES>
__device__ __forceinline__ void load_to_lds(const Source<SIDES>& src, uint32_t s, char* slot) {
#pragma unroll
    for (int n = 0; n < SIDES * 2; ++n)
        __builtin_amdgcn_global_load_lds((const HCCL_AS1 void*)(src.code[n] + (uint64_t)s * 128), (lds_ptr)(slot + n * 1024), 16, 0, 0);
#pragma unroll
    for (int n = 0; n < (SIDES + 1) / 2; ++n)
        __builtin_amdgcn_global_load_lds((const HCCL_AS1 void*)(src.scale[n] + (uint64_t)s * 8), (lds_ptr)(slot + SIDES * 2048 + n * 256), 4, 0, 0);
}
// (in one block with the wait, as the compiler would have a read wait for every load to LDS there is)
__device__ __forceinline__ void read_from_lds(Codes (&c)[1], uint32_t at0, uint32_t at1, uint32_t scale) {
    asm volatile("ds_read_b128 %0, %3\n\tds_read_b128 %1, %4\n\tds_read_u16 %2, %5\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(c[0].c[0]), "=&v"(c[0].c[1]), "=&v"(c[0].scale)
                 : "v"(at0), "v"(at1), "v"(scale)
                 : "memory");
}
__device__ __forceinline__ void read_from_lds(Codes (&c)[2], uint32_t at0, uint32_t at1, uint32_t scale) {
    asm volatile("ds_read_b128 %0, %6\n\tds_read_b128 %1, %7\n\tds_read_b128 %3, %6 offset:2048\n\tds_read_b128 %4, %7 offset:2048\n\t"
                 "ds_read_u16 %2, %8\n\tds_read_u16 %5, %8 offset:128\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(c[0].c[0]), "=&v"(c[0].c[1]), "=&v"(c[0].scale), "=&v"(c[1].c[0]), "=&v"(c[1].c[1]), "=&v"(c[1].scale)
                 : "v"(at0), "v"(at1), "v"(scale)
                 : "memory");
}
__device__ __forceinline__ void read_from_lds(Codes (&c)[4], uint32_t at0, uint32_t at1, uint32_t scale) {
    Codes two[2];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        read_from_lds(two, at0 + n * 4096, at1 + n * 4096, scale + n * 256);
        c[n * 2] = two[0], c[n * 2 + 1] = two[1];
    }
}
template <int N>
__device__ __forceinline__ void wait_steps() {  // until at most N are on their way
    static_assert(N < 64, "the counter");
    __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | (N & 48) << 10);
}

}  // namespace
}  // namespace hccl
