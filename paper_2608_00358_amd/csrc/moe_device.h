// moe_device.h -- loads, stores and reductions that the kernels of the mixture-of-experts operators share.
#pragma once
#include <hip/hip_runtime.h>

#include <stdint.h>

#include "moe.h"

namespace hccl {
namespace {

constexpr uint32_t kWave = 64;
constexpr float kInf = __builtin_inff();

#define HCCL_AS1 __attribute__((address_space(1)))
template <typename T>
__device__ __forceinline__ const HCCL_AS1 T* gptr(const void* p) { return (const HCCL_AS1 T*)p; }
template <typename T>
__device__ __forceinline__ HCCL_AS1 T* gptr(void* p) { return (HCCL_AS1 T*)p; }

typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef __bf16 b2 __attribute__((ext_vector_type(2)));

// 16 bytes at the alignment of the elements: global accesses may be unaligned, so rows of any length
// and stride keep one wide access per lane.
template <int ES> struct Loose;
template <> struct Loose<1> { typedef uint32_t x4 __attribute__((ext_vector_type(4), aligned(1))); typedef uint32_t x2 __attribute__((ext_vector_type(2), aligned(1))); typedef uint32_t x1 __attribute__((aligned(1))); };
template <> struct Loose<2> { typedef uint32_t x4 __attribute__((ext_vector_type(4), aligned(2))); typedef uint32_t x2 __attribute__((ext_vector_type(2), aligned(2))); };
template <> struct Loose<4> { typedef uint32_t x4 __attribute__((ext_vector_type(4), aligned(4))); typedef uint32_t x2 __attribute__((ext_vector_type(2), aligned(4))); };

template <int DT> constexpr int kSize = DT == hcclFp32 ? 4 : 2;
template <int DT> constexpr int kVecOf = 16 / kSize<DT>;  // elements of a 16-byte vector

template <int DT>
__device__ __forceinline__ float widen1(uint32_t bits) {
    if constexpr (DT == hcclBf16) return __uint_as_float(bits << 16);
    else if constexpr (DT == hcclFp16) return (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
    else return __uint_as_float(bits);
}
// One rounding, to nearest with ties to even; values beyond the type's range become infinite.
template <int DT>
__device__ __forceinline__ uint32_t narrow1(float x) {
    if constexpr (DT == hcclBf16) return __builtin_bit_cast(uint16_t, (__bf16)x);
    else if constexpr (DT == hcclFp16) return __builtin_bit_cast(uint16_t, (_Float16)x);
    else return __float_as_uint(x);
}
template <int DT>
__device__ __forceinline__ void widen(const v4u& r, float (&x)[kVecOf<DT>]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (DT == hcclFp32) {
            x[i] = __uint_as_float(r[i]);
        } else if constexpr (DT == hcclBf16) {
            x[2 * i] = __uint_as_float(r[i] << 16);
            x[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
        } else {
            x[2 * i] = widen1<DT>(r[i] & 0xffffu);
            x[2 * i + 1] = widen1<DT>(r[i] >> 16);
        }
    }
}
template <int DT>
__device__ __forceinline__ v4u narrow(const float (&x)[kVecOf<DT>]) {
    v4u w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (DT == hcclFp32) {
            w[i] = __float_as_uint(x[i]);
        } else if constexpr (DT == hcclBf16) {
            const f2 v = {x[2 * i], x[2 * i + 1]};
            w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, b2));
        } else {
            w[i] = narrow1<DT>(x[2 * i]) | (narrow1<DT>(x[2 * i + 1]) << 16);
        }
    }
    return w;
}

template <int ES>
__device__ __forceinline__ v4u load16(const void* p) { return (v4u)*gptr<typename Loose<ES>::x4>(p); }
template <int ES>
__device__ __forceinline__ void store16(void* p, v4u v) { *gptr<typename Loose<ES>::x4>(p) = (typename Loose<ES>::x4)v; }

template <int ES>
__device__ __forceinline__ uint32_t load1(const void* p) {
    if constexpr (ES == 2) return *gptr<uint16_t>(p);
    else return *gptr<uint32_t>(p);
}
template <int ES>
__device__ __forceinline__ void store1(void* p, uint32_t v) {
    if constexpr (ES == 2) *gptr<uint16_t>(p) = (uint16_t)v;
    else *gptr<uint32_t>(p) = v;
}

// Vector `e / V` of a row of `cols` elements that begins at p; elements past the end are zero.
template <int ES>
__device__ __forceinline__ v4u load_row(const char* p, uint64_t e, uint64_t cols) {
    constexpr int V = 16 / ES;
    if (e + V <= cols) return load16<ES>(p + e * ES);
    v4u r = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (e + i < cols) {
            const uint32_t b = load1<ES>(p + (e + i) * ES);
            if constexpr (ES == 2) r[i / 2] |= b << (16 * (i & 1));
            else r[i] = b;
        }
    return r;
}
template <int ES>
__device__ __forceinline__ void store_row(char* p, uint64_t e, uint64_t cols, const v4u& r) {
    constexpr int V = 16 / ES;
    if (e + V <= cols) return store16<ES>(p + e * ES, r);
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (e + i < cols) {
            if constexpr (ES == 2) store1<ES>(p + (e + i) * ES, (r[i / 2] >> (16 * (i & 1))) & 0xffffu);
            else store1<ES>(p + (e + i) * ES, r[i]);
        }
}

// ---- reductions over groups of L lanes (16, 32 or 64); every lane gets the result
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);  // (every lane has a source)
}
constexpr int kQuadSwap = 0xB1, kQuadHalf = 0x4E, kHalfMirror = 0x141, kMirror = 0x140;

template <int L, typename OP>
__device__ __forceinline__ uint32_t fold_lanes(uint32_t v, OP op) {
    v = op(v, dpp<kQuadSwap>(v));
    v = op(v, dpp<kQuadHalf>(v));
    v = op(v, dpp<kHalfMirror>(v));  // (a quad's lanes agree by now, so mirrored lanes are as good as shifted ones)
    v = op(v, dpp<kMirror>(v));
    // the halves of 32 lanes, and of the wave, side by side in two registers
    if constexpr (L >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        v = op(r[0], r[1]);
    }
    if constexpr (L >= 64) {
        const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        v = op(r[0], r[1]);
    }
    return v;
}
template <int L>
__device__ __forceinline__ float max_lanes(float v) {
    return __uint_as_float(fold_lanes<L>(__float_as_uint(v), [](uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }));
}
template <int L>
__device__ __forceinline__ float sum_lanes(float v) {
    return __uint_as_float(fold_lanes<L>(__float_as_uint(v), [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}
template <int L>
__device__ __forceinline__ uint32_t maxu_lanes(uint32_t v) { return fold_lanes<L>(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; }); }
template <int L>
__device__ __forceinline__ uint32_t minu_lanes(uint32_t v) { return fold_lanes<L>(v, [](uint32_t a, uint32_t b) { return a < b ? a : b; }); }

__device__ __forceinline__ uint32_t first_lane(uint32_t v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ uint32_t at_lane(uint32_t v, uint32_t lane) { return __builtin_amdgcn_readlane(v, lane); }

}  // namespace
}  // namespace hccl
