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

// The 16 bytes of v moved down by `bits` (0 .. 127), with zeros from above. In 32-bit operations: a 64-bit shift
// whose amount lies in the last register that a wave has gives wrong bits now and then, and the compiler does put
// it there (products of 16-bit results and 256 x 256 tiles with rows of odd strides were wrong by it).
__device__ __forceinline__ v4u shift_down(const v4u& v, uint32_t bits) {
    const bool two = bits & 64, one = bits & 32;
    const uint32_t a0 = two ? v[2] : v[0], a1 = two ? v[3] : v[1], a2 = two ? 0 : v[2], a3 = two ? 0 : v[3];
    const uint32_t b0 = one ? a1 : a0, b1 = one ? a2 : a1, b2 = one ? a3 : a2, b3 = one ? 0 : a3;
    return v4u{__builtin_amdgcn_alignbit(b1, b0, bits), __builtin_amdgcn_alignbit(b2, b1, bits),
               __builtin_amdgcn_alignbit(b3, b2, bits), __builtin_amdgcn_alignbit(0, b3, bits)};
}

// The vector at element e of a row of `cols` elements (at least one) that begins at p; elements past the end
// are zero. The row's last vector is read where the one asked for would pass the end, and moved down: one
// load for every lane, where element by element each would wait for the one before.
template <int ES>
__device__ __forceinline__ v4u load_row(const char* p, uint64_t e, uint64_t cols) {
    constexpr int V = 16 / ES;
    if (cols >= V) {
        const uint64_t at = e + V <= cols ? e : cols - V;
        const v4u v = load16<ES>(p + at * ES);
        if (e == at) return v;
        return e >= cols ? v4u{0, 0, 0, 0} : shift_down(v, (uint32_t)(e - at) * ES * 8);
    }
    v4u r = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const uint64_t at = e + i < cols ? e + i : cols - 1;
        const uint32_t b = e + i < cols ? load1<ES>(p + at * ES) : 0u;
        if constexpr (ES == 2) r[i / 2] |= b << (16 * (i & 1));
        else r[i] = b;
    }
    return r;
}
// The same for a store: the last elements of a row in pieces of 8, 4 and 2 bytes.
template <int ES>
__device__ __forceinline__ void store_row(char* p, uint64_t e, uint64_t cols, const v4u& r) {
    constexpr int V = 16 / ES;
    if (e + V <= cols) return store16<ES>(p + e * ES, r);
    if (e >= cols) return;
    const uint32_t n = (uint32_t)(cols - e);  // 1 .. V - 1
    char* at = p + e * ES;
    v4u v = r;
    if (n * ES >= 8) {
        typedef typename Loose<ES>::x2 x2;
        *gptr<x2>(at) = x2{v[0], v[1]};
        v = v4u{v[2], v[3], 0, 0};
        at += 8;
    }
    if constexpr (ES == 4) {
        if (n & 1) store1<4>(at, v[0]);
    } else {
        typedef uint32_t x1 __attribute__((aligned(2)));
        if (n & 2) {
            *gptr<x1>(at) = v[0];
            v[0] = v[1];
            at += 4;
        }
        if (n & 1) store1<2>(at, v[0] & 0xffffu);
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
