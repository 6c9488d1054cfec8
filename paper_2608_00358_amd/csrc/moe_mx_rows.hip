// moe_mx_rows.hip -- rows to microscaled 4-bit floats (quantize, dispatch) and back (dequantize).
//
// A block of 32 neighbours needs nothing beyond itself: four lanes take one, 8 elements each, find its greatest
// magnitude among themselves, and store 4 bytes of codes a lane and the block's scale byte. Blocks are numbered
// through all rows, so that rows of any length fill the waves. All of it is bound by memory: 3 001 x 2 051 fp32 to codes
// 7.0 us and back 8.8 us (28 MB each), 32 768 x 4 096 codes to bf16 60 us (340 MB, 5.7 TB/s).
#include "moe_mx_device.h"

namespace hccl {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr uint32_t kUnits = 2;                      // of 16 blocks each that a wave has on their way together
constexpr uint32_t kWaveBlocks = 16 * kUnits;

// Row and block of the lane's quad in unit u of its wave, of `blocks` a row.
struct Place {
    uint32_t t, b;
};
__device__ __forceinline__ Place place(uint32_t unit, uint32_t blocks) {
    const uint32_t first = unit * 16, quad = (threadIdx.x & 63) / 4;
    uint32_t t = first / blocks, b = first % blocks + quad;
    if (blocks >= 16) {
        const bool next = b >= blocks;
        return {next ? t + 1 : t, next ? b - blocks : b};
    }
    return {t + b / blocks, b % blocks};
}

// Eight elements of a row of `cols`, from e on, in 32 bits; those behind the last are 0.
template <int DT>
__device__ __forceinline__ void load8(const char* row, uint64_t e, uint64_t cols, float (&x)[8]) {
    constexpr int ES = kSize<DT>;
    if constexpr (ES == 2) {
        widen<DT>(load_row<2>(row, e, cols), x);
    } else {
        float lo[4], hi[4];
        widen<DT>(load_row<4>(row, e, cols), lo);
        widen<DT>(load_row<4>(row, e + 4, cols), hi);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = lo[i], x[4 + i] = hi[i];
    }
}

// The scale byte of the lane's quad, and the codes of its 8 values.
template <int DT, bool GATED>
__device__ __forceinline__ void encode(float (&x)[8], const float (&up)[8], uint32_t& b, uint32_t& codes) {
    if constexpr (GATED) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = mx_gate(x[i], up[i]);
    }
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
    top = max(top, dpp<kQuadSwap>(top));
    top = max(top, dpp<kQuadHalf>(top));
    b = mx_scale(top);
    codes = b == 255u ? 0u : mx_encode(x, mx_power(b));
}

// Rows that are whole units: a wave is at one row, whose places are on their way with it. Its codes go through LDS, so that a
// lane stores 16 bytes of them and not 4, and its scales are one store. (8 192 x 4 096 bf16 to 4 rows each, 139 MB: 36 us; by 4 bytes, with the
// places looked up before each store, 43 us. 16 384 x 4 096 to one row 32 us for 170 MB.)
constexpr uint32_t kWide = 4;  // units
struct WideRow {               // of a wave, aligned for what it reads back
    v4u codes[kWide * 16];
    uint32_t scales[kWide * 4];
};
static_assert(alignof(WideRow) == 16 && sizeof(WideRow) % 16 == 0, "16 bytes a lane");
template <int DT, bool GATED>
__global__ __launch_bounds__(kThreads) void hccl_moe_quantize_mx_wide_kernel(QuantizeMxArgs a) {
    constexpr int ES = kSize<DT>;
    __shared__ WideRow own[kWaves];
    const uint32_t lane = threadIdx.x & 63, w = first_lane(threadIdx.x >> 6), pieces = a.blocks / (kWide * 16);
    const uint32_t id = blockIdx.x * kWaves + w, t = id / pieces, b0 = id % pieces * (kWide * 16);
    const uint64_t rows = a.limit && *a.limit < (int64_t)a.rows ? (*a.limit < 0 ? 0 : (uint64_t)*a.limit) : a.rows;
    if (t >= rows) return;
    const uint32_t mine = !a.row ? t : lane < a.top_k ? (uint32_t)a.row[(uint64_t)t * a.top_k + lane] : ~0u;
    const char* src = (const char*)a.x + t * a.ldx * ES;
    float x[kWide][8], up[kWide][8];
#pragma unroll
    for (uint32_t u = 0; u < kWide; ++u) {
        const uint64_t e = (b0 + u * 16) * kMxBlock + lane * 8;
        load8<DT>(src, e, a.cols, x[u]);
        if constexpr (GATED) load8<DT>(src + a.cols * ES, e, a.cols, up[u]);
    }
#pragma unroll
    for (uint32_t u = 0; u < kWide; ++u) {
        uint32_t b, codes;
        encode<DT, GATED>(x[u], up[u], b, codes);
        ((uint32_t*)own[w].codes)[u * 64 + lane] = codes;
        if (lane % 4 == 0) ((uint8_t*)own[w].scales)[u * 16 + lane / 4] = (uint8_t)b;
    }
    // (a wave's own part of LDS, which it reads in the order of its writes; the fence keeps the compiler to that)
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const v4u codes = own[w].codes[lane];
    const uint32_t scales = own[w].scales[lane % 16];
    const uint32_t copies = a.row ? a.top_k : 1u;
    for (uint32_t k = 0; k < copies; ++k) {
        const uint32_t r = a.row ? at_lane(mine, k) : t;
        if (r >= a.capacity) continue;
        store16<1>(a.codes + r * a.ldq + b0 * 16 + lane * 16, codes);
        if (lane < 16) *gptr<typename Loose<1>::x1>(a.scale + r * a.lds + b0 + lane * 4) = scales;
    }
}

template <int DT, bool GATED>
__global__ __launch_bounds__(kThreads) void hccl_moe_quantize_mx_kernel(QuantizeMxArgs a) {
    constexpr int ES = kSize<DT>;
    const uint32_t lane = threadIdx.x & 63, unit0 = (blockIdx.x * kWaves + first_lane(threadIdx.x >> 6)) * kUnits;
    const uint64_t rows = a.limit && *a.limit < (int64_t)a.rows ? (*a.limit < 0 ? 0 : (uint64_t)*a.limit) : a.rows;
    float x[kUnits][8], up[kUnits][8];
    Place p[kUnits];
    uint32_t first[kUnits];  // places, on their way with the rows: the first, and others as they are needed
#pragma unroll
    for (uint32_t u = 0; u < kUnits; ++u) {
        p[u] = place(unit0 + u, a.blocks);
        const uint64_t e = (uint64_t)p[u].b * kMxBlock + lane % 4 * 8;
        const char* src = (const char*)a.x + p[u].t * a.ldx * ES;
        if (p[u].t < rows) {
            load8<DT>(src, e, a.cols, x[u]);
            if constexpr (GATED) load8<DT>(src + a.cols * ES, e, a.cols, up[u]);
            first[u] = a.row ? (uint32_t)a.row[(uint64_t)p[u].t * a.top_k] : p[u].t;
        }
    }
#pragma unroll
    for (uint32_t u = 0; u < kUnits; ++u) {
        if (p[u].t >= rows) continue;  // (a quad's lanes are of one row)
        uint32_t b, codes;
        encode<DT, GATED>(x[u], up[u], b, codes);
        const uint32_t e = p[u].b * kMxBlock + lane % 4 * 8, left = (uint32_t)a.cols > e ? (uint32_t)a.cols - e : 0;
        auto put = [&](uint32_t r) {
            if (r >= a.capacity) return;
            uint8_t* dst = a.codes + r * a.ldq + e / 2;
            if (left >= 7) {
                *gptr<typename Loose<1>::x1>(dst) = codes;
            } else {
#pragma unroll
                for (uint32_t i = 0; i < 3; ++i)
                    if (2 * i < left) *gptr<uint8_t>(dst + i) = (uint8_t)(codes >> (8 * i));
            }
            if (lane % 4 == 0) *gptr<uint8_t>(a.scale + r * a.lds + p[u].b) = (uint8_t)b;
        };
        put(first[u]);
        if (!a.row) continue;
        const int32_t* row = a.row + (uint64_t)p[u].t * a.top_k;
#pragma unroll 4
        for (uint32_t k = 1; k < a.top_k; ++k) put((uint32_t)row[k]);
    }
}

template <int DT>
__global__ __launch_bounds__(kThreads) void hccl_moe_dequantize_mx_kernel(DequantizeMxArgs a) {
    constexpr int ES = kSize<DT>;
    const uint32_t lane = threadIdx.x & 63, unit0 = (blockIdx.x * kWaves + first_lane(threadIdx.x >> 6)) * kUnits;
    const uint64_t rows = a.limit && *a.limit < (int64_t)a.rows ? (*a.limit < 0 ? 0 : (uint64_t)*a.limit) : a.rows;
    uint32_t codes[kUnits] = {}, b[kUnits] = {};
    Place p[kUnits];
#pragma unroll
    for (uint32_t u = 0; u < kUnits; ++u) {
        p[u] = place(unit0 + u, a.blocks);
        const uint32_t e = p[u].b * kMxBlock + lane % 4 * 8, left = (uint32_t)a.cols > e ? (uint32_t)a.cols - e : 0;
        if (p[u].t < rows && left) {
            const uint8_t* src = a.codes + p[u].t * a.ldq + e / 2;
            if (left >= 7) {
                codes[u] = *gptr<typename Loose<1>::x1>(src);
            } else {
#pragma unroll
                for (uint32_t i = 0; i < 3; ++i)
                    if (2 * i < left) codes[u] |= (uint32_t)*gptr<uint8_t>(src + i) << (8 * i);
            }
            b[u] = *gptr<uint8_t>(a.scale + p[u].t * a.lds + p[u].b);
        }
    }
#pragma unroll
    for (uint32_t u = 0; u < kUnits; ++u) {
        const uint64_t e = (uint64_t)p[u].b * kMxBlock + lane % 4 * 8;
        if (p[u].t >= rows || e >= a.cols) continue;
        float x[8];
        mx_decode(codes[u], mx_power(b[u]), x);
        char* dst = (char*)a.out + p[u].t * a.ldo * ES;
        if constexpr (ES == 2) {
            store_row<2>(dst, e, a.cols, narrow<DT>(x));
        } else {
            const float lo[4] = {x[0], x[1], x[2], x[3]}, hi[4] = {x[4], x[5], x[6], x[7]};
            store_row<4>(dst, e, a.cols, narrow<DT>(lo));
            store_row<4>(dst, e + 4, a.cols, narrow<DT>(hi));
        }
    }
}

// Blocks of a launch; 0 where a wave's units or the launch's threads would pass 32 bits.
uint32_t grid_of(uint64_t rows, uint64_t blocks) {
    if (rows > 0xffffffffull / blocks) return 0;
    const uint64_t n = (rows * blocks + kWaveBlocks * kWaves - 1) / (kWaveBlocks * kWaves);
    return n * kThreads <= 0xffffffffull && n * kWaves * kWaveBlocks <= 0xffffffffull ? (uint32_t)n : 0;
}

template <typename F>
hipError_t by_type(hcclDataType_t dt, F f) {
    if (dt == hcclBf16) f(std::integral_constant<int, hcclBf16>());
    else if (dt == hcclFp16) f(std::integral_constant<int, hcclFp16>());
    else f(std::integral_constant<int, hcclFp32>());
    return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize_mx(const QuantizeMxArgs& a, hcclDataType_t dt, bool gated, hipStream_t s) {
    const uint32_t grid = grid_of(a.rows, a.blocks);
    if (!grid) return hipErrorInvalidConfiguration;
    if (a.cols % (kWide * 16 * kMxBlock) == 0) {
        const uint64_t waves = a.rows * (a.blocks / (kWide * 16));
        const dim3 wide((uint32_t)((waves + kWaves - 1) / kWaves));
        return by_type(dt, [&](auto type) {
            constexpr int DT = decltype(type)::value;
            if (gated) hipLaunchKernelGGL((hccl_moe_quantize_mx_wide_kernel<DT, true>), wide, dim3(kThreads), 0, s, a);
            else hipLaunchKernelGGL((hccl_moe_quantize_mx_wide_kernel<DT, false>), wide, dim3(kThreads), 0, s, a);
        });
    }
    return by_type(dt, [&](auto type) {
        constexpr int DT = decltype(type)::value;
        if (gated) hipLaunchKernelGGL((hccl_moe_quantize_mx_kernel<DT, true>), dim3(grid), dim3(kThreads), 0, s, a);
        else hipLaunchKernelGGL((hccl_moe_quantize_mx_kernel<DT, false>), dim3(grid), dim3(kThreads), 0, s, a);
    });
}

hipError_t launch_dequantize_mx(const DequantizeMxArgs& a, hcclDataType_t dt, hipStream_t s) {
    const uint32_t grid = grid_of(a.rows, a.blocks);
    if (!grid) return hipErrorInvalidConfiguration;
    return by_type(dt, [&](auto type) {
        constexpr int DT = decltype(type)::value;
        hipLaunchKernelGGL(hccl_moe_dequantize_mx_kernel<DT>, dim3(grid), dim3(kThreads), 0, s, a);
    });
}

}  // namespace hccl
