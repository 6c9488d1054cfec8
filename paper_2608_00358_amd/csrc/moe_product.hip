// moe_product.hip -- the experts' product in 8-bit integers:
//   out[m, n] = a_scale[m] * b_scale[e, n] * sum_k a[m, k] b[e, n, k],   e the expert of row m's segment
// on the matrix instructions for 8-bit integers, with whole sums in 32 bits (exact: at most
// 131 071 products of at most 2^14). The rows of a segment follow each other; where segments begin is
// read on the device, so the grid is sized for the worst case and surplus blocks end at once.
//
// The weights are the instruction's first operand: a lane then holds neighbouring columns of one row.
// The order of k within an instruction does not matter as long as both operands have the same.
#include "moe_device.h"

namespace hccl {
namespace {

typedef int32_t v4i __attribute__((ext_vector_type(4)));

// Rows [first, end) of tile `tile` of BM rows, and its expert; false where there are fewer tiles.
// One lane a segment: tiles of a segment, their running sum, and the segment that holds the tile.
struct Rows {
    uint64_t first, end;
    uint32_t expert;
};
template <uint32_t BM>
__device__ __forceinline__ bool find_rows(const ProductArgs& a, uint32_t tile, Rows& out) {
    if (!a.offsets) {
        out.first = (uint64_t)tile * BM;
        out.end = a.rows;
        out.expert = 0;
        return out.first < a.rows;
    }
    const uint32_t lane = threadIdx.x & 63;
    uint32_t left = tile;
    for (uint32_t s0 = 0; s0 < a.segments; s0 += kWave) {
        const uint32_t s = s0 + lane;
        uint64_t first = 0, end = 0;
        if (s < a.segments) {
            const int64_t lo = a.offsets[s], hi = a.offsets[s + 1];
            first = lo < 0 ? 0 : (uint64_t)lo < a.rows ? (uint64_t)lo : a.rows;
            end = hi < (int64_t)first ? first : (uint64_t)hi < a.rows ? (uint64_t)hi : a.rows;
        }
        const uint32_t n = (uint32_t)((end - first + BM - 1) / BM);
        uint32_t incl = n;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const uint32_t v = (uint32_t)__shfl_up((int)incl, d);
            if (lane >= (uint32_t)d) incl += v;
        }
        const uint32_t all = at_lane(incl, 63);
        if (left < all) {
            const uint32_t l = first_lane((uint32_t)__popcll(__ballot(incl <= left)));
            const uint32_t skip = left - (at_lane(incl, l) - at_lane(n, l));
            out.first = ((uint64_t)at_lane((uint32_t)(first >> 32), l) << 32 | at_lane((uint32_t)first, l)) + (uint64_t)skip * BM;
            out.end = (uint64_t)at_lane((uint32_t)(end >> 32), l) << 32 | at_lane((uint32_t)end, l);
            out.expert = (s0 + l) % a.experts;
            return true;
        }
        left -= all;
    }
    return false;
}

// 16 bytes of a row at k; bytes from `inner` on are zero.
__device__ __forceinline__ v4i load_k(const int8_t* row, uint32_t k, uint32_t inner) {
    if (k + 16 <= inner) return (v4i)load16<1>(row + k);
    v4i r = {0, 0, 0, 0};
    if (k < inner) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (k + i < inner) r[i / 4] |= (int32_t)((uint32_t)(uint8_t)*gptr<int8_t>(row + k + i) << (8 * (i & 3)));
    }
    return r;
}

// Four neighbouring columns of a row.
template <int DT>
__device__ __forceinline__ void store_four(const ProductArgs& a, uint64_t m, uint32_t n, const v4i& acc, float as, const float* bs) {
    constexpr int ES = kSize<DT>;
    char* dst = (char*)a.out + (m * a.ldo + n) * ES;
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = n + i < a.cols ? (float)acc[i] * as * bs[n + i] : 0.0f;
    if (n + 4 <= a.cols) {
        if constexpr (DT == hcclFp32) {
            store16<4>(dst, v4u{__float_as_uint(y[0]), __float_as_uint(y[1]), __float_as_uint(y[2]), __float_as_uint(y[3])});
        } else {
            const uint32_t lo = narrow1<DT>(y[0]) | narrow1<DT>(y[1]) << 16, hi = narrow1<DT>(y[2]) | narrow1<DT>(y[3]) << 16;
            *gptr<typename Loose<2>::x2>(dst) = typename Loose<2>::x2{lo, hi};
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n + i < a.cols) store1<ES>(dst + i * ES, narrow1<DT>(y[i]));
    }
}

// Few rows a segment: 16 MB rows by 16 NB columns a block, whose W waves share out the k axis in
// steps of 128 and join their sums through LDS. Weights go from memory to registers: each is used
// by one block only. A lane reads 32 neighbouring bytes of a row, four lanes the 128 of a step.
template <int DT, int MB, int NB, int W>
__global__ __launch_bounds__(W * 64) void hccl_moe_product_few_kernel(ProductArgs a, uint32_t nblocks) {
    constexpr uint32_t BM = 16 * MB, BN = 16 * NB;
    __shared__ v4i part[W][MB * NB][64];
    const uint32_t lane = threadIdx.x & 63, w = first_lane(threadIdx.x >> 6);
    const uint32_t tile = blockIdx.x / nblocks, n0 = blockIdx.x % nblocks * BN;
    Rows rows;
    if (!find_rows<BM>(a, tile, rows)) return;
    const uint32_t i = lane & 15, q = lane >> 4;
    const int8_t* pa[MB];
    const int8_t* pb[NB];
#pragma unroll
    for (int x = 0; x < MB; ++x) {
        const uint64_t m = rows.first + x * 16 + i;
        pa[x] = a.a + (m < rows.end ? m : rows.end - 1) * a.lda;
    }
#pragma unroll
    for (int y = 0; y < NB; ++y) {
        const uint32_t n = n0 + y * 16 + i;
        pb[y] = a.b + ((uint64_t)rows.expert * a.cols + (n < a.cols ? n : a.cols - 1)) * a.ldb;
    }
    v4i acc[MB][NB];
#pragma unroll
    for (int x = 0; x < MB; ++x)
#pragma unroll
        for (int y = 0; y < NB; ++y) acc[x][y] = v4i{0, 0, 0, 0};
    for (uint32_t k0 = w * 128; k0 < a.inner; k0 += W * 128) {
        const uint32_t k = k0 + q * 32;
        v4i va[MB][2], vb[NB][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int y = 0; y < NB; ++y) vb[y][h] = load_k(pb[y], k + 16 * h, a.inner);
#pragma unroll
            for (int x = 0; x < MB; ++x) va[x][h] = load_k(pa[x], k + 16 * h, a.inner);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int x = 0; x < MB; ++x)
#pragma unroll
                for (int y = 0; y < NB; ++y) acc[x][y] = __builtin_amdgcn_mfma_i32_16x16x64_i8(vb[y][h], va[x][h], acc[x][y], 0, 0, 0);
    }
#pragma unroll
    for (int x = 0; x < MB; ++x)
#pragma unroll
        for (int y = 0; y < NB; ++y) part[w][x * NB + y][lane] = acc[x][y];
    __syncthreads();
    const float* bs = a.b_scale + (uint64_t)rows.expert * a.cols;
    for (uint32_t p = w; p < MB * NB; p += W) {
        v4i sum = part[0][p][lane];
#pragma unroll
        for (int v = 1; v < W; ++v) sum += part[v][p][lane];
        const uint64_t m = rows.first + p / NB * 16 + i;
        const uint32_t n = n0 + p % NB * 16 + q * 4;
        if (m < rows.end && n < a.cols) store_four<DT>(a, m, n, sum, a.a_scale[m], bs);
    }
}

template <int DT>
hipError_t product_type(const ProductArgs& a, int cus, hipStream_t s) {
    const uint32_t nblocks = (a.cols + 63) / 64;
    const uint64_t tiles = (a.rows + 15) / 16 + (a.offsets ? a.segments : 0);
    if (tiles * nblocks > 0xffffffffull / 256) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL((hccl_moe_product_few_kernel<DT, 1, 4, 4>), dim3((uint32_t)(tiles * nblocks)), dim3(256), 0, s, a, nblocks);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_product(const ProductArgs& a, hcclDataType_t dt, int cus, hipStream_t s) {
    return dt == hcclBf16 ? product_type<hcclBf16>(a, cus, s) : dt == hcclFp16 ? product_type<hcclFp16>(a, cus, s) : product_type<hcclFp32>(a, cus, s);
}

}  // namespace hccl
