// moe_mx_product.hip -- the experts' product in microscaled 4-bit floats:
//   out[m, n] = sum_k a[m, k] b[e, n, k],   e the expert of row m's segment
// on the matrix instructions that take 4-bit floats with a scale byte for every 32 of them. Products of two codes are
// multiples of 1/4 up to 36, so a block's sum is exact; blocks are added up in 32 bits. Segments, tiles and the order of
// operands are those of the 8-bit product: 16 bytes, which are 16 elements there, are 32 here, and one block.
#include <type_traits>

#include "moe_mx_device.h"
#include "moe_segments.h"

namespace hccl {
namespace {

typedef int32_t v4i __attribute__((ext_vector_type(4)));
typedef int32_t v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));

constexpr int kFp4 = 4;  // the operands' format

// (4-bit operands take half of the instruction's registers)
__device__ __forceinline__ v8i whole(const v4i& v) { return __builtin_shufflevector(v, v, 0, 1, 2, 3, -1, -1, -1, -1); }

// f(the type of the results): a uniform branch at a kernel's end, where a kernel for each type would be the same before it.
template <typename F>
__device__ __forceinline__ void by_result(uint32_t dt, F f) {
    if (dt == hcclBf16) f(std::integral_constant<int, hcclBf16>());
    else if (dt == hcclFp16) f(std::integral_constant<int, hcclFp16>());
    else f(std::integral_constant<int, hcclFp32>());
}

// Four neighbouring columns of a row.
template <int DT>
__device__ __forceinline__ void store_four(const ProductMxArgs& a, uint64_t m, uint32_t n, const v4f& y) {
    constexpr int ES = kSize<DT>;
    char* dst = (char*)a.out + (m * a.ldo + n) * ES;
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

// Few rows a segment: 16 MB rows by 16 NB columns a block, whose W waves share out the k axis in steps of 128 bytes
// (256 elements) and join their sums through LDS, in the waves' order. Each weight is used by one wave only, and comes by
// loads to LDS of its own (ALIGNED), or to registers. A lane has 32 neighbouring bytes of a row, two blocks, and their
// two scale bytes; four lanes the 128 bytes of a step.
// Bound by the weights' bytes: 256 rows, 64 experts of 2048 x 2048 bf16, 143 MB, 26.0 us (5.5 TB/s; 22.6 us out of the last
// cache); 256 x 4096 x 4096 x 64, 570 MB, 107 us (5.3 TB/s). One step a wave and more waves: two steps on their way took 32.4,
// four waves of one step 24.7 us where two took 24.3.
template <int MB, int NB, int W, bool ALIGNED>
__global__ __launch_bounds__(W * 64) void hccl_moe_product_mx_few_kernel(ProductMxArgs a, uint32_t nblocks) {
    constexpr uint32_t BM = 16 * MB, BN = 16 * NB;
    constexpr uint32_t kOwn = ALIGNED && kSlot<NB> > MB * NB * 1024 ? kSlot<NB> : MB * NB * 1024;  // LDS of a wave: a step, then its sums
    __shared__ __attribute__((aligned(256))) char lds[W * kOwn];
    const uint32_t lane = threadIdx.x & 63, w = first_lane(threadIdx.x >> 6);
    const uint32_t tile = blockIdx.x / nblocks, n0 = blockIdx.x % nblocks * BN;
    Rows rows;
    if (!find_rows<BM>(a, Segments<BM>(a, 0), tile, rows)) return;
    const uint32_t i = lane & 15, q = lane >> 4;
    const uint8_t *pa[MB], *sa[MB], *pb[NB], *sb[NB];
#pragma unroll
    for (int x = 0; x < MB; ++x) {
        uint64_t m = rows.first + x * 16 + i;
        m = m < rows.end ? m : rows.end - 1;
        pa[x] = a.a + m * a.lda;
        sa[x] = a.a_scale + m * a.ldas;
    }
#pragma unroll
    for (int y = 0; y < NB; ++y) {
        uint64_t n = n0 + y * 16 + i;
        n = (uint64_t)rows.expert * a.cols + (n < a.cols ? n : a.cols - 1);
        pb[y] = a.b + n * a.ldb;
        sb[y] = a.b_scale + n * a.ldbs;
    }
    v4f acc[MB][NB];
#pragma unroll
    for (int x = 0; x < MB; ++x)
#pragma unroll
        for (int y = 0; y < NB; ++y) acc[x][y] = v4f{0, 0, 0, 0};
    char* mine = lds + w * kOwn;
    struct Step {
        v4i a[MB][2];
        uint32_t sa[MB];
        Codes b[NB];
    };
    const uint32_t blocks = (a.inner + kMxBlock - 1) / kMxBlock;
    auto fetch_rows = [&](Step& f, uint32_t s, auto inside) {  // INSIDE: the step lies inside the rows
        constexpr bool INSIDE = decltype(inside)::value;
        typedef uint16_t loose __attribute__((aligned(1)));
        const uint32_t k = s * 128 + q * 32, b = k / 16;
#pragma unroll
        for (int x = 0; x < MB; ++x) {
#pragma unroll
            for (int h = 0; h < 2; ++h) f.a[x][h] = (v4i)(INSIDE ? load16<1>(pa[x] + k + 16 * h) : load_codes<false, true>(pa[x], k + 16 * h, a.inner));
            f.sa[x] = INSIDE || b + 2 <= blocks ? *gptr<loose>(sa[x] + b) : b < blocks ? *gptr<uint8_t>(sa[x] + b) : 0u;
        }
    };
    auto fetch_weights = [&](Step& f, uint32_t s, auto inside) {
#pragma unroll
        for (int y = 0; y < NB; ++y) f.b[y] = load_pair<decltype(inside)::value>(pb[y], sb[y], s * 128 + q * 32, a.inner);
    };
    auto multiply = [&](const Step& f) {
#pragma unroll
        for (int x = 0; x < MB; ++x)
#pragma unroll
            for (int y = 0; y < NB; ++y) {
                acc[x][y] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(whole((v4i)f.b[y].c[0]), whole(f.a[x][0]), acc[x][y], kFp4, kFp4, 0, f.b[y].scale, 0, f.sa[x]);
                acc[x][y] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(whole((v4i)f.b[y].c[1]), whole(f.a[x][1]), acc[x][y], kFp4, kFp4, 1, f.b[y].scale, 1, f.sa[x]);
            }
    };
    const uint32_t steps = ((a.inner + 1) / 2 + 127) / 128, whole_steps = a.inner / 256;
    uint32_t s = w;
    if constexpr (ALIGNED) {
        const Source<NB> src = source_of<NB>(a.b, a.ldb, a.b_scale, a.ldbs, [&](uint32_t y, uint32_t r) {
            const uint64_t n = n0 + y * 16 + r;
            return (uint64_t)rows.expert * a.cols + (n < a.cols ? n : a.cols - 1);
        });
        const uint32_t at0 = lds_address(mine) + code_place(lane), at_scale = lds_address(mine) + scale_place(NB, lane);
#pragma unroll 1
        for (; s < whole_steps; s += W) {
            Step f;
            load_to_lds<NB>(src, s, mine);
            fetch_rows(f, s, std::true_type());
            wait_steps<0>();
            read_from_lds(f.b, at0, at0 ^ 16, at_scale);
            multiply(f);
        }
    } else {
        Step f[2];
        for (; s + W < whole_steps; s += 2 * W) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                fetch_weights(f[u], s + u * W, std::true_type());
                fetch_rows(f[u], s + u * W, std::true_type());
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < 2; ++u) multiply(f[u]);
        }
        if (s < whole_steps) {
            fetch_weights(f[0], s, std::true_type());
            fetch_rows(f[0], s, std::true_type());
            multiply(f[0]);
        }
    }
    if (whole_steps < steps && whole_steps % W == w) {
        Step f;
        fetch_weights(f, whole_steps, std::false_type());
        fetch_rows(f, whole_steps, std::false_type());
        multiply(f);
    }
    v4f* sums = (v4f*)mine;
#pragma unroll
    for (int x = 0; x < MB; ++x)
#pragma unroll
        for (int y = 0; y < NB; ++y) sums[(x * NB + y) * 64 + lane] = acc[x][y];
    __syncthreads();
    for (uint32_t p = w; p < MB * NB; p += W) {
        v4f sum = ((const v4f*)lds)[p * 64 + lane];
#pragma unroll
        for (int v = 1; v < W; ++v) {
            const v4f more = ((const v4f*)(lds + v * kOwn))[p * 64 + lane];
#pragma unroll
            for (int j = 0; j < 4; ++j) sum[j] += more[j];
        }
        const uint64_t m = rows.first + p / NB * 16 + i;
        const uint32_t n = n0 + p % NB * 16 + q * 4;
        if (m < rows.end && n < a.cols) by_result(a.type, [&](auto type) { store_four<decltype(type)::value>(a, m, n, sum); });
    }
}

// Many rows a segment: BM rows by BN columns a block, in WM x WN waves, k in steps of 64 bytes (128 elements, four blocks)
// through BUFFERS LDS buffers: one is multiplied while the others are filled, by loads that go to LDS directly (DIRECT:
// rows and weights are 16-byte aligned) or through registers (any alignment, and the last step of an inner size that is no
// multiple of 128, where codes past the end are zero).
//
// Bound by the matrix units' power (codes of 0: 226 and 165 us in the first two) and by the starts and ends of tiles, 9 us each
// of 256 x 256: 8192 x 8192 x 8192 294-325 us (3.4-3.7 PFLOP/s), 16384 x 4096 x 4096 through 16 experts 194-201 us (2.8), 2999 x
// 1407 x 2050 through 12 16-18 us (1.0).
//
// A wave reads a step's fragments from LDS, waits for them, and multiplies them. With two GROUPS, waves 0 to 3 and 4 to 7,
// which share the SIMDs, the second is half a step behind: one reads while the other multiplies, and barriers between the
// halves keep it so. With one, other blocks on the CU fill the gap. Reads are one block of assembly with its wait: the
// compiler, which cannot tell which loads to LDS a read depends on, would have each wait for all of them.
//
// LDS holds a row's 64 bytes as 4 chunks of 16; chunk c of row r lies in slot c ^ (r / 4 & 3), so that the
// 16 lanes served together, which read one chunk of 16 rows, use different banks. A direct load writes its 64 lanes one
// after the other, so a lane reads the chunk that belongs in its slot. The lanes' halves take chunks 0 and 2 in a step's
// first part and 1 and 3 in its second, so that a half's two scale bytes are neighbours.
//
// Scales: a thread has kRows rows, of the tile's rows or columns, whose next 16 scale bytes (four steps) it reads into a
// register a step after those before went to LDS, each half's 8 bytes together. A wave has its fragments' scales of four
// steps in registers, so one buffer does.
constexpr uint32_t kStep = 64;
constexpr uint32_t kBand = 4;

template <int N>
__device__ __forceinline__ void wait_loads() {  // until at most N loads are on their way, and LDS is done
    static_assert(N < 16, "the counter's low bits");
    __builtin_amdgcn_s_waitcnt(0x70 | N);
}
// A barrier that leaves loads to LDS in flight; nothing that touches memory moves across it.
__device__ __forceinline__ void meet() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}
__device__ __forceinline__ void lds_write(uint32_t at, const v4u& v) { asm volatile("ds_write_b128 %0, %1" ::"v"(at), "v"(v) : "memory"); }

// A step's fragments of a wave: TM of rows, TN of columns, two parts each; and the scales of four steps, 16 bits each.
template <int TM, int TN>
struct Fragments {
    v4i a[2][TM], b[2][TN];
    v2u sa[TM], sb[TN];
};
// (the distance of fragments is 32 rows: 2048 bytes of codes, 512 of scales)
__device__ __forceinline__ void read_codes(Fragments<4, 2>& f, uint32_t a0, uint32_t a1, uint32_t b0, uint32_t b1) {
    asm volatile(
        "ds_read_b128 %0, %12\n\tds_read_b128 %8, %14\n\tds_read_b128 %9, %14 offset:2048\n\tds_read_b128 %1, %12 offset:2048\n\t"
        "ds_read_b128 %2, %12 offset:4096\n\tds_read_b128 %3, %12 offset:6144\n\tds_read_b128 %4, %13\n\tds_read_b128 %10, %15\n\t"
        "ds_read_b128 %11, %15 offset:2048\n\tds_read_b128 %5, %13 offset:2048\n\tds_read_b128 %6, %13 offset:4096\n\t"
        "ds_read_b128 %7, %13 offset:6144\n\ts_waitcnt lgkmcnt(0)"
        : "=&v"(f.a[0][0]), "=&v"(f.a[0][1]), "=&v"(f.a[0][2]), "=&v"(f.a[0][3]), "=&v"(f.a[1][0]), "=&v"(f.a[1][1]), "=&v"(f.a[1][2]), "=&v"(f.a[1][3]),
          "=&v"(f.b[0][0]), "=&v"(f.b[0][1]), "=&v"(f.b[1][0]), "=&v"(f.b[1][1])
        : "v"(a0), "v"(a1), "v"(b0), "v"(b1)
        : "memory");
}
__device__ __forceinline__ void read_codes(Fragments<2, 2>& f, uint32_t a0, uint32_t a1, uint32_t b0, uint32_t b1) {
    asm volatile(
        "ds_read_b128 %0, %8\n\tds_read_b128 %4, %10\n\tds_read_b128 %5, %10 offset:2048\n\tds_read_b128 %1, %8 offset:2048\n\t"
        "ds_read_b128 %2, %9\n\tds_read_b128 %6, %11\n\tds_read_b128 %7, %11 offset:2048\n\tds_read_b128 %3, %9 offset:2048\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(f.a[0][0]), "=&v"(f.a[0][1]), "=&v"(f.a[1][0]), "=&v"(f.a[1][1]), "=&v"(f.b[0][0]), "=&v"(f.b[0][1]), "=&v"(f.b[1][0]), "=&v"(f.b[1][1])
        : "v"(a0), "v"(a1), "v"(b0), "v"(b1)
        : "memory");
}
__device__ __forceinline__ void read_codes(Fragments<2, 1>& f, uint32_t a0, uint32_t a1, uint32_t b0, uint32_t b1) {
    asm volatile(
        "ds_read_b128 %0, %6\n\tds_read_b128 %4, %8\n\tds_read_b128 %1, %6 offset:2048\n\t"
        "ds_read_b128 %2, %7\n\tds_read_b128 %5, %9\n\tds_read_b128 %3, %7 offset:2048\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(f.a[0][0]), "=&v"(f.a[0][1]), "=&v"(f.a[1][0]), "=&v"(f.a[1][1]), "=&v"(f.b[0][0]), "=&v"(f.b[1][0])
        : "v"(a0), "v"(a1), "v"(b0), "v"(b1)
        : "memory");
}
template <int TM, int TN>
__device__ __forceinline__ void read_scales(Fragments<TM, TN>& f, uint32_t a, uint32_t b) {
    static_assert((TM == 4 && TN == 2) || (TM == 2 && TN <= 2), "the fragments above");
    if constexpr (TM == 4)
        asm volatile("ds_read_b64 %0, %6\n\tds_read_b64 %1, %6 offset:512\n\tds_read_b64 %2, %6 offset:1024\n\tds_read_b64 %3, %6 offset:1536\n\t"
                     "ds_read_b64 %4, %7\n\tds_read_b64 %5, %7 offset:512\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(f.sa[0]), "=&v"(f.sa[1]), "=&v"(f.sa[2]), "=&v"(f.sa[3]), "=&v"(f.sb[0]), "=&v"(f.sb[1])
                     : "v"(a), "v"(b)
                     : "memory");
    else if constexpr (TN == 2)
        asm volatile("ds_read_b64 %0, %4\n\tds_read_b64 %1, %4 offset:512\n\tds_read_b64 %2, %5\n\tds_read_b64 %3, %5 offset:512\n\t"
                     "s_waitcnt lgkmcnt(0)"
                     : "=&v"(f.sa[0]), "=&v"(f.sa[1]), "=&v"(f.sb[0]), "=&v"(f.sb[1])
                     : "v"(a), "v"(b)
                     : "memory");
    else
        asm volatile("ds_read_b64 %0, %3\n\tds_read_b64 %1, %3 offset:512\n\tds_read_b64 %2, %4\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(f.sa[0]), "=&v"(f.sa[1]), "=&v"(f.sb[0])
                     : "v"(a), "v"(b)
                     : "memory");
}

template <int BM, int BN, int WM, int WN, int GROUPS, int BUFFERS, bool DIRECT>
__global__ __launch_bounds__(WM * WN * 64, 2) void hccl_moe_product_mx_many_kernel(ProductMxArgs a, uint32_t nblocks) {
    constexpr int W = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32;
    constexpr int LA = BM / 16 / W, LB = BN / 16 / W, LN = LA + LB;  // loads a wave makes for a step: 16 rows each
    constexpr uint32_t kAhead = BUFFERS - 1;
    static_assert(BM % (16 * W) == 0 && BN % (16 * W) == 0 && (BUFFERS - 2) * LN < 16, "whole loads, and a counter that holds them");
    static_assert(GROUPS == 1 || W == 8, "two groups of a wave a SIMD");
    constexpr int kRows = (BM + BN + W * 64 - 1) / (W * 64);
    constexpr uint32_t kBuffer = (BM + BN) * kStep;
    __shared__ __attribute__((aligned(256))) char lds[BUFFERS * kBuffer];
    __shared__ __attribute__((aligned(256))) char lds_scale[(BM + BN) * 16];
    const uint32_t lane = threadIdx.x & 63, w = first_lane(threadIdx.x >> 6);

    // Blocks go to the XCDs in turn; each XCD gets neighbouring tiles, in bands of kBand column blocks, so
    // that the tiles it works on at a time share their rows and weights in its L2.
    const Segments<BM> segments(a, 0);
    uint32_t tile, nb;
    {
        const uint32_t tiles = count_tiles<BM>(a, segments);
        const uint64_t all = (uint64_t)tiles * nblocks, share = (all + 7) / 8;
        const uint64_t id = (blockIdx.x & 7) * share + blockIdx.x / 8;
        if (blockIdx.x / 8 >= share || id >= all) return;
        const uint64_t banded = (uint64_t)(nblocks / kBand * kBand) * tiles;
        const uint32_t width = id < banded ? kBand : nblocks % kBand;
        const uint64_t at = id < banded ? id % ((uint64_t)kBand * tiles) : id - banded;
        tile = (uint32_t)(at / width);
        nb = (id < banded ? (uint32_t)(id / ((uint64_t)kBand * tiles)) * kBand : nblocks / kBand * kBand) + (uint32_t)(at % width);
    }
    Rows rows;
    if (!find_rows<BM>(a, segments, tile, rows)) return;
    const uint32_t n0 = nb * BN;
    auto row_of = [&](uint32_t r) { return rows.first + r < rows.end ? rows.first + r : rows.end - 1; };
    auto col_of = [&](uint32_t c) { return (uint64_t)rows.expert * a.cols + (n0 + c < a.cols ? n0 + c : a.cols - 1); };

    // where this lane's part of each load comes from, and where in a buffer each load goes
    const uint32_t lrow = lane >> 2, chunk = ((lane & 3) ^ (lrow >> 2)) * 16;
    auto source = [&](int i) { return i < LA ? a.a + row_of((w * LA + i) * 16 + lrow) * a.lda : a.b + col_of((w * LB + i - LA) * 16 + lrow) * a.ldb; };
    const uint8_t* src[LN];
#pragma unroll
    for (int i = 0; i < LN; ++i) src[i] = source(i) + chunk;
    auto slot = [&](uint32_t s, int i) { return lds + (s % BUFFERS) * kBuffer + (i < LA ? (w * LA + i) * 16 : BM + (w * LB + i - LA) * 16) * kStep; };
    const uint8_t* scale_src[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const uint32_t at = r * W * 64 + threadIdx.x;
        scale_src[r] = at < BM ? a.a_scale + row_of(at) * a.ldas : a.b_scale + col_of(at < BM + BN ? at - BM : 0) * a.ldbs;
    }
    const uint32_t scale_bytes = (a.inner + kMxBlock - 1) / kMxBlock;

    v16f acc[TN][TM];
#pragma unroll
    for (int y = 0; y < TN; ++y)
#pragma unroll
        for (int x = 0; x < TM; ++x)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[y][x][r] = 0;

    const uint32_t steps = (a.inner + 2 * kStep - 1) / (2 * kStep), whole_steps = a.inner / (2 * kStep);
    // Waves of the same rows are neighbours, and so on different SIMDs: where an end of a segment leaves
    // waves without rows, those that have some share out the matrix units.
    const uint32_t wm = w / WN, wn = w % WN;
    const bool second = GROUPS == 2 && w >= 4;
    v4u held[LN];           // on their way through registers
    v4u held_scale[kRows];  // scales of four steps, on their way
    auto put = [&](uint32_t s, int i, const v4u& v) { lds_write(lds_address(slot(s, i)) + lane * 16, v); };
    // Load i of those that bring in step s, a whole one; through registers, the one before goes to its buffer meanwhile.
    auto fetch = [&](uint32_t s, int i) {
        if constexpr (DIRECT) {
            __builtin_amdgcn_global_load_lds((const HCCL_AS1 void*)(src[i] + (uint64_t)s * kStep), (lds_ptr)slot(s, i), 16, 0, 0);
        } else {
            put(s - 1, i, held[i]);
            held[i] = load16<1>(src[i] + (uint64_t)s * kStep);
        }
    };
    auto bring = [&](uint32_t s) {  // any step, at once
#pragma unroll 1
        for (int i = 0; i < LN; ++i)
            put(s, i, i < LA ? load_codes<true, true>(source(i), s * kStep + chunk, a.inner) : load_codes<true, false>(source(i), s * kStep + chunk, a.inner));
    };
    auto fetch_scales = [&](uint32_t four) {
#pragma unroll
        for (int r = 0; r < kRows; ++r) held_scale[r] = load_bytes<false>(scale_src[r], four * 16, scale_bytes);
    };
    auto put_scales = [&] {
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const v4u& v = held_scale[r];
            const v4u halves = {__builtin_amdgcn_perm(v[1], v[0], 0x05040100u), __builtin_amdgcn_perm(v[3], v[2], 0x05040100u),
                                __builtin_amdgcn_perm(v[1], v[0], 0x07060302u), __builtin_amdgcn_perm(v[3], v[2], 0x07060302u)};
            const uint32_t at = r * W * 64 + threadIdx.x;
            if ((r + 1) * W * 64 <= BM + BN || at < BM + BN) lds_write(lds_address(lds_scale) + at * 16, halves);
        }
    };

    // a lane's places in a buffer: its row of the wave's first fragment, the chunk of its half
    const uint32_t place = (lane & 31) * kStep + ((lane >> 5) * 2 ^ (lane >> 2 & 3)) * 16;
    const uint32_t at_a = lds_address(lds) + wm * TM * 32 * kStep + place, at_b = lds_address(lds) + (BM + wn * TN * 32) * kStep + place;
    const uint32_t at_sa = lds_address(lds_scale) + (wm * TM * 32 + (lane & 31)) * 16 + (lane >> 5) * 8;
    const uint32_t at_sb = at_sa + (BM + wn * TN * 32 - wm * TM * 32) * 16;
    Fragments<TM, TN> f;
    // A step's matrix instructions, with the loads that bring in step s + kAhead (INNER: a whole one) between them: a wave that
    // makes its loads in one go waits for the units that take them, and its SIMD with it. PHASE: the step's place among four.
    auto multiply = [&](uint32_t s, auto phase, auto inner) {
        constexpr int kMfmas = 2 * TM * TN, P = decltype(phase)::value;
        int next = 0;
#pragma unroll
        for (int i = 0; i < kMfmas; ++i) {
            const int x = i / TN % TM, y = i % TN;
            if (i < kMfmas / 2)
                acc[y][x] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(whole(f.b[0][y]), whole(f.a[0][x]), acc[y][x], kFp4, kFp4, P % 2 * 2, f.sb[y][P / 2], P % 2 * 2,
                                                                            f.sa[x][P / 2]);
            else
                acc[y][x] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(whole(f.b[1][y]), whole(f.a[1][x]), acc[y][x], kFp4, kFp4, P % 2 * 2 + 1, f.sb[y][P / 2],
                                                                            P % 2 * 2 + 1, f.sa[x][P / 2]);
            __builtin_amdgcn_sched_barrier(0);
            if (inner.value)
                for (; next < LN && next * kMfmas < (i + 1) * LN; ++next) fetch(s + kAhead, next);
            __builtin_amdgcn_sched_barrier(0);
        }
        // (here, and not sunk behind what follows)
#pragma unroll
        for (int y = 0; y < TN; ++y)
#pragma unroll
            for (int x = 0; x < TM; ++x) {
                if constexpr (TM * TN >= 8) asm volatile("" : "+v"(acc[y][x]));
                else asm volatile("" : "+a"(acc[y][x]));
            }
    };
    // One step. ON: the wave has rows. Loads of step s + 1 have to be there for all waves when the first group reads it: that
    // group waits for its own at the end of step s, when those of the steps behind may be on their way, and the second in the
    // middle of it, when it has made one step's less.
    auto pass = [&](uint32_t s, auto phase, auto on, auto inner) {
        constexpr int P = decltype(phase)::value;
        if (on.value) {
            const uint32_t at = (s % BUFFERS) * kBuffer;
            if (P == 0) read_scales(f, at_sa, at_sb);
            read_codes(f, at_a + at, (at_a ^ 16) + at, at_b + at, (at_b ^ 16) + at);
        }
        if constexpr (GROUPS == 2) {
            if (second && DIRECT) {
                if (inner.value) wait_loads<(BUFFERS - 3) * LN>();
                else wait_loads<0>();
            }
            meet();
        }
        if (!inner.value) {  // what is left to bring in
            if (!DIRECT && s + kAhead - 1 < whole_steps) {
#pragma unroll
                for (int i = 0; i < LN; ++i) put(s + kAhead - 1, i, held[i]);
            }
            if (s + kAhead < whole_steps) {
#pragma unroll
                for (int i = 0; i < LN; ++i) {
                    if constexpr (DIRECT) fetch(s + kAhead, i);
                    else held[i] = load16<1>(src[i] + (uint64_t)(s + kAhead) * kStep);
                }
            } else if (s + kAhead == whole_steps && whole_steps < steps) {
                bring(whole_steps);
            }
        }
        if (P == 1) {  // every wave has the scales of these four steps
            put_scales();
            fetch_scales(s / 4 + 2);
        }
        if (on.value) multiply(s, phase, inner);
        else if (inner.value) {
#pragma unroll
            for (int i = 0; i < LN; ++i) fetch(s + kAhead, i);
        }
        if (!DIRECT || second) __builtin_amdgcn_s_waitcnt(0xc07f);  // LDS alone
        else if (inner.value) wait_loads<(BUFFERS - 2) * LN>();
        else wait_loads<0>();
        if (inner.value || !second || s + 1 < steps) meet();  // (the last barrier is the first group's)
    };
    auto walk = [&](auto on) {
        const std::integral_constant<int, 0> p0;
        const std::integral_constant<int, 1> p1;
        const std::integral_constant<int, 2> p2;
        const std::integral_constant<int, 3> p3;
        if (second) meet();
        uint32_t s = 0;
#pragma unroll 1
        for (; s + 3 + kAhead < whole_steps; s += 4) {
            pass(s, p0, on, std::true_type());
            pass(s + 1, p1, on, std::true_type());
            pass(s + 2, p2, on, std::true_type());
            pass(s + 3, p3, on, std::true_type());
        }
#pragma unroll 1
        for (; s < steps; s += 4) {
            pass(s, p0, on, std::false_type());
            if (s + 1 < steps) pass(s + 1, p1, on, std::false_type());
            if (s + 2 < steps) pass(s + 2, p2, on, std::false_type());
            if (s + 3 < steps) pass(s + 3, p3, on, std::false_type());
        }
    };
    if (steps) {
        fetch_scales(0);
        if constexpr (DIRECT) {
            const uint32_t n = whole_steps < kAhead ? whole_steps : kAhead;
            for (uint32_t s = 0; s < n; ++s)
#pragma unroll
                for (int i = 0; i < LN; ++i) fetch(s, i);
        } else {
            for (uint32_t s = 0; s < kAhead - 1 && s < whole_steps; ++s) bring(s);
            if (whole_steps >= kAhead) {
#pragma unroll
                for (int i = 0; i < LN; ++i) held[i] = load16<1>(src[i] + (kAhead - 1) * kStep);
            }
        }
        if (whole_steps < kAhead && whole_steps < steps) bring(whole_steps);
        put_scales();
        fetch_scales(1);
        wait_loads<0>();
        meet();
        if (rows.first + wm * TM * 32 >= rows.end) {
            walk(std::false_type());
            return;
        }
        walk(std::true_type());
    }

    // The wave's TM x TN blocks leave through its own part of LDS, as rows of TN * 32 results: lanes that hold
    // four results each of 32 rows would store 16 bytes of a line at a time.
    by_result(a.type, [&](auto type) {
        constexpr int DT = decltype(type)::value;
        constexpr int ES = kSize<DT>;
        constexpr uint32_t kLine = TN * 32 * ES, kChunks = kLine / 16;  // bytes of a row
        constexpr int kRowsEach = BUFFERS * kBuffer / W / kLine >= TM * 32 ? TM : BUFFERS * kBuffer / W / kLine / 32;  // blocks of 32 rows at a time
        static_assert(kRowsEach >= 1 && TM % kRowsEach == 0, "a block of rows fits");
        // (nothing reads the buffers any more: the last barrier is behind the last read)
        char* mine = lds + w * (BUFFERS * kBuffer / W);
        const uint32_t c0 = n0 + wn * TN * 32;
#pragma unroll
        for (int x0 = 0; x0 < TM; x0 += kRowsEach) {
            const uint64_t m0 = rows.first + (wm * TM + x0) * 32;
#pragma unroll
            for (int x = 0; x < kRowsEach; ++x) {
                const uint32_t r = x * 32 + (lane & 31);
#pragma unroll
                for (int y = 0; y < TN; ++y)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        float v[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[i] = acc[y][x0 + x][4 * g + i];
                        // columns y * 32 + g * 8 + (lane / 32) * 4 of row r; a row's 16-byte chunks lie in another order in
                        // each pair of rows
                        if constexpr (ES == 2) {
                            const uint32_t at = ((y * 4 + g) ^ (r >> 1)) % kChunks * 16 + (lane >> 5) * 8;
                            *(v2u*)(mine + r * kLine + at) = v2u{narrow1<DT>(v[0]) | narrow1<DT>(v[1]) << 16, narrow1<DT>(v[2]) | narrow1<DT>(v[3]) << 16};
                        } else {
                            const uint32_t at = ((y * 8 + g * 2 + (lane >> 5)) ^ (r >> 1)) % kChunks * 16;
                            *(v4u*)(mine + r * kLine + at) = v4u{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
                        }
                    }
            }
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_waitcnt(0xc07f);
            constexpr uint32_t kRowsAtOnce = 64 / kChunks, V = 16 / ES;
            const uint32_t c = lane % kChunks;
#pragma unroll
            for (uint32_t r0 = 0; r0 < kRowsEach * 32; r0 += kRowsAtOnce) {
                const uint32_t r = r0 + lane / kChunks;
                const v4u v = *(const v4u*)(mine + r * kLine + (c ^ (r >> 1)) % kChunks * 16);
                if (m0 + r < rows.end) store_row<ES>((char*)a.out + (m0 + r) * a.ldo * ES, c0 + c * V, a.cols, v);
            }
            asm volatile("" ::: "memory");
        }
    });
}

template <int BM, int BN, int WM, int WN, int GROUPS, int BUFFERS, bool DIRECT>
hipError_t launch_many(const ProductMxArgs& a, hipStream_t s) {
    const uint32_t nblocks = (a.cols + BN - 1) / BN, threads = WM * WN * 64;
    const uint64_t blocks = most_tiles(a, BM) * nblocks;
    if (blocks + 8 > 0xffffffffull / threads) return hipErrorInvalidConfiguration;
    const dim3 grid((uint32_t)((blocks + 7) / 8 * 8));
    hipLaunchKernelGGL((hccl_moe_product_mx_many_kernel<BM, BN, WM, WN, GROUPS, BUFFERS, DIRECT>), grid, dim3(threads), 0, s, a, nblocks);
    return hipGetLastError();
}

template <int MB, int NB, int W>
hipError_t launch_few(const ProductMxArgs& a, hipStream_t s) {
    const uint64_t nblocks = (a.cols + 16 * NB - 1) / (16 * NB), tiles = most_tiles(a, 16 * MB);
    if (tiles * nblocks > 0xffffffffull / (W * 64)) return hipErrorInvalidConfiguration;
    const dim3 grid((uint32_t)(tiles * nblocks)), block(W * 64);
    const bool aligned = (((uintptr_t)a.b | a.ldb) % 16 | ((uintptr_t)a.b_scale | a.ldbs) % 4) == 0;
    if (aligned) hipLaunchKernelGGL((hccl_moe_product_mx_few_kernel<MB, NB, W, true>), grid, block, 0, s, a, (uint32_t)nblocks);
    else hipLaunchKernelGGL((hccl_moe_product_mx_few_kernel<MB, NB, W, false>), grid, block, 0, s, a, (uint32_t)nblocks);
    return hipGetLastError();
}

}  // namespace

// Which kernel, by the rows of a segment and the blocks that leaves (microseconds; rows x inner x columns x experts; weights
// that lie in no cache where none is said). Tiles: as large as keep most CUs busy and are mostly full.
//   256 x 256 or 128 x 128: 4096 x 4096 x 4096 x 1 45 : 62 (256 blocks), 2048 rows 36 : 34 (128); 16384 x 2048 x 2048 x 64
//     75 : 86 (256 rows a segment), 12800 rows 51 : 53 (200; in cache 47 : 45). Rows that are not 16-byte aligned go through
//     registers, of which the largest tile has none left.
//   128 x 128 or 64 x 128: 3000 x 2048 x 1408 x 16 18.5 : 19.3 (187 rows a segment), 2048 rows 20 : 16 (128), 8192 rows of 64
//     experts 44 : 43 (128; in cache 39 : 35), 1024 x 4096 x 4096 x 1 22.3 : 22.6, 8192 x 8192 x 8192 x 1 417 : 557.
//   64 x 128 or few rows: 512 x 4096 x 4096 x 1 19 : 25; 1024 x 2048 x 2048 x 64 31.3 : 32.5 (16 rows a segment), 512 rows 30.6 :
//     28 (8). 64 x 64 or few rows: 256 x 4096 x 4096 x 1 16.5 : 15.2, in cache 10.7 : 13.1 (256 blocks), 128 rows 16 : 10.8 (128).
// Few rows: 16 a block cost less than 32 up to 12 a segment (768 x 2048 x 2048 x 64 31 : 33). As many columns a block as
// leave blocks enough: 64 or 32, the inner size shared by 2 or 4 waves: 1024 x 1024 x 4096 x 256 97 : 147 (20 480 blocks of 64),
// 256 x 2048 x 2048 x 64 27.6 : 26.0 (2 560); 32 or 16: 1 x 8192 x 12288 x 1 13.9 : 15.3 (384 blocks of 32), 1 x 4096 x 4096 x 1
// 6.0 : 4.8 (128), 24 x 4096 x 8192 x 1 7.6 : 8.7 (256).
hipError_t launch_product_mx(const ProductMxArgs& a, int cus, hipStream_t s) {
    const uint64_t each = a.rows / a.segments, spread = a.offsets ? (a.rows < a.segments ? a.rows : a.segments) : 0;
    auto blocks = [&](uint64_t bm, uint64_t bn) {  // about; half a tile more for every segment
        return (a.offsets ? a.rows / bm + (spread + 1) / 2 : (a.rows + bm - 1) / bm) * ((a.cols + bn - 1) / bn);
    };
    const bool direct = (((uintptr_t)a.a | a.lda | (uintptr_t)a.b | a.ldb) % 16) == 0;
    const uint64_t most = a.inner >= kMxBlock ? (uint64_t)cus * 3 / 4 : ~0ull;  // (tiles want 16 bytes of codes a row)
    if (each >= 256 && direct && blocks(256, 256) >= most) return launch_many<256, 256, 2, 4, 2, 4, true>(a, s);
    if (each >= 192 && blocks(128, 128) >= most) return direct ? launch_many<128, 128, 2, 2, 1, 3, true>(a, s) : launch_many<128, 128, 2, 2, 1, 3, false>(a, s);
    if (each >= 16 && blocks(64, 128) >= most) return direct ? launch_many<64, 128, 1, 4, 1, 3, true>(a, s) : launch_many<64, 128, 1, 4, 1, 3, false>(a, s);
    if (each > 64 && a.inner >= kMxBlock && blocks(64, 64) >= (uint64_t)cus)
        return direct ? launch_many<64, 64, 1, 2, 1, 3, true>(a, s) : launch_many<64, 64, 1, 2, 1, 3, false>(a, s);
    const uint64_t cols16 = (a.cols + 15) / 16;
    if (a.offsets ? each <= 12 : a.rows <= 16) {
        const uint64_t tiles = a.offsets ? a.rows / 16 + spread : 1;
        if (tiles * (cols16 / 4) >= (uint64_t)cus * 16) return launch_few<1, 4, 2>(a, s);
        if (tiles * (cols16 / 2) >= (uint64_t)cus) return launch_few<1, 2, 4>(a, s);
        return launch_few<1, 1, 8>(a, s);
    }
    const uint64_t tiles = a.offsets ? a.rows / 32 + spread : (a.rows + 31) / 32;
    if (tiles * (cols16 / 4) >= (uint64_t)cus * 16) return launch_few<2, 4, 2>(a, s);
    if (tiles * (cols16 / 2) >= (uint64_t)cus) return launch_few<2, 2, 4>(a, s);
    return launch_few<2, 1, 4>(a, s);
}

}  // namespace hccl
