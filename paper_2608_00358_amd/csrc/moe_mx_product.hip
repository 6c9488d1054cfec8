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
// (256 elements) and join their sums through LDS, in the waves' order. Weights go from memory to registers: each is used
// by one block only. A lane reads 32 neighbouring bytes of a row, two blocks, and their two scale bytes; four lanes
// the 128 bytes of a step. The loads of U steps are on their way together.
template <int MB, int NB, int W, int U>
__global__ __launch_bounds__(W * 64) void hccl_moe_product_mx_few_kernel(ProductMxArgs a, uint32_t nblocks) {
    constexpr uint32_t BM = 16 * MB, BN = 16 * NB;
    __shared__ v4f part[W][MB * NB][64];
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
    v4i va[U][MB][2], vb[U][NB][2];
    uint32_t ra[U][MB], rb[U][NB];
    const uint32_t blocks = (a.inner + kMxBlock - 1) / kMxBlock;
    auto scales = [&](const uint8_t* p, uint32_t b, auto inside) -> uint32_t {  // of the blocks b and b + 1
        typedef uint16_t loose __attribute__((aligned(1)));
        if (inside.value || b + 2 <= blocks) return *gptr<loose>(p + b);
        return b < blocks ? *gptr<uint8_t>(p + b) : 0u;
    };
    auto fetch = [&](int u, uint32_t k0, auto inside) {  // INSIDE: the step lies inside the rows
        const uint32_t k = k0 + q * 32;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int y = 0; y < NB; ++y) vb[u][y][h] = inside.value ? (v4i)load16<1>(pb[y] + k + 16 * h) : (v4i)load_codes<false, false>(pb[y], k + 16 * h, a.inner);
#pragma unroll
            for (int x = 0; x < MB; ++x) va[u][x][h] = inside.value ? (v4i)load16<1>(pa[x] + k + 16 * h) : (v4i)load_codes<false, true>(pa[x], k + 16 * h, a.inner);
        }
#pragma unroll
        for (int y = 0; y < NB; ++y) rb[u][y] = scales(sb[y], k / 16, inside);
#pragma unroll
        for (int x = 0; x < MB; ++x) ra[u][x] = scales(sa[x], k / 16, inside);
    };
    auto multiply = [&](int u) {
#pragma unroll
        for (int x = 0; x < MB; ++x)
#pragma unroll
            for (int y = 0; y < NB; ++y) {
                acc[x][y] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(whole(vb[u][y][0]), whole(va[u][x][0]), acc[x][y], kFp4, kFp4, 0, rb[u][y], 0, ra[u][x]);
                acc[x][y] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(whole(vb[u][y][1]), whole(va[u][x][1]), acc[x][y], kFp4, kFp4, 1, rb[u][y], 1, ra[u][x]);
            }
    };
    const uint32_t bytes = a.inner / 2, all = (a.inner + 1) / 2;  // (whole bytes)
    uint32_t k0 = w * 128;
    for (; k0 + (U - 1) * (W * 128) + 128 <= bytes; k0 += U * (W * 128)) {
#pragma unroll
        for (int u = 0; u < U; ++u) fetch(u, k0 + u * (W * 128), std::true_type());
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = 0; u < U; ++u) multiply(u);
    }
#pragma unroll 1
    for (; k0 < all; k0 += W * 128) {
        if (k0 + 128 <= bytes) fetch(0, k0, std::true_type());
        else fetch(0, k0, std::false_type());
        multiply(0);
    }
#pragma unroll
    for (int x = 0; x < MB; ++x)
#pragma unroll
        for (int y = 0; y < NB; ++y) part[w][x * NB + y][lane] = acc[x][y];
    __syncthreads();
    for (uint32_t p = w; p < MB * NB; p += W) {
        v4f sum = part[0][p][lane];
#pragma unroll
        for (int v = 1; v < W; ++v) {
            const v4f more = part[v][p][lane];
#pragma unroll
            for (int j = 0; j < 4; ++j) sum[j] += more[j];
        }
        const uint64_t m = rows.first + p / NB * 16 + i;
        const uint32_t n = n0 + p % NB * 16 + q * 4;
        if (m < rows.end && n < a.cols) by_result(a.type, [&](auto type) { store_four<decltype(type)::value>(a, m, n, sum); });
    }
}

// Many rows a segment: BM rows by BN columns a block, in WM x WN waves, k in steps of 64 bytes (128 elements, four blocks)
// through four LDS buffers: one is multiplied while the next three are filled, by loads that go to LDS directly
// (DIRECT: 1 for rows, 2 for weights that are 16-byte aligned) or through registers (any alignment, and the
// last step of an inner size that is no multiple of 128, where codes past the end are zero).
//
// LDS holds a row's 64 bytes as 4 chunks of 16; chunk c of row r lies in slot c ^ (r / 4 & 3), so that the
// 16 lanes served together, which read one chunk of 16 rows, use different banks. A direct load writes its 64 lanes one
// after the other, so a lane reads the chunk that belongs in its slot.
//
// Scales: a thread has one row, of the tile's rows or columns, whose next 16 scale bytes (four steps) it reads into a
// register four steps ahead and puts into LDS two steps before they count, there being two such buffers. A step's four
// bytes of a row are one 32-bit word; a lane moves it down by its half's chunk, and the instructions take byte 0 or 2.
//
// Fragments are read one part (32 of the 64 bytes) ahead of the matrix instructions. The barrier stands
// inside a step's last part: by then all its fragments have been read, so the next step's buffer can be
// read and the old one refilled while that part is still being multiplied.
constexpr uint32_t kStep = 64;
constexpr uint32_t kBuffers = 4;
constexpr uint32_t kBand = 4;

typedef __attribute__((address_space(3))) void* lds_ptr;

template <int N>
__device__ __forceinline__ void wait_loads() {  // until at most N loads are on their way, and LDS is done
    __builtin_amdgcn_s_waitcnt(0x70 | N);
}
// A barrier that leaves loads to LDS in flight; nothing that touches memory moves across it.
__device__ __forceinline__ void meet() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

template <int BM, int BN, int WM, int WN, int DIRECT>
__global__ __launch_bounds__(WM * WN * 64) void hccl_moe_product_mx_many_kernel(ProductMxArgs a, uint32_t nblocks) {
    constexpr int W = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32;
    constexpr int LA = BM / 16 / W, LB = BN / 16 / W, LN = LA + LB;  // loads a wave makes for a step: 16 rows each
    static_assert(BM % (16 * W) == 0 && BN % (16 * W) == 0 && 3 * LN < 16, "whole loads, and a counter that holds them");
    static_assert(BM + BN <= W * 64, "a thread has the scales of one row");
    constexpr uint32_t kBuffer = (BM + BN) * kStep, kScales = (BM + BN) * 16;
    __shared__ __attribute__((aligned(256))) char lds[kBuffers * kBuffer];
    __shared__ __attribute__((aligned(256))) char lds_scale[2 * kScales];
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
    const uint8_t* src[LN];
#pragma unroll
    for (int i = 0; i < LA; ++i) src[i] = a.a + row_of((w * LA + i) * 16 + lrow) * a.lda + chunk;
#pragma unroll
    for (int i = 0; i < LB; ++i) src[LA + i] = a.b + col_of((w * LB + i) * 16 + lrow) * a.ldb + chunk;
    auto slot = [&](uint32_t s, int i) { return lds + (s % kBuffers) * kBuffer + (i < LA ? (w * LA + i) * 16 : BM + (w * LB + i - LA) * 16) * kStep; };
    const uint8_t* scale_src = threadIdx.x < BM ? a.a_scale + row_of(threadIdx.x) * a.ldas : a.b_scale + col_of(threadIdx.x < BM + BN ? threadIdx.x - BM : 0) * a.ldbs;
    const uint32_t scale_bytes = threadIdx.x < BM + BN ? (a.inner + kMxBlock - 1) / kMxBlock : 0;

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
    constexpr bool kAll = DIRECT == 3;
    auto direct = [](int i) { return (DIRECT & (i < LA ? 1 : 2)) != 0; };
    v4u held[2][LN];  // on their way through registers: steps of either parity
    v4u held_scale;   // scales of four steps, on their way
    // Load i of those that bring in step s. INNER: it and the steps before it are whole.
    auto fetch = [&](uint32_t s, int parity, auto inner, int i) {
        if (direct(i) && (inner.value || s < whole_steps)) {
            __builtin_amdgcn_global_load_lds((const HCCL_AS1 void*)(src[i] + (uint64_t)s * kStep), (lds_ptr)slot(s, i), 16, 0, 0);
        } else if (inner.value || s < steps) {
            const v4u v = inner.value || s < whole_steps ? load16<1>(src[i] + (uint64_t)s * kStep) : i < LA ? load_codes<true, true>(src[i] - chunk, s * kStep + chunk, a.inner)
                                                                                                                  : load_codes<true, false>(src[i] - chunk, s * kStep + chunk, a.inner);
            if (direct(i)) *(v4u*)(slot(s, i) + lane * 16) = v;
            else held[parity][i] = v;
        }
    };
    auto fetch_all = [&](uint32_t s, int parity, auto inner) {
#pragma unroll
        for (int i = 0; i < LN; ++i) fetch(s, parity, inner, i);
    };
    auto put = [&](uint32_t s, int parity) {  // what registers hold of step s goes to its buffer
#pragma unroll
        for (int i = 0; i < LN; ++i)
            if (!direct(i)) *(v4u*)(slot(s, i) + lane * 16) = held[parity][i];
    };
    auto fetch_scales = [&](uint32_t four) { held_scale = load_bytes<false>(scale_src, four * 16, scale_bytes); };
    auto put_scales = [&](uint32_t four) {
        if (BM + BN == W * 64 || threadIdx.x < BM + BN) *(v4u*)(lds_scale + (four & 1) * kScales + threadIdx.x * 16) = held_scale;
    };
    // In the second of four steps s: the scales of the next four go to LDS, those after them on their way.
    auto stage = [&](uint32_t s) {
        put_scales(s / 4 + 1);
        fetch_scales(s / 4 + 2);
    };
    v4i va[2][TM], vb[2][TN];
    uint32_t sa[2][TM], sb[2][TN];
    auto read = [&](uint32_t s, uint32_t part, int i) {  // fragment i of a part, in the order of their use
        const uint32_t at = (s % kBuffers) * kBuffer + ((part * 2 + (lane >> 5)) ^ (lane >> 2 & 3)) * 16 + (lane & 31) * kStep;
        if (i == 0) va[part][0] = *(const v4i*)(lds + wm * TM * 32 * kStep + at);
        else if (i <= TN) vb[part][i - 1] = *(const v4i*)(lds + (BM + (wn * TN + i - 1) * 32) * kStep + at);
        else va[part][i - TN] = *(const v4i*)(lds + (wm * TM + i - TN) * 32 * kStep + at);
    };
    auto read_scale = [&](uint32_t s, int parity, int i) {
        const char* at = lds_scale + (s / 4 & 1) * kScales + (s & 3) * 4 + (lane & 31) * 16;
        if (i < TN) sb[parity][i] = *(const uint32_t*)(at + (BM + (wn * TN + i) * 32) * 16) >> (lane >> 5) * 8;
        else sa[parity][i - TN] = *(const uint32_t*)(at + (wm * TM + i - TN) * 32 * 16) >> (lane >> 5) * 8;
    };
    // A part's matrix instructions, one after the other, each followed by a load or a read or two: a wave
    // that makes its loads in one go waits for the units that take them, and its SIMD with it.
    constexpr int kMfmas = TM * TN, kReads = TM + TN, kFirst = kMfmas >= 8 ? 2 : 1;
    auto multiply = [&](auto part, int parity, int from, int to, auto between) {
        constexpr int P = decltype(part)::value;
#pragma unroll
        for (int i = from; i < to; ++i) {
            acc[i % TN][i / TN] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(whole(vb[P][i % TN]), whole(va[P][i / TN]), acc[i % TN][i / TN], kFp4, kFp4,
                                                                                2 * P, sb[parity][i % TN], 2 * P, sa[parity][i / TN]);
            __builtin_amdgcn_sched_barrier(0);
            between(i);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // Those of n operations that go behind instruction i, spread over `slots` of them from `from` on.
    auto spread = [](int i, int from, int slots, int n, auto f) {
        const int at = i - from;
        if (at < 0 || at >= slots) return;
#pragma unroll
        for (int r = at * n / slots; r < (at + 1) * n / slots; ++r) f(r);
    };
    // reads end two instructions before the part does, so that they are there when the next one begins
    constexpr int kReadSlots = kMfmas >= 8 ? kMfmas - kFirst - 2 : kMfmas >= 4 ? 2 : 1;
    const std::integral_constant<int, 0> first_part;
    const std::integral_constant<int, 1> second_part;
    // Step s + 1 has landed for all waves, and all have read step s, whose buffer step s + 4 takes. Loads of
    // the steps s + 2 and s + 3 stay on their way (where all are direct loads; where some pass through registers,
    // step s + 2 is needed there, and only those of step s + 3 do).
    auto land = [&](uint32_t s, int parity, auto inner) {
        if (inner.value || s + 2 < steps) put(s + 2, parity);
        if (DIRECT == 0) __builtin_amdgcn_s_waitcnt(0xc07f);  // LDS alone
        else if (inner.value || s + 3 < whole_steps) wait_loads<kAll ? 2 * LN : LN>();
        else wait_loads<0>();
        meet();
    };
    auto step = [&](uint32_t s, int phase, auto inner) {
        const int parity = phase & 1;
        multiply(first_part, parity, 0, kMfmas, [&](int i) {
            spread(i, kFirst - 1, kReadSlots, kReads, [&](int r) { read(s, 1, r); });
            spread(i, kFirst - 1, kMfmas - kFirst + 1, LN, [&](int r) { fetch(s + 3, parity ^ 1, inner, r); });
        });
        multiply(second_part, parity, 0, kFirst, [](int) {});
        if (inner.value ? phase == 1 : (s & 3) == 1) stage(s);
        land(s, parity, inner);
        const bool more = inner.value || s + 1 < steps;
        multiply(second_part, parity, kFirst, kMfmas, [&](int i) {
            if (more) spread(i, kFirst, kReadSlots, 2 * kReads, [&](int r) {
                if (r & 1) read(s + 1, 0, r / 2);
                else read_scale(s + 1, parity ^ 1, r / 2);
            });
        });
    };
    auto idle = [&](uint32_t s, int phase, auto inner) {  // a step of a wave without rows: brings in its part for the others
        const int parity = phase & 1;
        fetch_all(s + 3, parity ^ 1, inner);
        if (inner.value ? phase == 1 : (s & 3) == 1) stage(s);
        land(s, parity, inner);
    };
    auto walk = [&](auto each) {
        uint32_t s = 0;
        for (; s + 6 < whole_steps; s += 4) {
            each(s, 0, std::true_type());
            each(s + 1, 1, std::true_type());
            each(s + 2, 2, std::true_type());
            each(s + 3, 3, std::true_type());
        }
#pragma unroll 1
        for (; s < steps; s += 2) {
            each(s, 0, std::false_type());
            if (s + 1 < steps) each(s + 1, 1, std::false_type());
        }
    };
    if (steps) {
        const std::false_type any;
        fetch_scales(0);
        fetch_all(0, 0, any), fetch_all(1, 1, any);
        put_scales(0);
        put(0, 0);
        if (steps > 1) put(1, 1);
        fetch_all(2, 0, any);
        fetch_scales(1);
        wait_loads<0>();
        meet();
        if (rows.first + wm * TM * 32 >= rows.end) {
            walk(idle);
            return;
        }
#pragma unroll
        for (int r = 0; r < kReads; ++r) read(0, 0, r), read_scale(0, 0, r);
        walk(step);
    }

    // The wave's TM x TN blocks leave through its own part of LDS, as rows of TN * 32 results: lanes that hold
    // four results each of 32 rows would store 16 bytes of a line at a time.
    by_result(a.type, [&](auto type) {
        constexpr int DT = decltype(type)::value;
        constexpr int ES = kSize<DT>;
        constexpr uint32_t kLine = TN * 32 * ES, kChunks = kLine / 16;  // bytes of a row
        constexpr int kRowsEach = kBuffers * kBuffer / W / kLine >= TM * 32 ? TM : kBuffers * kBuffer / W / kLine / 32;  // blocks of 32 rows at a time
        static_assert(kRowsEach >= 1 && TM % kRowsEach == 0, "a block of rows fits");
        // (nothing reads the buffers after the last step's barrier)
        char* mine = lds + w * (kBuffers * kBuffer / W);
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

template <int BM, int BN, int WM, int WN>
hipError_t launch_many(const ProductMxArgs& a, hipStream_t s) {
    const uint32_t nblocks = (a.cols + BN - 1) / BN, threads = WM * WN * 64;
    const uint64_t blocks = most_tiles(a, BM) * nblocks;
    if (blocks + 8 > 0xffffffffull / threads) return hipErrorInvalidConfiguration;
    const dim3 grid((uint32_t)((blocks + 7) / 8 * 8));
    const int direct = (((uintptr_t)a.a | a.lda) % 16 == 0 ? 1 : 0) | (((uintptr_t)a.b | a.ldb) % 16 == 0 ? 2 : 0);
    if (direct == 3) hipLaunchKernelGGL((hccl_moe_product_mx_many_kernel<BM, BN, WM, WN, 3>), grid, dim3(threads), 0, s, a, nblocks);
    else if (direct == 2) hipLaunchKernelGGL((hccl_moe_product_mx_many_kernel<BM, BN, WM, WN, 2>), grid, dim3(threads), 0, s, a, nblocks);
    else if (direct == 1) hipLaunchKernelGGL((hccl_moe_product_mx_many_kernel<BM, BN, WM, WN, 1>), grid, dim3(threads), 0, s, a, nblocks);
    else hipLaunchKernelGGL((hccl_moe_product_mx_many_kernel<BM, BN, WM, WN, 0>), grid, dim3(threads), 0, s, a, nblocks);
    return hipGetLastError();
}

template <int MB, int NB, int W, int U>
hipError_t launch_few(const ProductMxArgs& a, hipStream_t s) {
    const uint64_t nblocks = (a.cols + 16 * NB - 1) / (16 * NB), tiles = most_tiles(a, 16 * MB);
    if (tiles * nblocks > 0xffffffffull / (W * 64)) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL((hccl_moe_product_mx_few_kernel<MB, NB, W, U>), dim3((uint32_t)(tiles * nblocks)), dim3(W * 64), 0, s, a, (uint32_t)nblocks);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_product_mx(const ProductMxArgs& a, int cus, hipStream_t s) {
    const uint64_t each = a.rows / a.segments, spread = a.offsets ? (a.rows < a.segments ? a.rows : a.segments) : 0;
    auto blocks = [&](uint64_t bm, uint64_t bn) {  // about; half a tile more for every segment
        return (a.offsets ? a.rows / bm + (spread + 1) / 2 : (a.rows + bm - 1) / bm) * ((a.cols + bn - 1) / bn);
    };
    const uint64_t most = a.inner >= kMxBlock ? (uint64_t)cus * 3 / 4 : ~0ull;  // (tiles want 16 bytes of codes a row)
    if (each >= 128 && blocks(256, 256) >= most) return launch_many<256, 256, 2, 4>(a, s);
    if (each >= 32 && blocks(128, 128) >= most) return launch_many<128, 128, 2, 2>(a, s);
    if (each >= 16 && blocks(64, 128) >= most) return launch_many<64, 128, 1, 4>(a, s);
    if (each > 64 && a.inner >= kMxBlock && blocks(64, 64) >= (uint64_t)cus / 2) return launch_many<64, 64, 1, 2>(a, s);
    if (a.offsets ? each <= 8 : a.rows <= 16) {
        const uint64_t tiles = a.offsets ? a.rows / 16 + spread : 1, cols16 = (a.cols + 15) / 16;
        if (tiles * (cols16 / 4) >= (uint64_t)cus) return launch_few<1, 4, 4, 2>(a, s);
        if (tiles * (cols16 / 2) >= (uint64_t)cus) return launch_few<1, 2, 4, 4>(a, s);
        return launch_few<1, 1, 16, 2>(a, s);
    }
    const uint64_t tiles = a.offsets ? a.rows / 32 + spread : (a.rows + 31) / 32, cols16 = (a.cols + 15) / 16;
    if (tiles * (cols16 / 4) >= (uint64_t)cus) return launch_few<2, 4, 4, 2>(a, s);
    if (tiles * (cols16 / 2) >= (uint64_t)cus) return launch_few<2, 2, 8, 2>(a, s);
    return launch_few<2, 1, 16, 2>(a, s);
}

}  // namespace hccl
