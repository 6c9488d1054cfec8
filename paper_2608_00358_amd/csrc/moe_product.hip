// moe_product.hip -- the experts' product in 8-bit integers:
//   out[m, n] = a_scale[m] * b_scale[e, n] * sum_k a[m, k] b[e, n, k],   e the expert of row m's segment
// on the matrix instructions for 8-bit integers, with whole sums in 32 bits (exact: at most 131 071 products of at
// most 2^14), which become 32-bit floats only for the scales (a sum above 2^24 is rounded there, by 2^-24 of itself at
// most, as each of the two products with the scales is). The rows of a segment follow each other; where segments begin
// is read on the device, so the grid is sized for the worst case and surplus blocks end at once. A tile holds rows of one
// segment: where several segments use one expert (rows of several sources), its weights are read for each of them.
//
// The weights are the instruction's first operand: a lane then holds neighbouring columns of one row.
// The order of k within an instruction does not matter as long as both operands have the same.
//
// Bounds: with few rows a segment, the weights' bytes (256 rows over 64 experts of 2048 x 2048, of which about 53 have
// a row: 235 MB in 42 us, 5.6 TB/s, where a large copy reaches 6.2); with many, power and the loads from L2 to LDS
// (8192 x 8192 x 8192 in 475-490 us, 2.25-2.3 POPS, where a library product takes 518 us; in long products the matrix
// units alone, without any load, bring the clock down to 1.9 GHz, and the whole kernel to 1.7).
#include <type_traits>

#include "moe_device.h"

namespace hccl {
namespace {

typedef int32_t v4i __attribute__((ext_vector_type(4)));
typedef int32_t v16i __attribute__((ext_vector_type(16)));

struct Rows {
    uint64_t first, end;
    uint32_t expert;
};

// (offsets outside 0 .. rows are clipped, and a segment that ends before it begins is empty)
__device__ __forceinline__ void segment(const ProductArgs& a, uint32_t s, uint64_t& first, uint64_t& end) {
    const int64_t lo = a.offsets[s], hi = a.offsets[s + 1];
    first = lo < 0 ? 0 : (uint64_t)lo < a.rows ? (uint64_t)lo : a.rows;
    end = hi < (int64_t)first ? first : (uint64_t)hi < a.rows ? (uint64_t)hi : a.rows;
}

// 64 segments, one a lane: their rows, their tiles of BM rows and the running sum of those (which 32 bits hold even
// where all 64 have every row: that is at most 2^25 tiles of 64 rows each, or, by the limit of a launch, 2^24 of fewer).
template <uint32_t BM>
struct Segments {
    uint64_t first, end;
    uint32_t n, incl, all;
    __device__ __forceinline__ Segments(const ProductArgs& a, uint32_t s0) {
        const uint32_t lane = threadIdx.x & 63, s = s0 + lane;
        first = end = 0;
        if (!a.offsets) {  // one segment, which find_rows does not look for
            all = (uint32_t)((a.rows + BM - 1) / BM);
            return;
        }
        if (s < a.segments) segment(a, s, first, end);
        n = (uint32_t)((end - first + BM - 1) / BM);
        incl = n;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const uint32_t v = (uint32_t)__shfl_up((int)incl, d);
            if (lane >= (uint32_t)d) incl += v;
        }
        all = at_lane(incl, 63);
    }
};

// Tiles that the segments have; `s` holds the first 64 of them.
template <uint32_t BM>
__device__ __forceinline__ uint32_t count_tiles(const ProductArgs& a, const Segments<BM>& s) {
    uint32_t n = s.all;
    for (uint32_t s0 = kWave; s0 < a.segments; s0 += kWave) n += Segments<BM>(a, s0).all;
    return n;
}

// Rows [first, end) of tile `tile`, and its expert; false where there are fewer tiles.
template <uint32_t BM>
__device__ __forceinline__ bool find_rows(const ProductArgs& a, Segments<BM> s, uint32_t tile, Rows& out) {
    if (!a.offsets) {
        out.first = (uint64_t)tile * BM;
        out.end = a.rows;
        out.expert = 0;
        return tile < s.all;
    }
    uint32_t left = tile;
    for (uint32_t s0 = 0;;) {
        if (left < s.all) {
            const uint32_t l = first_lane((uint32_t)__popcll(__ballot(s.incl <= left)));
            const uint32_t skip = left - (at_lane(s.incl, l) - at_lane(s.n, l));
            out.first = ((uint64_t)at_lane((uint32_t)(s.first >> 32), l) << 32 | at_lane((uint32_t)s.first, l)) + (uint64_t)skip * BM;
            out.end = (uint64_t)at_lane((uint32_t)(s.end >> 32), l) << 32 | at_lane((uint32_t)s.end, l);
            out.expert = (s0 + l) % a.experts;
            return true;
        }
        left -= s.all;
        s0 += kWave;
        if (s0 >= a.segments) return false;
        s = Segments<BM>(a, s0);
    }
}

// 16 bytes of a row at k; bytes from `inner` on are zero: the row's last 16 bytes, shifted down.
__device__ __forceinline__ v4i load_k(const int8_t* row, uint32_t k, uint32_t inner) {
    if (k + 16 <= inner) return (v4i)load16<1>(row + k);
    v4i r = {0, 0, 0, 0};
    if (k >= inner) return r;
    if (inner >= 16) return (v4i)shift_down(load16<1>(row + inner - 16), 8 * (k + 16 - inner));
    for (uint32_t i = 0; k + i < inner; ++i) {  // (a row of fewer than 16 bytes; k is 0)
        const uint32_t v = (uint32_t)(uint8_t)*gptr<int8_t>(row + k + i) << (8 * (i & 3));
        r[0] |= i / 4 == 0 ? v : 0;
        r[1] |= i / 4 == 1 ? v : 0;
        r[2] |= i / 4 == 2 ? v : 0;
        r[3] |= i / 4 == 3 ? v : 0;
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
// by one block only. A lane reads 32 neighbouring bytes of a row, four lanes the 128 of a step; the loads
// of U steps are on their way together.
template <int DT, int MB, int NB, int W, int U>
__global__ __launch_bounds__(W * 64) void hccl_moe_product_few_kernel(ProductArgs a, uint32_t nblocks) {
    constexpr uint32_t BM = 16 * MB, BN = 16 * NB;
    __shared__ v4i part[W][MB * NB][64];
    const uint32_t lane = threadIdx.x & 63, w = first_lane(threadIdx.x >> 6);
    const uint32_t tile = blockIdx.x / nblocks, n0 = blockIdx.x % nblocks * BN;
    Rows rows;
    if (!find_rows<BM>(a, Segments<BM>(a, 0), tile, rows)) return;
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
    v4i va[U][MB][2], vb[U][NB][2];
    auto fetch = [&](int u, uint32_t k0, auto inner) {  // INNER: the step lies inside the rows
        const uint32_t k = k0 + q * 32;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int y = 0; y < NB; ++y) vb[u][y][h] = inner.value ? (v4i)load16<1>(pb[y] + k + 16 * h) : load_k(pb[y], k + 16 * h, a.inner);
#pragma unroll
            for (int x = 0; x < MB; ++x) va[u][x][h] = inner.value ? (v4i)load16<1>(pa[x] + k + 16 * h) : load_k(pa[x], k + 16 * h, a.inner);
        }
    };
    auto multiply = [&](int u) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int x = 0; x < MB; ++x)
#pragma unroll
                for (int y = 0; y < NB; ++y) acc[x][y] = __builtin_amdgcn_mfma_i32_16x16x64_i8(vb[u][y][h], va[u][x][h], acc[x][y], 0, 0, 0);
    };
    uint32_t k0 = w * 128;
    for (; k0 + (U - 1) * (W * 128) + 128 <= a.inner; k0 += U * (W * 128)) {
#pragma unroll
        for (int u = 0; u < U; ++u) fetch(u, k0 + u * (W * 128), std::true_type());
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = 0; u < U; ++u) multiply(u);
    }
#pragma unroll 1
    for (; k0 < a.inner; k0 += W * 128) {
        if (k0 + 128 <= a.inner) fetch(0, k0, std::true_type());
        else fetch(0, k0, std::false_type());
        multiply(0);
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

// Many rows a segment: BM rows by BN columns a block, in WM x WN waves, k in steps of 64 through four
// LDS buffers: one is multiplied while the next three are filled, by loads that go to LDS directly
// (DIRECT: 1 for rows, 2 for weights that are 16-byte aligned) or through registers (any alignment, and the
// last step of an inner size that is no multiple of 64, where bytes past the end are zero).
//
// LDS holds a row's 64 bytes as 4 chunks of 16; chunk c of row r lies in slot c ^ (r / 4 & 3), so that the
// 16 lanes served together, which read one chunk of 16 rows, use different banks (four rows fill the 256
// bytes of all banks; with conflicts LDS was busy twice as long). A direct load writes its 64 lanes one
// after the other, so a lane reads the chunk that belongs in its slot.
//
// Fragments are read one part (32 of the 64 k) ahead of the matrix instructions. The barrier stands
// inside a step's last part: by then all its fragments have been read, so the next step's buffer can be
// read and the old one refilled while that part is still being multiplied.
constexpr uint32_t kStep = 64;
constexpr uint32_t kBuffers = 4;
constexpr uint32_t kBand = 4;  // (4, 8 and 16: 328, 332 and 348 us for 16 384 rows through 16 experts)

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

template <int DT, int BM, int BN, int WM, int WN, int DIRECT>
__global__ __launch_bounds__(WM * WN * 64) void hccl_moe_product_many_kernel(ProductArgs a, uint32_t nblocks) {
    constexpr int W = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32;
    constexpr int LA = BM / 16 / W, LB = BN / 16 / W, LN = LA + LB;  // loads a wave makes for a step: 16 rows each
    static_assert(BM % (16 * W) == 0 && BN % (16 * W) == 0 && 3 * LN < 16, "whole loads, and a counter that holds them");
    constexpr uint32_t kBuffer = (BM + BN) * kStep;
    __shared__ __attribute__((aligned(256))) char lds[kBuffers * kBuffer];
    const uint32_t lane = threadIdx.x & 63, w = first_lane(threadIdx.x >> 6);

    // Blocks go to the XCDs in turn; each XCD gets neighbouring tiles, in bands of kBand column blocks, so
    // that the tiles it works on at a time share their rows and weights in its L2. (Ends of segments, which are
    // less work, in a turn of their own after the whole tiles read the weights twice: 346 us against 337 for
    // 16 384 rows through 16 experts.)
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

    // where this lane's part of each load comes from, and where in a buffer each load goes
    const uint32_t lrow = lane >> 2, chunk = ((lane & 3) ^ (lrow >> 2)) * 16;
    const int8_t* src[LN];
#pragma unroll
    for (int i = 0; i < LA; ++i) {
        const uint64_t m = rows.first + (w * LA + i) * 16 + lrow;
        src[i] = a.a + (m < rows.end ? m : rows.end - 1) * a.lda + chunk;
    }
#pragma unroll
    for (int i = 0; i < LB; ++i) {
        const uint32_t n = n0 + (w * LB + i) * 16 + lrow;
        src[LA + i] = a.b + ((uint64_t)rows.expert * a.cols + (n < a.cols ? n : a.cols - 1)) * a.ldb + chunk;
    }
    auto slot = [&](uint32_t s, int i) { return lds + (s % kBuffers) * kBuffer + (i < LA ? (w * LA + i) * 16 : BM + (w * LB + i - LA) * 16) * kStep; };

    v16i acc[TN][TM];
#pragma unroll
    for (int y = 0; y < TN; ++y)
#pragma unroll
        for (int x = 0; x < TM; ++x)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[y][x][r] = 0;

    const uint32_t steps = (a.inner + kStep - 1) / kStep, whole = a.inner / kStep;
    // Waves of the same rows are neighbours, and so on different SIMDs: where an end of a segment leaves
    // waves without rows, those that have some share out the matrix units.
    const uint32_t wm = w / WN, wn = w % WN;
    constexpr bool kAll = DIRECT == 3;
    auto direct = [](int i) { return (DIRECT & (i < LA ? 1 : 2)) != 0; };
    v4u held[2][LN];  // on their way through registers: steps of either parity
    // Load i of those that bring in step s. INNER: it and the steps before it are whole.
    auto fetch = [&](uint32_t s, int parity, auto inner, int i) {
        if (direct(i) && (inner.value || s < whole)) {
            __builtin_amdgcn_global_load_lds((const HCCL_AS1 void*)(src[i] + (uint64_t)s * kStep), (lds_ptr)slot(s, i), 16, 0, 0);
        } else if (inner.value || s < steps) {
            const v4u v = inner.value || s < whole ? load16<1>(src[i] + (uint64_t)s * kStep) : (v4u)load_k(src[i] - chunk, s * kStep + chunk, a.inner);
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
    v4i va[2][TM], vb[2][TN];
    auto read = [&](uint32_t s, uint32_t part, int i) {  // fragment i of a part, in the order of their use
        const uint32_t at = (s % kBuffers) * kBuffer + ((part * 2 + (lane >> 5)) ^ (lane >> 2 & 3)) * 16 + (lane & 31) * kStep;
        if (i == 0) va[part][0] = *(const v4i*)(lds + wm * TM * 32 * kStep + at);
        else if (i <= TN) vb[part][i - 1] = *(const v4i*)(lds + (BM + (wn * TN + i - 1) * 32) * kStep + at);
        else va[part][i - TN] = *(const v4i*)(lds + (wm * TM + i - TN) * 32 * kStep + at);
    };
    // A part's matrix instructions, one after the other, each followed by a load or a read or two: a wave
    // that makes its loads in one go waits for the units that take them, and its SIMD with it.
    constexpr int kMfmas = TM * TN, kReads = TM + TN, kFirst = kMfmas >= 8 ? 2 : 1;
    auto multiply = [&](uint32_t part, int from, int to, auto between) {
#pragma unroll
        for (int i = from; i < to; ++i) {
            acc[i % TN][i / TN] = __builtin_amdgcn_mfma_i32_32x32x32_i8(vb[part][i % TN], va[part][i / TN], acc[i % TN][i / TN], 0, 0, 0);
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
    // Step s + 1 has landed for all waves, and all have read step s, whose buffer step s + 4 takes. Loads of
    // the steps s + 2 and s + 3 stay on their way (where all are direct loads; where some pass through registers,
    // step s + 2 is needed there, and only those of step s + 3 do).
    auto land = [&](uint32_t s, int parity, auto inner) {
        if (inner.value || s + 2 < steps) put(s + 2, parity);
        if (DIRECT == 0) __builtin_amdgcn_s_waitcnt(0xc07f);  // LDS alone
        else if (inner.value || s + 3 < whole) wait_loads<kAll ? 2 * LN : LN>();
        else wait_loads<0>();
        meet();
    };
    auto step = [&](uint32_t s, int parity, auto inner) {
        multiply(0, 0, kMfmas, [&](int i) {
            spread(i, kFirst - 1, kReadSlots, kReads, [&](int r) { read(s, 1, r); });
            spread(i, kFirst - 1, kMfmas - kFirst + 1, LN, [&](int r) { fetch(s + 3, parity ^ 1, inner, r); });
        });
        multiply(1, 0, kFirst, [](int) {});
        land(s, parity, inner);
        const bool more = inner.value || s + 1 < steps;
        multiply(1, kFirst, kMfmas, [&](int i) {
            if (more) spread(i, kFirst, kReadSlots, kReads, [&](int r) { read(s + 1, 0, r); });
        });
    };
    auto idle = [&](uint32_t s, int parity, auto inner) {  // a step of a wave without rows: brings in its part for the others
        fetch_all(s + 3, parity ^ 1, inner);
        land(s, parity, inner);
    };
    auto walk = [&](auto each) {
        uint32_t s = 0;
        for (; s + 4 < whole; s += 2) {
            each(s, 0, std::true_type());
            each(s + 1, 1, std::true_type());
        }
#pragma unroll 1
        for (; s < steps; s += 2) {
            each(s, 0, std::false_type());
            if (s + 1 < steps) each(s + 1, 1, std::false_type());
        }
    };
    if (steps) {
        const std::false_type any;
        fetch_all(0, 0, any), fetch_all(1, 1, any);
        put(0, 0);
        if (steps > 1) put(1, 1);
        fetch_all(2, 0, any);
        if (kAll && whole >= kBuffers - 1) wait_loads<2 * LN>();
        else wait_loads<0>();
        meet();
        if (rows.first + wm * TM * 32 >= rows.end) {
            walk(idle);
            return;
        }
#pragma unroll
        for (int r = 0; r < kReads; ++r) read(0, 0, r);
        walk(step);
    }

    // The wave's TM x TN blocks leave through its own part of LDS, as rows of TN * 32 results: lanes that hold
    // four results each of 32 rows would store 16 bytes of a line at a time.
    constexpr int ES = kSize<DT>;
    constexpr uint32_t kLine = TN * 32 * ES, kChunks = kLine / 16;  // bytes of a row
    constexpr int kRowsEach = kBuffers * kBuffer / W / kLine >= TM * 32 ? TM : kBuffers * kBuffer / W / kLine / 32;  // blocks of 32 rows at a time
    static_assert(kRowsEach >= 1 && TM % kRowsEach == 0, "a block of rows fits");
    // (nothing reads the buffers after the last step's barrier)
    char* mine = lds + w * (kBuffers * kBuffer / W);
    const float* bs = a.b_scale + (uint64_t)rows.expert * a.cols;
    const uint32_t c0 = n0 + wn * TN * 32;
    float scale[TN][4][4];
#pragma unroll
    for (int y = 0; y < TN; ++y)
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t n = c0 + y * 32 + g * 8 + (lane >> 5) * 4 + i;
                scale[y][g][i] = bs[n < a.cols ? n : a.cols - 1];
            }
#pragma unroll
    for (int x0 = 0; x0 < TM; x0 += kRowsEach) {
        const uint64_t m0 = rows.first + (wm * TM + x0) * 32;
#pragma unroll
        for (int x = 0; x < kRowsEach; ++x) {
            const uint64_t m = m0 + x * 32 + (lane & 31);
            const float as = a.a_scale[m < rows.end ? m : rows.end - 1];
            const uint32_t r = x * 32 + (lane & 31);
#pragma unroll
            for (int y = 0; y < TN; ++y)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    float v[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = (float)acc[y][x0 + x][4 * g + i] * as * scale[y][g][i];
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
}

// Tiles that rows in segments can make at most: a segment adds a part of one, and each has a row.
uint64_t most_tiles(const ProductArgs& a, uint64_t bm) {
    const uint64_t n = (a.rows + bm - 1) / bm + (a.offsets ? a.segments : 0);
    return n < a.rows ? n : a.rows;
}

template <int DT, int BM, int BN, int WM, int WN>
hipError_t launch_many(const ProductArgs& a, hipStream_t s) {
    const uint32_t nblocks = (a.cols + BN - 1) / BN, threads = WM * WN * 64;
    const uint64_t blocks = most_tiles(a, BM) * nblocks;
    if (blocks + 8 > 0xffffffffull / threads) return hipErrorInvalidConfiguration;
    const dim3 grid((uint32_t)((blocks + 7) / 8 * 8));
    const int direct = (((uintptr_t)a.a | a.lda) % 16 == 0 ? 1 : 0) | (((uintptr_t)a.b | a.ldb) % 16 == 0 ? 2 : 0);
    if (direct == 3) hipLaunchKernelGGL((hccl_moe_product_many_kernel<DT, BM, BN, WM, WN, 3>), grid, dim3(threads), 0, s, a, nblocks);
    else if (direct == 2) hipLaunchKernelGGL((hccl_moe_product_many_kernel<DT, BM, BN, WM, WN, 2>), grid, dim3(threads), 0, s, a, nblocks);
    else if (direct == 1) hipLaunchKernelGGL((hccl_moe_product_many_kernel<DT, BM, BN, WM, WN, 1>), grid, dim3(threads), 0, s, a, nblocks);
    else hipLaunchKernelGGL((hccl_moe_product_many_kernel<DT, BM, BN, WM, WN, 0>), grid, dim3(threads), 0, s, a, nblocks);
    return hipGetLastError();
}

template <int DT, int MB, int NB, int W, int U>
hipError_t launch_few(const ProductArgs& a, hipStream_t s) {
    const uint64_t nblocks = (a.cols + 16 * NB - 1) / (16 * NB), tiles = most_tiles(a, 16 * MB);
    if (tiles * nblocks > 0xffffffffull / (W * 64)) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL((hccl_moe_product_few_kernel<DT, MB, NB, W, U>), dim3((uint32_t)(tiles * nblocks)), dim3(W * 64), 0, s, a, (uint32_t)nblocks);
    return hipGetLastError();
}

// The largest tiles that leave at least 3/4 of the CUs a block and are not mostly empty: a tile is at most
// twice as high as a segment has rows on average (4 times for 16 rows, where weights are all that counts). us, bf16:
//   rows x inner x columns x experts   256 x 256   128 x 128   64 x 128   64 x 64   few rows
//       16384 x 4096 x 4096 x 16           321         390        496        599      1379
//       12000 x 1024 x 1024 x 16            23          29         31         36        84
//        2999 x 1408 x 2050 x 12            25          22         25         29        65
//        2048 x 2048 x 2048 x 64            65          61         61         68        76
//        1024 x 2048 x 2048 x 64            61          55         55         60        58
//         512 x 2048 x 2048 x 64            59          54         52         55        50
//         256 x 2048 x 2048 x 64            57          52         49         52        46
//        1024 x 4096 x 4096 x 1             42          24         31         41        87
//         256 x 4096 x 4096 x 1             40          19         16         14        24
//          64 x 4096 x 4096 x 1             30          17         15         13        10
//         128 x 4096 x 1024 x 1              -          18         15         13         8
//         505 x 4672 x  185 x 1              -          27         19         14         7
// Few rows, or too few blocks for half the CUs: 32 rows a block from 9 rows a segment on (16 where one expert has
// no more), and of 64, 32 and 16 columns the most that leave every CU a block, with k shared out over more waves
// the fewer columns there are (1 x 4096 x 4096: 16 columns 5.4 us, 32 columns 7.0, 64 columns 10.5;
// 256 x 2048 x 2048 x 64: 80, 48 and 46 us).
// All of this goes by the rows of the array, which are known on the host; where it has room for more rows than its
// segments hold, the tiles are those of the room.
// Short inner sizes leave most of 16 waves without k, at no cost (inner 64-1024, 16 against 4 waves, both within 0.1 us:
// 9 x 300 columns 3.6-3.9 us, 505 x 185 3.9 us, 100 x 512 over 16 experts 3.9-4.1 us).
template <int DT>
hipError_t product_type(const ProductArgs& a, int cus, hipStream_t s) {
    const uint64_t each = a.rows / a.segments, spread = a.offsets ? (a.rows < a.segments ? a.rows : a.segments) : 0;
    auto blocks = [&](uint64_t bm, uint64_t bn) {  // about; half a tile more for every segment
        return (a.offsets ? a.rows / bm + (spread + 1) / 2 : (a.rows + bm - 1) / bm) * ((a.cols + bn - 1) / bn);
    };
    const uint64_t most = (uint64_t)cus * 3 / 4;
    if (each >= 128 && blocks(256, 256) >= most) return launch_many<DT, 256, 256, 2, 4>(a, s);
    if (each >= 32 && blocks(128, 128) >= most) return launch_many<DT, 128, 128, 2, 2>(a, s);
    if (each >= 16 && blocks(64, 128) >= most) return launch_many<DT, 64, 128, 1, 4>(a, s);
    if (each > 64 && blocks(64, 64) >= (uint64_t)cus / 2) return launch_many<DT, 64, 64, 1, 2>(a, s);
    if (a.offsets ? each <= 8 : a.rows <= 16) {
        const uint64_t tiles = a.offsets ? a.rows / 16 + spread : 1, cols16 = (a.cols + 15) / 16;
        if (tiles * (cols16 / 4) >= (uint64_t)cus) return launch_few<DT, 1, 4, 4, 2>(a, s);
        if (tiles * (cols16 / 2) >= (uint64_t)cus) return launch_few<DT, 1, 2, 4, 4>(a, s);
        return launch_few<DT, 1, 1, 16, 2>(a, s);
    }
    const uint64_t tiles = a.offsets ? a.rows / 32 + spread : (a.rows + 31) / 32, cols16 = (a.cols + 15) / 16;
    if (tiles * (cols16 / 4) >= (uint64_t)cus) return launch_few<DT, 2, 4, 4, 2>(a, s);
    if (tiles * (cols16 / 2) >= (uint64_t)cus) return launch_few<DT, 2, 2, 8, 2>(a, s);
    return launch_few<DT, 2, 1, 16, 2>(a, s);
}

}  // namespace

hipError_t launch_product(const ProductArgs& a, hcclDataType_t dt, int cus, hipStream_t s) {
    return dt == hcclBf16 ? product_type<hcclBf16>(a, cus, s) : dt == hcclFp16 ? product_type<hcclFp16>(a, cus, s) : product_type<hcclFp32>(a, cus, s);
}

}  // namespace hccl
