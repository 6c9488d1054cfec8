// moe_rows.hip -- the rows of a mixture-of-experts layer: their order by expert (plan), the tokens'
// rows copied there (dispatch), quantised to 8 bits (quantize, dispatch), and the experts' rows added
// up for each token (combine) with its gradients. All of them are bound by memory.
#include "moe_device.h"

namespace hccl {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;

// ------------------------------------------------------------------------------------------ plan
// Routes are ordered by expert, then as they come (token, slot). The row of a route is the number of
// routes of lower experts, plus that of earlier routes of its own. Blocks take consecutive routes;
// the first kernel counts every block's routes per expert, and in the second a block adds up the
// counts before its own and ranks its routes among themselves: wave by wave, a lane's peers (equal
// expert) are found by one ballot for each bit of the expert's number. Only sums of whole numbers
// are taken in no fixed order. Bound by launches and latency: 148 routes over 64 experts 4.2 us in one
// launch, 32 768 routes (0.26 MB) 3.7 + 4.7 us in two.

__global__ __launch_bounds__(kPlanThreads) void hccl_moe_count_kernel(PlanArgs a) {
    __shared__ uint32_t n[HCCL_MAX_EXPERTS];
    for (uint32_t e = threadIdx.x; e < a.experts; e += kPlanThreads) n[e] = 0;
    __syncthreads();
    for (uint32_t s = 0; s < a.steps; ++s) {
        const uint64_t i = ((uint64_t)blockIdx.x * a.steps + s) * kPlanThreads + threadIdx.x;
        const uint32_t e = i < a.routes ? (uint32_t)a.index[i] : ~0u;
        if (e < a.experts) atomicAdd(&n[e], 1u);
    }
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < a.experts; e += kPlanThreads) a.hist[(uint64_t)blockIdx.x * a.experts + e] = n[e];
}

static_assert(kPlanThreads == HCCL_MAX_EXPERTS, "the second kernel has a thread for every expert");

__global__ __launch_bounds__(kPlanThreads) void hccl_moe_plan_kernel(PlanArgs a) {
    constexpr uint32_t kPlanWaves = kPlanThreads / 64;
    __shared__ uint32_t before[HCCL_MAX_EXPERTS];   // routes of an expert in earlier blocks, then its next row
    __shared__ uint32_t first[HCCL_MAX_EXPERTS + 1];  // routes of an expert, then its first row
    __shared__ uint16_t seen[kPlanWaves][HCCL_MAX_EXPERTS];
    __shared__ uint32_t sums[kPlanWaves];
    const uint32_t tid = threadIdx.x, lane = tid & 63, w = tid >> 6, E = a.experts;
    before[tid] = 0;
    first[tid] = 0;
    __syncthreads();
    if (a.blocks == 1) {
        for (uint32_t s = 0; s < a.steps; ++s) {
            const uint64_t i = (uint64_t)s * kPlanThreads + tid;
            const uint32_t e = i < a.routes ? (uint32_t)a.index[i] : ~0u;
            if (e < E) atomicAdd(&first[e], 1u);
        }
    } else {
        uint32_t width = 64;
        while (width < E) width *= 2;
        const uint32_t e = tid & (width - 1), stride = kPlanThreads / width;
        if (e < E) {
            uint32_t all = 0, mine = 0;
            for (uint32_t b = tid / width; b < a.blocks; b += stride) {
                const uint32_t v = a.hist[(uint64_t)b * E + e];
                all += v;
                if (b < blockIdx.x) mine += v;
            }
            atomicAdd(&first[e], all);
            atomicAdd(&before[e], mine);
        }
    }
    __syncthreads();
    // exclusive sum over the experts, one per thread
    const uint32_t n = first[tid];
    uint32_t incl = n;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t v = (uint32_t)__shfl_up((int)incl, d);
        if (lane >= (uint32_t)d) incl += v;
    }
    if (lane == 63) sums[w] = incl;
    __syncthreads();
    uint32_t base = 0;
#pragma unroll
    for (uint32_t q = 0; q < kPlanWaves; ++q)
        if (q < w) base += sums[q];
    const uint32_t at = base + incl - n;
    first[tid] = at;  // (nobody else reads it before the barrier)
    if (tid == kPlanThreads - 1) first[kPlanThreads] = at + n;
    before[tid] += at;
    __syncthreads();
    if (blockIdx.x == 0) {
        auto clip = [&](uint32_t v) { return (int64_t)(v < a.capacity ? v : a.capacity); };
        for (uint32_t e = tid; e <= E; e += kPlanThreads) a.offsets[e] = clip(first[e]);
        if (a.rank_counts && tid < a.ranks) {
            const uint32_t each = E / a.ranks;
            a.rank_counts[tid] = clip(first[(tid + 1) * each]) - clip(first[tid * each]);
        }
    }
    const uint32_t bits = 32 - __builtin_clz(E);  // (E itself stands for no expert)
    for (uint32_t s = 0; s < a.steps; ++s) {
        const uint64_t i = ((uint64_t)blockIdx.x * a.steps + s) * kPlanThreads + tid;
        for (uint32_t e = lane; e < E; e += 64) seen[w][e] = 0;
        __syncthreads();
        uint32_t e = i < a.routes ? (uint32_t)a.index[i] : E;
        if (e > E) e = E;
        uint64_t peers = ~0ull;
        for (uint32_t b = 0; b < bits; ++b) {
            const uint64_t set = __ballot((e >> b) & 1u);
            peers &= ((e >> b) & 1u) ? set : ~set;
        }
        const uint32_t rank = (uint32_t)__popcll(peers & ((1ull << lane) - 1));
        if (e < E && rank == 0) seen[w][e] = (uint16_t)__popcll(peers);
        __syncthreads();
        uint32_t run = 0;
        if (tid < E) {
#pragma unroll
            for (uint32_t q = 0; q < kPlanWaves; ++q) {
                const uint32_t c = seen[q][tid];
                seen[q][tid] = (uint16_t)run;
                run += c;
            }
        }
        __syncthreads();
        if (i < a.routes) {
            int32_t r = -1;
            if (e < E) {
                const uint32_t at_row = before[e] + seen[w][e] + rank;
                if (at_row < a.capacity) r = (int32_t)at_row;
            }
            a.row[i] = r;
        }
        __syncthreads();
        if (tid < E) before[tid] += run;
    }
}

// -------------------------------------------------------------------------------------- dispatch
// Vectors of rows. WHOLE: every lane's vector lies inside the row, so that none looks where it ends.
// STREAM: with the non-temporal hint, for calls that move more than the last-level cache holds. That
// keeps their results from pushing out what the call still reads: dispatch of 8 192 x 4 096 bf16 to 4
// rows each 67 -> 53 us, gradients of the combination of 8 192 x 4 rows of 2 048 60 -> 52 us. It costs
// a consumer that reads the rows at once (dispatch and quantisation 151 -> 158 us), and in calls that
// the cache holds it costs more than it gives (2 048 x 4 096 to 4 rows each, and quantised, 40 -> 45 us).
constexpr uint64_t kLastLevelCache = 256ull << 20;

template <int ES, bool WHOLE, bool STREAM>
__device__ __forceinline__ v4u piece_load(const char* row, uint64_t e, uint64_t cols) {
    if constexpr (WHOLE && STREAM) return (v4u)__builtin_nontemporal_load(gptr<typename Loose<ES>::x4>(row + e * ES));
    else if constexpr (WHOLE) return load16<ES>(row + e * ES);
    else return load_row<ES>(row, e, cols);
}
template <int ES, bool WHOLE, bool STREAM>
__device__ __forceinline__ void piece_store(char* row, uint64_t e, uint64_t cols, const v4u& v) {
    if constexpr (WHOLE && STREAM) __builtin_nontemporal_store((typename Loose<ES>::x4)v, gptr<typename Loose<ES>::x4>(row + e * ES));
    else if constexpr (WHOLE) store16<ES>(row + e * ES, v);
    else store_row<ES>(row, e, cols, v);
}

// A wave copies 1 KiB of a token's row to every row that the token has: it is read once, and few
// tokens still make many waves. Rows that begin at any alignment are read and written as they lie:
// stores brought to 16 bytes, which read the token again at another shift for every row, took 60 us
// against 43 (16 384 x 1 001 bf16 to 4 rows each).
template <int ES, bool WHOLE, bool STREAM>
__device__ __forceinline__ void dispatch_piece(const DispatchArgs& a, uint64_t t, uint64_t e, uint32_t mine) {
    const v4u v = piece_load<ES, WHOLE, false>((const char*)a.x + t * a.ldx * ES, e, a.cols);
    for (uint32_t k = 0; k < a.top_k; ++k) {
        const uint32_t r = at_lane(mine, k);
        if (r < a.capacity) piece_store<ES, WHOLE, STREAM>((char*)a.out + (uint64_t)r * a.ldo * ES, e, a.cols, v);
    }
}

template <int ES, bool STREAM>
__global__ __launch_bounds__(kThreads) void hccl_moe_dispatch_kernel(DispatchArgs a, uint32_t pieces) {
    constexpr uint64_t V = 16 / ES, kPiece = kWave * V;
    const uint32_t lane = threadIdx.x & 63;
    const uint64_t id = (uint64_t)blockIdx.x * kWaves + first_lane(threadIdx.x >> 6);
    const uint64_t t = id / pieces, c0 = (id % pieces) * kPiece;
    if (t >= a.tokens) return;
    const uint32_t mine = lane < a.top_k ? (uint32_t)a.row[t * a.top_k + lane] : ~0u;
    if (c0 + kPiece <= a.cols) dispatch_piece<ES, true, STREAM>(a, t, c0 + lane * V, mine);
    else dispatch_piece<ES, false, STREAM>(a, t, c0 + lane * V, mine);
}

// Rows of up to G vectors: a wave takes 64 / G tokens, G lanes each.
template <int ES, int G>
__global__ __launch_bounds__(kThreads) void hccl_moe_dispatch_narrow_kernel(DispatchArgs a) {
    const uint64_t t = (uint64_t)blockIdx.x * (kThreads / G) + threadIdx.x / G, e = threadIdx.x % G * (16 / ES);
    if (t >= a.tokens || e >= a.cols) return;
    const v4u v = load_row<ES>((const char*)a.x + t * a.ldx * ES, e, a.cols);
    const int32_t* row = a.row + t * a.top_k;
#pragma unroll 4
    for (uint32_t k = 0; k < a.top_k; ++k) {
        const uint32_t r = (uint32_t)row[k];
        if (r < a.capacity) store_row<ES>((char*)a.out + (uint64_t)r * a.ldo * ES, e, a.cols, v);
    }
}

// -------------------------------------------------------------------------------------- quantize
// code = rint(x * (1 / max|x| * 127)), scale = max|x| / 127: the reciprocal once for a row. The maximum is
// taken of the values' bits without their sign, which orders infinities and NaN above the rest: such
// a row gets codes of 0 and that scale, so that its products are NaN. Rows below 2^-119 count as 0
// (127 over them would overflow).
__device__ __forceinline__ void row_scale(uint32_t top, float& inv, float& scale) {
    const float m = __uint_as_float(top);
    const bool none = top < 0x04000000u;  // 2^-119
    const bool finite = top < 0x7f800000u;
    inv = none || !finite ? 0.0f : 1.0f / m * 127.0f;
    scale = none ? 0.0f : finite ? m / 127.0f : m;
}

__device__ __forceinline__ uint32_t code4(float a, float b, float c, float d, float inv) {
    const int32_t i = (int32_t)rintf(a * inv), j = (int32_t)rintf(b * inv), k = (int32_t)rintf(c * inv), l = (int32_t)rintf(d * inv);
    return ((uint32_t)i & 0xffu) | ((uint32_t)j & 0xffu) << 8 | ((uint32_t)k & 0xffu) << 16 | (uint32_t)l << 24;
}

// What a lane keeps of a vector between the two passes: its bits, or the gated values, silu(x) * (the row's
// second half), which cost more to make than registers. silu(x) = x / (1 + 2^(-x log2 e)); the exponent's
// rounding is |x| 2^-24 of a term that is small where |x| is large.
template <int DT, bool GATED>
struct Held {
    float x[kVecOf<DT>];
    __device__ __forceinline__ void values(float (&y)[kVecOf<DT>]) const {
#pragma unroll
        for (int i = 0; i < kVecOf<DT>; ++i) y[i] = x[i];
    }
};
template <int DT>
struct Held<DT, false> {
    v4u x;
    __device__ __forceinline__ void values(float (&y)[kVecOf<DT>]) const { widen<DT>(x, y); }
};
template <int DT, bool GATED, bool WHOLE>
__device__ __forceinline__ Held<DT, GATED> hold(const char* src, uint64_t e, uint64_t cols) {
    constexpr int ES = kSize<DT>;
    Held<DT, GATED> h;
    if constexpr (GATED) {
        float up[kVecOf<DT>];
        const v4u g = piece_load<ES, WHOLE, false>(src, e, cols), u = piece_load<ES, WHOLE, false>(src + cols * ES, e, cols);
        widen<DT>(g, h.x);
        widen<DT>(u, up);
#pragma unroll
        for (int i = 0; i < kVecOf<DT>; ++i) h.x[i] *= __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(h.x[i] * -1.44269504088896340736f)) * up[i];
    } else {
        h.x = piece_load<ES, WHOLE, false>(src, e, cols);
    }
    return h;
}

// The greatest magnitude's bits among the values of a vector.
template <int DT, bool GATED>
__device__ __forceinline__ uint32_t top_of(const Held<DT, GATED>& h, uint32_t top) {
    float x[kVecOf<DT>];
    h.values(x);
#pragma unroll
    for (int i = 0; i < kVecOf<DT>; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
    return top;
}

constexpr int kKeep = 4;

// A row that lane `at` of `step / V` shares: its vectors are at e = at * V, + step, ...; the first kKeep of them
// stay in registers between the two passes, those of longer rows are read twice.
template <int DT, bool GATED, int W, bool WHOLE>
__device__ __forceinline__ void quantize_row(const QuantizeArgs& a, uint64_t t, uint32_t at, uint32_t* tops, bool on) {
    constexpr int V = kVecOf<DT>, ES = kSize<DT>;
    constexpr uint64_t step = (uint64_t)W * kWave * V;
    const uint32_t lane = threadIdx.x & 63, w = first_lane(threadIdx.x >> 6);
    const char* src = (const char*)a.x + t * a.ldx * ES;
    Held<DT, GATED> x[kKeep];
    const uint32_t copies = a.row ? a.top_k : 1u;
    const uint32_t mine = !a.row ? (uint32_t)t : on && lane < copies ? (uint32_t)a.row[t * a.top_k + lane] : ~0u;
    uint32_t top = 0;
    if (on) {
#pragma unroll
        for (int u = 0; u < kKeep; ++u)
            if (u * step + at * V < a.cols) x[u] = hold<DT, GATED, WHOLE>(src, u * step + at * V, a.cols);
#pragma unroll
        for (int u = 0; u < kKeep; ++u)
            if (u * step + at * V < a.cols) top = top_of<DT, GATED>(x[u], top);
        for (uint64_t e = kKeep * step + at * V; e < a.cols; e += step) top = top_of<DT, GATED>(hold<DT, GATED, WHOLE>(src, e, a.cols), top);
    }
    top = maxu_lanes<64>(top);
    if constexpr (W > 1) {
        if (lane == 0) tops[w] = top;
        __syncthreads();
#pragma unroll
        for (int q = 0; q < W; ++q) top = max(top, tops[w / W * W + q]);
    }
    if (!on) return;
    float inv, scale;
    row_scale(top, inv, scale);
    auto store = [&](uint64_t e, const Held<DT, GATED>& h) {
        float y[V];
        h.values(y);
        uint32_t lo = 0, hi = 0;
        if (inv != 0.0f) {  // (infinity times 0 is no number, and no number has no code)
            lo = code4(y[0], y[1], y[2], y[3], inv);
            if constexpr (V == 8) hi = code4(y[4], y[5], y[6], y[7], inv);
        }
        for (uint32_t k = 0; k < copies; ++k) {
            const uint32_t r = a.row ? at_lane(mine, k) : (uint32_t)t;
            if (r >= a.capacity) continue;
            char* dst = (char*)a.codes + (uint64_t)r * a.ldq + e;
            if (WHOLE || e + V <= a.cols) {
                if constexpr (V == 8) *gptr<typename Loose<1>::x2>(dst) = typename Loose<1>::x2{lo, hi};
                else *gptr<typename Loose<1>::x1>(dst) = lo;
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (e + i < a.cols) *gptr<uint8_t>(dst + i) = (uint8_t)((i < 4 ? lo : hi) >> (8 * (i & 3)));
            }
        }
    };
#pragma unroll
    for (int u = 0; u < kKeep; ++u)
        if (u * step + at * V < a.cols) store(u * step + at * V, x[u]);
    for (uint64_t e = kKeep * step + at * V; e < a.cols; e += step) store(e, hold<DT, GATED, WHOLE>(src, e, a.cols));
    if (at < copies && w % W == 0) {
        const uint32_t r = a.row ? mine : (uint32_t)t;
        if (r < a.capacity) a.scale[r] = scale;
    }
}

template <int DT, bool GATED, int W>
__global__ __launch_bounds__(kThreads) void hccl_moe_quantize_kernel(QuantizeArgs a) {
    __shared__ uint32_t tops[kWaves];
    const uint64_t t = (uint64_t)blockIdx.x * (kWaves / W) + first_lane(threadIdx.x >> 6) / W;
    const bool on = t < a.rows && (!a.limit || (int64_t)t < *a.limit);
    const uint32_t at = threadIdx.x & (W * kWave - 1);
    if (a.cols % kVecOf<DT> == 0) quantize_row<DT, GATED, W, true>(a, t, at, tops, on);
    else quantize_row<DT, GATED, W, false>(a, t, at, tops, on);
}

// --------------------------------------------------------------------------------------- combine
// y_t = sum_k w_k z_{row k}, added up in 32 bits in the order of the slots. A wave takes a piece of a
// token; the loads of kBatch rows are in flight together. Bound by memory: 8 192 tokens x 4 rows of 2 048
// bf16 (168 MB) 31 us, 5.4 TB/s; 256 tokens x 4 rows of 4 096 3.3 us, little more than an empty launch.
constexpr int kBatch = 4;
constexpr int kCombineVecs = 2;

template <int DT, bool WHOLE>
__device__ __forceinline__ void combine_piece(const CombineArgs& a, uint64_t t, uint64_t c0, uint32_t lane) {
    constexpr int V = kVecOf<DT>, ES = kSize<DT>;
    const uint32_t mine = lane < a.top_k ? (uint32_t)a.row[t * a.top_k + lane] : ~0u;
    const float weight = a.weight && lane < a.top_k ? a.weight[t * a.top_k + lane] : 1.0f;
    float acc[kCombineVecs][V];
#pragma unroll
    for (int u = 0; u < kCombineVecs; ++u)
#pragma unroll
        for (int i = 0; i < V; ++i) acc[u][i] = 0.0f;
    for (uint32_t k = 0; k < a.top_k; k += kBatch) {
        v4u z[kBatch][kCombineVecs];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const uint32_t r = at_lane(mine, k + j);  // (lanes from top_k on have no row)
            if (r >= a.capacity) continue;
            const char* src = (const char*)a.z + (uint64_t)r * a.ldz * ES;
#pragma unroll
            for (int u = 0; u < kCombineVecs; ++u) z[j][u] = piece_load<ES, WHOLE, false>(src, c0 + (u * kWave + lane) * V, a.cols);
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            if (at_lane(mine, k + j) >= a.capacity) continue;
            const float w = __uint_as_float(at_lane(__float_as_uint(weight), k + j));
#pragma unroll
            for (int u = 0; u < kCombineVecs; ++u) {
                float x[V];
                widen<DT>(z[j][u], x);
#pragma unroll
                for (int i = 0; i < V; ++i) acc[u][i] += w * x[i];
            }
        }
    }
    char* dst = (char*)a.out + t * a.ldo * ES;
#pragma unroll
    for (int u = 0; u < kCombineVecs; ++u) piece_store<ES, WHOLE, false>(dst, c0 + (u * kWave + lane) * V, a.cols, narrow<DT>(acc[u]));
}

template <int DT>
__global__ __launch_bounds__(kThreads) void hccl_moe_combine_kernel(CombineArgs a, uint32_t pieces) {
    constexpr uint64_t kPiece = kCombineVecs * kWave * kVecOf<DT>;
    const uint32_t lane = threadIdx.x & 63;
    const uint64_t id = (uint64_t)blockIdx.x * kWaves + first_lane(threadIdx.x >> 6);
    const uint64_t t = id / pieces, c0 = (id % pieces) * kPiece;
    if (t >= a.tokens) return;
    if (c0 + kPiece <= a.cols) combine_piece<DT, true>(a, t, c0, lane);
    else combine_piece<DT, false>(a, t, c0, lane);
}

// Rows of up to G vectors: a wave takes 64 / G tokens, G lanes each.
template <int DT, int G>
__global__ __launch_bounds__(kThreads) void hccl_moe_combine_narrow_kernel(CombineArgs a) {
    constexpr int V = kVecOf<DT>, ES = kSize<DT>;
    const uint64_t t = (uint64_t)blockIdx.x * (kThreads / G) + threadIdx.x / G, e = threadIdx.x % G * V;
    if (t >= a.tokens || e >= a.cols) return;
    const int32_t* row = a.row + t * a.top_k;
    float acc[V];
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] = 0.0f;
    for (uint32_t k = 0; k < a.top_k; k += kBatch) {
        uint32_t r[kBatch];
        float w[kBatch];
        v4u z[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            r[j] = k + j < a.top_k ? (uint32_t)row[k + j] : ~0u;
            w[j] = a.weight && k + j < a.top_k ? a.weight[t * a.top_k + k + j] : 1.0f;
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
            if (r[j] < a.capacity) z[j] = load_row<ES>((const char*)a.z + (uint64_t)r[j] * a.ldz * ES, e, a.cols);
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            if (r[j] >= a.capacity) continue;
            float x[V];
            widen<DT>(z[j], x);
#pragma unroll
            for (int i = 0; i < V; ++i) acc[i] += w[j] * x[i];
        }
    }
    store_row<ES>((char*)a.out + t * a.ldo * ES, e, a.cols, narrow<DT>(acc));
}

// dz_{row k} = w_k dy_t, dw_k = <dy_t, z_{row k}>. A block of W waves takes a token, as many as its row
// has vectors for, up to 4 (3 001 tokens x 2 rows of 1 003 fp16: 2 waves 9 us, 4 waves 12 us). The
// products are added up in a lane, over the lanes and then over the waves, always in the same order.
// Bound by memory: 8 192 tokens x 4 rows of 2 048 bf16 (302 MB) 46 us, 6.6 TB/s.
template <int DT, bool WHOLE, bool STREAM>
__device__ __forceinline__ void backward_piece(const CombineBackwardArgs& a, const char* dy, const uint32_t (&r)[kBatch], const float (&wk)[kBatch],
                                               uint64_t e, float (&dot)[kBatch]) {
    constexpr int V = kVecOf<DT>, ES = kSize<DT>;
    const v4u g = piece_load<ES, WHOLE, false>(dy, e, a.cols);
    v4u z[kBatch];
    if (a.grad_weight) {
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
            if (r[j] < a.capacity) z[j] = piece_load<ES, WHOLE, STREAM>((const char*)a.z + (uint64_t)r[j] * a.ldz * ES, e, a.cols);
    }
    float x[V];
    widen<DT>(g, x);
    if (a.grad_z) {
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            if (r[j] >= a.capacity) continue;
            float d[V];
#pragma unroll
            for (int i = 0; i < V; ++i) d[i] = wk[j] * x[i];
            piece_store<ES, WHOLE, STREAM>((char*)a.grad_z + (uint64_t)r[j] * a.ldo * ES, e, a.cols, narrow<DT>(d));
        }
    }
    if (a.grad_weight) {
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            if (r[j] >= a.capacity) continue;
            float y[V];
            widen<DT>(z[j], y);
#pragma unroll
            for (int i = 0; i < V; ++i) dot[j] += x[i] * y[i];
        }
    }
}

template <int DT, int W, bool STREAM>
__global__ __launch_bounds__(W * 64) void hccl_moe_combine_backward_kernel(CombineBackwardArgs a) {
    constexpr uint64_t V = kVecOf<DT>, ES = kSize<DT>;
    __shared__ float parts[W][kBatch];
    const uint32_t lane = threadIdx.x & 63, w = first_lane(threadIdx.x >> 6);
    const uint64_t t = blockIdx.x;
    const uint32_t mine = lane < a.top_k ? (uint32_t)a.row[t * a.top_k + lane] : ~0u;
    const float weight = lane < a.top_k ? a.weight[t * a.top_k + lane] : 0.0f;
    const char* dy = (const char*)a.grad + t * a.ldg * ES;
    for (uint32_t k = 0; k < a.top_k; k += kBatch) {
        uint32_t r[kBatch];
        float wk[kBatch], dot[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            r[j] = at_lane(mine, k + j);  // (lanes from top_k on have no row)
            wk[j] = __uint_as_float(at_lane(__float_as_uint(weight), k + j));
            dot[j] = 0.0f;
        }
        for (uint64_t e = w * kWave * V; e < a.cols; e += W * kWave * V) {
            if (e + kWave * V <= a.cols) backward_piece<DT, true, STREAM>(a, dy, r, wk, e + lane * V, dot);
            else backward_piece<DT, false, STREAM>(a, dy, r, wk, e + lane * V, dot);
        }
        if (!a.grad_weight) continue;
#pragma unroll
        for (int j = 0; j < kBatch; ++j) dot[j] = sum_lanes<64>(dot[j]);
        if constexpr (W > 1) {
            if (lane == 0) {
#pragma unroll
                for (int j = 0; j < kBatch; ++j) parts[w][j] = dot[j];
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                dot[j] = parts[0][j];
#pragma unroll
                for (int q = 1; q < W; ++q) dot[j] += parts[q][j];
            }
            __syncthreads();
        }
        if (threadIdx.x == 0) {
#pragma unroll
            for (int j = 0; j < kBatch; ++j)
                if (k + j < a.top_k) a.grad_weight[t * a.top_k + k + j] = r[j] < a.capacity ? dot[j] : 0.0f;
        }
    }
}

// Rows of up to G vectors: a wave takes 64 / G tokens, G lanes each (all of them until the sums are made).
template <int DT, int G>
__global__ __launch_bounds__(kThreads) void hccl_moe_combine_backward_narrow_kernel(CombineBackwardArgs a) {
    constexpr int V = kVecOf<DT>, ES = kSize<DT>;
    const uint64_t t = (uint64_t)blockIdx.x * (kThreads / G) + threadIdx.x / G, e = threadIdx.x % G * V;
    const bool on = t < a.tokens && e < a.cols;
    const uint64_t route = t < a.tokens ? t * a.top_k : 0;
    float x[V];
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = 0.0f;
    if (on) widen<DT>(load_row<ES>((const char*)a.grad + t * a.ldg * ES, e, a.cols), x);
    for (uint32_t k = 0; k < a.top_k; k += kBatch) {
        uint32_t r[kBatch];
        float w[kBatch];
        v4u z[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            r[j] = k + j < a.top_k ? (uint32_t)a.row[route + k + j] : ~0u;
            w[j] = k + j < a.top_k ? a.weight[route + k + j] : 0.0f;
        }
        if (a.grad_weight) {
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                z[j] = v4u{0, 0, 0, 0};
                if (on && r[j] < a.capacity) z[j] = load_row<ES>((const char*)a.z + (uint64_t)r[j] * a.ldz * ES, e, a.cols);
            }
        }
        if (a.grad_z) {
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                if (!on || r[j] >= a.capacity) continue;
                float d[V];
#pragma unroll
                for (int i = 0; i < V; ++i) d[i] = w[j] * x[i];
                store_row<ES>((char*)a.grad_z + (uint64_t)r[j] * a.ldo * ES, e, a.cols, narrow<DT>(d));
            }
        }
        if (!a.grad_weight) continue;
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            float y[V], dot = 0.0f;
            widen<DT>(z[j], y);
#pragma unroll
            for (int i = 0; i < V; ++i) dot += x[i] * y[i];
            dot = sum_lanes<G>(dot);
            if (t < a.tokens && threadIdx.x % G == 0 && k + j < a.top_k) a.grad_weight[route + k + j] = r[j] < a.capacity ? dot : 0.0f;
        }
    }
}

// Lanes for a token whose row has few vectors, 0 where a wave or more takes it: with one wave a token most of its
// lanes would idle. us in bf16 (tokens x columns x rows a token), lanes / a wave: dispatch 12 691 x 64 x 6 4.4 / 6.6;
// combine 15 168 x 128 x 8 7.8 / 24; gradients 12 213 x 256 x 6 15 / 21.
int narrow_lanes(uint64_t cols, uint64_t es) {
    const uint64_t vecs = (cols * es + 15) / 16;
    return vecs <= 16 ? 16 : vecs <= 32 ? 32 : 0;
}

// A launch's threads are counted in 32 bits.
bool too_many(uint64_t blocks, uint32_t threads) { return blocks * threads > 0xffffffffull; }

template <typename F>
hipError_t by_type(hcclDataType_t dt, F f) {
    if (dt == hcclBf16) f(std::integral_constant<int, hcclBf16>());
    else if (dt == hcclFp16) f(std::integral_constant<int, hcclFp16>());
    else f(std::integral_constant<int, hcclFp32>());
    return hipGetLastError();
}

}  // namespace

void plan_shape(uint64_t routes, uint32_t* blocks, uint32_t* steps) {
    // One launch for up to 4 096 routes, then two with at most 128 blocks: a block of the second
    // reads every block's counts.
    const uint64_t n = (routes + kPlanThreads - 1) / kPlanThreads;
    if (n <= 4) {
        *blocks = 1;
        *steps = (uint32_t)n;
    } else {
        *steps = (uint32_t)((n + 127) / 128);
        *blocks = (uint32_t)((n + *steps - 1) / *steps);
    }
}

hipError_t launch_plan(const PlanArgs& a, hipStream_t s) {
    if (a.blocks > 1) hipLaunchKernelGGL(hccl_moe_count_kernel, dim3(a.blocks), dim3(kPlanThreads), 0, s, a);
    hipLaunchKernelGGL(hccl_moe_plan_kernel, dim3(a.blocks), dim3(kPlanThreads), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_dispatch(const DispatchArgs& a, hcclDataType_t dt, hipStream_t s) {
    const uint32_t es = dt == hcclFp32 ? 4 : 2, per = kWave * 16 / es;
    if (const int lanes = narrow_lanes(a.cols, es)) {
        if (too_many(a.tokens / kThreads + 1, kThreads * lanes)) return hipErrorInvalidConfiguration;
        const dim3 grid((uint32_t)((a.tokens * lanes + kThreads - 1) / kThreads)), block(kThreads);
        if (es == 2 && lanes == 16) hipLaunchKernelGGL((hccl_moe_dispatch_narrow_kernel<2, 16>), grid, block, 0, s, a);
        else if (es == 2) hipLaunchKernelGGL((hccl_moe_dispatch_narrow_kernel<2, 32>), grid, block, 0, s, a);
        else if (lanes == 16) hipLaunchKernelGGL((hccl_moe_dispatch_narrow_kernel<4, 16>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((hccl_moe_dispatch_narrow_kernel<4, 32>), grid, block, 0, s, a);
        return hipGetLastError();
    }
    const uint32_t pieces = (uint32_t)((a.cols + per - 1) / per);
    const uint64_t blocks = (a.tokens * pieces + kWaves - 1) / kWaves;
    if (too_many(blocks, kThreads)) return hipErrorInvalidConfiguration;
    const bool stream = a.tokens * (a.top_k + 1) * a.cols * es > kLastLevelCache;
    const dim3 grid((uint32_t)blocks), block(kThreads);
    if (es == 2 && stream) hipLaunchKernelGGL((hccl_moe_dispatch_kernel<2, true>), grid, block, 0, s, a, pieces);
    else if (es == 2) hipLaunchKernelGGL((hccl_moe_dispatch_kernel<2, false>), grid, block, 0, s, a, pieces);
    else if (stream) hipLaunchKernelGGL((hccl_moe_dispatch_kernel<4, true>), grid, block, 0, s, a, pieces);
    else hipLaunchKernelGGL((hccl_moe_dispatch_kernel<4, false>), grid, block, 0, s, a, pieces);
    return hipGetLastError();
}

template <int DT, bool GATED, int W>
void launch_quantize_rows(const QuantizeArgs& a, hipStream_t s) {
    hipLaunchKernelGGL((hccl_moe_quantize_kernel<DT, GATED, W>), dim3((uint32_t)((a.rows * W + kWaves - 1) / kWaves)), dim3(kThreads), 0, s, a);
}

// As many waves a row as leave its lanes at most kKeep vectors, up to 4; one for up to 2 vectors a lane
// (16 384 rows of bf16: 512 columns 1 / 2 / 4 waves 7.3 / 9.9 / 14 us, 4 096 columns 50 / 37 / 38 us, 8 192
// columns 106 / 87 / 71 us).
uint32_t quantize_waves(uint64_t cols, hcclDataType_t dt) {
    const uint64_t per = kWave * (dt == hcclFp32 ? 4 : 8), vecs = (cols + per - 1) / per;
    return vecs <= 2 ? 1 : vecs <= 2 * kKeep ? 2 : 4;
}

template <int DT, bool GATED>
void quantize_type(const QuantizeArgs& a, uint32_t waves, hipStream_t s) {
    if (waves == 1) launch_quantize_rows<DT, GATED, 1>(a, s);
    else if (waves == 2) launch_quantize_rows<DT, GATED, 2>(a, s);
    else launch_quantize_rows<DT, GATED, 4>(a, s);
}

hipError_t launch_quantize(const QuantizeArgs& a, hcclDataType_t dt, bool gated, hipStream_t s) {
    const uint32_t waves = quantize_waves(a.cols, dt);
    if (too_many((a.rows * waves + kWaves - 1) / kWaves, kThreads)) return hipErrorInvalidConfiguration;
    return by_type(dt, [&](auto type) {
        constexpr int DT = decltype(type)::value;
        if (gated) quantize_type<DT, true>(a, waves, s);
        else quantize_type<DT, false>(a, waves, s);
    });
}

hipError_t launch_combine(const CombineArgs& a, hcclDataType_t dt, hipStream_t s) {
    if (const int lanes = narrow_lanes(a.cols, dt == hcclFp32 ? 4 : 2)) {
        if (too_many(a.tokens / kThreads + 1, kThreads * lanes)) return hipErrorInvalidConfiguration;
        return by_type(dt, [&](auto type) {
            constexpr int DT = decltype(type)::value;
            const dim3 grid((uint32_t)((a.tokens * lanes + kThreads - 1) / kThreads)), block(kThreads);
            if (lanes == 16) hipLaunchKernelGGL((hccl_moe_combine_narrow_kernel<DT, 16>), grid, block, 0, s, a);
            else hipLaunchKernelGGL((hccl_moe_combine_narrow_kernel<DT, 32>), grid, block, 0, s, a);
        });
    }
    const uint32_t per = kCombineVecs * kWave * (dt == hcclFp32 ? 4 : 8), pieces = (uint32_t)((a.cols + per - 1) / per);
    const uint64_t blocks = (a.tokens * pieces + kWaves - 1) / kWaves;
    if (too_many(blocks, kThreads)) return hipErrorInvalidConfiguration;
    return by_type(dt, [&](auto type) {
        constexpr int DT = decltype(type)::value;
        const dim3 grid((uint32_t)blocks);
        hipLaunchKernelGGL(hccl_moe_combine_kernel<DT>, grid, dim3(kThreads), 0, s, a, pieces);
    });
}

hipError_t launch_combine_backward(const CombineBackwardArgs& a, hcclDataType_t dt, hipStream_t s) {
    const uint64_t es = dt == hcclFp32 ? 4 : 2, vecs = a.cols * es / (kWave * 16);
    const uint64_t arrays = (a.grad_z ? 1 : 0) + (a.grad_weight ? 1 : 0);
    const bool stream = a.tokens * (a.top_k * arrays + 1) * a.cols * es > kLastLevelCache;
    const int lanes = narrow_lanes(a.cols, es);
    // (16 waves for tokens for no more than one block a CU: 64 tokens x 8 rows of 7 040 fp32 30 -> 15 us)
    const uint32_t waves = vecs < 1 ? 1 : vecs < 2 ? 2 : vecs >= 16 && a.tokens <= 256 ? 16 : 4;
    if (lanes ? too_many(a.tokens / kThreads + 1, kThreads * lanes) : too_many(a.tokens, waves * kWave)) return hipErrorInvalidConfiguration;
    return by_type(dt, [&](auto type) {
        constexpr int DT = decltype(type)::value;
        const dim3 grid((uint32_t)a.tokens), narrow_grid((uint32_t)((a.tokens * lanes + kThreads - 1) / kThreads)), block(waves * kWave);
        if (lanes == 16) hipLaunchKernelGGL((hccl_moe_combine_backward_narrow_kernel<DT, 16>), narrow_grid, dim3(kThreads), 0, s, a);
        else if (lanes == 32) hipLaunchKernelGGL((hccl_moe_combine_backward_narrow_kernel<DT, 32>), narrow_grid, dim3(kThreads), 0, s, a);
        else if (waves == 1) hipLaunchKernelGGL((hccl_moe_combine_backward_kernel<DT, 1, false>), grid, block, 0, s, a);
        else if (waves == 2) hipLaunchKernelGGL((hccl_moe_combine_backward_kernel<DT, 2, false>), grid, block, 0, s, a);
        else if (waves == 16) hipLaunchKernelGGL((hccl_moe_combine_backward_kernel<DT, 16, false>), grid, block, 0, s, a);
        else if (stream) hipLaunchKernelGGL((hccl_moe_combine_backward_kernel<DT, 4, true>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((hccl_moe_combine_backward_kernel<DT, 4, false>), grid, block, 0, s, a);
    });
}

}  // namespace hccl
