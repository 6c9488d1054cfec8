// moe_route.hip -- routing: logits to chosen experts and weights, and the logits' gradient.
//
// A token's experts lie in the registers of L neighbouring lanes, N consecutive ones each, so a wave
// routes 64 / L tokens and nothing is exchanged beyond those lanes. One round of the top k is a
// maximum over N registers and L lanes; the maximum of the exponentials' argument, their sum and the
// chosen weights' sum are reductions over the same lanes. All of it is held in 32 bits.
// Bound by launch and latency up to thousands of tokens (one token of 64 experts 2.1-2.5 us, 4 099 of 192 fp32 with
// bias and groups 5.7-7.2 us), then by the arithmetic of the rounds: 32 768 tokens x 128 bf16 experts, top 8, 5.6-7.2 us
// for 10.5 MB, their gradient 4.7-5.7 us for 18.9 MB, also without renormalisation (512 experts 14 us for 69 MB);
// 32 768 x 256 fp32 sigmoids with a bias 21 us for 36 MB: two reductions a round where 16-bit logits have one.
//
//   s_e = exp(l_e - max l) / sum, or 1 / (1 + exp(-l_e))
//   w_k = scale * s_{i_k} (/ sum_j s_{i_j})
#include "moe_device.h"

namespace hccl {
namespace {

constexpr int kRouteThreads = 256;

// N logits of a lane, the first of them expert e0; experts past the end, and those whose logit is
// minus infinity or no number, are -inf: never chosen, with score 0.
template <int DT, int N>
__device__ __forceinline__ void load_logits(const char* row, uint32_t e0, uint32_t experts, bool on, float (&l)[N]) {
    constexpr int ES = kSize<DT>;
#pragma unroll
    for (int j = 0; j < N; ++j) l[j] = -kInf;
    if (!on || e0 >= experts) return;
    if (e0 + N <= experts) {
        constexpr int V = kVecOf<DT>;
#pragma unroll
        for (int q = 0; q < N / V; ++q) {
            float x[V];
            widen<DT>(load16<ES>(row + (uint64_t)(e0 + q * V) * ES), x);
#pragma unroll
            for (int i = 0; i < V; ++i) l[q * V + i] = x[i];
        }
        if constexpr (N % V == 4) {  // four 16-bit logits
            const typename Loose<ES>::x2 r = *gptr<typename Loose<ES>::x2>(row + (uint64_t)(e0 + N - 4) * ES);
#pragma unroll
            for (int j = 0; j < 4; ++j) l[N - 4 + j] = widen1<DT>((r[j / 2] >> (16 * (j & 1))) & 0xffffu);
        }
    } else {
        constexpr int V = kVecOf<DT>;
#pragma unroll
        for (int q = 0; q < (N + V - 1) / V; ++q) {
            float x[V];
            widen<DT>(load_row<ES>(row, e0 + q * V, experts), x);
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (q * V + i < N && e0 + q * V + i < experts) l[q * V + i] = x[i];
        }
    }
#pragma unroll
    for (int j = 0; j < N; ++j) l[j] = fmaxf(l[j], -kInf);  // (the greater of NaN and -inf is -inf)
}

constexpr float kLog2e = 1.44269504088896340736f;

// e^(l - m), m the greatest logit, as 2^((l - m) log2 e): the product's rounding makes the error |l - m| 2^-24
// of the value, and the values that count are near m. (One fused product l log2 e - m log2 e would be off by
// m 2^-24, which is anything where all logits are a mask's -1e9.) Logits of +inf share the weight among
// themselves: inf - inf is NaN, and the lesser of NaN and 0 is 0. Without any logit (m = -inf) all are 0.
struct Exponential {
    float top;
    __device__ __forceinline__ explicit Exponential(float m) : top(m > -kInf ? m : 0.0f) {}
    __device__ __forceinline__ float operator()(float l) const { return __builtin_amdgcn_exp2f(fminf(l - top, 0.0f) * kLog2e); }
};
// (0 at -inf)
__device__ __forceinline__ float sigmoid(float l) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-l * kLog2e)); }

// Sigmoids of a token's choices (a lane has one choice's logit, -inf without one), for shares of their sum. Where the
// sum r is small, some or all of them may be too small for 32 bits, and 1 / r too great; so there they are taken without a
// factor that they have in common: e^l / (1 + e^l) = e^m e^(l - m) s(-l), m the greatest logit. (Above 2^-24 a share that
// is lost is below 2^-102.) Below e^-708, the least normal number of 64 bits, they are 0 all the same: a mask by a
// great negative number leaves nothing to share. The branch is a wave's, the choice between the two each token's.
constexpr float kSmallSum = 0x1p-24f, kNoScore = -708.0f;
template <int L>
__device__ __forceinline__ void small_sigmoids(float logit, float& u, float& r) {
    if (!__ballot(r < kSmallSum)) return;
    const float m = max_lanes<L>(logit), v = m < kNoScore ? 0.0f : Exponential(m)(logit) * sigmoid(-logit), sum = sum_lanes<L>(v);
    u = r < kSmallSum ? v : u;
    r = r < kSmallSum ? sum : r;
}

// A 16-bit float widened to 32 bits has its 13 lowest bits free: the order of the float as an unsigned
// number there, and 1023 less the expert below it. -0 counts as 0. And back.
constexpr uint32_t kFree = 0x1fffu;
__device__ __forceinline__ uint32_t order16(float l, uint32_t e) {
    const int32_t x = __float_as_int(l + 0.0f);
    return ((uint32_t)x ^ (((uint32_t)(x >> 31) & 0x7fffffffu & ~kFree) | 0x80000000u)) | (HCCL_MAX_EXPERTS - 1 - e);
}
__device__ __forceinline__ float value16(uint32_t key) {
    const uint32_t o = key & ~kFree;
    return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o & ~kFree);
}

// PACK: the choice is by 16-bit logits, so logit and expert fit one 32-bit key, greater for the
// lower expert among equals: a round is one maximum. Otherwise a round is the greatest choice score,
// then the lowest expert that has it.
template <int DT, int L, int N, bool PACK, bool GROUPED>
__global__ __launch_bounds__(kRouteThreads) void hccl_moe_route_kernel(RouteArgs a) {
    constexpr int ES = kSize<DT>;
    const uint32_t sub = threadIdx.x & (L - 1), slot = threadIdx.x / L;
    const uint64_t t = (uint64_t)blockIdx.x * (kRouteThreads / L) + slot;
    const bool on = t < a.tokens;
    const char* row = (const char*)a.logits + t * a.ld * ES;
    const uint32_t e0 = sub * N;
    float bias[PACK ? 1 : N] = {};
    if constexpr (!PACK) {
        if (a.bias) {  // (on their way together with the logits; no branch for each)
#pragma unroll
            for (int j = 0; j < N; ++j) bias[j] = a.bias[e0 + j < a.experts ? e0 + j : 0];
        }
    }
    float l[N];
    load_logits<DT, N>(row, e0, a.experts, on, l);

    float m = -kInf, inv = 1.0f;  // greatest logit, 1 / the sum of the exponentials
    if (!a.sigmoid) {
#pragma unroll
        for (int j = 0; j < N; ++j) m = fmaxf(m, l[j]);
        m = max_lanes<L>(m);
    }
    const Exponential exponential(m);
    // Renormalised weights of a choice by logit have no need of the sum over all experts: it cancels.
    if (!a.sigmoid && a.whole_sum) {
        float total = 0.0f;
#pragma unroll
        for (int j = 0; j < N; ++j) total += exponential(l[j]);
        total = sum_lanes<L>(total);
        inv = total > 0.0f ? 1.0f / total : 0.0f;
    }
    auto score = [&](float x) { return a.sigmoid ? sigmoid(x) : exponential(x) * inv; };

    uint32_t mine = ~0u;   // lane k keeps choice k
    float logit = -kInf;
    if constexpr (PACK) {
        uint32_t key[N];
#pragma unroll
        for (int j = 0; j < N; ++j) key[j] = order16(l[j], e0 + j);
        // Keys already chosen are the last one and those above it. Less the last one, modulo 2^32, they
        // come below all the others, in their order: one subtraction takes them all out. (-inf is chosen
        // like any other value, behind them all, and stands for no expert.)
        uint32_t last = 0;
        for (uint32_t k = 0; k < a.top_k; ++k) {
            uint32_t best = key[0] - last;
#pragma unroll
            for (int j = 1; j < N; ++j) best = max(best, key[j] - last);
            last += maxu_lanes<L>(best);
            mine = sub == k ? last : mine;
        }
        if (sub < a.top_k) {
            logit = value16(mine);
            mine = logit > -kInf ? HCCL_MAX_EXPERTS - 1 - (mine & kFree) : ~0u;
        }
    } else {
        // the chosen logits are looked up here at the end
        __shared__ float logits[kRouteThreads * N];
        float* own = logits + slot * (L * N);
        float c[N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
            c[j] = l[j];
            own[e0 + j] = l[j];
        }
        // Choice values: logits, or with a bias scores and bias. Groups are judged by them, or by scores.
        float v[N];
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = l[j];
        if (a.bias || (GROUPED && a.group_top == 2)) {
            if (a.sigmoid) {
#pragma unroll
                for (int j = 0; j < N; ++j) v[j] = sigmoid(l[j]) + bias[j];
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j) v[j] = exponential(l[j]) * inv + bias[j];
            }
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = l[j] > -kInf ? fmaxf(v[j], -kInf) : -kInf;
        }
        if (a.bias) {
#pragma unroll
            for (int j = 0; j < N; ++j) c[j] = v[j];
        }
        if constexpr (GROUPED) {
            // lane g: the greatest one or two values of group g, of those that may be chosen. Where groups
            // are whole lanes, a lane has found its own two first.
            __shared__ float seen[kRouteThreads * N];
            float* part = seen + slot * (L * N);
            float one = -kInf, two = -kInf;
            auto take = [&](float x) {
                two = fmaxf(two, fminf(one, x));
                one = fmaxf(one, x);
            };
            uint32_t each = a.group_size;  // values of a group in LDS
            if (a.group_lanes) {
                each = a.group_lanes * 2;
#pragma unroll
                for (int j = 0; j < N; ++j) take(v[j]);
                part[sub * 2] = one;
                part[sub * 2 + 1] = two;
                one = two = -kInf;
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j) part[e0 + j] = v[j];
            }
            __syncthreads();
            if (sub < a.groups) {
                const float* group = part + sub * each;
#pragma unroll 4
                for (uint32_t n = 0; n < each; ++n) take(group[n]);
            }
            float left = a.group_top == 2 && two > -kInf ? one + two : one;
            uint32_t kept = 0;
            for (uint32_t k = 0; k < a.top_groups; ++k) {
                const float best = max_lanes<L>(left);
                const uint32_t g = minu_lanes<L>(best > -kInf && left == best ? sub : 255u);
                if (g < 32u) kept |= 1u << g;
                if (sub == g) left = -kInf;
            }
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const uint32_t g = ((e0 + j) * a.group_magic) >> 20;
                if (g < 32u && !((kept >> g) & 1u)) c[j] = -kInf;
            }
        }
        for (uint32_t k = 0; k < a.top_k; ++k) {
            float best = c[0];
#pragma unroll
            for (int j = 1; j < N; ++j) best = fmaxf(best, c[j]);
            best = max_lanes<L>(best);
            uint32_t e = ~0u;
#pragma unroll
            for (int j = N - 1; j >= 0; --j) e = c[j] == best ? e0 + j : e;
            e = minu_lanes<L>(e);
            if (best == -kInf) e = ~0u;  // none is left
            if (sub == k) mine = e;
#pragma unroll
            for (int j = 0; j < N; ++j) c[j] = e0 + j == e ? -kInf : c[j];
        }
        __syncthreads();
        if (mine != ~0u) logit = own[mine];
    }

    if (on && a.mask && !a.mask[t]) {
        mine = ~0u;
        logit = -kInf;
    }
    float w = score(logit);
    if (a.renormalize) {
        // Where the greatest logit of all need not be among the chosen (a bias, groups by two values) their
        // scores may all be too small for 32 bits; their shares are not, by the greatest logit among them.
        if (!a.sigmoid && a.whole_sum) w = Exponential(max_lanes<L>(logit))(logit);
        float sum = sum_lanes<L>(w);
        if (a.sigmoid) small_sigmoids<L>(logit, w, sum);
        w = sum > 0.0f ? w / sum : 0.0f;
    }
    if (on && sub < a.top_k) {
        a.index[t * a.top_k + sub] = (int32_t)mine;
        a.weight[t * a.top_k + sub] = w * a.scale;
    }
}

// With r = sum_k u_k (or 1), u_k = s_{i_k}, w_k = scale u_k / r:
//   du_k = scale (g_k - sum_j g_j u_j / r) / r (the second term only with the sum)
//   softmax: dl_e = s_e (du_e - sum_k du_k u_k)     sigmoid: dl_e = du_e s_e (1 - s_e)
// Scores are computed again from the logits: reading them costs less than storing them would.
// DENSE: a softmax without renormalisation, where every expert's logit moves the weights. Otherwise only
// the chosen ones' do: with the sum, sum_k du_k u_k is nothing, and with the shares p_k = u_k / r
//   dl_e = scale (g_e - sum_j g_j p_j) p_e   (times 1 - s_e: sigmoid)
// so a lane needs its choice's logit and no other. The gradients of the chosen go to the lanes that hold
// those experts through LDS.
template <int DT, int L, int N, bool DENSE>
__global__ __launch_bounds__(kRouteThreads) void hccl_moe_route_backward_kernel(RouteBackwardArgs a) {
    constexpr int ES = kSize<DT>;
    __shared__ float slope[kRouteThreads * N];
    const uint32_t sub = threadIdx.x & (L - 1), slot = threadIdx.x / L;
    const uint64_t t = (uint64_t)blockIdx.x * (kRouteThreads / L) + slot;
    const bool on = t < a.tokens;
    const char* row = (const char*)a.logits + t * a.ld * ES;
    const uint32_t e0 = sub * N;
    float* part = slope + slot * (L * N);
    uint32_t mine = ~0u;
    float g = 0.0f, logit = -kInf;
    if (on && sub < a.top_k) {
        mine = (uint32_t)a.index[t * a.top_k + sub];
        g = a.grad_weight[t * a.top_k + sub] * a.scale;
    }
    const bool some = mine < a.experts;
    if (some) logit = fmaxf(widen1<DT>(load1<ES>(row + (uint64_t)mine * ES)), -kInf);
    else g = 0.0f;
    float l[DENSE ? N : 1];
    if constexpr (DENSE) load_logits<DT, N>(row, e0, a.experts, on, l);
#pragma unroll
    for (int j = 0; j < N; ++j) part[e0 + j] = 0.0f;
    __syncthreads();
    float common = 0.0f;
    if constexpr (DENSE) {
        float m = -kInf;
#pragma unroll
        for (int j = 0; j < N; ++j) m = fmaxf(m, l[j]);
        m = max_lanes<L>(m);
        const Exponential exponential(m);
        float total = 0.0f;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            l[j] = exponential(l[j]);
            total += l[j];
        }
        total = sum_lanes<L>(total);
        const float inv = total > 0.0f ? 1.0f / total : 0.0f;
#pragma unroll
        for (int j = 0; j < N; ++j) l[j] *= inv;
        common = sum_lanes<L>(g * (exponential(logit) * inv));
    } else {
        // 1 - s = s(-l), without its cancellation. (0 at -inf)
        float u = sigmoid(logit), d = u, slope = a.sigmoid ? sigmoid(-logit) : 1.0f;
        if (!a.sigmoid) u = Exponential(max_lanes<L>(logit))(logit);
        if (a.renormalize) {
            float r = sum_lanes<L>(u), mean = sum_lanes<L>(g * u);
            if (a.sigmoid && __ballot(r < kSmallSum)) {
                small_sigmoids<L>(logit, u, r);
                mean = sum_lanes<L>(g * u);
            }
            d = r > 0.0f ? u / r : 0.0f;
            g = r > 0.0f ? g - mean / r : 0.0f;
        }
        g *= d * slope;
    }
    if (some) atomicAdd(&part[mine], g);  // (a router names an expert once)
    __syncthreads();
    if (!on || e0 >= a.experts) return;
    float d[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        d[j] = part[e0 + j];
        if constexpr (DENSE) d[j] = l[j] * (d[j] - common);
    }
    char* out = (char*)a.grad_logits + t * a.ldg * ES;
    if (e0 + N <= a.experts) {
        constexpr int V = kVecOf<DT>;
#pragma unroll
        for (int q = 0; q < N / V; ++q) {
            float x[V];
#pragma unroll
            for (int i = 0; i < V; ++i) x[i] = d[q * V + i];
            store16<ES>(out + (uint64_t)(e0 + q * V) * ES, narrow<DT>(x));
        }
        if constexpr (N % V == 4) {
            typedef typename Loose<ES>::x2 v2;
            *gptr<v2>(out + (uint64_t)(e0 + N - 4) * ES) = v2{narrow1<DT>(d[N - 4]) | narrow1<DT>(d[N - 3]) << 16, narrow1<DT>(d[N - 2]) | narrow1<DT>(d[N - 1]) << 16};
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < N; ++j)
        if (e0 + j < a.experts) store1<ES>(out + (uint64_t)(e0 + j) * ES, narrow1<DT>(d[j]));
}

// Lanes for a token: 16 where they hold its choices and groups one each and its experts 16 each, else 32
// or 64. Few lanes leave little to exchange between them; a wave then routes four tokens.
template <int L, int N>
struct Shape {
    static constexpr int lanes = L, each = N;
};
template <typename F>
hipError_t by_lanes(uint32_t experts, uint32_t across, F f) {
    if (across <= 16 && experts <= 64) return f(Shape<16, 4>());
    if (across <= 16 && experts <= 128) return f(Shape<16, 8>());
    if (across <= 16 && experts <= 192) return f(Shape<16, 12>());
    if (across <= 16 && experts <= 256) return f(Shape<16, 16>());
    if (experts <= 256) return f(Shape<32, 8>());
    if (experts <= 512) return f(Shape<32, 16>());
    return f(Shape<64, 16>());
}

// A launch's threads are counted in 32 bits.
bool too_many(uint64_t tokens, uint32_t lanes) { return (tokens + kRouteThreads) * lanes > 0xffffffffull; }

template <int DT>
hipError_t route_type(RouteArgs a, hipStream_t s) {
    const bool grouped = a.top_groups < a.groups;
    return by_lanes(a.experts, a.top_k > a.groups ? a.top_k : a.groups, [&](auto shape) {
        constexpr int L = decltype(shape)::lanes, N = decltype(shape)::each;
        if (too_many(a.tokens, L)) return hipErrorInvalidConfiguration;
        const dim3 grid((uint32_t)((a.tokens + kRouteThreads / L - 1) / (kRouteThreads / L))), block(kRouteThreads);
        if (grouped) {
            a.group_lanes = a.group_size % N ? 0 : a.group_size / N;
            hipLaunchKernelGGL((hccl_moe_route_kernel<DT, L, N, false, true>), grid, block, 0, s, a);
        } else if (DT != hcclFp32 && !a.bias) {
            hipLaunchKernelGGL((hccl_moe_route_kernel<DT, L, N, DT != hcclFp32, false>), grid, block, 0, s, a);
        } else {
            hipLaunchKernelGGL((hccl_moe_route_kernel<DT, L, N, false, false>), grid, block, 0, s, a);
        }
        return hipGetLastError();
    });
}

template <int DT>
hipError_t backward_type(const RouteBackwardArgs& a, hipStream_t s) {
    return by_lanes(a.experts, a.top_k, [&](auto shape) {
        constexpr int L = decltype(shape)::lanes, N = decltype(shape)::each;
        if (too_many(a.tokens, L)) return hipErrorInvalidConfiguration;
        const dim3 grid((uint32_t)((a.tokens + kRouteThreads / L - 1) / (kRouteThreads / L))), block(kRouteThreads);
        if (!a.sigmoid && !a.renormalize) hipLaunchKernelGGL((hccl_moe_route_backward_kernel<DT, L, N, true>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((hccl_moe_route_backward_kernel<DT, L, N, false>), grid, block, 0, s, a);
        return hipGetLastError();
    });
}

}  // namespace

hipError_t launch_route(const RouteArgs& a, hcclDataType_t dt, hipStream_t s) {
    return dt == hcclBf16 ? route_type<hcclBf16>(a, s) : dt == hcclFp16 ? route_type<hcclFp16>(a, s) : route_type<hcclFp32>(a, s);
}

hipError_t launch_route_backward(const RouteBackwardArgs& a, hcclDataType_t dt, hipStream_t s) {
    return dt == hcclBf16 ? backward_type<hcclBf16>(a, s) : dt == hcclFp16 ? backward_type<hcclFp16>(a, s) : backward_type<hcclFp32>(a, s);
}

}  // namespace hccl
