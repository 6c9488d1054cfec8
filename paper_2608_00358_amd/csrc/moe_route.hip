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
#include "moe_route_device.h"

namespace hccl {
namespace {

constexpr int kRouteThreads = 256;

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

    __shared__ float logits[PACK ? 1 : kRouteThreads * N], seen[GROUPED ? kRouteThreads * N : 1];
    route_token<L, N, PACK, GROUPED>(a, t, sub, on, l, bias, logits + (PACK ? 0 : slot * (L * N)), seen + (GROUPED ? slot * (L * N) : 0), [&](int32_t index, float weight) {
        a.index[t * a.top_k + sub] = index;
        a.weight[t * a.top_k + sub] = weight;
    });
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
