// moe_route_device.h -- a token's choice of experts, as the kernels that route share it.
#pragma once
#include "moe_device.h"

namespace hccl {
namespace {

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
//
// A token's lane `sub` of L, with its logits and biases: lane k gets choice k and its weight without the scale. In LDS a token has L * N values
// of its own: where the chosen logits are looked up (not PACK), and where groups are judged (GROUPED). All threads of the block
// call it together.
template <int L, int N, bool PACK, bool GROUPED, typename F>
__device__ __forceinline__ void route_token(const RouteArgs& a, uint64_t t, uint32_t sub, bool on, const float (&l)[N], const float (&bias)[PACK ? 1 : N], float* own,
                                            float* part, F store) {
    const uint32_t e0 = sub * N;
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
    if (on && sub < a.top_k) store((int32_t)mine, w * a.scale);
}

}  // namespace
}  // namespace hccl
