// moe_mx_layer.hip -- a whole mixture-of-experts layer for few tokens, with weights in microscaled 4-bit floats:
//   h_tk = silu(G_e x_t) * (U_e x_t),   y_t = sum_k w_tk D_e h_tk,   e = the token's choice k
// in two launches behind the choice. Tokens keep their own type: codes become 16-bit floats exactly (an e2m1 code times
// a power of two has two bits), rows that 16-bit floats do not hold are split into two or three that add up to them, and
// the matrix instructions add up the products in 32 bits. Bound by the weights' bytes.
#include "moe_mx_device.h"

namespace hccl {
namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));

constexpr int kTerms(int dt) { return dt == hcclBf16 ? 1 : dt == hcclFp16 ? 2 : 3; }   // bf16 terms that hold a value of a type
constexpr int kPlanes(int dt) { return dt == hcclFp32 ? 3 : 2; }                       // bf16 planes of the hidden values

__device__ __forceinline__ uint32_t padded(uint32_t inner) { return (inner + 31) / 32 * 32; }

// Eight codes times 2^(b - 127) as 16-bit floats.
__device__ __forceinline__ b8 decode8(uint32_t c, float power) {
    const b2 p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, power, 0), q = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, power, 1);
    const b2 r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, power, 2), s = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, power, 3);
    return b8{p[0], p[1], q[0], q[1], r[0], r[1], s[0], s[1]};
}

// Eight values as terms of 16 bits: the upper halves of what is left, which is exact until nothing is.
template <int TERMS>
__device__ __forceinline__ void split8(const float (&x)[8], b8 (&t)[TERMS]) {
    float left[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) left[i] = x[i];
#pragma unroll
    for (int n = 0; n < TERMS; ++n) {
        v4u w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __builtin_amdgcn_perm(__float_as_uint(left[2 * i + 1]), __float_as_uint(left[2 * i]), 0x07060302u);
        t[n] = __builtin_bit_cast(b8, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) left[i] -= __uint_as_float(__float_as_uint(left[i]) & 0xffff0000u);
    }
}

// Eight elements of a row at e, as terms; those behind the last are 0.
template <int DT, bool INSIDE>
__device__ __forceinline__ void load_terms(const char* row, uint32_t e, uint32_t cols, b8 (&t)[kTerms(DT)]) {
    constexpr int ES = kSize<DT>;
    if constexpr (DT == hcclBf16) {
        t[0] = __builtin_bit_cast(b8, INSIDE ? load16<2>(row + (uint64_t)e * 2) : load_row<2>(row, e, cols));
    } else {
        float x[8];
        if constexpr (ES == 2) {
            widen<DT>(INSIDE ? load16<2>(row + (uint64_t)e * 2) : load_row<2>(row, e, cols), x);
        } else {
            float lo[4], hi[4];
            widen<DT>(INSIDE ? load16<4>(row + (uint64_t)e * 4) : load_row<4>(row, e, cols), lo);
            widen<DT>(INSIDE ? load16<4>(row + (uint64_t)e * 4 + 16) : load_row<4>(row, e + 4, cols), hi);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = lo[i], x[4 + i] = hi[i];
        }
        split8<kTerms(DT)>(x, t);
    }
}

// The routes of expert e, in their order, into `list` (LDS); their number.
__device__ __forceinline__ uint32_t list_routes(const LayerMxArgs& a, uint32_t e, uint16_t* list, bool write) {
    const uint32_t lane = threadIdx.x & 63, routes = a.tokens * a.top_k;
    uint32_t n = 0;
    for (uint32_t r0 = 0; r0 < routes; r0 += 64) {
        const bool mine = r0 + lane < routes && (uint32_t)a.index[r0 + lane] - a.first == e;
        const uint64_t all = __ballot(mine);
        if (mine && write) list[n + (uint32_t)__popcll(all & ((1ull << lane) - 1))] = (uint16_t)(r0 + lane);
        n += (uint32_t)__popcll(all);
    }
    return n;
}

// Two blocks of codes of a weight row and their scales.
struct Codes {
    v4u c[2];
    uint32_t scale;
};
template <bool INSIDE>
__device__ __forceinline__ Codes load_pair(const uint8_t* row, const uint8_t* scales, uint32_t k, uint32_t cols) {
    typedef uint16_t loose __attribute__((aligned(1)));
    const uint32_t b = k / 16, blocks = (cols + kMxBlock - 1) / kMxBlock;
    Codes r;
#pragma unroll
    for (int h = 0; h < 2; ++h) r.c[h] = INSIDE ? load16<1>(row + k + 16 * h) : load_codes<false, true>(row, k + 16 * h, cols);
    r.scale = INSIDE || b + 2 <= blocks ? *gptr<loose>(scales + b) : b < blocks ? *gptr<uint8_t>(scales + b) : 0u;
    return r;
}
__device__ __forceinline__ float power_of(const Codes& c, int h) { return mx_power(h ? c.scale >> 8 : c.scale & 0xffu); }

// Hidden values: a block takes 16 gates and their 16 ups of one expert, for all of its tokens, 16 at a time; its W waves
// share out the tokens' columns in steps of 256 and join their sums through LDS, in the waves' order.
template <int DT, int W>
__global__ __launch_bounds__(W * 64) void hccl_moe_layer_mx_up_kernel(LayerMxArgs a, uint32_t tiles, uint32_t by_route) {
    constexpr int TERMS = kTerms(DT), PLANES = kPlanes(DT), ES = kSize<DT>;
    __shared__ v4f part[W][2][64];
    __shared__ uint16_t list[HCCL_MAX_LAYER_TOKENS];
    const uint32_t lane = threadIdx.x & 63, w = first_lane(threadIdx.x >> 6), i = lane & 15, q = lane >> 4;
    const uint32_t slot = blockIdx.x / tiles, f0 = blockIdx.x % tiles * 16;
    uint32_t e = slot;
    if (by_route) {  // the block of the first route to an expert takes all of them
        e = (uint32_t)a.index[slot] - a.first;
        if (e >= a.held) return;
    }
    const uint32_t n = list_routes(a, e, list, w == 0);
    __syncthreads();
    if (n == 0 || (by_route && list[0] != slot)) return;

    const uint8_t *pw[2], *ps[2];
#pragma unroll
    for (int y = 0; y < 2; ++y) {
        const uint32_t f = f0 + i < a.inner ? f0 + i : a.inner - 1;
        const uint64_t row = (uint64_t)e * 2 * a.inner + y * a.inner + f;
        pw[y] = a.w_in + row * a.ld_in;
        ps[y] = a.w_in_scale + row * a.ld_in_scale;
    }
#pragma unroll 1
    for (uint32_t x0 = 0; x0 < n; x0 += 16) {
        const bool on = x0 + i < n;
        const uint32_t route = list[on ? x0 + i : x0];
        const char* px = (const char*)a.x + (uint64_t)(route / a.top_k) * a.ldx * ES;
        v4f acc[2] = {v4f{0, 0, 0, 0}, v4f{0, 0, 0, 0}};
        auto step = [&](uint32_t k0, auto inside) {
            constexpr bool INSIDE = decltype(inside)::value;
            const uint32_t k = k0 + q * 32;
            const Codes c[2] = {load_pair<INSIDE>(pw[0], ps[0], k, a.cols), load_pair<INSIDE>(pw[1], ps[1], k, a.cols)};
            b8 t[8][TERMS] = {};
            if (on) {
#pragma unroll
                for (int j = 0; j < 8; ++j) load_terms<DT, INSIDE>(px, k * 2 + j * 8, a.cols, t[j]);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const b8 v = decode8(c[y].c[j / 4][j % 4], power_of(c[y], j / 4));
#pragma unroll
                    for (int m = 0; m < TERMS; ++m) acc[y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, t[j][m], acc[y], 0, 0, 0);
                }
        };
        const uint32_t bytes = (a.cols + 1) / 2;
#pragma unroll 1
        for (uint32_t k0 = w * 128; k0 < bytes; k0 += W * 128) {
            if (k0 + 128 <= a.cols / 2) step(k0, std::true_type());
            else step(k0, std::false_type());
        }
        if (x0) __syncthreads();  // (the sums of the tokens before have been read)
#pragma unroll
        for (int y = 0; y < 2; ++y) part[w][y][lane] = acc[y];
        __syncthreads();
        if (w == 0 && on) {
            v4f g = part[0][0][lane], u = part[0][1][lane];
#pragma unroll
            for (int v = 1; v < W; ++v) {
                const v4f gv = part[v][0][lane], uv = part[v][1][lane];
#pragma unroll
                for (int j = 0; j < 4; ++j) g[j] += gv[j], u[j] += uv[j];
            }
            const uint32_t f = f0 + q * 4, ldh = padded(a.inner);
            uint16_t* to = a.hidden + (uint64_t)route * PLANES * ldh + f;
            float h[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) h[j] = f + j < a.inner ? mx_gate(g[j], u[j]) : 0.0f;
#pragma unroll
            for (int p = 0; p < PLANES; ++p) {
                uint32_t b[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    // (the last of two planes is rounded, after which 2^-16 of the value is missing at most; three are exact)
                    b[j] = p == 1 && PLANES == 2 ? narrow1<hcclBf16>(h[j]) : __float_as_uint(h[j]) >> 16;
                    h[j] -= __uint_as_float(b[j] << 16);
                }
                *gptr<typename Loose<2>::x2>(to + (uint64_t)p * ldh) = typename Loose<2>::x2{b[0] | b[1] << 16, b[2] | b[3] << 16};
            }
        }
    }
}

// Results: a block takes 16 columns of all tokens. Its W waves share out the experts that have a token, and where those are
// fewer the hidden values of each, in steps of 256; a wave adds its weighted results up in its own part of LDS, and
// these are added up at the end in the waves' order.
template <int DT, int W>
__global__ __launch_bounds__(W * 64) void hccl_moe_layer_mx_down_kernel(LayerMxArgs a) {
    constexpr int PLANES = kPlanes(DT), ES = kSize<DT>;
    __shared__ float sums[W][HCCL_MAX_LAYER_TOKENS][16];
    __shared__ uint8_t used[HCCL_MAX_EXPERTS];
    __shared__ uint16_t experts[HCCL_MAX_EXPERTS], lists[W][HCCL_MAX_LAYER_TOKENS];
    __shared__ uint32_t number;
    const uint32_t lane = threadIdx.x & 63, w = first_lane(threadIdx.x >> 6), i = lane & 15, q = lane >> 4;
    const uint32_t n0 = blockIdx.x * 16, routes = a.tokens * a.top_k;
    for (uint32_t e = threadIdx.x; e < a.held; e += W * 64) used[e] = 0;
    for (uint32_t r = lane; r < a.tokens * 16; r += 64) sums[w][r / 16][r % 16] = 0.0f;
    __syncthreads();
    for (uint32_t r = threadIdx.x; r < routes; r += W * 64) {
        const uint32_t e = (uint32_t)a.index[r] - a.first;
        if (e < a.held) used[e] = 1;
    }
    __syncthreads();
    if (w == 0) {
        uint32_t all = 0;
        for (uint32_t e0 = 0; e0 < a.held; e0 += 64) {
            const bool some = e0 + lane < a.held && used[e0 + lane];
            const uint64_t mask = __ballot(some);
            if (some) experts[all + (uint32_t)__popcll(mask & ((1ull << lane) - 1))] = (uint16_t)(e0 + lane);
            all += (uint32_t)__popcll(mask);
        }
        number = all;
    }
    __syncthreads();
    const uint32_t some = first_lane(number), ldh = padded(a.inner), steps = (ldh + 255) / 256;
    uint32_t shares = some && some < W ? W / some : 1;  // of an expert's hidden values
    shares = shares < steps ? shares : steps;
    for (uint32_t unit = w; unit < some * shares; unit += W) {
        const uint32_t e = first_lane(experts[unit / shares]), share = unit % shares;
        const uint32_t n = list_routes(a, e, lists[w], true);
        const uint32_t col = n0 + i < a.cols ? n0 + i : a.cols - 1;
        const uint8_t* pw = a.w_out + ((uint64_t)e * a.cols + col) * a.ld_out;
        const uint8_t* ps = a.w_out_scale + ((uint64_t)e * a.cols + col) * a.ld_out_scale;
#pragma unroll 1
        for (uint32_t x0 = 0; x0 < n; x0 += 16) {
            const bool on = x0 + i < n;
            const uint32_t route = lists[w][on ? x0 + i : x0];
            const uint16_t* ph = a.hidden + (uint64_t)route * PLANES * ldh;
            v4f acc = v4f{0, 0, 0, 0};
            auto step = [&](uint32_t k0, auto inside) {
                constexpr bool INSIDE = decltype(inside)::value;
                const uint32_t k = k0 + q * 32;
                const Codes c = load_pair<INSIDE>(pw, ps, k, a.inner);
                b8 t[8][PLANES] = {};
                if (on) {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
#pragma unroll
                        for (int p = 0; p < PLANES; ++p)
                            if (INSIDE || k * 2 + j * 8 < ldh) t[j][p] = __builtin_bit_cast(b8, load16<2>(ph + (uint64_t)p * ldh + k * 2 + j * 8));
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const b8 v = decode8(c.c[j / 4][j % 4], power_of(c, j / 4));
#pragma unroll
                    for (int p = 0; p < PLANES; ++p) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, t[j][p], acc, 0, 0, 0);
                }
            };
            const uint32_t bytes = (a.inner + 1) / 2;
#pragma unroll 1
            for (uint32_t k0 = share * 128; k0 < bytes; k0 += shares * 128) {
                if (k0 + 128 <= a.inner / 2) step(k0, std::true_type());
                else step(k0, std::false_type());
            }
            if (on) {
                const float weight = a.weight[route];
                float* to = &sums[w][route / a.top_k][q * 4];
#pragma unroll
                for (int j = 0; j < 4; ++j) to[j] += weight * acc[j];
            }
        }
    }
    __syncthreads();
    for (uint32_t r = threadIdx.x; r < a.tokens * 16; r += W * 64) {
        const uint32_t t = r / 16, n = n0 + r % 16;
        if (n >= a.cols) continue;
        float y = sums[0][t][r % 16];
#pragma unroll
        for (int v = 1; v < W; ++v) y += sums[v][t][r % 16];
        store1<ES>((char*)a.out + (t * a.ldo + n) * ES, narrow1<DT>(y));
    }
}

constexpr int kUpWaves = 4, kDownWaves = 16;

template <int DT>
hipError_t layer_type(const LayerMxArgs& a, hipStream_t s) {
    const uint32_t routes = a.tokens * a.top_k, tiles = ((a.inner + 31) / 32 * 32) / 16;
    const bool by_route = routes <= a.held;
    const uint64_t up = (uint64_t)(by_route ? routes : a.held) * tiles, down = ((uint64_t)a.cols + 15) / 16;
    if (up * kUpWaves * 64 > 0xffffffffull || down * kDownWaves * 64 > 0xffffffffull) return hipErrorInvalidConfiguration;
    if (up) hipLaunchKernelGGL((hccl_moe_layer_mx_up_kernel<DT, kUpWaves>), dim3((uint32_t)up), dim3(kUpWaves * 64), 0, s, a, tiles, by_route ? 1u : 0u);
    hipLaunchKernelGGL((hccl_moe_layer_mx_down_kernel<DT, kDownWaves>), dim3((uint32_t)down), dim3(kDownWaves * 64), 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_layer_mx(const LayerMxArgs& a, hcclDataType_t dt, hipStream_t s) {
    return dt == hcclBf16 ? layer_type<hcclBf16>(a, s) : dt == hcclFp16 ? layer_type<hcclFp16>(a, s) : layer_type<hcclFp32>(a, s);
}

}  // namespace hccl
