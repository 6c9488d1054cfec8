// moe_mx_layer.hip -- a whole mixture-of-experts layer for few tokens, with weights in microscaled 4-bit floats:
//   h_tk = silu(G_e x_t) * (U_e x_t),   y_t = sum_k w_tk D_e h_tk,   e = the token's choice k
// in two launches, the first of which makes the choice too. Tokens keep their own type: codes become 16-bit floats exactly (an e2m1
// code times a power of two has two bits; from 2^128 on it is infinite), rows and hidden values that 16-bit floats do not hold are
// split into two or three that add up to them (down to 2^-133, the least 16-bit float), and the matrix instructions add up
// the products in 32 bits. Bound by latency up to some MB of weights (one token, 4 experts of 2048 x 1024, 15.1 us for 13 MB),
// then by their bytes and by what rows and hidden values take to reach the matrix instructions: 8 tokens, 8 of 128 experts of
// 4096 x 1024, 74-92 us for 355 MB; 32 tokens, 4 of 64 experts of 4096 x 2048, 183-217 us for 766 MB, and 262 where an expert has
// more than 8 of them. (Ranges are those of eight batches.)
#include <type_traits>

#include "moe_mx_device.h"
#include "moe_route_device.h"

namespace hccl {
namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));

constexpr int kTerms(int dt) { return dt == hcclBf16 ? 1 : dt == hcclFp16 ? 2 : 3; }   // bf16 terms that hold a value of a type
// bf16 planes of the hidden values: 32 bits of them, as rows of fp32 have. With two the last would be rounded, 2^-16 of a value
// away, for 1.5 times fewer loads in the second launch (8 tokens 25 : 28 us, 32 tokens 80 : 91 us).
constexpr int kPlanes = 3;

__device__ __forceinline__ uint32_t padded(uint32_t inner) { return (inner + 31) / 32 * 32; }

// Eight codes times 2^(b - 127) as 16-bit floats: subnormal ones from the least scales, infinite ones from the greatest two.
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

// Eight elements of a row as they lie in memory; those behind the last are 0.
template <int DT>
struct Raw {
    v4u v[kSize<DT> / 2];
};
template <int DT, bool INSIDE>
__device__ __forceinline__ void load_raw(const char* row, uint32_t e, uint32_t cols, Raw<DT>& r) {
    constexpr int ES = kSize<DT>;
    r.v[0] = INSIDE ? load16<ES>(row + (uint64_t)e * ES) : load_row<ES>(row, e, cols);
    if constexpr (ES == 4) r.v[1] = INSIDE ? load16<4>(row + (uint64_t)e * 4 + 16) : load_row<4>(row, e + 4, cols);
}
template <int DT>
__device__ __forceinline__ void terms_of(const Raw<DT>& r, b8 (&t)[kTerms(DT)]) {
    if constexpr (DT == hcclBf16) {
        t[0] = __builtin_bit_cast(b8, r.v[0]);
    } else {
        float x[8];
        if constexpr (DT == hcclFp16) {
            widen<DT>(r.v[0], x);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(r.v[0][i]), x[4 + i] = __uint_as_float(r.v[1][i]);
        }
        split8<kTerms(DT)>(x, t);
    }
}

constexpr int kWaves = 8;  // of a block
constexpr uint32_t kMostRoutes = HCCL_MAX_LAYER_TOKENS * HCCL_MAX_TOP_K;
constexpr uint32_t kMostEntries = HCCL_MAX_EXPERTS + kMostRoutes / 16;  // (of 4 rows an expert has one at most)
constexpr int kLists = 8;  // more than the entries that a wave has begun: one a step on its way, one that is multiplied and one ahead

// LDS by assembly: the compiler would have a read or write of its own wait for every load to LDS that is on its way, as it
// cannot tell that they have nothing to do with each other. Reads have their wait in the block.
__device__ __forceinline__ uint32_t lds_u16(const uint16_t* p) {
    uint32_t v;
    asm volatile("ds_read_u16 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=&v"(v) : "v"(lds_address(p)) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t lds_u32(const void* p) {
    uint32_t v;
    asm volatile("ds_read_b32 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=&v"(v) : "v"(lds_address(p)) : "memory");
    return v;
}
__device__ __forceinline__ void lds_put16(uint16_t* p, uint32_t v) { asm volatile("ds_write_b16 %0, %1" ::"v"(lds_address(p)), "v"(v) : "memory"); }
__device__ __forceinline__ void lds_add4(float* p, float x, float y, float z, float w) {
    asm volatile("ds_add_f32 %0, %1\n\tds_add_f32 %0, %2 offset:4\n\tds_add_f32 %0, %3 offset:8\n\tds_add_f32 %0, %4 offset:12" ::"v"(lds_address(p)), "v"(x), "v"(y), "v"(z),
                 "v"(w)
                 : "memory");
}

// What the blocks of both kernels find out about the choices: the held expert of every route, its weight, and the entries: experts
// that have a route, with `rows` of their routes each, ascending. An entry is the expert, and the first of its routes << 16.
// Entries have 4, 8 or 16 rows: the least that the expert of most routes needs, so that hardly ever one takes its weights twice.
struct Choices {
    uint16_t expert[kMostRoutes];  // 0xffff without one
    float weight[kMostRoutes];
    uint32_t entries[kMostEntries], count[HCCL_MAX_EXPERTS], number, rows;
    uint16_t lists[kWaves][kLists][16];
};
// ROUTES: and makes them, where the launch found that it may (LayerMxArgs::routes), for rounds that every block does over again
// while it would wait for the routes; block 0 stores them. A launch less: one token 15.6 -> 15.1 us in a row of calls, whose
// launches overlap, and 27.7 -> 26.9 us by itself; 5 tokens by themselves 38.7 -> 37.2 us; 24 and more within a percent. 16 lanes a
// token keep it at one pass for 32 tokens; more experts than 128, 17 choices or groups would not fit those, and are a launch of
// their own.
constexpr int kRouteLanes = 16, kRouteEach = 8;  // a token's lanes, experts of each
constexpr uint32_t kRouteValues = kWaves * 64 * kRouteEach;
template <bool ROUTES>
__device__ __forceinline__ void find_choices(const LayerMxArgs& a, Choices& c, float* values) {
    const uint32_t lane = threadIdx.x & 63, w = first_lane(threadIdx.x >> 6), routes = a.tokens * a.top_k;
    auto note = [&](uint32_t r, int32_t index, float weight) {
        const uint32_t e = (uint32_t)index - a.first;
        c.expert[r] = e < a.held ? (uint16_t)e : 0xffffu;
        c.weight[r] = weight;
        if (e < a.held) atomicAdd(&c.count[e], 1u);
    };
    for (uint32_t e = threadIdx.x; e < a.held; e += kWaves * 64) c.count[e] = 0;
    if (ROUTES && a.routes) {
        __syncthreads();
        const uint32_t sub = threadIdx.x % kRouteLanes, slot = threadIdx.x / kRouteLanes, e0 = sub * kRouteEach;
        for (uint32_t t0 = 0; t0 < a.tokens; t0 += kWaves * 64 / kRouteLanes) {
            const uint32_t t = t0 + slot;
            const bool on = t < a.tokens;
            float l[kRouteEach], bias[kRouteEach] = {};
            if (a.route.bias) {
#pragma unroll
                for (int j = 0; j < kRouteEach; ++j) bias[j] = a.route.bias[e0 + j < a.route.experts ? e0 + j : 0];
            }
            auto load = [&](auto type) {
                constexpr int DT = decltype(type)::value;
                load_logits<DT, kRouteEach>((const char*)a.route.logits + t * a.route.ld * kSize<DT>, e0, a.route.experts, on, l);
            };
            if (a.logits_type == hcclBf16) load(std::integral_constant<int, hcclBf16>());
            else if (a.logits_type == hcclFp16) load(std::integral_constant<int, hcclFp16>());
            else load(std::integral_constant<int, hcclFp32>());
            route_token<kRouteLanes, kRouteEach, false, false>(a.route, t, sub, on, l, bias, values + slot * (kRouteLanes * kRouteEach), nullptr, [&](int32_t index, float weight) {
                const uint32_t r = t * a.top_k + sub;
                note(r, index, weight);
                if (blockIdx.x == 0) a.index[r] = index, a.weight[r] = weight;
            });
        }
    } else {
        constexpr int kEach = (kMostRoutes + kWaves * 64 - 1) / (kWaves * 64);
        int32_t index[kEach];  // (on their way together)
        float weight[kEach];
#pragma unroll
        for (int n = 0; n < kEach; ++n) {
            const uint32_t r = n * kWaves * 64 + threadIdx.x;
            if (r < routes) index[n] = a.index[r], weight[n] = a.weight[r];
        }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < kEach; ++n) {
            const uint32_t r = n * kWaves * 64 + threadIdx.x;
            if (r >= routes) break;
            note(r, index[n], weight[n]);
        }
    }
    __syncthreads();
    if (w == 0) {
        uint32_t most = 0, all = 0;
        for (uint32_t e = lane; e < a.held; e += 64) most = max(most, c.count[e]);
        most = maxu_lanes<64>(most);
        const uint32_t shift = most <= 4 ? 2 : most <= 8 ? 3 : 4;
        for (uint32_t e0 = 0; e0 < a.held; e0 += 64) {
            uint32_t left = e0 + lane < a.held ? c.count[e0 + lane] : 0, first = 0;
            // an expert's entries: the first of all experts, then the second of those that have one, ...
            for (uint64_t mask = __ballot(left > 0); mask; mask = __ballot(left > 0)) {
                if (left) c.entries[all + (uint32_t)__popcll(mask & ((1ull << lane) - 1))] = e0 + lane | first << 16;
                all += (uint32_t)__popcll(mask);
                first += 1u << shift;
                left = left > 1u << shift ? left - (1u << shift) : 0;
            }
        }
        c.number = all;
        c.rows = 1u << shift;
    }
    __syncthreads();
}
// An entry's routes, in their order, into a list of the wave; 0xffff where there are fewer.
__device__ __forceinline__ void list_entry(const LayerMxArgs& a, Choices& c, uint32_t w, uint32_t entry, uint32_t what) {
    const uint32_t lane = threadIdx.x & 63, routes = a.tokens * a.top_k, e = what & 0xffffu;
    uint16_t* list = c.lists[w][entry % kLists];
    if (lane < 16) lds_put16(list + lane, 0xffffu);
    uint32_t at = 0u - (what >> 16);
    for (uint32_t r0 = 0; r0 < routes; r0 += 64) {
        const bool mine = lds_u16(c.expert + (r0 + lane < routes ? r0 + lane : 0)) == e && r0 + lane < routes;
        const uint64_t all = __ballot(mine);
        const uint32_t rank = at + (uint32_t)__popcll(all & ((1ull << lane) - 1));
        if (mine && rank < 16) lds_put16(list + rank, r0 + lane);
        at += (uint32_t)__popcll(all);
    }
}
// The route of row r of an entry; the first one's where there are fewer.
__device__ __forceinline__ uint32_t route_of(Choices& c, uint32_t w, uint32_t entry, uint32_t r) {
    const uint16_t* list = c.lists[w][entry % kLists];
    const uint32_t own = lds_u16(list + r), first = lds_u16(list);
    return own != 0xffffu ? own : first;
}

__device__ __forceinline__ float power_of(const Codes& c, int h) { return mx_power(h ? c.scale >> 8 : c.scale & 0xffu); }

// How rows reach the matrix instructions. A lane of 16 holds 8 elements of its row, 8 times for the 64 that its quarter of the
// wave has of a step. Lanes 4 r to 4 r + 3 load four of the 8 pieces of row r of every four rows, 64 bytes side by side, so
// that two loads do for them instead of 8 whose lanes would each be an access of its own. For an instruction the piece moves from
// its lane to lane 4 r + g, g the four that the row is one of, so that up to 16 rows are 16 columns of one instruction. Columns
// of rows that are not there have nothing that counts.
constexpr uint32_t row_of_lane(uint32_t i) { return i % 4 * 4 + i / 4; }
template <int J, int FOURS, int N>
__device__ __forceinline__ b8 piece(const b8 (&t)[FOURS][N], int n, uint32_t lane) {
    constexpr int kAll = J * 0x55;  // the quad's lane J to all of it
    v4u v = __builtin_bit_cast(v4u, t[0][n]);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = dpp<kAll>(v[k]);
#pragma unroll
    for (int g = 1; g < FOURS; ++g) {
        const v4u u = __builtin_bit_cast(v4u, t[g][n]);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t moved = dpp<kAll>(u[k]);
            v[k] = (lane & 3) == (uint32_t)g ? moved : v[k];
        }
    }
    return __builtin_bit_cast(b8, v);
}
// p[j] of lane 4 r + g: t[g] of lane 4 r + j, for the N that there are. So with several planes or rows for a lane all of its pieces
// move at once, in two exchanges.
template <int N>
__device__ __forceinline__ void turn(const b8 (&t)[N], b8 (&p)[4], uint32_t lane) {
    static_assert(N >= 2 && N <= 4, "lanes of a quad");
    const bool odd = lane & 1, high = lane & 2;
    v4u x[4], y[4];
#pragma unroll
    for (int n = 0; n < N; ++n) x[n] = __builtin_bit_cast(v4u, t[n]);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t s0 = dpp<kQuadSwap>(x[0][k]), s1 = dpp<kQuadSwap>(x[1][k]);
        const uint32_t a0 = odd ? s1 : x[0][k], a1 = odd ? x[1][k] : s0;
        const uint32_t h0 = dpp<kQuadHalf>(a0), h1 = dpp<kQuadHalf>(a1);
        if constexpr (N == 2) {
            y[0][k] = a0, y[1][k] = a1, y[2][k] = h0, y[3][k] = h1;
        } else {
            const uint32_t s2 = dpp<kQuadSwap>(x[2][k]);
            uint32_t a2 = x[2][k], a3 = s2;
            if constexpr (N == 4) {
                const uint32_t s3 = dpp<kQuadSwap>(x[3][k]);
                a2 = odd ? s3 : x[2][k], a3 = odd ? x[3][k] : s2;
            }
            const uint32_t h2 = dpp<kQuadHalf>(a2), h3 = dpp<kQuadHalf>(a3);
            y[0][k] = high ? h2 : a0, y[1][k] = high ? h3 : a1, y[2][k] = high ? a2 : h0, y[3][k] = high ? a3 : h1;
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) p[j] = __builtin_bit_cast(b8, y[j]);
}
// f(which of four pieces) for each
template <typename F>
__device__ __forceinline__ void each_piece(F f) {
    f(std::integral_constant<int, 0>());
    f(std::integral_constant<int, 1>());
    f(std::integral_constant<int, 2>());
    f(std::integral_constant<int, 3>());
}

// Both kernels walk along whole steps of 256 elements, kAhead of which are on their way while one is multiplied: with no branch
// around a load, which would leave the compiler unable to tell how many are, and all of them waited for. So lanes without a
// row read their first one, steps behind the last are the last once more, and what is left of a row behind its whole steps
// is a second, plain pass.

// Hidden values. An item is 16 gates and their 16 ups of one expert, for the rows of an entry; `shares` waves of a block
// take one, each a part of the tokens' columns in steps of 256, and join their sums through LDS, in the waves' order. As many
// shares as leave the waves least to do in all of their rounds.
template <int DT, int FOURS, int AHEAD, bool ALIGNED>
__device__ __forceinline__ void layer_up(const LayerMxArgs& a, Choices& choices, char* buffers, v4f (*part)[2][64]) {
    constexpr int TERMS = kTerms(DT), ES = kSize<DT>;
    const uint32_t lane = threadIdx.x & 63, w = first_lane(threadIdx.x >> 6), i = lane & 15, q = lane >> 4;
    const uint32_t ldh = padded(a.inner), tiles = ldh / 16, items = first_lane(choices.number) * tiles;
    const uint32_t steps = ((a.cols + 1) / 2 + 127) / 128, whole_steps = a.cols / 256;
    uint32_t shares = 1;
    {
        uint32_t least = ~0u;
#pragma unroll
        for (uint32_t n = 1; n <= kWaves; n *= 2) {  // steps of all rounds (a step's time and a half for each round's beginning and end)
            const uint32_t each = gridDim.x * (kWaves / n), time = (items + each - 1) / each * (2 * ((steps + n - 1) / n) + 3);
            if (time < least) least = time, shares = n;
        }
    }
    const uint32_t at_a_time = kWaves / shares, share = w % shares;
    char* mine = buffers + w * (AHEAD * kSlot<2>);
    const uint32_t at0 = lds_address(mine) + code_place(lane), at_scale = lds_address(mine) + scale_place(2, lane);
    for (uint32_t item0 = blockIdx.x * at_a_time; item0 < items; item0 += gridDim.x * at_a_time) {
        const bool some = item0 + w / shares < items;
        const uint32_t item = some ? item0 + w / shares : items - 1, entry = item / tiles, f0 = item % tiles * 16;
        const uint32_t what = first_lane(lds_u32(choices.entries + entry)), e = what & 0xffffu;
        list_entry(a, choices, w, entry, what);
        const char* px[FOURS];
#pragma unroll
        for (int r = 0; r < FOURS; ++r) px[r] = (const char*)a.x + (uint64_t)(route_of(choices, w, entry, r * 4 + i / 4) / a.top_k) * a.ldx * ES;
        auto row_of = [&](int y, uint32_t f) { return (uint64_t)e * 2 * a.inner + y * a.inner + (f < a.inner ? f : a.inner - 1); };
        const uint8_t *pw[2], *ps[2];
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            pw[y] = a.w_in + row_of(y, f0 + i) * a.ld_in;
            ps[y] = a.w_in_scale + row_of(y, f0 + i) * a.ld_in_scale;
        }
        Source<2> src;
        if constexpr (ALIGNED) src = source_of<2>(a.w_in, a.ld_in, a.w_in_scale, a.ld_in_scale, [&](uint32_t y, uint32_t r) { return row_of(y, f0 + r); });
        v4f acc[2] = {v4f{0, 0, 0, 0}, v4f{0, 0, 0, 0}};
        Codes c[ALIGNED ? 1 : AHEAD][2];
        Raw<DT> x[AHEAD][FOURS][2];
        auto fetch_x = [&](int u, uint32_t s, auto inside) {
#pragma unroll
            for (int r = 0; r < FOURS; ++r)
#pragma unroll
                for (int h = 0; h < 2; ++h) load_raw<DT, decltype(inside)::value>(px[r], s * 256 + q * 64 + h * 32 + (i & 3) * 8, a.cols, x[u][r][h]);
        };
        auto fetch_codes = [&](int u, uint32_t s, auto inside) {
#pragma unroll
            for (int y = 0; y < 2; ++y) c[u][y] = load_pair<decltype(inside)::value>(pw[y], ps[y], s * 128 + q * 32, a.cols);
        };
        auto fetch = [&](int u, uint32_t s) {
            if constexpr (ALIGNED) load_to_lds<2>(src, s, mine + u * kSlot<2>);
            else fetch_codes(u, s, std::true_type());
            fetch_x(u, s, std::true_type());
            asm volatile("" ::: "memory");  // (steps' loads are made in the steps' order, which the waits count on)
        };
        auto multiply = [&](int u, const Codes (&codes)[2]) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                b8 terms[FOURS][TERMS];
#pragma unroll
                for (int r = 0; r < FOURS; ++r) terms_of<DT>(x[u][r][h], terms[r]);
                each_piece([&](auto j) {
                    constexpr int J = decltype(j)::value;
                    const b8 v[2] = {decode8(codes[0].c[h][J], power_of(codes[0], h)), decode8(codes[1].c[h][J], power_of(codes[1], h))};
#pragma unroll
                    for (int m = 0; m < TERMS; ++m) {
                        const b8 rows = piece<J>(terms, m, lane);
#pragma unroll
                        for (int y = 0; y < 2; ++y) acc[y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[y], rows, acc[y], 0, 0, 0);
                    }
                });
            }
        };
        if (some && share < whole_steps) {
            const uint32_t n = (whole_steps - share + shares - 1) / shares;  // this wave's steps
            auto step = [&](uint32_t m) { return share + (m < n ? m : n - 1) * shares; };
            auto take = [&](int u) {
                if constexpr (ALIGNED) {
                    wait_steps<(AHEAD - 1) * (kSlotLoads<2> + FOURS * ES)>();
                    const uint32_t at = u * kSlot<2>;
                    read_from_lds(c[0], at0 + at, (at0 ^ 16) + at, at_scale + at);
                    // (used from here on, and not sooner, which would be another wait)
#pragma unroll
                    for (int r = 0; r < FOURS; ++r)
#pragma unroll
                        for (int h = 0; h < 2; ++h)
#pragma unroll
                            for (int n = 0; n < ES / 2; ++n) asm volatile("" : "+v"(x[u][r][h].v[n]));
                    multiply(u, c[0]);
                } else {
                    multiply(u, c[u]);
                }
            };
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) fetch(u, step(u));
            uint32_t m = 0;
#pragma unroll 1
            for (; m + AHEAD <= n; m += AHEAD) {
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    take(u);
                    fetch(u, step(m + u + AHEAD));
                }
            }
#pragma unroll
            for (int u = 0; u < AHEAD - 1; ++u) {
                if (m + u >= n) break;
                take(u);
            }
            if (ALIGNED) wait_steps<0>();  // (those behind the last step)
        }
        if (some && whole_steps < steps && whole_steps % shares == share) {
            fetch_codes(0, whole_steps, std::false_type());
            fetch_x(0, whole_steps, std::false_type());
            multiply(0, c[0]);
        }
        if (shares > 1) {
#pragma unroll
            for (int y = 0; y < 2; ++y) part[w][y][lane] = acc[y];
            __syncthreads();
            if (share == 0) {
                for (uint32_t v = 1; v < shares; ++v)
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const v4f more = part[w + v][y][lane];
#pragma unroll
                        for (int j = 0; j < 4; ++j) acc[y][j] += more[j];
                    }
            }
            __syncthreads();
        }
        const uint32_t route = lds_u16(choices.lists[w][entry % kLists] + row_of_lane(i));
        if (!some || share != 0 || route == 0xffffu) continue;
        const uint32_t f = f0 + q * 4;
        uint16_t* to = a.hidden + (uint64_t)route * kPlanes * ldh + f;
        float h[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) h[j] = f + j < a.inner ? mx_gate(acc[0][j], acc[1][j]) : 0.0f;
#pragma unroll
        for (int p = 0; p < kPlanes; ++p) {
            uint32_t b[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                b[j] = __float_as_uint(h[j]) >> 16;
                h[j] -= __uint_as_float(b[j] << 16);
            }
            *gptr<typename Loose<2>::x2>(to + (uint64_t)p * ldh) = typename Loose<2>::x2{b[0] | b[1] << 16, b[2] | b[3] << 16};
        }
    }
}

constexpr int steps_ahead(int dt, int fours) { return fours == 4 && dt == hcclFp32 ? 1 : 2; }  // (registers)

template <int DT, bool ALIGNED>
__global__ __launch_bounds__(kWaves * 64, 2) void hccl_moe_layer_mx_up_kernel(LayerMxArgs a) {
    __shared__ Choices choices;
    __shared__ v4f part[kWaves][2][64];
    __shared__ __attribute__((aligned(256))) char buffers[ALIGNED ? kWaves * 2 * kSlot<2> : 16];
    static_assert(sizeof(part) >= kRouteValues * sizeof(float), "room for the logits of a round");
    find_choices<true>(a, choices, (float*)part);
    if (choices.number == 0) return;
    const uint32_t rows = first_lane(choices.rows);
    if (rows == 4) layer_up<DT, 1, steps_ahead(DT, 1), ALIGNED>(a, choices, buffers, part);
    else if (rows == 8) layer_up<DT, 2, steps_ahead(DT, 2), ALIGNED>(a, choices, buffers, part);
    else layer_up<DT, 4, steps_ahead(DT, 4), ALIGNED>(a, choices, buffers, part);
}

// Results. A block takes 16 columns of all tokens. The whole steps of all entries, one entry behind the other, are shared out
// evenly among its waves, and so is what is left of each; a wave adds its weighted results up in its own part of LDS, and these
// are added up at the end in the waves' order. An instruction's 16 columns are up to 4 rows in three planes, up to 8 in the
// first two (and another's the third), or up to 16 in one; a row's columns are added up when its entry ends.
template <int FOURS, int AHEAD, bool ALIGNED>
__device__ __forceinline__ void layer_down(const LayerMxArgs& a, Choices& choices, char* buffers, float (*sums)[HCCL_MAX_LAYER_TOKENS][16]) {
    const uint32_t lane = threadIdx.x & 63, w = first_lane(threadIdx.x >> 6), i = lane & 15, q = lane >> 4;
    const uint32_t n0 = blockIdx.x * 16;
    const uint32_t ldh = padded(a.inner), whole_steps = a.inner / 256, entries = first_lane(choices.number);
    char* mine = buffers + w * (AHEAD * kSlot<1>);
    const uint32_t at0 = lds_address(mine) + code_place(lane), at_scale = lds_address(mine) + scale_place(1, lane);
    Codes c[ALIGNED ? 1 : AHEAD][1];
    b8 hidden[AHEAD][FOURS][2][kPlanes];
    const uint8_t *pw, *ps;
    Source<1> src;
    const uint16_t* ph[FOURS];
    auto look = [&](uint32_t entry) {  // turns the pointers to an entry
        const uint32_t what = first_lane(lds_u32(choices.entries + entry));
        const uint64_t first = (uint64_t)(what & 0xffffu) * a.cols;
        auto row_of = [&](uint32_t r) { return first + (n0 + r < a.cols ? n0 + r : a.cols - 1); };
        pw = a.w_out + row_of(i) * a.ld_out;
        ps = a.w_out_scale + row_of(i) * a.ld_out_scale;
        if constexpr (ALIGNED) src = source_of<1>(a.w_out, a.ld_out, a.w_out_scale, a.ld_out_scale, [&](uint32_t, uint32_t r) { return row_of(r); });
        list_entry(a, choices, w, entry, what);
#pragma unroll
        for (int r = 0; r < FOURS; ++r) ph[r] = a.hidden + (uint64_t)route_of(choices, w, entry, r * 4 + i / 4) * kPlanes * ldh;
    };
    auto fetch_h = [&](int u, uint32_t s, auto inside) {
#pragma unroll
        for (int r = 0; r < FOURS; ++r)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int p = 0; p < kPlanes; ++p) {
                    const uint32_t k = s * 256 + q * 64 + h * 32 + (i & 3) * 8;
                    hidden[u][r][h][p] = decltype(inside)::value || k < ldh ? __builtin_bit_cast(b8, load16<2>(ph[r] + (uint64_t)p * ldh + k)) : b8{};
                }
    };
    auto fetch_codes = [&](int u, uint32_t s, auto inside) { c[u][0] = load_pair<decltype(inside)::value>(pw, ps, s * 128 + q * 32, a.inner); };
    auto fetch = [&](int u, uint32_t s) {
        if constexpr (ALIGNED) load_to_lds<1>(src, s, mine + u * kSlot<1>);
        else fetch_codes(u, s, std::true_type());
        fetch_h(u, s, std::true_type());
        asm volatile("" ::: "memory");  // (steps' loads are made in the steps' order, which the waits count on)
    };
    v4f acc[2] = {v4f{0, 0, 0, 0}, v4f{0, 0, 0, 0}};
    auto multiply = [&](int u, const Codes& codes) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            b8 v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = decode8(codes.c[h][j], power_of(codes, h));
            auto with = [&](int y, const auto& t) {
                b8 p[4];
                turn(t, p, lane);
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[j], p[j], acc[y], 0, 0, 0);
            };
            auto& x = hidden[u];
            if constexpr (FOURS == 1) {
                with(0, x[0][h]);
            } else if constexpr (FOURS == 2) {
                const b8 two[4] = {x[0][h][0], x[1][h][0], x[0][h][1], x[1][h][1]}, last[2] = {x[0][h][2], x[1][h][2]};
                with(0, two);
                with(1, last);
            } else {
#pragma unroll
                for (int p = 0; p < kPlanes; ++p) {
                    const b8 four[4] = {x[0][h][p], x[1][h][p], x[2][h][p], x[3][h][p]};
                    with(0, four);
                }
            }
        }
    };
    auto add = [&](uint32_t entry) {
        // (the columns' terms, small ones first)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t y = __float_as_uint(acc[0][j]);
            if constexpr (FOURS == 1) acc[0][j] += __uint_as_float(dpp<kQuadSwap>(y)) + __uint_as_float(dpp<kQuadHalf>(y));
            if constexpr (FOURS == 2) acc[0][j] += __uint_as_float(dpp<kQuadHalf>(y)) + acc[1][j];
        }
        const uint32_t route = lds_u16(choices.lists[w][entry % kLists] + row_of_lane(i));
        if (route != 0xffffu) {
            const float weight = __uint_as_float(lds_u32(choices.weight + route));
            lds_add4(&sums[w][route / a.top_k][q * 4], weight * acc[0][0], weight * acc[0][1], weight * acc[0][2], weight * acc[0][3]);
        }
        acc[0] = acc[1] = v4f{0, 0, 0, 0};
    };
    const uint64_t all = (uint64_t)entries * whole_steps;
    uint32_t g = (uint32_t)(all * w / kWaves);
    const uint32_t end = (uint32_t)(all * (w + 1) / kWaves);
    if (g < end) {
        uint32_t entry = g / whole_steps, s = g % whole_steps;  // that are multiplied
        uint32_t next = entry, next_s = s, left = end - g;      // that are read
        look(next);
        auto fetch_next = [&](int u) {
            fetch(u, next_s);
            if (left > 1) {
                --left;
                if (++next_s == whole_steps) next_s = 0, look(++next);
            }
        };
        auto take = [&](int u) {
            if constexpr (ALIGNED) {
                wait_steps<(AHEAD - 1) * (kSlotLoads<1> + FOURS * 2 * kPlanes)>();
                const uint32_t at = u * kSlot<1>;
                read_from_lds(c[0], at0 + at, (at0 ^ 16) + at, at_scale + at);
                // (used from here on, and not sooner, which would be another wait)
#pragma unroll
                for (int r = 0; r < FOURS; ++r)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int p = 0; p < kPlanes; ++p) asm volatile("" : "+v"(hidden[u][r][h][p]));
                multiply(u, c[0][0]);
            } else {
                multiply(u, c[u][0]);
            }
            ++g;
            if (++s == whole_steps || g == end) {
                add(entry);
                s = 0, ++entry;
            }
        };
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) fetch_next(u);
#pragma unroll 1
        while (g + AHEAD <= end) {
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                take(u);
                fetch_next(u);
            }
        }
#pragma unroll
        for (int u = 0; u < AHEAD - 1; ++u) {
            if (g >= end) break;
            take(u);
        }
        if (ALIGNED) wait_steps<0>();  // (those behind the last step)
    }
    if (whole_steps * 256 < a.inner) {
        for (uint32_t entry = w; entry < entries; entry += kWaves) {
            look(entry);
            fetch_codes(0, whole_steps, std::false_type());
            fetch_h(0, whole_steps, std::false_type());
            multiply(0, c[0][0]);
            add(entry);
        }
    }
}

template <int DT, bool ALIGNED>
__global__ __launch_bounds__(kWaves * 64, 2) void hccl_moe_layer_mx_down_kernel(LayerMxArgs a) {
    constexpr int ES = kSize<DT>;
    __shared__ Choices choices;
    __shared__ float sums[kWaves][HCCL_MAX_LAYER_TOKENS][16];
    __shared__ __attribute__((aligned(256))) char buffers[ALIGNED ? kWaves * 2 * kSlot<1> : 16];
    const uint32_t lane = threadIdx.x & 63, w = first_lane(threadIdx.x >> 6), n0 = blockIdx.x * 16;
    for (uint32_t r = lane; r < a.tokens * 16; r += 64) sums[w][r / 16][r % 16] = 0.0f;
    find_choices<false>(a, choices, nullptr);
    const uint32_t rows = first_lane(choices.rows);
    if (rows == 4) layer_down<1, 2, ALIGNED>(a, choices, buffers, sums);
    else if (rows == 8) layer_down<2, 2, ALIGNED>(a, choices, buffers, sums);
    else layer_down<4, 1, ALIGNED>(a, choices, buffers, sums);  // (registers)
    __builtin_amdgcn_s_waitcnt(0xc07f);  // (LDS alone: the compiler does not know of the sums' additions)
    __syncthreads();
    for (uint32_t r = threadIdx.x; r < a.tokens * 16; r += kWaves * 64) {
        const uint32_t t = r / 16, n = n0 + r % 16;
        if (n >= a.cols) continue;
        float y = sums[0][t][r % 16];
#pragma unroll
        for (int v = 1; v < kWaves; ++v) y += sums[v][t][r % 16];
        store1<ES>((char*)a.out + (t * a.ldo + n) * ES, narrow1<DT>(y));
    }
}

bool aligned(const uint8_t* codes, uint64_t ld, const uint8_t* scale, uint64_t ld_scale) {
    return ((uintptr_t)codes | ld) % 16 == 0 && ((uintptr_t)scale | ld_scale) % 4 == 0;
}

template <int DT>
hipError_t layer_type(LayerMxArgs a, int cus, hipStream_t s) {
    const uint64_t routes = a.cols ? a.tokens * a.top_k : 0, items = routes * ((a.inner + 31) / 32 * 2);  // at most
    const uint64_t down = ((uint64_t)a.cols + 15) / 16;
    if (down * kWaves * 64 > 0xffffffffull || items > 0x7fffffffull) return hipErrorInvalidConfiguration;
    a.routes = items && a.route.experts <= kRouteLanes * kRouteEach && a.top_k <= kRouteLanes && a.route.top_groups == a.route.groups;
    if (!a.routes) {
        const hipError_t e = launch_route(a.route, a.logits_type, s);
        if (e != hipSuccess || a.cols == 0) return e;
    }
    const dim3 block(kWaves * 64), up_grid((uint32_t)(items < (uint64_t)cus ? items : (uint64_t)cus)), down_grid((uint32_t)down);
    if (items) {
        if (aligned(a.w_in, a.ld_in, a.w_in_scale, a.ld_in_scale)) hipLaunchKernelGGL((hccl_moe_layer_mx_up_kernel<DT, true>), up_grid, block, 0, s, a);
        else hipLaunchKernelGGL((hccl_moe_layer_mx_up_kernel<DT, false>), up_grid, block, 0, s, a);
    }
    if (aligned(a.w_out, a.ld_out, a.w_out_scale, a.ld_out_scale)) hipLaunchKernelGGL((hccl_moe_layer_mx_down_kernel<DT, true>), down_grid, block, 0, s, a);
    else hipLaunchKernelGGL((hccl_moe_layer_mx_down_kernel<DT, false>), down_grid, block, 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_layer_mx(const LayerMxArgs& a, hcclDataType_t dt, int cus, hipStream_t s) {
    return dt == hcclBf16 ? layer_type<hcclBf16>(a, cus, s) : dt == hcclFp16 ? layer_type<hcclFp16>(a, cus, s) : layer_type<hcclFp32>(a, cus, s);
}

}  // namespace hccl
