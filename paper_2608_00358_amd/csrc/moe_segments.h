// moe_segments.h -- the tiles of rows in segments, for the products: ARGS has offsets, rows, segments and experts.
#pragma once
#include "moe_device.h"

namespace hccl {
namespace {

struct Rows {
    uint64_t first, end;
    uint32_t expert;
};

// (offsets outside 0 .. rows are clipped, and a segment that ends before it begins is empty)
template <typename ARGS>
__device__ __forceinline__ void segment(const ARGS& a, uint32_t s, uint64_t& first, uint64_t& end) {
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
    template <typename ARGS>
    __device__ __forceinline__ Segments(const ARGS& a, uint32_t s0) {
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
template <uint32_t BM, typename ARGS>
__device__ __forceinline__ uint32_t count_tiles(const ARGS& a, const Segments<BM>& s) {
    uint32_t n = s.all;
    for (uint32_t s0 = kWave; s0 < a.segments; s0 += kWave) n += Segments<BM>(a, s0).all;
    return n;
}

// Rows [first, end) of tile `tile`, and its expert; false where there are fewer tiles.
template <uint32_t BM, typename ARGS>
__device__ __forceinline__ bool find_rows(const ARGS& a, Segments<BM> s, uint32_t tile, Rows& out) {
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

// Tiles that rows in segments can make at most: a segment adds a part of one, and each has a row.
template <typename ARGS>
uint64_t most_tiles(const ARGS& a, uint64_t bm) {
    const uint64_t n = (a.rows + bm - 1) / bm + (a.offsets ? a.segments : 0);
    return n < a.rows ? n : a.rows;
}

}  // namespace
}  // namespace hccl
