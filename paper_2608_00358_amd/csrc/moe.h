// moe.h -- the launches of the mixture-of-experts operators: routing, dispatch and combine, and the
// experts' 8-bit product. The entry points (moe_api.cpp) check a call and fill one of these structs,
// which travels in the launch packet; each operator's kernels are in a file of their own.
#pragma once
#include <hip/hip_runtime.h>

#include <stdint.h>

#include "hccl.h"

namespace hccl {

// what moe_api.cpp needs of a communicator and of the error record (api.cpp)
hcclResult_t api_fail(hcclResult_t code, const char* msg);
hcclResult_t api_hip_fail(hipError_t e, const char* what);
hcclResult_t operator_device(hcclComm_t comm, int* device);  // fails where a launch of its own is not possible
int api_ranks(hcclComm_t comm);
int api_cus(hcclComm_t comm);

struct RouteArgs {
    const void* logits;
    const float* bias;     // NULL: experts are chosen by logit, the order of the scores
    const uint8_t* mask;   // NULL: every token is routed
    int32_t* index;
    float* weight;
    uint64_t tokens, ld;
    float scale;
    uint32_t experts, top_k;
    uint32_t groups, top_groups, group_top, group_size;
    uint32_t group_magic;  // ceil(2^20 / group_size): e / group_size = e * group_magic >> 20 for e < 1024
    uint32_t group_lanes;  // lanes of a group where groups are whole lanes, else 0 (set by launch_route)
    uint32_t sigmoid, renormalize;
    uint32_t whole_sum;    // the softmax needs its sum over all experts
};

struct RouteBackwardArgs {
    const void* logits;
    const int32_t* index;
    const float* grad_weight;
    void* grad_logits;
    uint64_t tokens, ld, ldg;
    float scale;
    uint32_t experts, top_k, sigmoid, renormalize;
};

struct PlanArgs {
    const int32_t* index;
    int32_t* row;
    int64_t* offsets;
    int64_t* rank_counts;  // NULL: not wanted
    uint32_t* hist;        // [blocks][experts], where there are several blocks
    uint64_t routes, capacity;
    uint32_t experts, ranks;
    uint32_t blocks, steps;  // a block takes steps * kPlanThreads routes
};
constexpr uint32_t kPlanThreads = 1024;
void plan_shape(uint64_t routes, uint32_t* blocks, uint32_t* steps);

struct DispatchArgs {
    const void* x;
    const int32_t* row;
    void* out;
    uint64_t tokens, cols, ldx, ldo, capacity;
    uint32_t top_k;
};

// Rows to 8-bit codes: row t goes to the rows that `row` names, or to row t where it is NULL.
struct QuantizeArgs {
    const void* x;
    const int32_t* row;
    const int64_t* limit;  // NULL, or the number of rows that hold anything
    int8_t* codes;
    float* scale;
    uint64_t rows, cols, ldx, ldq, capacity;
    uint32_t top_k;
};

// Rows to microscaled 4-bit floats, `blocks` blocks of 32 a row: row t goes to the rows that `row` names, or to row t.
struct QuantizeMxArgs {
    const void* x;
    const int32_t* row;
    const int64_t* limit;  // NULL, or the number of rows that hold anything
    uint8_t* codes;
    uint8_t* scale;
    uint64_t rows, cols, ldx, ldq, lds, capacity;
    uint32_t top_k, blocks;
};

struct DequantizeMxArgs {
    const uint8_t* codes;
    const uint8_t* scale;
    const int64_t* limit;
    void* out;
    uint64_t rows, cols, ldq, lds, ldo;
    uint32_t blocks;
};

struct CombineArgs {
    const void* z;
    const int32_t* row;
    const float* weight;  // NULL: all 1
    void* out;
    uint64_t tokens, cols, ldz, ldo, capacity;
    uint32_t top_k;
};

struct CombineBackwardArgs {
    const void* grad;
    const void* z;
    const int32_t* row;
    const float* weight;
    void* grad_z;         // NULL: not wanted
    float* grad_weight;   // NULL: not wanted
    uint64_t tokens, cols, ldg, ldz, ldo, capacity;
    uint32_t top_k;
};

struct ProductMxArgs {
    const uint8_t* a;
    const uint8_t* a_scale;
    const uint8_t* b;
    const uint8_t* b_scale;
    const int64_t* offsets;  // NULL: one segment with every row
    void* out;
    uint64_t rows, lda, ldas, ldb, ldbs, ldo;
    uint32_t inner, cols, segments, experts;
    uint32_t type;  // hcclDataType_t of the results
};

// A whole layer for few tokens. Row f of an expert's w_in is a gate's, row inner + f the up's.
struct LayerMxArgs {
    const void* x;
    const uint8_t* w_in;
    const uint8_t* w_in_scale;
    const uint8_t* w_out;
    const uint8_t* w_out_scale;
    int32_t* index;  // the routes
    float* weight;
    void* out;
    uint16_t* hidden;  // [route][plane][inner padded to 32], three bf16 planes whose sum is the hidden value
    uint64_t ldx, ld_in, ld_in_scale, ld_out, ld_out_scale, ldo;
    uint32_t tokens, top_k, cols, inner;
    uint32_t first, held;  // experts whose weights are there
    RouteArgs route;       // what the routes are made of
    hcclDataType_t logits_type;
    uint32_t routes;  // the first kernel makes them (set by launch_layer_mx)
};

struct ProductArgs {
    const int8_t* a;
    const float* a_scale;
    const int8_t* b;
    const float* b_scale;
    const int64_t* offsets;  // NULL: one segment with every row
    void* out;
    uint64_t rows, lda, ldb, ldo;
    uint32_t inner, cols, segments, experts;
};

hipError_t launch_route(const RouteArgs& a, hcclDataType_t dt, hipStream_t s);
hipError_t launch_route_backward(const RouteBackwardArgs& a, hcclDataType_t dt, hipStream_t s);
hipError_t launch_plan(const PlanArgs& a, hipStream_t s);
hipError_t launch_dispatch(const DispatchArgs& a, hcclDataType_t dt, hipStream_t s);
hipError_t launch_quantize(const QuantizeArgs& a, hcclDataType_t dt, bool gated, hipStream_t s);
hipError_t launch_combine(const CombineArgs& a, hcclDataType_t dt, hipStream_t s);
hipError_t launch_combine_backward(const CombineBackwardArgs& a, hcclDataType_t dt, hipStream_t s);
hipError_t launch_quantize_mx(const QuantizeMxArgs& a, hcclDataType_t dt, bool gated, hipStream_t s);
hipError_t launch_dequantize_mx(const DequantizeMxArgs& a, hcclDataType_t dt, hipStream_t s);
hipError_t launch_product_mx(const ProductMxArgs& a, int cus, hipStream_t s);
hipError_t launch_layer_mx(const LayerMxArgs& a, hcclDataType_t dt, int cus, hipStream_t s);
hipError_t launch_product(const ProductArgs& a, hcclDataType_t dt, int cus, hipStream_t s);

}  // namespace hccl
