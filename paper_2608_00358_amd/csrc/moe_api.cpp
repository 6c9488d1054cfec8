// moe_api.cpp -- entry points of the mixture-of-experts operators: argument checks and launches.
//
// Unlike a collective, an operator is no work packet: nothing is compiled, cached or kept between
// calls, every array is the caller's, and a call is one or two kernel launches on the caller's
// stream, from the launch packet alone. So it may be captured into a HIP graph as it is.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdio>
#include <cstring>

#include "moe.h"

using namespace hccl;

namespace {

constexpr uint64_t kMaxCount = 0x7fffffffull;  // rows and routes are numbered in 32 bits, -1 is none
constexpr uint64_t kMaxBytes = 1ull << 62;
constexpr uint32_t kMaxInner = 131071;         // * 2^14 < 2^31: sums of products never wrap

// Rows of an array: `rows` of `width` bytes, `pitch` bytes apart.
struct Rows2D {
    uintptr_t at;
    uint64_t rows, width, pitch;
    bool written;
    const char* name;
    uint64_t bytes() const { return rows && width ? (rows - 1) * pitch + width : 0; }
};

bool overlap(const Rows2D& a, const Rows2D& b) {
    const uint64_t na = a.bytes(), nb = b.bytes();
    if (!na || !nb || a.at + na <= b.at || b.at + nb <= a.at) return false;
    if (a.rows > 1 && b.rows > 1 && a.pitch == b.pitch) {  // columns of one array, side by side
        const uint64_t d = a.at <= b.at ? (b.at - a.at) % a.pitch : a.pitch - (a.at - b.at) % a.pitch;
        if (d >= a.width && d + b.width <= a.pitch) return false;
    }
    return true;
}

class Check {
public:
    explicit Check(hcclComm_t comm) { result_ = operator_device(comm, &device_); }
    bool ok() const { return result_ == hcclSuccess; }
    hcclResult_t result() const { return result_; }
    bool host_only() const { return device_ == HCCL_NO_DEVICE; }
    int device() const { return device_; }

    Check& that(bool good, const char* msg) {
        if (ok() && !good) result_ = api_fail(hcclInvalidArgument, msg);
        return *this;
    }
    // rows of `width` elements of `es` bytes, `ld` elements apart
    Check& rows(const void* p, uint64_t rows, uint64_t width, uint64_t ld, uint64_t es, bool written, const char* name) {
        if (!ok()) return *this;
        if (rows == 0 || width == 0) return *this;
        if (!p) return refuse("null array: ", name);
        if ((uintptr_t)p % es) return refuse("array not aligned to its elements: ", name);
        if (rows > 1 && ld < width) return refuse("rows overlap (the stride is below the row length): ", name);
        if (width > kMaxBytes / es || (rows > 1 && ld > kMaxBytes / es / rows)) return refuse("array too large: ", name);
        const Rows2D v = {(uintptr_t)p, rows, width * es, rows > 1 ? ld * es : width * es, written, name};
        for (int i = 0; i < n_; ++i)
            if ((written || seen_[i].written) && overlap(v, seen_[i])) return refuse("buffers overlap: ", name);
        if (n_ < (int)(sizeof(seen_) / sizeof(seen_[0]))) seen_[n_++] = v;
        return *this;
    }
    Check& list(const void* p, uint64_t n, uint64_t es, bool written, const char* name) { return rows(p, 1, n, n, es, written, name); }

private:
    Check& refuse(const char* what, const char* name) {
        char msg[160];
        std::snprintf(msg, sizeof(msg), "%s%s", what, name);
        result_ = api_fail(hcclInvalidArgument, msg);
        return *this;
    }
    hcclResult_t result_;
    int device_ = HCCL_NO_DEVICE;
    Rows2D seen_[10];
    int n_ = 0;
};

uint64_t float_size(hcclDataType_t dt) { return dt == hcclFp32 ? 4 : 2; }
bool is_float(hcclDataType_t dt) { return dt == hcclBf16 || dt == hcclFp16 || dt == hcclFp32; }

template <typename F>
hcclResult_t enqueue(const Check& c, F launch) {
    if (c.host_only()) return hcclSuccess;
    int prev = -1;
    const bool changed = hipGetDevice(&prev) == hipSuccess && prev != c.device() && hipSetDevice(c.device()) == hipSuccess;
    const hipError_t e = launch();
    if (changed) (void)hipSetDevice(prev);
    if (e == hipErrorInvalidConfiguration) return api_fail(hcclUnsupported, "call too large for one launch");
    if (e != hipSuccess) return api_hip_fail(e, "launch of an operator");
    return hcclSuccess;
}

// The entry points' bodies: nothing is thrown across the boundary.
template <typename F>
hcclResult_t guarded(F body) {
    try {
        return body();
    } catch (...) {
        return hcclOutOfMemory;
    }
}

void check_router(Check& c, const hcclRouter_t* r) {
    c.that(r != nullptr, "null router");
    if (!c.ok()) return;
    c.that(r->experts >= 1 && r->experts <= HCCL_MAX_EXPERTS, "experts must be 1 to 1024")
        .that(r->top_k >= 1 && r->top_k <= HCCL_MAX_TOP_K && r->top_k <= r->experts, "top_k must be 1 to 32 and no more than the experts")
        .that(r->score == hcclScoreSoftmax || r->score == hcclScoreSigmoid, "unknown score")
        .that(r->groups >= 1 && r->groups <= HCCL_MAX_GROUPS, "groups must be 1 to 32")
        .that(r->groups == 0 || r->experts % r->groups == 0, "groups must divide the experts")
        .that(r->top_groups >= 1 && r->top_groups <= r->groups, "top_groups must be 1 to groups")
        .that(r->group_top == 1 || r->group_top == 2, "group_top must be 1 or 2")
        .that(r->groups == 0 || r->top_k <= r->top_groups * (r->experts / r->groups), "top_k is more than the kept groups hold")
        .that(std::isfinite(r->scale), "scale must be finite");
}

Check& check_routes(Check& c, size_t tokens, uint32_t top_k) {
    return c.that(top_k >= 1 && top_k <= HCCL_MAX_TOP_K, "top_k must be 1 to 32")
        .that(tokens <= kMaxCount / (top_k ? top_k : 1), "more than 2^31 - 1 routes");
}

}  // namespace

extern "C" {

hcclResult_t hccl_router_init(hcclRouter_t* router) {
    return guarded([&] {
        if (!router) return api_fail(hcclInvalidArgument, "null router");
        std::memset(router, 0, sizeof(*router));
        router->top_k = 1;
        router->score = hcclScoreSoftmax;
        router->groups = router->top_groups = router->group_top = 1;
        router->scale = 1.0f;
        return hcclSuccess;
    });
}

hcclResult_t hccl_moe_route(hcclComm_t comm, const hcclRouter_t* router, const void* logits, size_t ld,
                            hcclDataType_t dtype, size_t tokens, const float* bias, const uint8_t* mask, int32_t* index,
                            float* weight, void* stream) {
    return guarded([&] {
        Check c(comm);
        check_router(c, router);
        if (!c.ok()) return c.result();
        c.that(is_float(dtype), "logits must be bf16, fp16 or fp32");
        check_routes(c, tokens, router->top_k)
            .rows(logits, tokens, router->experts, ld, float_size(dtype), false, "logits")
            .list(index, tokens * router->top_k, 4, true, "index")
            .list(weight, tokens * router->top_k, 4, true, "weight");
        if (bias) c.list(bias, router->experts, 4, false, "bias");
        if (mask) c.list(mask, tokens, 1, false, "mask");
        if (!c.ok() || tokens == 0) return c.result();
        RouteArgs a{};
        a.logits = logits;
        a.bias = bias;
        a.mask = mask;
        a.index = index;
        a.weight = weight;
        a.tokens = tokens;
        a.ld = ld;
        a.scale = router->scale;
        a.experts = router->experts;
        a.top_k = router->top_k;
        a.groups = router->groups;
        a.top_groups = router->top_groups;
        a.group_top = router->group_top;
        a.group_size = router->experts / router->groups;
        a.group_magic = ((1u << 20) + a.group_size - 1) / a.group_size;
        a.sigmoid = router->score == hcclScoreSigmoid;
        a.renormalize = router->renormalize != 0;
        a.whole_sum = bias || !a.renormalize || (a.top_groups < a.groups && a.group_top == 2);
        return enqueue(c, [&] { return launch_route(a, dtype, (hipStream_t)stream); });
    });
}

hcclResult_t hccl_moe_route_backward(hcclComm_t comm, const hcclRouter_t* router, const void* logits, size_t ld,
                                     hcclDataType_t dtype, size_t tokens, const int32_t* index, const float* grad_weight,
                                     void* grad_logits, size_t ldg, void* stream) {
    return guarded([&] {
        Check c(comm);
        check_router(c, router);
        if (!c.ok()) return c.result();
        c.that(is_float(dtype), "logits must be bf16, fp16 or fp32");
        const uint64_t es = float_size(dtype);
        check_routes(c, tokens, router->top_k)
            .rows(logits, tokens, router->experts, ld, es, false, "logits")
            .list(index, tokens * router->top_k, 4, false, "index")
            .list(grad_weight, tokens * router->top_k, 4, false, "grad_weight")
            .rows(grad_logits, tokens, router->experts, ldg, es, true, "grad_logits");
        if (!c.ok() || tokens == 0) return c.result();
        RouteBackwardArgs a{};
        a.logits = logits;
        a.index = index;
        a.grad_weight = grad_weight;
        a.grad_logits = grad_logits;
        a.tokens = tokens;
        a.ld = ld;
        a.ldg = ldg;
        a.scale = router->scale;
        a.experts = router->experts;
        a.top_k = router->top_k;
        a.sigmoid = router->score == hcclScoreSigmoid;
        a.renormalize = router->renormalize != 0;
        return enqueue(c, [&] { return launch_route_backward(a, dtype, (hipStream_t)stream); });
    });
}

hcclResult_t hccl_moe_plan_bytes(size_t tokens, uint32_t top_k, uint32_t experts, size_t* bytes) {
    return guarded([&] {
        if (!bytes) return api_fail(hcclInvalidArgument, "null argument");
        if (top_k < 1 || top_k > HCCL_MAX_TOP_K) return api_fail(hcclInvalidArgument, "top_k must be 1 to 32");
        if (tokens > kMaxCount / top_k) return api_fail(hcclInvalidArgument, "more than 2^31 - 1 routes");
        if (experts < 1 || experts > HCCL_MAX_EXPERTS) return api_fail(hcclInvalidArgument, "experts must be 1 to 1024");
        uint32_t blocks, steps;
        plan_shape(tokens * top_k, &blocks, &steps);
        *bytes = blocks > 1 ? (size_t)blocks * experts * sizeof(uint32_t) : 0;
        return hcclSuccess;
    });
}

hcclResult_t hccl_moe_plan(hcclComm_t comm, const int32_t* index, size_t tokens, uint32_t top_k, uint32_t experts,
                           size_t capacity, int32_t* row, int64_t* offsets, int64_t* rank_counts, void* workspace,
                           size_t workspace_bytes, void* stream) {
    return guarded([&] {
        Check c(comm);
        check_routes(c, tokens, top_k)
            .that(experts >= 1 && experts <= HCCL_MAX_EXPERTS, "experts must be 1 to 1024")
            .that(capacity <= kMaxCount, "capacity is more than 2^31 - 1 rows")
            .that(offsets != nullptr, "null array: offsets");
        if (!c.ok()) return c.result();
        size_t need = 0;
        const hcclResult_t r = hccl_moe_plan_bytes(tokens, top_k, experts, &need);
        if (r != hcclSuccess) return r;
        const int ranks = api_ranks(comm);
        c.list(index, tokens * top_k, 4, false, "index")
            .list(row, tokens * top_k, 4, true, "row")
            .list(offsets, experts + 1, 8, true, "offsets");
        if (rank_counts)
            c.that(experts % (uint32_t)ranks == 0, "rank counts need the experts divided evenly over the ranks")
                .list(rank_counts, (uint64_t)ranks, 8, true, "rank_counts");
        if (need) c.that(workspace != nullptr && workspace_bytes >= need, "workspace too small (hccl_moe_plan_bytes)").list(workspace, need / 4, 4, true, "workspace");
        if (!c.ok()) return c.result();
        PlanArgs a{};
        a.index = index;
        a.row = row;
        a.offsets = offsets;
        a.rank_counts = rank_counts;
        a.hist = need ? (uint32_t*)workspace : nullptr;
        a.routes = tokens * top_k;
        a.capacity = capacity;
        a.experts = experts;
        a.ranks = (uint32_t)ranks;
        plan_shape(a.routes, &a.blocks, &a.steps);
        return enqueue(c, [&] { return launch_plan(a, (hipStream_t)stream); });
    });
}

hcclResult_t hccl_moe_dispatch(hcclComm_t comm, const void* x, size_t ldx, hcclDataType_t dtype, size_t tokens,
                               size_t cols, const int32_t* row, uint32_t top_k, void* out, size_t ldo, size_t capacity,
                               float* scale, void* stream) {
    return guarded([&] {
        Check c(comm);
        c.that(is_float(dtype), "rows must be bf16, fp16 or fp32");
        const uint64_t es = float_size(dtype);
        check_routes(c, tokens, top_k)
            .that(capacity <= kMaxCount, "capacity is more than 2^31 - 1 rows")
            .that(cols <= kMaxCount, "more than 2^31 - 1 columns")
            .rows(x, tokens, cols, ldx, es, false, "x")
            .list(row, tokens * top_k, 4, false, "row")
            .rows(out, capacity, cols, ldo, scale ? 1 : es, true, "out");
        if (scale) c.list(scale, capacity, 4, true, "scale");
        if (!c.ok() || tokens == 0 || capacity == 0 || (cols == 0 && !scale)) return c.result();
        if (scale) {
            QuantizeArgs a{};
            a.x = x;
            a.row = row;
            a.codes = (int8_t*)out;
            a.scale = scale;
            a.rows = tokens;
            a.cols = cols;
            a.ldx = ldx;
            a.ldq = ldo;
            a.capacity = capacity;
            a.top_k = top_k;
            return enqueue(c, [&] { return launch_quantize(a, dtype, false, (hipStream_t)stream); });
        }
        DispatchArgs a{};
        a.x = x;
        a.row = row;
        a.out = out;
        a.tokens = tokens;
        a.cols = cols;
        a.ldx = ldx;
        a.ldo = ldo;
        a.capacity = capacity;
        a.top_k = top_k;
        return enqueue(c, [&] { return launch_dispatch(a, dtype, (hipStream_t)stream); });
    });
}

hcclResult_t hccl_moe_combine(hcclComm_t comm, const void* z, size_t ldz, hcclDataType_t dtype, size_t capacity,
                              const int32_t* row, uint32_t top_k, const float* weight, size_t tokens, size_t cols,
                              void* out, size_t ldo, void* stream) {
    return guarded([&] {
        Check c(comm);
        c.that(is_float(dtype), "rows must be bf16, fp16 or fp32");
        const uint64_t es = float_size(dtype);
        check_routes(c, tokens, top_k)
            .that(capacity <= kMaxCount, "capacity is more than 2^31 - 1 rows")
            .that(cols <= kMaxCount, "more than 2^31 - 1 columns")
            .rows(z, capacity, cols, ldz, es, false, "z")
            .list(row, tokens * top_k, 4, false, "row")
            .rows(out, tokens, cols, ldo, es, true, "out");
        if (weight) c.list(weight, tokens * top_k, 4, false, "weight");
        if (!c.ok() || tokens == 0 || cols == 0) return c.result();
        CombineArgs a{};
        a.z = z;
        a.row = row;
        a.weight = weight;
        a.out = out;
        a.tokens = tokens;
        a.cols = cols;
        a.ldz = ldz;
        a.ldo = ldo;
        a.capacity = capacity;
        a.top_k = top_k;
        return enqueue(c, [&] { return launch_combine(a, dtype, (hipStream_t)stream); });
    });
}

hcclResult_t hccl_moe_combine_backward(hcclComm_t comm, const void* grad, size_t ldg, hcclDataType_t dtype,
                                       size_t tokens, size_t cols, const void* z, size_t ldz, size_t capacity,
                                       const int32_t* row, uint32_t top_k, const float* weight, void* grad_z,
                                       size_t ldgz, float* grad_weight, void* stream) {
    return guarded([&] {
        Check c(comm);
        c.that(is_float(dtype), "rows must be bf16, fp16 or fp32");
        const uint64_t es = float_size(dtype);
        check_routes(c, tokens, top_k)
            .that(capacity <= kMaxCount, "capacity is more than 2^31 - 1 rows")
            .that(cols <= kMaxCount, "more than 2^31 - 1 columns")
            .rows(grad, tokens, cols, ldg, es, false, "grad")
            .list(row, tokens * top_k, 4, false, "row")
            .list(weight, tokens * top_k, 4, false, "weight");
        if (grad_weight) c.rows(z, capacity, cols, ldz, es, false, "z").list(grad_weight, tokens * top_k, 4, true, "grad_weight");
        if (grad_z) c.rows(grad_z, capacity, cols, ldgz, es, true, "grad_z");
        if (!c.ok() || tokens == 0 || (!grad_z && !grad_weight)) return c.result();
        CombineBackwardArgs a{};
        a.grad = grad;
        a.z = z;
        a.row = row;
        a.weight = weight;
        a.grad_z = grad_z;
        a.grad_weight = grad_weight;
        a.tokens = tokens;
        a.cols = cols;
        a.ldg = ldg;
        a.ldz = ldz;
        a.ldo = ldgz;
        a.capacity = capacity;
        a.top_k = top_k;
        return enqueue(c, [&] { return launch_combine_backward(a, dtype, (hipStream_t)stream); });
    });
}

hcclResult_t hccl_moe_quantize(hcclComm_t comm, const void* x, size_t ldx, hcclDataType_t dtype, size_t rows,
                               size_t cols, int gated, const int64_t* limit, int8_t* codes, size_t ldq, float* scale,
                               void* stream) {
    return guarded([&] {
        Check c(comm);
        c.that(is_float(dtype), "rows must be bf16, fp16 or fp32")
            .that(rows <= kMaxCount, "more than 2^31 - 1 rows")
            .that(cols <= kMaxCount, "more than 2^31 - 1 columns")
            .rows(x, rows, gated ? 2 * cols : cols, ldx, float_size(dtype), false, "x")
            .rows(codes, rows, cols, ldq, 1, true, "codes")
            .list(scale, rows, 4, true, "scale");
        if (limit) c.list(limit, 1, 8, false, "limit");
        if (!c.ok() || rows == 0) return c.result();
        QuantizeArgs a{};
        a.x = x;
        a.limit = limit;
        a.codes = codes;
        a.scale = scale;
        a.rows = rows;
        a.cols = cols;
        a.ldx = ldx;
        a.ldq = ldq;
        a.capacity = rows;
        a.top_k = 1;
        return enqueue(c, [&] { return launch_quantize(a, dtype, gated != 0, (hipStream_t)stream); });
    });
}

hcclResult_t hccl_moe_product(hcclComm_t comm, const int8_t* codes, size_t lda, const float* scale, size_t rows,
                              size_t inner, const int8_t* weights, size_t ldb, const float* weight_scale, size_t cols,
                              size_t experts, const int64_t* offsets, size_t segments, void* out, size_t ldo,
                              hcclDataType_t dtype, void* stream) {
    return guarded([&] {
        Check c(comm);
        c.that(is_float(dtype), "the result must be bf16, fp16 or fp32")
            .that(rows <= kMaxCount, "more than 2^31 - 1 rows")
            .that(cols <= kMaxCount, "more than 2^31 - 1 columns")
            .that(inner <= kMaxInner, "inner size above 131071: sums of products could wrap")
            .that(experts >= 1 && experts <= kMaxCount, "experts must be 1 or more")
            .that(offsets ? segments >= 1 && segments <= kMaxCount : true, "segments must be 1 or more")
            .that(offsets ? segments % (experts ? experts : 1) == 0 : experts == 1, offsets ? "segments must be a multiple of the experts" : "several experts need offsets");
        if (!c.ok()) return c.result();
        c.that(experts <= kMaxBytes / (cols ? cols : 1), "array too large: weights");
        if (!c.ok()) return c.result();
        c.rows(codes, rows, inner, lda, 1, false, "codes")
            .list(scale, rows, 4, false, "scale")
            .rows(weights, experts * cols, inner, ldb, 1, false, "weights")
            .list(weight_scale, experts * cols, 4, false, "weight_scale")
            .rows(out, rows, cols, ldo, float_size(dtype), true, "out");
        if (offsets) c.list(offsets, segments + 1, 8, false, "offsets");
        if (!c.ok() || rows == 0 || cols == 0) return c.result();
        ProductArgs a{};
        a.a = codes;
        a.a_scale = scale;
        a.b = weights;
        a.b_scale = weight_scale;
        a.offsets = offsets;
        a.out = out;
        a.rows = rows;
        a.lda = lda;
        a.ldb = ldb;
        a.ldo = ldo;
        a.inner = (uint32_t)inner;
        a.cols = (uint32_t)cols;
        a.segments = offsets ? (uint32_t)segments : 1u;
        a.experts = (uint32_t)experts;
        return enqueue(c, [&] { return launch_product(a, dtype, api_cus(comm), (hipStream_t)stream); });
    });
}

}  // extern "C"
