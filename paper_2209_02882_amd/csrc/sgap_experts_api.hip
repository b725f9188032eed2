// Entry points of the router, the products grouped by expert and the way back: argument checks and launches.
#include <climits>

#include "../../include/sgap.h"
#include "../../include/sgap_debug.h"
#include "sgap_experts.hpp"

namespace sgap {
// sgap_api.hip
int fail_call(int status, const char* detail);  // what sgap_last_error() says
int device_compute_units();
}

namespace {

using sgap::fail_call;

constexpr int64_t kMaxIndex = 2147483646LL;  // row numbers and their ends are 32-bit
// rows, inner values and columns of a product: its kernels step past the end by up to three tiles
constexpr int64_t kMaxSteps = 2147483647LL - 65535;

int invalid(const char* what) { return fail_call(SGAP_ERR_INVALID_ARG, what); }

int launched(hipError_t err)
{
    return err == hipSuccess ? SGAP_OK : fail_call(SGAP_ERR_HIP, hipGetErrorString(err));
}

bool any_type(int dtype) { return dtype == SGAP_F32 || dtype == SGAP_F16 || dtype == SGAP_BF16; }

int check_route(int64_t T, int64_t E, int64_t k)
{
    if (T < 0) return invalid("negative number of tokens");
    if (E < 1 || E > SGAP_MAX_EXPERTS) return invalid("the number of experts must be 1 to 1,024");
    if (k < 1 || k > SGAP_MAX_CHOSEN || k > E) return invalid("k must be 1 to 16, and no more than the experts");
    if (T > kMaxIndex / k) return invalid("dimension exceeds int32 index range");
    return SGAP_OK;
}

// the parts that both products share
int check_grouped(int64_t G, int64_t R, int64_t K, int64_t N, const int32_t* offsets, const void* X, int64_t ldx,
                  const int32_t* src, int64_t src_div, int64_t x_rows, const void* W, const void* Y, int64_t ldy)
{
    if (G < 1) return invalid("there must be at least one group");
    if (R < 0 || K < 0 || N < 0 || x_rows < 0) return invalid("negative dimension");
    if (G > (1 << 20)) return invalid("more than 1,048,576 groups");
    if (R > kMaxSteps || K > kMaxSteps || N > kMaxSteps || x_rows > kMaxIndex)
        return invalid("dimension exceeds int32 index range: R, K and N are at most 2^31 - 65536");
    if (!offsets && G != 1) return invalid("offsets may be null for one group only");
    if (src_div < 1 || src_div > kMaxIndex) return invalid("src_div must be positive");
    if (!src && src_div != 1 && R > 0) return invalid("src_div needs src");
    if (!src && x_rows < R) return invalid("X has fewer rows than the product");
    if (ldx < K) return invalid("ldx is less than a row");
    if (ldy < N) return invalid("ldy is less than a row");
    if (R > 0 && N > 0 && !Y) return invalid("Y must not be null");
    if (K > 0 && N > 0 && !W) return invalid("the weights must not be null");
    if (R > 0 && K > 0 && x_rows > 0 && !X) return invalid("X must not be null");
    return SGAP_OK;
}

}  // namespace

extern "C" {

int64_t sgap_route_topk_workspace_size(int64_t T, int64_t E, int64_t k)
{
    if (check_route(T, E, k) != SGAP_OK) return -1;
    return sgap::route_workspace_bytes(T, E);
}

int sgap_route_topk(int64_t T, int64_t E, int64_t k, int dtype, const void* logits, int64_t ld_logits, int renormalise,
                    float* gates, int32_t* experts, int32_t* slot, int32_t* order, int32_t* offsets, void* workspace,
                    int64_t workspace_bytes, void* stream)
{
    if (const int st = check_route(T, E, k)) return st;
    if (!any_type(dtype)) return invalid("unknown element type");
    if (renormalise != 0 && renormalise != 1) return invalid("renormalise must be 0 or 1");
    if (ld_logits < E) return invalid("ld_logits is less than a row");
    if (!offsets) return invalid("offsets must not be null");
    if (T > 0 && (!logits || !gates || !experts || !slot || !order)) return invalid("logits and the results must not be null");
    const int64_t need = sgap::route_workspace_bytes(T, E);
    if (need > 0 && (!workspace || workspace_bytes < need))
        return invalid("the workspace is smaller than sgap_route_topk_workspace_size says");
    if (need > 0 && (reinterpret_cast<uintptr_t>(workspace) & 15)) return invalid("the workspace must be 16-byte aligned");
    const sgap::RouteArgs a{T, (int)E, (int)k, dtype, renormalise != 0, logits, ld_logits, gates, experts, slot, order, offsets, workspace};
    return launched(sgap::launch_route(a, static_cast<hipStream_t>(stream)));
}

int sgap_route_topk_grad(int64_t T, int64_t E, int64_t k, int dtype, const void* logits, int64_t ld_logits, int renormalise,
                         const float* gates, const int32_t* experts, const float* dgates, void* dlogits, int64_t ld_dlogits,
                         void* stream)
{
    if (const int st = check_route(T, E, k)) return st;
    if (!any_type(dtype)) return invalid("unknown element type");
    if (renormalise != 0 && renormalise != 1) return invalid("renormalise must be 0 or 1");
    if (ld_logits < E || ld_dlogits < E) return invalid("ld_logits or ld_dlogits is less than a row");
    if (T == 0) return SGAP_OK;
    if (!logits || !gates || !experts || !dgates || !dlogits) return invalid("the arrays must not be null");
    const sgap::RouteGradArgs a{T, (int)E, (int)k, dtype, renormalise != 0, logits, ld_logits, gates, experts, dgates, dlogits, ld_dlogits};
    return launched(sgap::launch_route_grad(a, static_cast<hipStream_t>(stream)));
}

static int check_combine(int64_t T, int64_t k, int64_t D, int dtype)
{
    if (T < 0 || D < 0) return invalid("negative dimension");
    if (k < 1 || k > SGAP_MAX_CHOSEN) return invalid("k must be 1 to 16");
    if (T > kMaxIndex / k || D > kMaxIndex) return invalid("dimension exceeds int32 index range");
    if (!any_type(dtype)) return invalid("unknown element type");
    return SGAP_OK;
}

int sgap_route_combine(int64_t T, int64_t k, int64_t D, int dtype, const void* Z, const int32_t* slot, const float* gates,
                       void* out, void* stream)
{
    if (const int st = check_combine(T, k, D, dtype)) return st;
    if (T == 0 || D == 0) return SGAP_OK;
    if (!Z || !slot || !out) return invalid("Z, slot and out must not be null");
    const sgap::CombineArgs a{T, D, (int)k, dtype, Z, slot, nullptr, gates, nullptr, out, nullptr};
    return launched(sgap::launch_combine(a, static_cast<hipStream_t>(stream)));
}

int sgap_route_combine_grad(int64_t T, int64_t k, int64_t D, int dtype, const void* Z, const int32_t* slot,
                            const int32_t* order, const float* gates, const void* dout, void* dZ, float* dgates, void* stream)
{
    if (const int st = check_combine(T, k, D, dtype)) return st;
    if (T == 0) return SGAP_OK;
    if (!slot || !order || !gates || !dgates) return invalid("slot, order, gates and dgates must not be null");
    if (D > 0 && (!Z || !dout || !dZ)) return invalid("Z, dout and dZ must not be null");
    const sgap::CombineArgs a{T, D, (int)k, dtype, Z, slot, order, gates, dout, dZ, dgates};
    return launched(sgap::launch_combine_grad(a, static_cast<hipStream_t>(stream)));
}

int sgap_grouped_mm(int64_t G, int64_t R, int64_t K, int64_t N, int dtype, const int32_t* offsets, const void* X, int64_t ldx,
                    int64_t x_rows, const int32_t* src, int64_t src_div, const void* W, int layout, void* Y, int64_t ldy, void* stream)
{
    if (!any_type(dtype)) return invalid("unknown element type");
    if (layout != SGAP_WEIGHTS_NK && layout != SGAP_WEIGHTS_KN) return invalid("unknown layout of the weights");
    if (const int st = check_grouped(G, R, K, N, offsets, X, ldx, src, src_div, x_rows, W, Y, ldy)) return st;
    if (R == 0 || N == 0) return SGAP_OK;
    const sgap::GroupedArgs a{G, R, K, N, offsets, {src, src_div, x_rows}, X, ldx, W, Y, ldy, layout == SGAP_WEIGHTS_KN,
                              sgap::device_compute_units()};
    return launched(sgap::launch_grouped_mm(a, dtype, static_cast<hipStream_t>(stream)));
}

int sgap_grouped_mm_wgrad(int64_t G, int64_t R, int64_t K, int64_t N, int dtype, const int32_t* offsets, const void* X,
                          int64_t ldx, int64_t x_rows, const int32_t* src, int64_t src_div, const void* dY, int64_t lddy, void* dW, int layout,
                          void* stream)
{
    if (!any_type(dtype)) return invalid("unknown element type");
    if (layout != SGAP_WEIGHTS_NK && layout != SGAP_WEIGHTS_KN) return invalid("unknown layout of the weights");
    if (const int st = check_grouped(G, R, K, N, offsets, X, ldx, src, src_div, x_rows, dW, dY, lddy)) return st;
    if (K == 0 || N == 0) return SGAP_OK;
    const sgap::GroupedArgs a{G, R, K, N, offsets, {src, src_div, x_rows}, X, ldx, dW, const_cast<void*>(dY), lddy,
                              layout == SGAP_WEIGHTS_KN, sgap::device_compute_units()};
    return launched(sgap::launch_grouped_wgrad(a, dtype, static_cast<hipStream_t>(stream)));
}

int sgap_debug_grouped_plan(int64_t G, int64_t R, int64_t K, int64_t N, int dtype, int given_offsets, int64_t ldx, int64_t x_rows,
                            int64_t ldy, int layout, int gradient, int aligned, int compute_units, int* plan)
{
    if (!any_type(dtype) || G < 1 || R < 0 || K < 0 || N < 0 || x_rows < 0 || R > kMaxSteps || K > kMaxSteps || N > kMaxSteps ||
        x_rows > kMaxIndex || ldx < K || ldy < N || (layout != SGAP_WEIGHTS_NK && layout != SGAP_WEIGHTS_KN) || compute_units < 1 || !plan)
        return invalid("bad arguments");
    // only the addresses' alignment and whether there are offsets are looked at
    void* const at = reinterpret_cast<void*>(aligned ? 0x1000 : 0x1004);
    const int32_t* const offsets = given_offsets ? static_cast<const int32_t*>(at) : nullptr;
    const sgap::GroupedArgs a{G, R, K, N, offsets, {nullptr, 1, x_rows}, at, ldx, at, at, ldy, layout == SGAP_WEIGHTS_KN, compute_units};
    const sgap::GroupedPlan p = sgap::plan_grouped(a, dtype, gradient != 0);
    plan[0] = (int)p.way;
    plan[1] = p.rows;
    plan[2] = p.columns;
    plan[3] = p.wide ? 1 : 0;
    plan[4] = p.apart ? 1 : 0;
    plan[5] = p.short_rows ? 1 : 0;
    return SGAP_OK;
}

static int check_w4(int64_t G, int64_t K, int64_t N, int64_t group_k)
{
    if (G < 1 || K < 0 || N < 0) return invalid("negative dimension, or no group");
    if (G > (1 << 20)) return invalid("more than 1,048,576 groups");
    if (K > kMaxSteps || N > kMaxSteps) return invalid("dimension exceeds int32 index range: K and N are at most 2^31 - 65536");
    if (group_k != 32 && group_k != 64 && (group_k < 128 || group_k % 128)) return invalid("group_k must be 32, 64 or a multiple of 128");
    if (group_k > kMaxIndex || K % group_k) return invalid("K must be a multiple of group_k");
    // a tile of 16 columns by 128 values is 2 KB at most with its scales and zero points: their sizes and places stay in 64 bits
    if (G * ((N + 15) / 16) > INT64_MAX / 2048 / ((K + 127) / 128 + 1)) return invalid("the laid-out weights are larger than any memory");
    return SGAP_OK;
}

int64_t sgap_w4_layout_size(int64_t G, int64_t K, int64_t N, int64_t group_k, int zeros)
{
    if (zeros != 0 && zeros != 1) {
        invalid("zeros must be 0 or 1");
        return -1;
    }
    if (check_w4(G, K, N, group_k) != SGAP_OK) return -1;
    return sgap::w4_sizes(G, K, N, (int)group_k, zeros != 0).bytes;
}

int sgap_w4_layout(int64_t G, int64_t K, int64_t N, int64_t group_k, const uint8_t* codes, const void* scales,
                   const uint8_t* zeros, void* weights, int64_t weights_bytes, void* stream)
{
    if (const int st = check_w4(G, K, N, group_k)) return st;
    const int64_t need = sgap::w4_sizes(G, K, N, (int)group_k, zeros != nullptr).bytes;
    if (weights_bytes < need) return invalid("weights is smaller than sgap_w4_layout_size says");
    if (need == 0) return SGAP_OK;
    if (!codes || !scales || !weights) return invalid("codes, scales and weights must not be null");
    if (reinterpret_cast<uintptr_t>(weights) & 15) return invalid("weights must be 16-byte aligned");
    return launched(sgap::launch_w4_layout(G, K, N, (int)group_k, codes, scales, zeros, static_cast<uint8_t*>(weights),
                                           static_cast<hipStream_t>(stream)));
}

int sgap_grouped_mm_w4(int64_t G, int64_t R, int64_t K, int64_t N, int dtype, int64_t group_k, int zeros, const int32_t* offsets,
                       const void* X, int64_t ldx, int64_t x_rows, const int32_t* src, int64_t src_div, const void* weights,
                       int64_t weights_bytes, void* Y, int64_t ldy, void* stream)
{
    if (dtype != SGAP_F16 && dtype != SGAP_BF16) return invalid("the element type must be a 16-bit one");
    if (zeros != 0 && zeros != 1) return invalid("zeros must be 0 or 1");
    if (const int st = check_w4(G, K, N, group_k)) return st;
    if (const int st = check_grouped(G, R, K, N, offsets, X, ldx, src, src_div, x_rows, weights, Y, ldy)) return st;
    if (weights_bytes < sgap::w4_sizes(G, K, N, (int)group_k, zeros != 0).bytes)
        return invalid("weights is smaller than sgap_w4_layout_size says");
    if (reinterpret_cast<uintptr_t>(weights) & 15) return invalid("weights must be 16-byte aligned");
    if (R == 0 || N == 0) return SGAP_OK;
    const sgap::GroupedW4Args a{G, R, K, N, offsets, {src, src_div, x_rows}, X, ldx, static_cast<const uint8_t*>(weights),
                                (int)group_k, zeros != 0, Y, ldy};
    return launched(sgap::launch_grouped_w4(a, dtype, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
