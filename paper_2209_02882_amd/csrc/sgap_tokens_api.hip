// Entry points of the balance loss, embeddings, numbers of 8 bits and products in them: argument checks and launches.
#include <climits>
#include <cmath>

#include "../../include/sgap.h"
#include "../../include/sgap_debug.h"
#include "sgap_tokens.hpp"

namespace sgap {
// sgap_api.hip
int fail_call(int status, const char* detail);  // what sgap_last_error() says
int device_compute_units();
}

namespace {

using sgap::f8_blocks;
using sgap::fail_call;

constexpr int64_t kMaxIndex = 2147483646LL;  // row numbers and their ends are 32-bit
constexpr int64_t kMaxSteps = 2147483647LL - 65535;

int invalid(const char* what) { return fail_call(SGAP_ERR_INVALID_ARG, what); }

int launched(hipError_t err)
{
    return err == hipSuccess ? SGAP_OK : fail_call(SGAP_ERR_HIP, hipGetErrorString(err));
}

bool any_type(int dtype) { return dtype == SGAP_F32 || dtype == SGAP_F16 || dtype == SGAP_BF16; }

bool loose(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }

int check_balance(int64_t T, int64_t E, int64_t k, int64_t S)
{
    if (T < 0) return invalid("negative number of tokens");
    if (E < 1 || E > SGAP_MAX_EXPERTS) return invalid("the number of experts must be 1 to 1,024");
    if (k < 1 || k > SGAP_MAX_CHOSEN || k > E) return invalid("k must be 1 to 16, and no more than the experts");
    if (T > kMaxIndex / k) return invalid("dimension exceeds int32 index range");
    if (S < 1 || S > SGAP_MAX_SEQUENCES) return invalid("the number of sequences must be 1 to 65,536");
    return SGAP_OK;
}

int check_embed(int64_t T, int64_t V, int64_t D)
{
    if (T < 0 || D < 0) return invalid("negative dimension");
    if (V < 1) return invalid("the table must have a row");
    if (T > kMaxSteps || V > kMaxSteps || D > kMaxSteps) return invalid("dimension exceeds int32 index range: T, V and D are at most 2^31 - 65536");
    return SGAP_OK;
}

}  // namespace

extern "C" {

int64_t sgap_route_balance_workspace_size(int64_t T, int64_t E, int64_t k, int64_t S)
{
    if (check_balance(T, E, k, S) != SGAP_OK) return -1;
    return sgap::balance_workspace_bytes(T, E, S);
}

int sgap_route_balance(int64_t T, int64_t E, int64_t k, int64_t S, int dtype, const void* logits, int64_t ld_logits,
                       const int32_t* experts, const int32_t* segments, float* loss, int32_t* counts, int32_t* rows,
                       void* workspace, int64_t workspace_bytes, void* stream)
{
    if (const int st = check_balance(T, E, k, S)) return st;
    if (!any_type(dtype)) return invalid("unknown element type");
    if (ld_logits < E) return invalid("ld_logits is less than a row");
    if (!segments && S != 1) return invalid("segments may be null for one sequence only");
    if (!loss || !counts || !rows) return invalid("loss, counts and rows must not be null");
    if (T > 0 && (!logits || !experts)) return invalid("logits and experts must not be null");
    if (!workspace || workspace_bytes < sgap::balance_workspace_bytes(T, E, S))
        return invalid("the workspace is smaller than sgap_route_balance_workspace_size says");
    if (loose(workspace)) return invalid("the workspace must be 16-byte aligned");
    const sgap::BalanceArgs a{T, S, (int)E, (int)k, dtype, logits, ld_logits, experts, segments, loss, counts, rows,
                              static_cast<char*>(workspace)};
    return launched(sgap::launch_balance(a, static_cast<hipStream_t>(stream)));
}

int sgap_route_balance_grad(int64_t T, int64_t E, int64_t k, int64_t S, int dtype, const void* logits, int64_t ld_logits,
                            const int32_t* experts, const int32_t* segments, const int32_t* counts, const int32_t* rows,
                            const float* dloss, int accumulate, void* dlogits, int64_t ld_dlogits, void* stream)
{
    if (const int st = check_balance(T, E, k, S)) return st;
    if (!any_type(dtype)) return invalid("unknown element type");
    if (accumulate != 0 && accumulate != 1) return invalid("accumulate must be 0 or 1");
    if (ld_logits < E || ld_dlogits < E) return invalid("ld_logits or ld_dlogits is less than a row");
    if (!segments && S != 1) return invalid("segments may be null for one sequence only");
    if (T == 0) return SGAP_OK;
    if (!logits || !experts || !counts || !rows || !dloss || !dlogits) return invalid("the arrays must not be null");
    const sgap::BalanceGradArgs a{T, S, (int)E, (int)k, dtype, logits, ld_logits, experts, segments, counts, rows, dloss, accumulate != 0,
                                  dlogits, ld_dlogits};
    return launched(sgap::launch_balance_grad(a, static_cast<hipStream_t>(stream)));
}

int sgap_embed(int64_t T, int64_t V, int64_t D, int dtype, const int32_t* ids, const void* weights, int64_t ld_weights,
               float scale, void* out, int64_t ld_out, void* stream)
{
    if (const int st = check_embed(T, V, D)) return st;
    if (!any_type(dtype)) return invalid("unknown element type");
    if (ld_weights < D || ld_out < D) return invalid("ld_weights or ld_out is less than a row");
    if (!std::isfinite(scale)) return invalid("the scale must be finite");
    if (T == 0 || D == 0) return SGAP_OK;
    if (!ids || !weights || !out) return invalid("ids, weights and out must not be null");
    const sgap::EmbedArgs a{T, V, D, dtype, ids, weights, ld_weights, out, ld_out, scale};
    return launched(sgap::launch_embed(a, static_cast<hipStream_t>(stream)));
}

int64_t sgap_embed_grad_workspace_size(int64_t T, int64_t V, int64_t D)
{
    if (check_embed(T, V, D) != SGAP_OK) return -1;
    return sgap::embed_grad_workspace_bytes(T, V, D);
}

int sgap_embed_grad(int64_t T, int64_t V, int64_t D, int dtype, const int32_t* ids, const void* dout, int64_t ld_dout,
                    float scale, int accumulate, int grad_dtype, void* dweights, int64_t ld_dweights, void* workspace,
                    int64_t workspace_bytes, void* stream)
{
    if (const int st = check_embed(T, V, D)) return st;
    if (!any_type(dtype)) return invalid("unknown element type");
    if (grad_dtype != dtype && grad_dtype != SGAP_F32) return invalid("the gradient's type must be dout's or float");
    if (accumulate != 0 && accumulate != 1) return invalid("accumulate must be 0 or 1");
    if (ld_dout < D || ld_dweights < D) return invalid("ld_dout or ld_dweights is less than a row");
    if (!std::isfinite(scale)) return invalid("the scale must be finite");
    if (D == 0 || (T == 0 && accumulate)) return SGAP_OK;
    if ((T > 0 && (!ids || !dout)) || !dweights) return invalid("ids, dout and dweights must not be null");
    if (!workspace || workspace_bytes < sgap::embed_grad_workspace_bytes(T, V, D))
        return invalid("the workspace is smaller than sgap_embed_grad_workspace_size says");
    if (loose(workspace)) return invalid("the workspace must be 16-byte aligned");
    const sgap::EmbedGradArgs a{T, V, D, dtype, grad_dtype, ids, dout, ld_dout, scale, accumulate != 0, dweights, ld_dweights,
                                static_cast<char*>(workspace)};
    return launched(sgap::launch_embed_grad(a, static_cast<hipStream_t>(stream)));
}

int sgap_f8_rows(int64_t R, int64_t K, int dtype, const void* X, int64_t ldx, uint8_t* codes, float* scales, void* stream)
{
    if (R < 0 || K < 0) return invalid("negative dimension");
    if (R > kMaxIndex || K > kMaxSteps) return invalid("dimension exceeds int32 index range");
    if (!any_type(dtype)) return invalid("unknown element type");
    if (ldx < K) return invalid("ldx is less than a row");
    if (R == 0 || K == 0) return SGAP_OK;
    if (!X || !codes || !scales) return invalid("X, codes and scales must not be null");
    if (loose(codes)) return invalid("codes must be 16-byte aligned");
    const sgap::F8RowsArgs a{R, K, dtype, X, ldx, codes, scales};
    return launched(sgap::launch_f8_rows(a, static_cast<hipStream_t>(stream)));
}

static int check_f8_weights(int64_t G, int64_t K, int64_t N)
{
    if (G < 1 || K < 0 || N < 0) return invalid("negative dimension, or no group");
    if (G > (1 << 20)) return invalid("more than 1,048,576 groups");
    if (K > kMaxSteps || N > kMaxSteps) return invalid("dimension exceeds int32 index range: K and N are at most 2^31 - 65536");
    // a block of codes is 16 KB: sizes and places stay in 64 bits
    if (f8_blocks(K) > 0 && G * (f8_blocks(N) + 1) > INT64_MAX / 16384 / f8_blocks(K)) return invalid("the weights are larger than any memory");
    return SGAP_OK;
}

int sgap_f8_weights(int64_t G, int64_t K, int64_t N, int dtype, const void* W, uint8_t* codes, float* scales, uint8_t* codes_t,
                    float* scales_t, void* stream)
{
    if (const int st = check_f8_weights(G, K, N)) return st;
    if (!any_type(dtype)) return invalid("unknown element type");
    if (!codes_t != !scales_t) return invalid("codes_t and scales_t go together");
    if (K == 0 || N == 0) return SGAP_OK;
    if (!W || !codes || !scales) return invalid("W, codes and scales must not be null");
    if (loose(codes) || loose(codes_t)) return invalid("codes must be 16-byte aligned");
    const sgap::F8WeightsArgs a{G, K, N, dtype, W, codes, scales, codes_t, scales_t};
    return launched(sgap::launch_f8_weights(a, static_cast<hipStream_t>(stream)));
}

int sgap_grouped_mm_f8(int64_t G, int64_t R, int64_t K, int64_t N, int dtype, const int32_t* offsets, const uint8_t* X,
                       const float* x_scales, int64_t x_rows, const int32_t* src, int64_t src_div, const uint8_t* W,
                       const float* w_scales, void* Y, int64_t ldy, void* stream)
{
    if (const int st = check_f8_weights(G, K, N)) return st;
    if (!any_type(dtype)) return invalid("unknown element type");
    if (R < 0 || x_rows < 0) return invalid("negative dimension");
    if (R > kMaxSteps || x_rows > kMaxIndex) return invalid("dimension exceeds int32 index range: R is at most 2^31 - 65536");
    if (!offsets && G != 1) return invalid("offsets may be null for one group only");
    if (src_div < 1 || src_div > kMaxIndex) return invalid("src_div must be positive");
    if (!src && src_div != 1 && R > 0) return invalid("src_div needs src");
    if (!src && x_rows < R) return invalid("X has fewer rows than the product");
    if (ldy < N) return invalid("ldy is less than a row");
    if (R == 0 || N == 0) return SGAP_OK;
    if (!Y) return invalid("Y must not be null");
    if (K > 0 && (!W || !w_scales)) return invalid("the weights and their scales must not be null");
    if (K > 0 && x_rows > 0 && (!X || !x_scales)) return invalid("X and its scales must not be null");
    if (loose(X) || loose(W)) return invalid("codes must be 16-byte aligned");
    const sgap::GroupedF8Args a{G, R, K, N, offsets, {src, src_div, x_rows}, X, x_scales, W, w_scales, Y, ldy, sgap::device_compute_units()};
    return launched(sgap::launch_grouped_f8(a, dtype, static_cast<hipStream_t>(stream)));
}

int sgap_debug_f8_plan(int64_t G, int64_t R, int64_t K, int64_t N, int dtype, int given_offsets, int given_src, int64_t x_rows,
                       int compute_units, int* plan)
{
    if (check_f8_weights(G, K, N) != SGAP_OK || !any_type(dtype) || R < 0 || R > kMaxSteps || x_rows < 0 || compute_units < 1 || !plan)
        return invalid("bad arguments");
    // only whether there are lists is looked at
    const int32_t* const list = reinterpret_cast<const int32_t*>(0x1000);
    const sgap::GroupedF8Args a{G, R, K, N, given_offsets ? list : nullptr, {given_src ? list : nullptr, 1, x_rows}, nullptr, nullptr,
                                nullptr, nullptr, nullptr, N, compute_units};
    const sgap::GroupedF8Plan p = sgap::plan_grouped_f8(a, dtype);
    plan[0] = p.teams;
    plan[1] = p.rows;
    plan[2] = p.columns;
    plan[3] = p.teams == 0 ? (p.deep ? 2 : 0) : p.far ? 1 : 0;
    return SGAP_OK;
}

}  // extern "C"
