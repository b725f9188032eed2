// What stands around the products of a mixture of experts that is trained on tokens: embeddings, the balance loss, numbers
// of 8 bits.  Arguments and the host-side launch entry points.
#pragma once
#include "sgap_experts.hpp"

namespace sgap {

struct EmbedArgs {
    int64_t T, V, D;
    int dtype;
    const int32_t* __restrict__ ids;
    const void* __restrict__ weights;
    int64_t ldw;
    void* __restrict__ out;
    int64_t ldo;
    float scale;
};

struct EmbedGradArgs {
    int64_t T, V, D;
    int dtype, grad_dtype;
    const int32_t* __restrict__ ids;
    const void* __restrict__ dout;
    int64_t ldd;
    float scale;
    bool accumulate;
    void* __restrict__ dweights;
    int64_t ldw;
    char* workspace;
};

struct BalanceArgs {
    int64_t T, S;
    int E, k, dtype;
    const void* __restrict__ logits;
    int64_t ld;
    const int32_t* __restrict__ experts;
    const int32_t* __restrict__ segments;
    float* __restrict__ loss;
    int32_t *__restrict__ counts, *__restrict__ rows;
    char* workspace;
};

struct BalanceGradArgs {
    int64_t T, S;
    int E, k, dtype;
    const void* __restrict__ logits;
    int64_t ld;
    const int32_t* __restrict__ experts;
    const int32_t* __restrict__ segments;
    const int32_t *__restrict__ counts, *__restrict__ rows;
    const float* __restrict__ dloss;
    bool accumulate;
    void* __restrict__ dlogits;
    int64_t ldd;
};

// values that share a scale, along a row (and for weights, rows as well)
constexpr int kF8Block = 128;
inline __host__ __device__ int64_t f8_blocks(int64_t n) { return (n + kF8Block - 1) / kF8Block; }

struct F8RowsArgs {
    int64_t R, K;
    int dtype;
    const void* __restrict__ X;
    int64_t ldx;
    uint8_t* __restrict__ codes;
    float* __restrict__ scales;
};

struct F8WeightsArgs {
    int64_t G, K, N;
    int dtype;
    const void* __restrict__ W;
    uint8_t* __restrict__ codes;
    float* __restrict__ scales;
    uint8_t* __restrict__ codes_t;  // null: not wanted
    float* __restrict__ scales_t;
};

struct GroupedF8Args {
    int64_t G, R, K, N;
    const int32_t* __restrict__ offsets;
    RowSource from;
    const uint8_t* __restrict__ X;
    const float* __restrict__ x_scales;
    const uint8_t* __restrict__ W;
    const float* __restrict__ w_scales;
    void* __restrict__ Y;
    int64_t ldy;
    int compute_units;
};

int64_t embed_grad_workspace_bytes(int64_t T, int64_t V, int64_t D);
hipError_t launch_embed(const EmbedArgs& a, hipStream_t s);
hipError_t launch_embed_grad(const EmbedGradArgs& a, hipStream_t s);
int64_t balance_workspace_bytes(int64_t T, int64_t E, int64_t S);
hipError_t launch_balance(const BalanceArgs& a, hipStream_t s);
hipError_t launch_balance_grad(const BalanceGradArgs& a, hipStream_t s);
hipError_t launch_f8_rows(const F8RowsArgs& a, hipStream_t s);
hipError_t launch_f8_weights(const F8WeightsArgs& a, hipStream_t s);
// Which kernel a product takes.
struct GroupedF8Plan {
    int teams;          // that make tiles and share the inner dimension; 0: few rows, whose workgroups' wavefronts share it
    int rows, columns;  // of a workgroup's part of the result
    bool far;           // tiles: rows are gathered from more than 4 GiB
    bool deep;          // few rows: more blocks on their way
};
GroupedF8Plan plan_grouped_f8(const GroupedF8Args& a, int dtype);
hipError_t launch_grouped_f8(GroupedF8Args a, int dtype, hipStream_t s);

}  // namespace sgap
