// Numbers of 8 bits (e4m3: largest 448, steps of an eighth of a power of two, NaN but no infinity) with a scale for each block
// of 128: rows, where 128 neighbours in a row share one, and weights, where 128 x 128 do, so that the transposed weights are
// the same numbers with the same scales.
//
// A block's scale is the smallest power of two, 2^-126 at least, by which its largest value is 448 at most; so dividing by it
// and multiplying by it again are exact, and a value is rounded once, to the nearest code, ties to even.  (The largest value
// over 448 itself would spare half a bit of the range at most, and would round three times.)  A block of zeros has scale 1.
// What is no finite number becomes NaN and has no part in its block's scale.
//
// Bound by memory: a value is read once and its codes are written once, 128 bytes of a block side by side.
#include <type_traits>

#include "sgap_tokens.hpp"

namespace sgap {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float magnitude(float x)
{
    const float m = __builtin_fabsf(x);
    return m < __builtin_inff() ? m : 0.0f;  // (NaN: 0)
}

struct Scale {
    float by, back;  // the scale, and one over it
};
// 448 is 1.75 * 2^8: the scale of m is 2^(e - 8) where m = f 2^e with f up to 1.75, else twice that
__device__ __forceinline__ Scale scale_of(float most)
{
    const uint32_t u = __float_as_uint(most);
    const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
    const int power = u == 0 ? 0 : max(e, -126);
    return {__uint_as_float((uint32_t)(power + 127) << 23), __uint_as_float((uint32_t)(127 - power) << 23)};
}

// four codes of four values
__device__ __forceinline__ uint32_t encode(const float* x, float back)
{
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __builtin_fabsf(x[i]) < __builtin_inff() ? x[i] * back : __builtin_nanf("");
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], r, true);
}

// N values of a row from column c on, zeros from column K on
template <typename T, int N>
__device__ __forceinline__ void load_values(const T* __restrict__ row, int64_t c, int64_t K, float (&x)[N])
{
    constexpr int P = Piece<T>::kCount;
    static_assert(N % P == 0, "");
    if (c + N <= K) {
#pragma unroll
        for (int h = 0; h < N / P; ++h) {
            const piece_t<T> v = load_piece(row + c + h * P);
#pragma unroll
            for (int i = 0; i < P; ++i) x[h * P + i] = (float)v[i];
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = c + i < K ? (float)row[c + i] : 0.0f;
}

// Sixteen lanes have a block of a row, eight values each.
template <typename T>
__global__ __launch_bounds__(kThreads) void f8_rows_kernel(F8RowsArgs a, int64_t blocks_k, int64_t block0)
{
    const int64_t block = (block0 + blockIdx.x) * (kThreads / 16) + (threadIdx.x >> 4);
    if (block >= a.R * blocks_k) return;
    const int64_t r = block / blocks_k, kb = block - r * blocks_k;
    const int part = threadIdx.x & 15;
    float x[8];
    load_values<T, 8>(static_cast<const T*>(a.X) + r * a.ldx, kb * kF8Block + part * 8, a.K, x);
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = fmaxf(most, magnitude(x[i]));
#pragma unroll
    for (int d = 8; d; d >>= 1) most = fmaxf(most, __shfl_xor(most, d));
    const Scale s = scale_of(most);
    *reinterpret_cast<uint2*>(a.codes + block * kF8Block + part * 8) = make_uint2(encode(x, s.back), encode(x + 4, s.back));
    if (part == 0) a.scales[block] = s.by;
}

// A workgroup has a block of 128 x 128 weights: sixteen lanes a row of them, sixteen rows at a time.
template <typename T, bool BOTH>
__global__ __launch_bounds__(kThreads) void f8_weights_kernel(F8WeightsArgs a, int64_t blocks_n, int64_t blocks_k, int64_t block0)
{
    constexpr int kTurns = kF8Block / (kThreads / 16), kPitch = kF8Block + 4;
    __shared__ float wave_most[kThreads / 64];
    __shared__ __align__(16) uint8_t tile[BOTH ? kF8Block * kPitch : 16];
    const int64_t block = block0 + blockIdx.x, per = blocks_n * blocks_k, g = block / per, in = block - g * per;
    const int64_t nb = in / blocks_k, kb = in - nb * blocks_k;
    const int part = threadIdx.x & 15, line = threadIdx.x >> 4;
    const int64_t k0 = kb * kF8Block, n0 = nb * kF8Block;
    float x[kTurns][8], most = 0.0f;
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
        const int64_t n = n0 + i * (kThreads / 16) + line;
        if (n < a.N) {
            load_values<T, 8>(static_cast<const T*>(a.W) + (g * a.N + n) * a.K, k0 + part * 8, a.K, x[i]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) x[i][j] = 0.0f;
        }
    }
#pragma unroll
    for (int i = 0; i < kTurns; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) most = fmaxf(most, magnitude(x[i][j]));
#pragma unroll
    for (int d = 32; d; d >>= 1) most = fmaxf(most, __shfl_xor(most, d));
    if ((threadIdx.x & 63) == 0) wave_most[threadIdx.x >> 6] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) most = fmaxf(most, wave_most[w]);
    const Scale s = scale_of(most);
    if (threadIdx.x == 0) {
        a.scales[block] = s.by;
        if (BOTH) a.scales_t[(g * blocks_k + kb) * blocks_n + nb] = s.by;
    }
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
        const int n = i * (kThreads / 16) + line;
        const uint32_t lo = encode(x[i], s.back), hi = encode(x[i] + 4, s.back);
        if (n0 + n < a.N) *reinterpret_cast<uint2*>(a.codes + ((g * a.N + n0 + n) * blocks_k + kb) * kF8Block + part * 8) = make_uint2(lo, hi);
        if constexpr (BOTH) {
            *reinterpret_cast<uint32_t*>(tile + n * kPitch + part * 8) = lo;
            *reinterpret_cast<uint32_t*>(tile + n * kPitch + part * 8 + 4) = hi;
        }
    }
    if constexpr (BOTH) {
        __syncthreads();
        // the same tile by columns: sixteen lanes a column, eight of its rows each
#pragma unroll
        for (int i = 0; i < kTurns; ++i) {
            const int k = i * (kThreads / 16) + line;
            uint32_t v[2] = {0, 0};
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j >> 2] |= (uint32_t)tile[(part * 8 + j) * kPitch + k] << (8 * (j & 3));
            if (k0 + k < a.K)
                *reinterpret_cast<uint2*>(a.codes_t + ((g * a.K + k0 + k) * blocks_n + nb) * kF8Block + part * 8) = make_uint2(v[0], v[1]);
        }
    }
}

template <typename T>
hipError_t f8_rows(const F8RowsArgs& a, hipStream_t s)
{
    const int64_t blocks_k = f8_blocks(a.K), blocks = a.R * blocks_k;
    return launch_parts((blocks + kThreads / 16 - 1) / (kThreads / 16), kThreads, [&](unsigned grid, int64_t block0) {
        f8_rows_kernel<T><<<grid, kThreads, 0, s>>>(a, blocks_k, block0);
    });
}

template <typename T>
hipError_t f8_weights(const F8WeightsArgs& a, hipStream_t s)
{
    const int64_t blocks_n = f8_blocks(a.N), blocks_k = f8_blocks(a.K);
    return launch_parts(a.G * blocks_n * blocks_k, kThreads, [&](unsigned grid, int64_t block0) {
        if (a.codes_t) f8_weights_kernel<T, true><<<grid, kThreads, 0, s>>>(a, blocks_n, blocks_k, block0);
        else f8_weights_kernel<T, false><<<grid, kThreads, 0, s>>>(a, blocks_n, blocks_k, block0);
    });
}

}  // namespace

hipError_t launch_f8_rows(const F8RowsArgs& a, hipStream_t s)
{
    switch (a.dtype) {
        case 0: return f8_rows<float>(a, s);
        case 1: return f8_rows<half_t>(a, s);
        default: return f8_rows<bf16_t>(a, s);
    }
}

hipError_t launch_f8_weights(const F8WeightsArgs& a, hipStream_t s)
{
    switch (a.dtype) {
        case 0: return f8_weights<float>(a, s);
        case 1: return f8_weights<half_t>(a, s);
        default: return f8_weights<bf16_t>(a, s);
    }
}

}  // namespace sgap
