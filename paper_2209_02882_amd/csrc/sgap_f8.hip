// Numbers of 8 bits (e4m3: largest 448, steps of an eighth of a power of two, NaN but no infinity) with a scale for each block
// of 128: rows, where 128 neighbours in a row share one, and weights, where 128 x 128 do, so that the transposed weights are
// the same numbers with the same scales.
//
// A block's scale is the smallest power of two, 2^-126 at least, by which its largest value is 448 at most; so dividing by it
// and multiplying by it again are exact, and a value is rounded once, to the nearest code, ties to even.  (The largest value
// over 448 itself would spare half a bit of the range at most, and would round three times.)  A block of zeros has scale 1.
// What is no finite number becomes NaN and has no part in its block's scale.
//
// Bound by memory: a value is read once and its codes are written once, 128 bytes of a block side by side.  16,384 rows of 4,096,
// bf16: 39.0 us, 5.2 TB/s; weights of 16 x 4,096 x 2,048, bf16: 69 us, 5.9 TB/s, transposed too 93 us, 5.8 TB/s (a copy reaches 5.5).  A thread's loads are all on their way together: where a row's length makes each a branch of its own, the weights took 118 us.
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

// Eight values of a row from column c on as they lie in memory, and as numbers, zeros from column K on.  EIGHTS: K is a multiple of
// eight, so that there are all of them or none, and the loads go without a branch, all of a thread's together.
template <typename T, bool EIGHTS>
struct Eight {
    static constexpr int P = Piece<T>::kCount;
    piece_t<T> v[8 / P];
    template <bool PAST = false>
    __device__ __forceinline__ void load(const T* __restrict__ row, int64_t c, int64_t K)
    {
        if (EIGHTS || c + 8 <= K) {
            const T* const from = row + (!EIGHTS || c < K ? c : 0);
#pragma unroll
            for (int h = 0; h < 8 / P; ++h) {
                if constexpr (PAST) v[h] = __builtin_nontemporal_load(reinterpret_cast<const typename Piece<T>::loose*>(from + h * P));
                else v[h] = load_piece(from + h * P);
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i / P][i % P] = c + i < K ? row[c + i] : (T)0.0f;
    }
    __device__ __forceinline__ void numbers(float (&x)[8], bool there) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = there ? (float)v[i / P][i % P] : 0.0f;
    }
};

// Sixteen lanes have a block of a row, eight values each; TURNS blocks, all of them on their way together.
template <typename T, int TURNS, bool EIGHTS>
__global__ __launch_bounds__(kThreads) void f8_rows_kernel(F8RowsArgs a, int64_t blocks_k, int64_t block0)
{
    constexpr int kGroups = kThreads / 16;
    const int64_t first = (block0 + blockIdx.x) * (kGroups * TURNS) + (threadIdx.x >> 4), blocks = a.R * blocks_k;
    const int part = threadIdx.x & 15;
    Eight<T, EIGHTS> held[TURNS];
    int64_t c[TURNS];
#pragma unroll
    for (int u = 0; u < TURNS; ++u) {
        const int64_t block = min(first + u * kGroups, blocks - 1), r = block / blocks_k;
        c[u] = (block - r * blocks_k) * kF8Block + part * 8;
        held[u].load(static_cast<const T*>(a.X) + r * a.ldx, c[u], a.K);
    }
#pragma unroll
    for (int u = 0; u < TURNS; ++u) {
        const int64_t block = first + u * kGroups;
        float x[8], most = 0.0f;
        held[u].numbers(x, !EIGHTS || c[u] < a.K);
#pragma unroll
        for (int i = 0; i < 8; ++i) most = fmaxf(most, magnitude(x[i]));
#pragma unroll
        for (int d = 8; d; d >>= 1) most = fmaxf(most, __shfl_xor(most, d));
        if (block >= blocks) break;
        const Scale s = scale_of(most);
        *reinterpret_cast<uint2*>(a.codes + block * kF8Block + part * 8) = make_uint2(encode(x, s.back), encode(x + 4, s.back));
        if (part == 0) a.scales[block] = s.by;
    }
}

template <bool PAST>
__device__ __forceinline__ void store_codes(uint8_t* to, uint32_t lo, uint32_t hi)
{
    const uint64_t both = (uint64_t)hi << 32 | lo;
    if constexpr (PAST) __builtin_nontemporal_store(both, reinterpret_cast<uint64_t*>(to));
    else *reinterpret_cast<uint64_t*>(to) = both;
}

// A workgroup has a block of 128 x 128 weights: sixteen lanes a row of them, sixteen rows at a time.  PAST: past the caches.
template <typename T, bool BOTH, bool EIGHTS, bool PAST>
__global__ __launch_bounds__(kThreads) void f8_weights_kernel(F8WeightsArgs a, int64_t blocks_n, int64_t blocks_k, int64_t block0)
{
    constexpr int kTurns = kF8Block / (kThreads / 16), kPitch = kF8Block + 4;
    __shared__ float wave_most[kThreads / 64];
    __shared__ __align__(16) uint8_t tile[BOTH ? kF8Block * kPitch : 16];
    const int64_t block = block0 + blockIdx.x, per = blocks_n * blocks_k, g = block / per, in = block - g * per;
    const int64_t nb = in / blocks_k, kb = in - nb * blocks_k;
    const int part = threadIdx.x & 15, line = threadIdx.x >> 4;
    const int64_t k0 = kb * kF8Block, n0 = nb * kF8Block;
    Eight<T, EIGHTS> held[kTurns];
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
        const int64_t n = min(n0 + i * (kThreads / 16) + line, a.N - 1);
        held[i].template load<PAST>(static_cast<const T*>(a.W) + (g * a.N + n) * a.K, k0 + part * 8, a.K);
    }
    const auto numbers = [&](int i, float (&x)[8]) {
        held[i].numbers(x, n0 + i * (kThreads / 16) + line < a.N && (!EIGHTS || k0 + part * 8 < a.K));
    };
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
        float x[8];
        numbers(i, x);
#pragma unroll
        for (int j = 0; j < 8; ++j) most = fmaxf(most, magnitude(x[j]));
    }
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
        float x[8];
        numbers(i, x);
        const uint32_t lo = encode(x, s.back), hi = encode(x + 4, s.back);
        if (n0 + n < a.N) store_codes<PAST>(a.codes + ((g * a.N + n0 + n) * blocks_k + kb) * kF8Block + part * 8, lo, hi);
        if constexpr (BOTH) {
            *reinterpret_cast<uint32_t*>(tile + n * kPitch + part * 8) = lo;
            *reinterpret_cast<uint32_t*>(tile + n * kPitch + part * 8 + 4) = hi;
        }
    }
    if constexpr (BOTH) {
        __syncthreads();
        // The same tile by columns: a thread has four columns of eight rows, read as eight words and turned round in registers; eight
        // threads whose rows follow each other write half a line of each column.
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int rows8 = threadIdx.x & 15, columns4 = i * 16 + (threadIdx.x >> 4);
            uint32_t w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = *reinterpret_cast<const uint32_t*>(tile + (rows8 * 8 + j) * kPitch + columns4 * 4);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                // bytes (0, 1) and (2, 3) of two rows, then of four
                const uint32_t a01 = __builtin_amdgcn_perm(w[4 * h + 1], w[4 * h], 0x05010400), a23 = __builtin_amdgcn_perm(w[4 * h + 1], w[4 * h], 0x07030602);
                const uint32_t b01 = __builtin_amdgcn_perm(w[4 * h + 3], w[4 * h + 2], 0x05010400), b23 = __builtin_amdgcn_perm(w[4 * h + 3], w[4 * h + 2], 0x07030602);
                w[4 * h + 0] = __builtin_amdgcn_perm(b01, a01, 0x05040100);
                w[4 * h + 1] = __builtin_amdgcn_perm(b01, a01, 0x07060302);
                w[4 * h + 2] = __builtin_amdgcn_perm(b23, a23, 0x05040100);
                w[4 * h + 3] = __builtin_amdgcn_perm(b23, a23, 0x07060302);
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int64_t k = k0 + columns4 * 4 + c;
                if (k < a.K) store_codes<PAST>(a.codes_t + ((g * a.K + k) * blocks_n + nb) * kF8Block + rows8 * 8, w[c], w[4 + c]);
            }
        }
    }
}

template <typename T, int TURNS, bool EIGHTS>
hipError_t f8_rows(const F8RowsArgs& a, int64_t blocks_k, hipStream_t s)
{
    constexpr int kBlocks = kThreads / 16 * TURNS;
    return launch_parts((a.R * blocks_k + kBlocks - 1) / kBlocks, kThreads, [&](unsigned grid, int64_t block0) {
        f8_rows_kernel<T, TURNS, EIGHTS><<<grid, kThreads, 0, s>>>(a, blocks_k, block0);
    });
}
template <typename T>
hipError_t f8_rows(const F8RowsArgs& a, hipStream_t s)
{
    const int64_t blocks_k = f8_blocks(a.K);
    if (a.K % 8) return f8_rows<T, 1, false>(a, blocks_k, s);
    // one block and two (us, bf16): 3,001 rows of 1,000 4.2, 4.5; 8,192 of 2,048 14.4, 13.5; 16,384 of 4,096 45.0, 39.0
    return a.R * blocks_k < 65536 ? f8_rows<T, 1, true>(a, blocks_k, s) : f8_rows<T, 2, true>(a, blocks_k, s);
}

template <typename T, bool BOTH, bool PAST>
hipError_t f8_weights(const F8WeightsArgs& a, hipStream_t s)
{
    const int64_t blocks_n = f8_blocks(a.N), blocks_k = f8_blocks(a.K);
    return launch_parts(a.G * blocks_n * blocks_k, kThreads, [&](unsigned grid, int64_t block0) {
        if (a.K % 8) f8_weights_kernel<T, BOTH, false, PAST><<<grid, kThreads, 0, s>>>(a, blocks_n, blocks_k, block0);
        else f8_weights_kernel<T, BOTH, true, PAST><<<grid, kThreads, 0, s>>>(a, blocks_n, blocks_k, block0);
    });
}
template <typename T, bool BOTH>
hipError_t f8_weights(const F8WeightsArgs& a, hipStream_t s)
{
    // past the caches where values and codes are more than these hold (us through and past them, bf16, both ways round, alone and with a
    // product of 1,024 rows behind: 4 x 4,096 x 2,048 31.0, 27.0 and 49.2, 49.8; 8 x 53.7, 48.9 and 78.0, 73.8; 16 x 103, 93 and 134, 131;
    // 1 x 4,096 x 4,096 13.9, 13.4 and 44.0, 48.2)
    return a.G * a.N * a.K >= 1ll << 26 ? f8_weights<T, BOTH, true>(a, s) : f8_weights<T, BOTH, false>(a, s);
}
template <typename T>
hipError_t f8_weights(const F8WeightsArgs& a, hipStream_t s)
{
    return a.codes_t ? f8_weights<T, true>(a, s) : f8_weights<T, false>(a, s);
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
