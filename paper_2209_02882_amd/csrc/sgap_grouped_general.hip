// Products over ragged groups, for every shape, layout and alignment:
//   Y[r, :]  = X[src(r), :] * op(W[g])              r in group g; W[g] is N x K or K x N
//   dW[g]    = sum over the rows r of g of dY[r, :] (x) X[src(r), :]
// Tiles go through registers into LDS, so that rows may begin at any element; inner values past the end and rows that do
// not exist become zeros on the way.  Sums in 32 bits, rounded once when they are stored.
#include "sgap_grouped_tiles.hpp"

namespace sgap {

namespace {

constexpr int kThreads = 256;

// The 16 bytes at p, of which `count` elements are there (all of them, or fewer: one by one).
template <typename T>
__device__ __forceinline__ piece_t<T> part_of_piece(const T* __restrict__ p, int64_t count)
{
    if (count >= Piece<T>::kCount) return load_piece(p);
    piece_t<T> v = {};
#pragma unroll
    for (int j = 0; j < Piece<T>::kCount; ++j)
        if (j < count) v[j] = p[j];
    return v;
}

template <typename T>
__device__ __forceinline__ void store_four(T* __restrict__ p, f32x4 v, int64_t count)
{
    typedef T four __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    if (count >= 4) {
        four o;
#pragma unroll
        for (int r = 0; r < 4; ++r) o[r] = (T)v[r];
        *reinterpret_cast<four*>(p) = o;
    } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (r < count) p[r] = (T)v[r];
    }
}

// A tile of 128 columns (the weights) by BM rows: a lane ends up with four neighbouring columns of one row.
template <typename T, int BM, bool KN>
__global__ __launch_bounds__(kThreads) void grouped_general_kernel(GroupedArgs a, int64_t column_tiles)
{
    constexpr int BN = 128;
    using Wt = Tile<T, BN, !KN, kThreads>;
    using Xt = Tile<T, BM, true, kThreads>;
    constexpr int WN = BM >= 128 ? 2 : 4, WM = 4 / WN;  // wavefronts along the columns and the rows
    constexpr int MI = BN / WN / 16, NJ = BM / WM / 16;
    __shared__ __align__(16) char lds[2 * (Wt::kBytes + Xt::kBytes)];
    const int64_t tile = blockIdx.x / column_tiles, n0 = (blockIdx.x - tile * column_tiles) * BN;
    const RowTile rows = find_row_tile<BM>(a.offsets, a.G, a.R, tile);
    if (rows.rows <= 0) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wn = (wave % WN) * (BN / WN), wm = (wave / WN) * (BM / WM);
    f32x4 acc[MI][NJ];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (rows.g < a.G) {
        const T* const W = static_cast<const T*>(a.W) + rows.g * a.N * a.K;
        const T* x[Xt::kRounds];
#pragma unroll
        for (int i = 0; i < Xt::kRounds; ++i) {
            const int m = Xt::major(i);
            const int64_t r = m < rows.rows ? a.from.row(rows.first + m) : -1;
            x[i] = r >= 0 ? static_cast<const T*>(a.X) + r * a.ldx : nullptr;
        }
        const auto fetch = [&](int t, int i) -> piece_t<T> {
            const int64_t k0 = (int64_t)t * Wt::kInner;
            if (i >= Wt::kRounds) {
                const int r = i - Wt::kRounds;
                const int64_t k = k0 + Xt::minor(r) * Xt::P;
                return x[r] ? part_of_piece(x[r] + k, a.K - k) : piece_t<T>{};
            }
            const int64_t k = k0 + (KN ? Wt::major(i) : Wt::minor(i) * Wt::P);
            const int64_t n = n0 + (KN ? Wt::minor(i) * Wt::P : Wt::major(i));
            if (k >= a.K || n >= a.N) return piece_t<T>{};
            return KN ? part_of_piece(W + k * a.N + n, a.N - n) : part_of_piece(W + n * a.K + k, a.K - k);
        };
        multiply_tiles_staged<Wt, Xt, MI, NJ, T>(lds, (int)((a.K + Wt::kInner - 1) / Wt::kInner), fetch, wn, wm, acc);
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
        const int m = wm + 16 * j + (lane & 15);
        if (m >= rows.rows) continue;
        T* __restrict__ y = static_cast<T*>(a.Y) + (rows.first + m) * a.ldy;
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const int64_t n = n0 + wn + 16 * i + 4 * (lane >> 4);
            if (n < a.N) store_four(y + n, acc[i][j], a.N - n);
        }
    }
}

// A tile of the weights' gradient, 128 x 128, over all rows of its group: the rows of the result are N of N x K, K of K x N.
template <typename T, bool KN>
__global__ __launch_bounds__(kThreads) void grouped_wgrad_general_kernel(GroupedArgs a, int64_t tiles_m, int64_t tiles_n)
{
    constexpr int B = 128;
    using Bt = Tile<T, B, false, kThreads>;
    __shared__ __align__(16) char lds[4 * Bt::kBytes];
    const int64_t per = tiles_m * tiles_n, g = blockIdx.x / per, in = blockIdx.x - g * per;
    const int64_t lines = KN ? a.K : a.N, columns = KN ? a.N : a.K;
    const int64_t m0 = in / tiles_n * B, n0 = in % tiles_n * B;
    const GroupRows gr = group_rows(a.offsets, g, a.R);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wn = (wave & 1) * 64, wm = (wave >> 1) * 64;
    f32x4 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const T* const X = static_cast<const T*>(a.X);
    const T* const dY = static_cast<const T*>(a.Y);
    const auto fetch = [&](int t, int i) -> piece_t<T> {
        const int64_t r = gr.first + (int64_t)t * Bt::kInner + Bt::major(i % Bt::kRounds);
        const bool first = i < Bt::kRounds;  // the operand that has the result's columns
        const int64_t line = (first ? n0 : m0) + Bt::minor(i % Bt::kRounds) * Bt::P;
        if (r >= gr.end || line >= (first ? columns : lines)) return piece_t<T>{};
        if (first == KN) return part_of_piece(dY + r * a.ldy + line, a.N - line);
        const int64_t row = a.from.row(r);
        return row >= 0 ? part_of_piece(X + row * a.ldx + line, a.K - line) : piece_t<T>{};
    };
    multiply_tiles_staged<Bt, Bt, 4, 4, T>(lds, (int)((gr.end - gr.first + Bt::kInner - 1) / Bt::kInner), fetch, wn, wm, acc);
    T* __restrict__ dW = static_cast<T*>(const_cast<void*>(a.W)) + g * a.N * a.K;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t m = m0 + wm + 16 * j + (lane & 15);
        if (m >= lines) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t n = n0 + wn + 16 * i + 4 * (lane >> 4);
            if (n < columns) store_four(dW + m * columns + n, acc[i][j], columns - n);
        }
    }
}

template <typename T, int BM>
hipError_t general(const GroupedArgs& a, hipStream_t s)
{
    const int64_t columns = (a.N + 127) / 128, grid = columns * most_row_tiles(a.G, a.R, BM, a.offsets != nullptr);
    if (grid > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    if (a.weights_kn) grouped_general_kernel<T, BM, true><<<(unsigned)grid, kThreads, 0, s>>>(a, columns);
    else grouped_general_kernel<T, BM, false><<<(unsigned)grid, kThreads, 0, s>>>(a, columns);
    return hipGetLastError();
}

template <typename T>
hipError_t by_rows(const GroupedArgs& a, hipStream_t s)
{
    // tiles as long as a group is in the mean: an empty half of a tile costs as much as a full one
    if (a.R <= 48 * a.G) return general<T, 32>(a, s);
    return general<T, 128>(a, s);
}

template <typename T>
hipError_t wgrad(const GroupedArgs& a, hipStream_t s)
{
    const int64_t tm = ((a.weights_kn ? a.K : a.N) + 127) / 128, tn = ((a.weights_kn ? a.N : a.K) + 127) / 128;
    if (a.G * tm * tn > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    if (a.weights_kn) grouped_wgrad_general_kernel<T, true><<<(unsigned)(a.G * tm * tn), kThreads, 0, s>>>(a, tm, tn);
    else grouped_wgrad_general_kernel<T, false><<<(unsigned)(a.G * tm * tn), kThreads, 0, s>>>(a, tm, tn);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_grouped_mm(const GroupedArgs& a, int dtype, hipStream_t s)
{
    if (grouped_fast_applies(a, dtype)) return launch_grouped_fast(a, dtype, s);
    switch (dtype) {
        case 0: return by_rows<float>(a, s);
        case 1: return by_rows<half_t>(a, s);
        default: return by_rows<bf16_t>(a, s);
    }
}

hipError_t launch_grouped_wgrad(const GroupedArgs& a, int dtype, hipStream_t s)
{
    if (grouped_fast_applies(a, dtype)) return launch_grouped_wgrad_fast(a, dtype, s);
    switch (dtype) {
        case 0: return wgrad<float>(a, s);
        case 1: return wgrad<half_t>(a, s);
        default: return wgrad<bf16_t>(a, s);
    }
}

}  // namespace sgap
