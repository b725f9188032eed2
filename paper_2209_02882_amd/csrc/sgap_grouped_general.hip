// Products over ragged groups, for every shape, layout and alignment:
//   Y[r, :]  = X[src(r), :] * op(W[g])              r in group g; W[g] is N x K or K x N
//   dW[g]    = sum over the rows r of g of dY[r, :] (x) X[src(r), :]
// Tiles go through registers into LDS, so that rows may begin at any element; inner values past the end and rows that do
// not exist become zeros on the way.  Sums in 32 bits, rounded once when they are stored.
#include "sgap_grouped_tiles.hpp"

namespace sgap {

namespace {

constexpr int kThreads = 256;

// The 16 bytes at p, of which `count` elements are there, zeros behind them; `before`: elements of the row in front of p.
// At the end of a row the 16 bytes up to the end are read and moved down.
template <typename T>
__device__ __forceinline__ piece_t<T> part_of_piece(const T* __restrict__ p, int count, int before)
{
    constexpr int P = Piece<T>::kCount;
    if (count >= P) return load_piece(p);
    if (count <= 0) return piece_t<T>{};
    if (count + before >= P) {
        union {
            piece_t<T> v;
            uint64_t u[2];
        } r;
        r.v = load_piece(p - (P - count));
        const int down = (P - count) * (int)sizeof(T) * 8;  // bits, 16 to 112
        const uint64_t lo = down < 64 ? r.u[0] >> down | r.u[1] << (64 - down) : r.u[1] >> (down - 64);
        r.u[1] = down < 64 ? r.u[1] >> down : 0;
        r.u[0] = lo;
        return r.v;
    }
    piece_t<T> v = {};
#pragma unroll
    for (int j = 0; j < P; ++j)
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
    constexpr int WN = BM >= 64 ? 2 : 4, WM = 4 / WN;  // wavefronts along the columns and the rows
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
        // where each load of the next tile begins: the tiles come in their order, and a step from one to the next is the
        // same for all (64-bit products for every load are what this kernel was bound by)
        const int N = (int)a.N, K = (int)a.K;
        const int64_t down = KN ? Wt::kInner * a.N : Wt::kInner;
        const T* w[Wt::kRounds];
        const T* x[Xt::kRounds];
#pragma unroll
        for (int i = 0; i < Wt::kRounds; ++i) {
            const int64_t k = KN ? Wt::major(i) : Wt::minor(i) * Wt::P, n = n0 + (KN ? Wt::minor(i) * Wt::P : Wt::major(i));
            w[i] = static_cast<const T*>(a.W) + rows.g * a.N * a.K + (KN ? k * a.N + n : n * a.K + k);
        }
        uint32_t real = 0;  // rounds whose row of X there is
#pragma unroll
        for (int i = 0; i < Xt::kRounds; ++i) {
            const int m = Xt::major(i);
            const int64_t r = m < rows.rows ? a.from.row(rows.first + m) : -1;
            real |= r >= 0 ? 1u << i : 0u;
            x[i] = static_cast<const T*>(a.X) + r * a.ldx + Xt::minor(i) * Xt::P;
        }
        const auto fetch = [&](int t, int i) -> piece_t<T> {
            const int k0 = t * Wt::kInner;
            piece_t<T> v = {};
            if (i >= Wt::kRounds) {
                const int r = i - Wt::kRounds, k = k0 + Xt::minor(r) * Xt::P;
                if (real >> r & 1) v = part_of_piece(x[r], K - k, k);
                x[r] += Xt::kInner;
                return v;
            }
            const int k = k0 + (KN ? Wt::major(i) : Wt::minor(i) * Wt::P);
            const int n = (int)n0 + (KN ? Wt::minor(i) * Wt::P : Wt::major(i));
            if (k < K && n < N) v = KN ? part_of_piece(w[i], N - n, n) : part_of_piece(w[i], K - k, k);
            w[i] += down;
            return v;
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
    // The loads of a tile: rows of the first operand, which has the result's columns, then of the second.  Those of dY
    // begin a step further down with every tile; what the list says of X's rows is asked for a tile ahead.
    constexpr int kRounds = Bt::kRounds, kXAt = KN ? kRounds : 0, kYAt = KN ? 0 : kRounds;
    const int first = (int)gr.first, end = (int)gr.end, N = (int)a.N, K = (int)a.K;
    const int x0 = (int)(KN ? m0 : n0), y0 = (int)(KN ? n0 : m0);
    const T* y[kRounds];
    int32_t entry[kRounds];
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
        y[i] = static_cast<const T*>(a.Y) + (gr.first + Bt::major(i)) * a.ldy + y0 + Bt::minor(i) * Bt::P;
        entry[i] = first + Bt::major(i) < end ? a.from.entry(first + Bt::major(i)) : -1;
    }
    const auto fetch = [&](int t, int i) -> piece_t<T> {
        const int round = i % kRounds, r = first + t * Bt::kInner + Bt::major(round);
        piece_t<T> v = {};
        if (i - round == kYAt) {
            const int line = y0 + Bt::minor(round) * Bt::P;
            if (r < end && line < N) v = part_of_piece(y[round], N - line, line);
            y[round] += Bt::kInner * a.ldy;
        } else {
            const int line = x0 + Bt::minor(round) * Bt::P, row = a.from.row_of(entry[round]);
            if (r < end && line < K && row >= 0) v = part_of_piece(static_cast<const T*>(a.X) + row * a.ldx + line, K - line, line);
            entry[round] = r + Bt::kInner < end ? a.from.entry(r + Bt::kInner) : -1;
        }
        return v;
    };
    static_assert(kXAt + kYAt == kRounds, "");
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
    // Tiles no longer than a group is in the mean (an empty half of a tile costs as much as a full one), and shorter ones
    // where there are not enough for the chip.
    if (a.R <= 48 * a.G) return general<T, 32>(a, s);
    const int64_t columns = (a.N + 127) / 128;
    if ((a.R / 128 + a.G / 2) * columns < 3 * a.compute_units) return general<T, 64>(a, s);
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
