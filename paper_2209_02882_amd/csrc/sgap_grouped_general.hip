// Products over ragged groups, for every shape, layout and alignment:
//   Y[r, :]  = X[src(r), :] * op(W[g])              r in group g; W[g] is N x K or K x N
//   dW[g]    = sum over the rows r of g of dY[r, :] (x) X[src(r), :]
// Tiles go through registers into LDS, so that rows may begin at any element; inner values past the end and rows that do
// not exist become zeros on the way.  Sums in 32 bits, rounded once when they are stored.
// Bound by the way through registers: a row at an odd address is read in pieces that begin before it and moved down.
// 3,001 rows in 7 groups, 1,000 by 1,531, f16 (9.2 GF each): 36, 31 and 37 us, 250 to 300 TF/s.
#include "sgap_grouped_tiles.hpp"

namespace sgap {

namespace {

constexpr int kThreads = 256;

// The first `count` elements at p, zeros behind them: rows of fewer elements than a piece has (SHORT) are read one by one.
template <typename T>
__device__ __forceinline__ piece_t<T> few_of_piece(const T* __restrict__ p, int count)
{
    piece_t<T> v = {};
#pragma unroll
    for (int j = 0; j < Piece<T>::kCount; ++j)
        if (j < count) v[j] = p[j];
    return v;
}

// A piece that was read `by` elements too early, moved down by them, zeros behind; by = 0 .. a piece's elements.
template <typename T>
__device__ __forceinline__ piece_t<T> move_down(piece_t<T> v, int by)
{
    union {
        piece_t<T> v;
        uint64_t u[2];
    } r;
    r.v = v;
    const int bits = by * (int)sizeof(T) * 8, low = bits & 63;
    const uint64_t over = low ? r.u[1] << (64 - low) : 0;
    const uint64_t lo = bits < 64 ? (r.u[0] >> low) | over : r.u[1] >> low, hi = r.u[1] >> low;
    r.u[0] = bits < 128 ? lo : 0;
    r.u[1] = bits < 64 ? hi : 0;
    return r.v;
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

// A tile of 128 columns (the weights) by BM rows: a lane ends up with four neighbouring columns of one row.  Loads have no
// branches, or they would come one after the other: what would pass the end of a row is read from so much further in front
// and moved down when it has arrived, and what is behind the last row or column is read from the last.
template <typename T, int BM, bool KN, bool SHORT>
__global__ __launch_bounds__(kThreads) void grouped_general_kernel(GroupedArgs a, int64_t column_tiles, int64_t block0)
{
    constexpr int BN = 128;
    using Wt = Tile<T, BN, !KN, kThreads>;
    using Xt = Tile<T, BM, true, kThreads>;
    constexpr int WN = BM >= 64 ? 2 : 4, WM = 4 / WN;  // wavefronts along the columns and the rows
    constexpr int MI = BN / WN / 16, NJ = BM / WM / 16, P = Wt::P;
    __shared__ __align__(16) char lds[2 * (Wt::kBytes + Xt::kBytes)];
    const int64_t item = block0 + blockIdx.x, tile = item / column_tiles, n0 = (item - tile * column_tiles) * BN;
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
        // same for all (64-bit products for every load would take longer than the products of the matrices)
        const int N = (int)a.N, K = (int)a.K;
        const int64_t down = KN ? Wt::kInner * a.N : Wt::kInner;
        const T* w[Wt::kRounds];
        const T* x[Xt::kRounds];
        // lines contiguous: how far in front of its place a piece at the end of the rows of W is read
        const auto ahead = [&](int i) { return KN && !SHORT ? max((int)n0 + Wt::minor(i) * P - (N - P), 0) : 0; };
        // inner contiguous: the same for the tile that begins at k0
        const auto early = [&](int k0, int minor) { return SHORT ? 0 : max(k0 + minor * P - (K - P), 0); };
#pragma unroll
        for (int i = 0; i < Wt::kRounds; ++i) {
            const int64_t k = KN ? Wt::major(i) : Wt::minor(i) * P;
            const int64_t n = KN ? n0 + Wt::minor(i) * P - ahead(i) : min(n0 + Wt::major(i), a.N - 1);
            w[i] = static_cast<const T*>(a.W) + rows.g * a.N * a.K + (KN ? k * a.N + n : n * a.K + k);
        }
        uint32_t real = 0;  // rounds whose row of X there is
#pragma unroll
        for (int i = 0; i < Xt::kRounds; ++i) {
            const int64_t r = a.from.row(rows.first + min(Xt::major(i), rows.rows - 1));
            real |= r >= 0 ? 1u << i : 0u;
            x[i] = static_cast<const T*>(a.X) + max(r, (int64_t)0) * a.ldx + Xt::minor(i) * P;
        }
        const auto fetch = [&](int t, int i) -> piece_t<T> {
            const int k0 = t * Wt::kInner;
            piece_t<T> v;
            if (i >= Wt::kRounds) {
                const int r = i - Wt::kRounds;
                if (SHORT) v = few_of_piece(x[r], real >> r & 1 ? K - (k0 + Xt::minor(r) * P) : 0);
                else v = load_piece(x[r] - early(k0, Xt::minor(r)));
                x[r] += Xt::kInner;
                return v;
            }
            if constexpr (!KN) {
                if (SHORT) v = few_of_piece(w[i], K - (k0 + Wt::minor(i) * P));
                else v = load_piece(w[i] - early(k0, Wt::minor(i)));
            } else {
                const bool there = k0 + Wt::major(i) < K;
                if (SHORT) v = few_of_piece(w[i], there ? N - ((int)n0 + Wt::minor(i) * P) : 0);
                else v = load_piece(there ? w[i] : w[i] - (int64_t)Wt::major(i) * N);  // (the tile's first row is there)
            }
            w[i] += down;
            return v;
        };
        const auto mend = [&](int t, int i, piece_t<T> v) -> piece_t<T> {
            const int k0 = t * Wt::kInner;
            if (SHORT) return v;
            if (i >= Wt::kRounds || !KN) {
                if (k0 + Wt::kInner <= K) return v;
                return move_down<T>(v, min(early(k0, i >= Wt::kRounds ? Xt::minor(i - Wt::kRounds) : Wt::minor(i)), P));
            }
            if (k0 + Wt::kInner <= K && n0 + BN <= N) return v;
            return move_down<T>(v, k0 + Wt::major(i) < K ? min(ahead(i), P) : P);
        };
        multiply_tiles_staged<Wt, Xt, MI, NJ, T>(lds, (int)((a.K + Wt::kInner - 1) / Wt::kInner), fetch, mend, wn, wm, acc);
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
        const int m = wm + 16 * j + (lane & 15);
        if (m >= rows.rows) continue;
        const bool real = !a.from.src || a.from.row(rows.first + m) >= 0;
        T* __restrict__ y = static_cast<T*>(a.Y) + (rows.first + m) * a.ldy;
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const int64_t n = n0 + wn + 16 * i + 4 * (lane >> 4);
            if (n < a.N) store_four(y + n, real ? acc[i][j] : f32x4{0.0f, 0.0f, 0.0f, 0.0f}, a.N - n);
        }
    }
}

// A tile of the weights' gradient, 128 x 128, over all rows of its group: the rows of the result are N of N x K, K of K x N.
template <typename T, bool KN, bool SHORT>
__global__ __launch_bounds__(kThreads) void grouped_wgrad_general_kernel(GroupedArgs a, int64_t tiles_m, int64_t tiles_n, int64_t block0)
{
    constexpr int B = 128;
    using Bt = Tile<T, B, false, kThreads>;
    constexpr int P = Bt::P;
    __shared__ __align__(16) char lds[4 * Bt::kBytes];
    const int64_t item = block0 + blockIdx.x, per = tiles_m * tiles_n, g = item / per, in = item - g * per;
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
    constexpr int kRounds = Bt::kRounds, kYAt = KN ? 0 : kRounds;
    const int first = (int)gr.first, end = (int)gr.end, N = (int)a.N, K = (int)a.K;
    const int x0 = (int)(KN ? m0 : n0), y0 = (int)(KN ? n0 : m0);
    // how far in front of its place a piece at the end of a row is read
    const auto x_ahead = [&](int i) { return SHORT ? 0 : max(x0 + Bt::minor(i) * P - (K - P), 0); };
    const auto y_ahead = [&](int i) { return SHORT ? 0 : max(y0 + Bt::minor(i) * P - (N - P), 0); };
    const T* y[kRounds];
    int32_t entry[kRounds];
    uint32_t none = 0;  // rounds of the tile that comes which have no row of X
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
        y[i] = static_cast<const T*>(a.Y) + (gr.first + Bt::major(i)) * a.ldy + y0 + Bt::minor(i) * P - y_ahead(i);
        entry[i] = -1;
        if (first + Bt::major(i) < end) entry[i] = a.from.entry(first + Bt::major(i));
    }
    const auto fetch = [&](int t, int i) -> piece_t<T> {
        const int round = i % kRounds, r = first + t * Bt::kInner + Bt::major(round);
        piece_t<T> v;
        if (i - round == kYAt) {
            if (SHORT) v = few_of_piece(y[round], r < end ? N - (y0 + Bt::minor(round) * P) : 0);
            else v = load_piece(r < end ? y[round] : y[round] - (int64_t)Bt::major(round) * a.ldy);  // (the tile's first row is there)
            y[round] += Bt::kInner * a.ldy;
        } else {
            const int row = a.from.row_of(entry[round]), line = x0 + Bt::minor(round) * P;
            none = round == 0 ? 0 : none;
            none |= row < 0 ? 1u << round : 0u;
            const T* const p = static_cast<const T*>(a.X) + max(row, 0) * a.ldx + line - x_ahead(round);
            if (SHORT) v = few_of_piece(p, row >= 0 ? K - line : 0);
            else v = load_piece(p);
            entry[round] = -1;
            if (r + Bt::kInner < end) entry[round] = a.from.entry(r + Bt::kInner);
        }
        return v;
    };
    const auto mend = [&](int t, int i, piece_t<T> v) -> piece_t<T> {
        const int round = i % kRounds, r0 = first + t * Bt::kInner;
        if (SHORT) return v;
        if (i - round == kYAt) {
            if (r0 + Bt::kInner <= end && y0 + B <= N) return v;
            return move_down<T>(v, r0 + Bt::major(round) < end ? min(y_ahead(round), P) : P);
        }
        if (x0 + B <= K && !__any(none != 0)) return v;
        return move_down<T>(v, none >> round & 1 ? P : min(x_ahead(round), P));
    };
    multiply_tiles_staged<Bt, Bt, 4, 4, T>(lds, (end - first + Bt::kInner - 1) / Bt::kInner, fetch, mend, wn, wm, acc);
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

template <typename T, int BM, bool SHORT>
hipError_t general(const GroupedArgs& a, hipStream_t s)
{
    const int64_t columns = (a.N + 127) / 128;
    return launch_parts(columns * most_row_tiles(a.G, a.R, BM, a.offsets != nullptr), kThreads, [&](unsigned grid, int64_t block0) {
        if (a.weights_kn) grouped_general_kernel<T, BM, true, SHORT><<<grid, kThreads, 0, s>>>(a, columns, block0);
        else grouped_general_kernel<T, BM, false, SHORT><<<grid, kThreads, 0, s>>>(a, columns, block0);
    });
}

template <typename T>
hipError_t by_rows(const GroupedArgs& a, const GroupedPlan& p, hipStream_t s)
{
    if (p.short_rows) return general<T, 32, true>(a, s);
    return p.rows == 32 ? general<T, 32, false>(a, s) : p.rows == 64 ? general<T, 64, false>(a, s) : general<T, 128, false>(a, s);
}

template <typename T, bool SHORT>
hipError_t wgrad_as(const GroupedArgs& a, hipStream_t s)
{
    const int64_t tm = ((a.weights_kn ? a.K : a.N) + 127) / 128, tn = ((a.weights_kn ? a.N : a.K) + 127) / 128;
    return launch_parts(a.G * tm * tn, kThreads, [&](unsigned grid, int64_t block0) {
        if (a.weights_kn) grouped_wgrad_general_kernel<T, true, SHORT><<<grid, kThreads, 0, s>>>(a, tm, tn, block0);
        else grouped_wgrad_general_kernel<T, false, SHORT><<<grid, kThreads, 0, s>>>(a, tm, tn, block0);
    });
}

template <typename T>
hipError_t wgrad(const GroupedArgs& a, const GroupedPlan& p, hipStream_t s)
{
    return p.short_rows ? wgrad_as<T, true>(a, s) : wgrad_as<T, false>(a, s);
}

}  // namespace

GroupedPlan plan_grouped(const GroupedArgs& a, int dtype, bool gradient)
{
    if (grouped_few_applies(a, dtype, gradient)) return plan_grouped_few(a, dtype, gradient);
    if (grouped_fast_applies(a, dtype)) return plan_grouped_fast(a, dtype, gradient);
    GroupedPlan p = {GroupedPlan::kRegisters, 128, 128, false, false, false};
    const int64_t piece = dtype == 0 ? 4 : 8;
    p.short_rows = a.K < piece || a.N < piece || a.from.rows == 0;  // or no rows
    if (gradient) return p;
    // Tiles no longer than a group is in the mean (an empty half of a tile costs as much as a full one), and shorter ones
    // where there are not enough for the chip.
    if (p.short_rows || a.R <= 48 * a.G) p.rows = 32;
    else if ((a.R / 128 + a.G / 2) * ((a.N + 127) / 128) < 3 * a.compute_units) p.rows = 64;
    return p;
}

hipError_t launch_grouped_mm(const GroupedArgs& a, int dtype, hipStream_t s)
{
    const GroupedPlan p = plan_grouped(a, dtype, false);
    if (p.way == GroupedPlan::kFew) return launch_grouped_few(a, dtype, false, p, s);
    if (p.way == GroupedPlan::kTiles) return launch_grouped_fast(a, dtype, false, p, s);
    switch (dtype) {
        case 0: return by_rows<float>(a, p, s);
        case 1: return by_rows<half_t>(a, p, s);
        default: return by_rows<bf16_t>(a, p, s);
    }
}

hipError_t launch_grouped_wgrad(const GroupedArgs& a, int dtype, hipStream_t s)
{
    const GroupedPlan p = plan_grouped(a, dtype, true);
    if (p.way == GroupedPlan::kFew) return launch_grouped_few(a, dtype, true, p, s);
    if (p.way == GroupedPlan::kTiles) return launch_grouped_fast(a, dtype, true, p, s);
    switch (dtype) {
        case 0: return wgrad<float>(a, p, s);
        case 1: return wgrad<half_t>(a, p, s);
        default: return wgrad<bf16_t>(a, p, s);
    }
}

}  // namespace sgap
