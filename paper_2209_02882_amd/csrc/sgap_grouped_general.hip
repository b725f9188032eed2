// Products over ragged groups, for every shape, layout and alignment:
//   Y[r, :]  = X[src(r), :] * op(W[g])              r in group g; W[g] is N x K or K x N
//   dW[g]    = sum over the rows r of g of dY[r, :] (x) X[src(r), :]
// Both are C = A * B^T over tiles of 128 bytes of the inner dimension, kept in LDS row by row with their 16-byte pieces
// rotated (piece p of row r lies at p ^ (r & 7)), so that sixteen lanes reading one piece of sixteen rows meet in no bank.
// An operand whose inner dimension is not the contiguous one is turned while it is put into LDS, element by element.
// Sums in 32 bits, rounded once when they are stored.
#include "sgap_grouped.hpp"

namespace sgap {

namespace {

constexpr int kThreads = 256;
constexpr int kRowBytes = 128;  // inner bytes of a tile

// One operand: `lines` rows of it (columns of the result or rows), `inner` values each.
// INNER: the inner dimension is contiguous, line l starts at ptr(l); else inner value k starts at ptr(k) and the lines lie
// side by side.  `at(i)` gives the row number that is multiplied by ld: -1 for a row of zeros.
template <typename T, int LINES, bool INNER, bool WHOLE, typename RowAt>
__device__ __forceinline__ void stage(T* lds, const T* __restrict__ base, int64_t ld, int64_t line0, int lines, int64_t k0,
                                      int64_t K, RowAt&& at)
{
    constexpr int P = Piece<T>::kCount, kTileK = kRowBytes / (int)sizeof(T);
    const int tid = threadIdx.x;
    if constexpr (INNER) {
        const int piece = tid & 7;
#pragma unroll
        for (int i = 0; i < LINES / 32; ++i) {
            const int line = (tid >> 3) + 32 * i;
            const int64_t k = k0 + piece * P;
            piece_t<T> v = {};
            const int64_t row = line < lines ? at(line0 + line) : -1;
            if (row >= 0) {
                const T* __restrict__ p = base + row * ld + k;
                if (WHOLE || k + P <= K) {
                    if (k < K) v = load_piece(p);
                } else {
#pragma unroll
                    for (int j = 0; j < P; ++j)
                        if (k + j < K) v[j] = p[j];
                }
            }
            *reinterpret_cast<piece_t<T>*>(lds + line * kTileK + ((piece ^ (line & 7)) * P)) = v;
        }
    } else {
        constexpr int kAcross = LINES / P;  // pieces side by side
#pragma unroll
        for (int i = 0; i < kTileK * kAcross / kThreads; ++i) {
            const int id = tid + kThreads * i;
            const int kk = id / kAcross, line = (id % kAcross) * P;
            const int64_t k = k0 + kk;
            piece_t<T> v = {};
            const int64_t row = k < K ? at(k) : -1;
            if (row >= 0) {
                const T* __restrict__ p = base + row * ld + line0 + line;
                if (line + P <= lines) {
                    v = load_piece(p);
                } else {
#pragma unroll
                    for (int j = 0; j < P; ++j)
                        if (line + j < lines) v[j] = p[j];
                }
            }
#pragma unroll
            for (int j = 0; j < P; ++j) {
                const int l = line + j;
                lds[l * kTileK + (((kk / P) ^ (l & 7)) * P) + kk % P] = v[j];
            }
        }
    }
}

// acc[i][j] += (A lines 16 i ..) x (B lines 16 j ..) over the tile in LDS
template <typename T, int MI, int NJ>
__device__ __forceinline__ void multiply(const T* a, const T* b, f32x4 (&acc)[MI][NJ])
{
    constexpr int P = Piece<T>::kCount, kTileK = kRowBytes / (int)sizeof(T);
    const int lane = threadIdx.x & 63, row = lane & 15, part = lane >> 4;
#pragma unroll
    for (int kc = 0; kc < 2; ++kc) {
        const int at = ((kc * 4 + part) ^ (row & 7)) * P;
        piece_t<T> fa[MI], fb[NJ];
#pragma unroll
        for (int i = 0; i < MI; ++i) fa[i] = *reinterpret_cast<const piece_t<T>*>(a + (16 * i + row) * kTileK + at);
#pragma unroll
        for (int j = 0; j < NJ; ++j) fb[j] = *reinterpret_cast<const piece_t<T>*>(b + (16 * j + row) * kTileK + at);
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NJ; ++j) acc[i][j] = mma16(fa[i], fb[j], acc[i][j]);
    }
}

// A tile of BN columns (A, the weights) by BM rows (B): a lane ends up with four neighbouring columns of one row.
template <typename T, int BM, bool KN>
__global__ __launch_bounds__(kThreads) void grouped_general_kernel(GroupedArgs a, int64_t column_tiles)
{
    constexpr int BN = 128, kTileK = kRowBytes / (int)sizeof(T);
    constexpr int WN = BM >= 128 ? 2 : 4, WM = 4 / WN;  // wavefronts along the columns and the rows
    constexpr int MI = BN / WN / 16, NJ = BM / WM / 16;
    __shared__ __align__(16) T wt[BN * kTileK];
    __shared__ __align__(16) T xt[BM * kTileK];
    const int64_t tile = blockIdx.x / column_tiles, n0 = (blockIdx.x - tile * column_tiles) * BN;
    const RowTile rows = find_row_tile<BM>(a.offsets, a.G, a.R, tile);
    if (rows.rows <= 0) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wn = (wave % WN) * (BN / WN), wm = (wave / WN) * (BM / WM);
    f32x4 acc[MI][NJ];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (rows.g < a.G) {
        const T* __restrict__ W = static_cast<const T*>(a.W) + rows.g * a.N * a.K;
        const T* __restrict__ X = static_cast<const T*>(a.X);
        const int columns = (int)min((int64_t)BN, a.N - n0);
        for (int64_t k0 = 0; k0 < a.K; k0 += kTileK) {
            __syncthreads();
            stage<T, BN, !KN, false>(wt, W, KN ? a.N : a.K, n0, columns, k0, a.K, [](int64_t r) { return r; });
            stage<T, BM, true, false>(xt, X, a.ldx, 0, rows.rows, k0, a.K,
                                      [&](int64_t r) { return a.from.row(rows.first + r); });
            __syncthreads();
            multiply<T, MI, NJ>(wt + wn * kTileK, xt + wm * kTileK, acc);
        }
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
        const int m = wm + 16 * j + (lane & 15);
        if (m >= rows.rows) continue;
        T* __restrict__ y = static_cast<T*>(a.Y) + (rows.first + m) * a.ldy;
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const int64_t n = n0 + wn + 16 * i + 4 * (lane >> 4);
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (n + r < a.N) y[n + r] = (T)acc[i][j][r];
        }
    }
}

// A tile of the weights' gradient, 128 x 128, over all rows of its group.  FIRST lies along the rows of the result:
// N of N x K, K of K x N.
template <typename T, bool KN>
__global__ __launch_bounds__(kThreads) void grouped_wgrad_general_kernel(GroupedArgs a, int64_t tiles_m, int64_t tiles_n)
{
    constexpr int B = 128, kTileK = kRowBytes / (int)sizeof(T);
    __shared__ __align__(16) T lt[B * kTileK];
    __shared__ __align__(16) T rt[B * kTileK];
    const int64_t per = tiles_m * tiles_n, g = blockIdx.x / per, in = blockIdx.x - g * per;
    const int64_t rows = KN ? a.K : a.N, columns = KN ? a.N : a.K;
    const int64_t m0 = in / tiles_n * B, n0 = in % tiles_n * B;
    const int m_rows = (int)min((int64_t)B, rows - m0), n_columns = (int)min((int64_t)B, columns - n0);
    const GroupRows gr = group_rows(a.offsets, g, a.R);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wn = (wave & 1) * 64, wm = (wave >> 1) * 64;
    f32x4 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const T* __restrict__ X = static_cast<const T*>(a.X);
    const T* __restrict__ dY = static_cast<const T*>(a.Y);
    const auto x_row = [&](int64_t r) { return a.from.row(r); };
    const auto y_row = [](int64_t r) { return r; };
    for (int64_t r0 = gr.first; r0 < gr.end; r0 += kTileK) {
        __syncthreads();
        if constexpr (KN) {
            stage<T, B, false, false>(lt, dY, a.ldy, n0, n_columns, r0, gr.end, y_row);
            stage<T, B, false, false>(rt, X, a.ldx, m0, m_rows, r0, gr.end, x_row);
        } else {
            stage<T, B, false, false>(lt, X, a.ldx, n0, n_columns, r0, gr.end, x_row);
            stage<T, B, false, false>(rt, dY, a.ldy, m0, m_rows, r0, gr.end, y_row);
        }
        __syncthreads();
        multiply<T, 4, 4>(lt + wn * kTileK, rt + wm * kTileK, acc);
    }
    T* __restrict__ dW = static_cast<T*>(const_cast<void*>(a.W)) + g * a.N * a.K;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t m = m0 + wm + 16 * j + (lane & 15);
        if (m >= rows) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t n = n0 + wn + 16 * i + 4 * (lane >> 4);
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (n + r < columns) dW[m * columns + n + r] = (T)acc[i][j][r];
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
