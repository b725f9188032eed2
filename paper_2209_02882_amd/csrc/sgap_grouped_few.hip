// Products over ragged groups of few rows, or few columns: every weight is read for one row or a handful, and their bytes
// are the bound, where there are enough loads on their way.  A workgroup has 16 to 64 columns and 16 or 32 rows, so that one
// group alone fills the chip, and its wavefronts share the inner dimension, in blocks of some steps of the matrix
// instruction; the next block's loads are on their way while one is multiplied, straight into the registers that the
// instruction takes (weights K x N: and from there, turned round, into those), and the shares are summed up through LDS at
// the end.
// One row by 4,096 x 4,096 bf16: 9.3 us, 3.6 TB/s of weights, 32 rows 16.3 us; K x N 14.9 and 19.7.
#include <type_traits>
#include <utility>

#include "sgap_grouped.hpp"

namespace sgap {

namespace {

constexpr int kTileN = 16;

// Blocks wave, wave + waves, .. of so many: the next one fetched before one is multiplied.
template <typename Block, typename F, typename M>
__device__ __forceinline__ void share_blocks(int wave, int waves, int64_t blocks, F&& fetch, M&& multiply)
{
    if (wave >= blocks) return;
    Block one, two;
    int64_t kb = wave;
    fetch(kb, one);
    for (;;) {
        if (kb + waves < blocks) fetch(kb + waves, two);
        multiply(kb, one);
        if ((kb += waves) >= blocks) break;
        if (kb + waves < blocks) fetch(kb + waves, one);
        multiply(kb, two);
        if ((kb += waves) >= blocks) break;
    }
}

template <typename T, int NT, int MT>
__global__ __launch_bounds__(512) void grouped_few_kernel(GroupedArgs a, int64_t column_items, int64_t block0)
{
    constexpr int P = Piece<T>::kCount, kStep = 4 * P, kBlock = 4 * kStep;
    __shared__ f32x4 part[8][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int waves = blockDim.x >> 6, row = lane & 15, piece = lane >> 4;
    const int64_t item = block0 + blockIdx.x, g = item / column_items, n0 = (item - g * column_items) * (NT * kTileN);
    const GroupRows gr = group_rows(a.offsets, g, a.R);
    T* __restrict__ Y = static_cast<T*>(a.Y);
    const int64_t blocks = (a.K + kBlock - 1) / kBlock;
    // columns and rows past the last are read from the last, and not stored; a row of X that does not exist is read from
    // row 0, and zeros are stored
    const T* __restrict__ w[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
        w[nt] = static_cast<const T*>(a.W) + (g * a.N + min(n0 + nt * kTileN + row, a.N - 1)) * a.K + piece * P;
    for (int64_t m0 = gr.first + (int64_t)blockIdx.y * 16 * MT; m0 < gr.end; m0 += (int64_t)gridDim.y * 16 * MT) {
        const T* __restrict__ x[MT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            const int64_t r = a.from.row(min(m0 + mt * 16 + row, gr.end - 1));
            x[mt] = static_cast<const T*>(a.X) + (r < 0 ? 0 : r) * a.ldx + piece * P;
        }
        struct Block {
            piece_t<T> w[NT][4], x[MT][4];
        };
        const auto fetch = [&](int64_t kb, Block& b) {
            asm volatile("" : "+s"(kb));  // (or the compiler keeps a pointer for every load)
            const int64_t k0 = kb * kBlock;
            const bool whole = k0 + kBlock <= a.K;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                // what is behind the end of a row is read from the block's beginning: there the row has a piece for
                // every lane, or, in a block of less than a step, for the first
                const bool there = whole || k0 + i * kStep + piece * P < a.K;
                const int64_t at = there ? k0 + i * kStep : k0 - piece * P;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) b.x[mt][i] = *reinterpret_cast<const piece_t<T>*>(x[mt] + at);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) b.w[nt][i] = *reinterpret_cast<const piece_t<T>*>(w[nt] + at);
            }
        };
        f32x4 acc[NT][MT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) acc[nt][mt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        Runs<sizeof(T) == 4, NT, MT, 512 / kBlock> runs;
        int done = 0;
        const auto multiply = [&](int64_t kb, Block& b) {
            if ((kb + 1) * kBlock > a.K) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (kb * kBlock + i * kStep + piece * P < a.K) continue;
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) b.x[mt][i] = piece_t<T>{};
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) b.w[nt][i] = piece_t<T>{};
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) acc[nt][mt] = mma16(b.x[mt][i], b.w[nt][i], acc[nt][mt]);
            runs.end_of(done++, acc);
        };
        share_blocks<Block>(wave, waves, blocks, fetch, multiply);
        runs.finish(acc);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                __syncthreads();
                part[wave][lane] = acc[nt][mt];
                __syncthreads();
                for (int i = threadIdx.x; i < 256; i += blockDim.x) {
                    // element i: row i / 16 of the tile (rows 4 l + r lie with lane part l), column i % 16
                    const int m = i >> 4, n = i & 15, from = (m >> 2) * 16 + n;
                    float v = 0.0f;
                    for (int s = 0; s < waves; ++s) v += reinterpret_cast<const float*>(&part[s][from])[m & 3];
                    const int64_t at = m0 + mt * 16 + m, column = n0 + nt * kTileN + n;
                    if (at >= gr.end || column >= a.N) continue;
                    if (a.from.src && a.from.row(at) < 0) v = 0.0f;
                    Y[at * a.ldy + column] = (T)v;
                }
            }
    }
    // rows behind the last group
    if (a.offsets && g == a.G - 1) {
        const int columns = (int)min((int64_t)NT * kTileN, a.N - n0);
        for (int64_t r = gr.end + blockIdx.y; r < a.R; r += gridDim.y)
            for (int n = threadIdx.x; n < columns; n += blockDim.x) Y[r * a.ldy + n0 + n] = (T)0.0f;
    }
}

// A lane's piece of W[e] from P rows of it: value e of every row, in the order of the rows.
template <int E, typename T, int V>
__device__ __forceinline__ piece_t<T> column_of(const T __attribute__((ext_vector_type(V))) (&rows)[Piece<T>::kCount])
{
    if constexpr (sizeof(T) == 4) {
        return piece_t<T>{rows[0][E], rows[1][E], rows[2][E], rows[3][E]};
    } else {
        uint32_t d[8][V / 2], out[4];
        __builtin_memcpy(d, rows, sizeof(d));
#pragma unroll
        for (int q = 0; q < 4; ++q)
            out[q] = __builtin_amdgcn_perm(d[2 * q + 1][E / 2], d[2 * q][E / 2], E % 2 ? 0x07060302u : 0x05040100u);
        return __builtin_bit_cast(piece_t<T>, out);
    }
}

// The same by weights K x N.  A lane takes V columns of as many rows of W as it has values of a row of X, and value e of
// each, put together in registers, is its piece of column tile e: columns n0 + V * (0 .. 15) + e.
template <typename T, int V, int MT>
__global__ __launch_bounds__(512) void grouped_few_kn_kernel(GroupedArgs a, int64_t column_items, int64_t block0)
{
    typedef T row_t __attribute__((ext_vector_type(V)));
    // a block: so many steps that their rows of W are 32 registers
    constexpr int P = Piece<T>::kCount, kStep = 4 * P, S = 8 / V, kBlock = S * kStep, kColumns = 16 * V;
    __shared__ f32x4 part[8][V][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int waves = blockDim.x >> 6, row = lane & 15, piece = lane >> 4;
    const int64_t item = block0 + blockIdx.x, g = item / column_items, n0 = (item - g * column_items) * kColumns;
    const GroupRows gr = group_rows(a.offsets, g, a.R);
    T* __restrict__ Y = static_cast<T*>(a.Y);
    const int64_t blocks = (a.K + kBlock - 1) / kBlock;
    // columns and rows past the last are read from the last, and not stored; a row of X that does not exist is read from
    // row 0, and zeros are stored
    const T* __restrict__ W = static_cast<const T*>(a.W) + g * a.K * a.N;
    const uint32_t column = (uint32_t)min(n0 + row * V, a.N - V);
    const uint32_t own = (uint32_t)(piece * P) * (uint32_t)a.N + column;  // N is 2^22 at most
    for (int64_t m0 = gr.first + (int64_t)blockIdx.y * 16 * MT; m0 < gr.end; m0 += (int64_t)gridDim.y * 16 * MT) {
        const T* __restrict__ x[MT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            const int64_t r = a.from.row(min(m0 + mt * 16 + row, gr.end - 1));
            x[mt] = static_cast<const T*>(a.X) + (r < 0 ? 0 : r) * a.ldx + piece * P;
        }
        struct Block {
            row_t w[S][P];
            piece_t<T> x[MT][S];
        };
        const auto fetch = [&](int64_t kb, Block& b) {
            asm volatile("" : "+s"(kb));  // (or the compiler keeps a pointer for every load)
            const int64_t k0 = kb * kBlock;
            if (k0 + kBlock <= a.K) {
#pragma unroll
                for (int i = 0; i < S; ++i) {
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) b.x[mt][i] = *reinterpret_cast<const piece_t<T>*>(x[mt] + k0 + i * kStep);
#pragma unroll
                    for (int j = 0; j < P; ++j) b.w[i][j] = *reinterpret_cast<const row_t*>(W + (k0 + i * kStep + j) * a.N + own);
                }
            } else {  // what is behind the last row of W is read from the last rows
#pragma unroll
                for (int i = 0; i < S; ++i) {
                    const int64_t k = min(k0 + i * kStep + piece * P, a.K - P);
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) b.x[mt][i] = *reinterpret_cast<const piece_t<T>*>(x[mt] + k - piece * P);
#pragma unroll
                    for (int j = 0; j < P; ++j) b.w[i][j] = *reinterpret_cast<const row_t*>(W + (k + j) * a.N + column);
                }
            }
        };
        f32x4 acc[V][MT];
#pragma unroll
        for (int e = 0; e < V; ++e)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) acc[e][mt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        Runs<sizeof(T) == 4, V, MT, 512 / kBlock, (V * MT > 4)> runs;
        int done = 0;
        const auto multiply = [&](int64_t kb, Block& b) {
            if ((kb + 1) * kBlock > a.K) {
#pragma unroll
                for (int i = 0; i < S; ++i) {
                    if (kb * kBlock + i * kStep + piece * P < a.K) continue;
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) b.x[mt][i] = piece_t<T>{};
#pragma unroll
                    for (int j = 0; j < P; ++j) b.w[i][j] = row_t{};
                }
            }
#pragma unroll
            for (int i = 0; i < S; ++i) {
                const auto tile = [&](auto e) {
                    const piece_t<T> w = column_of<e, T, V>(b.w[i]);
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) acc[e][mt] = mma16(b.x[mt][i], w, acc[e][mt]);
                };
                [&]<int... e>(std::integer_sequence<int, e...>) {
                    (tile(std::integral_constant<int, e>()), ...);
                }(std::make_integer_sequence<int, V>());
            }
            runs.end_of(done++, acc);
        };
        share_blocks<Block>(wave, waves, blocks, fetch, multiply);
        runs.finish(acc);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < V; ++e) part[wave][e][lane] = acc[e][mt];
            __syncthreads();
            for (int i = threadIdx.x; i < 16 * kColumns; i += blockDim.x) {
                // element i: row i / kColumns of the tile (rows 4 l + r lie with lane part l), column i % kColumns
                const int m = i / kColumns, n = i % kColumns, from = (m >> 2) * 16 + n / V;
                float v = 0.0f;
                for (int s = 0; s < waves; ++s) v += reinterpret_cast<const float*>(&part[s][n % V][from])[m & 3];
                const int64_t at = m0 + mt * 16 + m, to = n0 + n;
                if (at >= gr.end || to >= a.N) continue;
                if (a.from.src && a.from.row(at) < 0) v = 0.0f;
                Y[at * a.ldy + to] = (T)v;
            }
        }
    }
    // rows behind the last group
    if (a.offsets && g == a.G - 1) {
        const int columns = (int)min((int64_t)kColumns, a.N - n0);
        for (int64_t r = gr.end + blockIdx.y; r < a.R; r += gridDim.y)
            for (int n = threadIdx.x; n < columns; n += blockDim.x) Y[r * a.ldy + n0 + n] = (T)0.0f;
    }
}

// The gradient of few weights from many rows, where tiles of 128 x 128 are too few for the chip: a workgroup has 16 V x 16 V
// weights, and its wavefronts share the group's rows.  Both operands come as W above does, V columns of P rows to a lane.
// KN: the gradient's rows are X's columns, otherwise dY's.
template <typename T, int V, bool KN>
__global__ __launch_bounds__(512) void grouped_few_wgrad_kernel(GroupedArgs a, int64_t tiles_m, int64_t tiles_n)
{
    typedef T row_t __attribute__((ext_vector_type(V)));
    constexpr int P = Piece<T>::kCount, kStep = 4 * P, S = 4 / V, kBlock = S * kStep, kSide = 16 * V;
    __shared__ f32x4 part[8][V][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    constexpr int waves = 8;
    const int place = lane & 15, piece = lane >> 4;
    const int64_t M = KN ? a.K : a.N, N = KN ? a.N : a.K;
    const int64_t g = blockIdx.x / (tiles_m * tiles_n), tile = blockIdx.x - g * tiles_m * tiles_n;
    const int64_t m0 = tile / tiles_n * kSide, n0 = (tile - tile / tiles_n * tiles_n) * kSide;
    const GroupRows gr = group_rows(a.offsets, g, a.R);
    const int64_t blocks = (gr.end - gr.first + kBlock - 1) / kBlock;
    // columns past the last are read from the last, and not stored
    const int64_t mc = min(m0 + place * V, M - V), nc = min(n0 + place * V, N - V);
    const T* __restrict__ X = static_cast<const T*>(a.X) + (KN ? mc : nc);
    const T* __restrict__ dY = static_cast<const T*>(a.Y) + (KN ? nc : mc);
    struct Block {
        row_t x[S][P], y[S][P];
        uint32_t none[S], past;  // rows of X that do not exist, and rows behind the group's last
    };
    // what the list says for the rows of the block that is fetched next, one to a lane: asked for a block ahead
    static_assert(kBlock <= 64, "a lane for every row");
    int32_t entry = 0;
    const auto ask = [&](int64_t kb) { entry = a.from.src[min(gr.first + kb * kBlock + lane % kBlock, gr.end - 1)]; };
    if (a.from.src && wave < blocks) ask(wave);
    const auto fetch = [&](int64_t kb, Block& b) {
        const int64_t r0 = gr.first + kb * kBlock + piece * P;
        int32_t row = 0;
        if (a.from.src) {
            row = a.from.row_of(entry);
            if (kb + waves < blocks) ask(kb + waves);
        }
        b.past = 0;
#pragma unroll
        for (int i = 0; i < S; ++i) {
            b.none[i] = 0;
#pragma unroll
            for (int j = 0; j < P; ++j) {
                const int64_t r = r0 + i * kStep + j, real = min(r, gr.end - 1);
                if (r > real) b.past |= 1u << (i * P + j);
                int64_t from = real;
                if (a.from.src) from = __shfl(row, i * kStep + piece * P + j);
                if (from < 0 || from >= a.from.rows) b.none[i] |= 1u << j, from = 0;
                b.y[i][j] = *reinterpret_cast<const row_t*>(dY + real * a.ldy);
                b.x[i][j] = *reinterpret_cast<const row_t*>(X + from * a.ldx);
            }
        }
    };
    f32x4 acc[V][V];
#pragma unroll
    for (int e = 0; e < V; ++e)
#pragma unroll
        for (int f = 0; f < V; ++f) acc[e][f] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    Runs<sizeof(T) == 4, V, V, 512 / kBlock, (V > 2)> runs;
    int done = 0;
    const auto multiply = [&](int64_t, Block& b) {
#pragma unroll
        for (int i = 0; i < S; ++i) {
            if (b.none[i] | b.past) {
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    const bool past = b.past >> (i * P + j) & 1;
                    if (past) b.y[i][j] = row_t{};
                    if (past || (b.none[i] >> j & 1)) b.x[i][j] = row_t{};
                }
            }
            piece_t<T> x[V], y[V];
            const auto turn = [&](auto e) {
                x[e] = column_of<e, T, V>(b.x[i]);
                y[e] = column_of<e, T, V>(b.y[i]);
            };
            [&]<int... e>(std::integer_sequence<int, e...>) {
                (turn(std::integral_constant<int, e>()), ...);
            }(std::make_integer_sequence<int, V>());
#pragma unroll
            for (int e = 0; e < V; ++e)
#pragma unroll
                for (int f = 0; f < V; ++f) acc[e][f] = KN ? mma16(x[e], y[f], acc[e][f]) : mma16(y[e], x[f], acc[e][f]);
        }
        runs.end_of(done++, acc);
    };
    share_blocks<Block>(wave, waves, blocks, fetch, multiply);
    runs.finish(acc);
    T* __restrict__ W = static_cast<T*>(const_cast<void*>(a.W)) + g * a.K * a.N;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        __syncthreads();
#pragma unroll
        for (int f = 0; f < V; ++f) part[wave][f][lane] = acc[e][f];
        __syncthreads();
        for (int i = threadIdx.x; i < 16 * kSide; i += blockDim.x) {
            // element i: row V * (i / kSide) + e of the tile (rows 4 l + r lie with lane part l), column i % kSide
            const int m = i / kSide, n = i % kSide, from = (m >> 2) * 16 + n / V;
            float v = 0.0f;
            for (int s = 0; s < waves; ++s) v += reinterpret_cast<const float*>(&part[s][n % V][from])[m & 3];
            const int64_t to = m0 + m * V + e, column = n0 + n;
            if (to < M && column < N) W[to * N + column] = (T)v;
        }
    }
}

// workgroups that share a group's rows, `rows` each
unsigned down(const GroupedArgs& a, int rows)
{
    const int64_t mean = (a.R + a.G - 1) / a.G, most = a.G == 1 ? mean : 2 * mean, n = (most + rows - 1) / rows;
    return (unsigned)(n < 1 ? 1 : n > 64 ? 64 : n);
}

template <typename T, int V, int MT>
hipError_t few_kn(const GroupedArgs& a, int waves, hipStream_t s)
{
    const int64_t items = (a.N + V * 16 - 1) / (V * 16);
    return launch_parts(a.G * items, 64 * waves, [&](unsigned grid, int64_t block0) {
        grouped_few_kn_kernel<T, V, MT><<<dim3(grid, down(a, 16 * MT)), 64 * waves, 0, s>>>(a, items, block0);
    });
}

template <typename T, int NT, int MT>
hipError_t few(const GroupedArgs& a, int waves, hipStream_t s)
{
    const int64_t items = (a.N + NT * kTileN - 1) / (NT * kTileN);
    return launch_parts(a.G * items, 64 * waves, [&](unsigned grid, int64_t block0) {
        grouped_few_kernel<T, NT, MT><<<dim3(grid, down(a, 16 * MT)), 64 * waves, 0, s>>>(a, items, block0);
    });
}

template <typename T>
hipError_t by_plan(const GroupedArgs& a, const GroupedPlan& p, hipStream_t s)
{
    const int64_t blocks = (a.K * (int64_t)sizeof(T) + 255) / 256;
    int waves = 8;
    while (waves > 1 && waves / 2 >= blocks) waves /= 2;
    if (a.weights_kn) {
        if (p.rows > 16) return p.columns == 32 ? few_kn<T, 2, 2>(a, waves, s) : few_kn<T, 4, 2>(a, waves, s);
        return p.columns == 32 ? few_kn<T, 2, 1>(a, waves, s) : few_kn<T, 4, 1>(a, waves, s);
    }
    if (p.rows > 16) return p.columns == 16 ? few<T, 1, 2>(a, waves, s) : few<T, 2, 2>(a, waves, s);
    return p.columns == 16 ? few<T, 1, 1>(a, waves, s) : few<T, 2, 1>(a, waves, s);
}

// (no more than 128 tiles of 128 x 128)
template <typename T, int V, bool KN>
hipError_t few_wgrad(const GroupedArgs& a, hipStream_t s)
{
    constexpr int kSide = 16 * V;
    const int64_t tm = ((KN ? a.K : a.N) + kSide - 1) / kSide, tn = ((KN ? a.N : a.K) + kSide - 1) / kSide;
    grouped_few_wgrad_kernel<T, V, KN><<<(unsigned)(a.G * tm * tn), 512, 0, s>>>(a, tm, tn);
    return hipGetLastError();
}

template <typename T>
hipError_t wgrad_by_plan(const GroupedArgs& a, const GroupedPlan& p, hipStream_t s)
{
    if (p.rows == 32) return a.weights_kn ? few_wgrad<T, 2, true>(a, s) : few_wgrad<T, 2, false>(a, s);
    return a.weights_kn ? few_wgrad<T, 4, true>(a, s) : few_wgrad<T, 4, false>(a, s);
}

// Where tiles of 64 x 128 are too few for the chip.  Up to sixteen rows a group: up to 256 of them; floats, whose tiles take
// longer, 512, and by weights K x N, which they have to turn round, 1,024.  More rows: 96 and 128; floats 128 and 192.
// Tiles and here, us, in brackets how many tiles; inner dimension first where there are groups:
//   bf16    one group, 4,096: 1 row by 4,096 (32) 44, 9.3, K x N 42.5, 14.9; 32 rows by 4,096 (32) 55.6, 16.3, K x N 43.1, 19.7;
//           few rows: 32 experts of 64 for 8 tokens, 4,096 x 1,024 (256) 63, 52, 8 groups of 4, 4,096 x 4,096 (256) 64, 67, K x N
//           63, 52; 16 experts for 32 rows, 2,048 x 4,096 (512) 47, 60, K x N 50, 57;
//           8 groups, 512 rows, 2,048 x 1,024 (96) 32.6, 24.7; 1,024 rows by 1,024 (128) 42.4, 71; K x N 42.7, 41.1, 64 groups,
//           2,048 rows, 1,024 x 256 (128) 18.7, 12.6, 16 groups, 1,024 rows, 1,024 x 1,024 (192) 19.5, 22.6
//   floats  64 groups of 4, 1,024 x 2,048 (1,024) 131, 139, K x N 131, 111; one group, 4,096: 1,024 rows by 1,024 (128) 174, 168;
//           8 groups, 1,024 rows, 2,048 x 1,024 (160) 81, 96, K x N 83, 66; 16 groups, 1,024 rows, 1,024 x 1,024 (192) K x N
//           44.0, 41.7; one group, 2,048 rows by 1,024 (256) K x N 170, 237
bool few_rows_apply(const GroupedArgs& a, int dtype)
{
    if (!grouped_fast_applies(a, dtype)) return false;
    const int64_t mean = (a.R + a.G - 1) / a.G, used = a.G < a.R ? a.G : a.R;  // groups that may have rows
    const int64_t rows = a.R / 64 + used / 2, tiles = (rows > used ? rows : used) * ((a.N + 127) / 128);
    const bool floats = dtype == 0;
    if ((a.G == 1 ? mean : 2 * mean) <= 16) return tiles <= (!floats ? 256 : a.weights_kn ? 1024 : 512);
    return tiles <= (floats ? (a.weights_kn ? 192 : 128) : a.weights_kn ? 128 : 96);
}

// Tiles of 128 x 128 and here, us, in brackets how many tiles:
//   bf16    8,192 rows by 256 x 256 (4) 143, 37; 1,024 x 1,024 (64) 146, 52; 512 rows by the same 14.2, 8.9, 128 rows 8.0, 7.4;
//           16 groups of 64 rows, 256 x 256 (64) 7.4, 7.3; 8,192 rows by 2,048 x 1,024 (128) 146, 97; 8 groups of 1,024, 512 x 512
//           (128) 23.1, 24.0; 1,024 rows by 2,048 x 2,048 (256) 25, 42
//   floats  8,192 rows by 256 x 256 504, 66; 1,024 x 1,024 519, 195; 2,048 x 1,024 526, 368; 8 groups of 1,024, 512 x 512 70, 55, of
//           128 14.4, 15.5; 1,024 rows by 2,048 x 2,048 76, 101
bool few_weights_apply(const GroupedArgs& a, int dtype)
{
    if (!grouped_fast_applies(a, dtype)) return false;
    const int64_t tiles = a.G * ((a.N + 127) / 128) * ((a.K + 127) / 128);
    return tiles <= 64 || (tiles <= 128 && a.R / a.G >= (dtype == 0 ? 1024 : 2048));
}

}  // namespace

bool grouped_few_applies(const GroupedArgs& a, int dtype, bool gradient)
{
    return gradient ? few_weights_apply(a, dtype) : few_rows_apply(a, dtype);
}

GroupedPlan plan_grouped_few(const GroupedArgs& a, int dtype, bool gradient)
{
    GroupedPlan p = {GroupedPlan::kFew, 16, 16, false, false, false};
    if (gradient) {
        // 32 x 32 weights to a workgroup while there is no more than one to a compute unit, then 64 x 64: 8,192 rows, bf16, by
        // 512 x 512 (256 of the small) 40 us and 48, 1,024 x 1,024 153 and 52; floats 70 and 175, 266 and 195
        p.rows = p.columns = a.G * ((a.N + 31) / 32) * ((a.K + 31) / 32) <= a.compute_units ? 32 : 64;
        return p;
    }
    const int64_t used = a.G < a.R ? a.G : a.R, tiles = used * ((a.N + 15) / 16);
    const int64_t mean = (a.R + a.G - 1) / a.G, most = a.G == 1 ? mean : 2 * mean;
    if (most > 16) p.rows = 32;
    // More columns to a workgroup where the narrow ones are more than one to a compute unit, so that rows of X are read less
    // often.  bf16: one group, inner dimension 4,096, by 16 and by 32 columns: 512 rows by 512 columns 27.2, 19.4; 128 by 4,096
    // 53.3, 38.3; 32 by 4,096 (256 workgroups) 16.3, 21.2.  Weights K x N, 32 and 64 columns: 128 by 4,096 36.3, 22.0; 32 experts
    // for 64 rows, 2,048 by 1,024 50.1, 30.6; 512 rows by 512 (256) 16.2, 21.2.  128 columns are never better.
    if (a.weights_kn) p.columns = used * ((a.N + 31) / 32) * down(a, p.rows) <= a.compute_units ? 32 : 64;
    else if (most > 16) p.columns = tiles * down(a, 32) <= a.compute_units ? 16 : 32;
    else p.columns = tiles < 1024 ? 16 : 32;
    return p;
}

hipError_t launch_grouped_few(const GroupedArgs& a, int dtype, bool gradient, const GroupedPlan& p, hipStream_t s)
{
    switch (dtype) {
        case 0: return gradient ? wgrad_by_plan<float>(a, p, s) : by_plan<float>(a, p, s);
        case 1: return gradient ? wgrad_by_plan<half_t>(a, p, s) : by_plan<half_t>(a, p, s);
        default: return gradient ? wgrad_by_plan<bf16_t>(a, p, s) : by_plan<bf16_t>(a, p, s);
    }
}

}  // namespace sgap
