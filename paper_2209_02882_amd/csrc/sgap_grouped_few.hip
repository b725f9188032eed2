// Products over ragged groups of few rows, or few columns, by weights N x K (a row of W is a column of the result): every
// weight is read for one row or a handful, and their bytes are the bound, where there are enough loads on their way.  A
// workgroup has 16 or 32 columns and rows, so that one group alone fills the chip, and its wavefronts share the inner
// dimension, in blocks of four steps of the matrix instruction; the next block's loads are on their way while one is
// multiplied, straight into the registers that the instruction takes, and the shares are summed up through LDS at the end.
// One row by 4,096 x 4,096 bf16: 9.3 us, 3.6 TB/s of weights.
#include "sgap_grouped.hpp"

namespace sgap {

namespace {

constexpr int kTileN = 16;

template <typename T, int NT, int MT>
__global__ __launch_bounds__(512) void grouped_few_kernel(GroupedArgs a, int64_t column_items)
{
    constexpr int P = Piece<T>::kCount, kStep = 4 * P, kBlock = 4 * kStep;
    __shared__ f32x4 part[8][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int waves = blockDim.x >> 6, row = lane & 15, piece = lane >> 4;
    const int64_t g = blockIdx.x / column_items, n0 = (blockIdx.x - g * column_items) * (NT * kTileN);
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
        };
        if (wave < blocks) {
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

template <typename T, int NT, int MT>
hipError_t few(const GroupedArgs& a, int waves, hipStream_t s)
{
    const int64_t items = (a.N + NT * kTileN - 1) / (NT * kTileN);
    if (a.G * items > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    const int64_t mean = (a.R + a.G - 1) / a.G, most = a.G == 1 ? mean : 2 * mean, down = (most + 16 * MT - 1) / (16 * MT);
    const dim3 grid((unsigned)(a.G * items), (unsigned)(down < 1 ? 1 : down > 64 ? 64 : down));
    grouped_few_kernel<T, NT, MT><<<grid, 64 * waves, 0, s>>>(a, items);
    return hipGetLastError();
}

template <typename T>
hipError_t by_columns(const GroupedArgs& a, hipStream_t s)
{
    const int64_t used = a.G < a.R ? a.G : a.R, tiles = used * ((a.N + 15) / 16);
    const int64_t blocks = (a.K * (int64_t)sizeof(T) + 255) / 256, mean = (a.R + a.G - 1) / a.G, most = a.G == 1 ? mean : 2 * mean;
    int waves = 8;
    while (waves > 1 && waves / 2 >= blocks) waves /= 2;
    if (most > 16) return few<T, 1, 2>(a, waves, s);
    if (tiles < 1024) return few<T, 1, 1>(a, waves, s);
    return few<T, 2, 1>(a, waves, s);
}

}  // namespace

// Where tiles of 64 x 128 are too few for the chip: up to 256 of them with up to sixteen rows a group, up to 48 with more
// (floats, whose tiles take longer: 512 and 100).  bf16, tiles and here, us:
//   one group, inner dimension 4,096: 1 row by 4,096 columns (32 tiles) 44, 9.3; 32 rows by 4,096 (32) 42.3, 14.6; 512 rows
//   by 512 (34) 42.1, 27.4; 1,024 rows by 512 (66) 43.0, 54.7; 64 rows by 1,024 (12) 40.3, 14.3
//   few rows a group: 32 experts of 64 for 8 tokens, 4,096 x 1,024 (256) 63, 52; 8 groups of 4 rows, 4,096 x 4,096 (256) 64, 67;
//   16 experts for 32 rows, 2,048 x 4,096 (512) 47, 60
// floats: 32 rows by 4,096 x 4,096 (32) 169, 28.5; 512 rows in 8 groups, 2,048 x 1,024 (96) 90, 73; 512 rows by 1,024 x 2,048 (136) 47, 67.
bool grouped_few_applies(const GroupedArgs& a, int dtype)
{
    if (a.weights_kn || !grouped_fast_applies(a, dtype)) return false;
    const int64_t mean = (a.R + a.G - 1) / a.G, used = a.G < a.R ? a.G : a.R;  // groups that may have rows
    const int64_t down = a.R / 64 + used / 2, tiles = (down > used ? down : used) * ((a.N + 127) / 128);
    if ((a.G == 1 ? mean : 2 * mean) <= 16) return tiles <= (dtype == 0 ? 512 : 256);
    return tiles <= (dtype == 0 ? 100 : 48);
}

hipError_t launch_grouped_few(const GroupedArgs& a, int dtype, hipStream_t s)
{
    switch (dtype) {
        case 0: return by_columns<float>(a, s);
        case 1: return by_columns<half_t>(a, s);
        default: return by_columns<bf16_t>(a, s);
    }
}

}  // namespace sgap
