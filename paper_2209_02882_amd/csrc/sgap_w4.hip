// Products over ragged groups with weights of 4 bits: W[n, k] = (q[n, k] - z[n, k / group]) * s[n, k / group].
//
// Made for few rows a group, where every weight is read for one row or a handful and the bytes of the weights are the
// bound.  A wavefront takes tiles of 16 columns and its share of the inner dimension; the codes of 16 columns by 128
// values lie in 1,024 consecutive bytes (launch_w4_layout puts them there once), 16 bytes to a lane, in the order in
// which the matrix instruction wants them.  No weight is ever rounded: a code goes into the top of the mantissa of the
// number 16 (16 + q, exact in both 16-bit types, one shift and one and-or for two codes), the matrix unit sums
// (16 + q) x and, against ones, x itself over a scale's values in 32 bits, and then
//     acc += s * (-(16 + z) * sum of x + sum of (16 + q) x).
// The wavefronts of a workgroup have shares of the inner dimension and are summed up through LDS at the end.
//
// Where x is infinite or so large that the sums overflow, that difference is no number although the definition may be
// one: an element that comes out not finite is computed again value by value.
#include <type_traits>

#include "sgap_grouped.hpp"

namespace sgap {

namespace {

constexpr int kTileN = 16, kBlockK = 128, kTileBytes = kTileN * kBlockK / 2;

template <typename T>
struct Code;  // 16 as a number of that type, and how far up its mantissa the four bits lie that count 1 to 15
template <>
struct Code<half_t> {
    static constexpr uint32_t kSixteen = 0x4c004c00u, kMask = 0x03c003c0u;
    static constexpr int kShift = 6;
};
template <>
struct Code<bf16_t> {
    static constexpr uint32_t kSixteen = 0x41804180u, kMask = 0x00780078u;
    static constexpr int kShift = 3;
};

// Eight codes to eight numbers 16 + q.  Nibble i holds value 2 i, nibble 4 + i value 2 i + 1 (i = 0 .. 3).
template <typename T>
__device__ __forceinline__ piece_t<T> decode(uint32_t d)
{
    union {
        uint32_t u[4];
        piece_t<T> v;
    } r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int up = Code<T>::kShift - 4 * i;
        const uint32_t x = up >= 0 ? d << (up & 31) : d >> ((-up) & 31);
        r.u[i] = (x & Code<T>::kMask) | Code<T>::kSixteen;
    }
    return r.v;
}

// (the code of column n, value k) of a group's tiles
__device__ __forceinline__ uint32_t code_at(const uint8_t* __restrict__ tiles, int64_t blocks_k, int64_t n, int64_t k)
{
    const int in = (int)(k % kBlockK), step = in >> 5, part = (in >> 3) & 3, j = in & 7;
    const uint8_t* at = tiles + ((n / kTileN) * blocks_k + k / kBlockK) * kTileBytes + (part * 16 + n % kTileN) * 16 + step * 4;
    const int nibble = (j >> 1) + 4 * (j & 1);
    return (at[nibble >> 1] >> (4 * (nibble & 1))) & 15;
}

// scales (and zero points) of a block of 128 values
inline __host__ __device__ int scales_of_block(int group_k) { return group_k >= 128 ? 1 : 128 / group_k; }

// One byte of the laid-out codes, one scale and one zero point per thread and turn.
__global__ __launch_bounds__(256) void w4_layout_kernel(int64_t G, int64_t K, int64_t N, int group_k, bool zeros, W4Sizes z,
                                                        const uint8_t* __restrict__ q, const uint16_t* __restrict__ scales,
                                                        const uint8_t* __restrict__ zero, uint8_t* __restrict__ out)
{
    const int64_t codes = G * z.tiles_n * z.blocks_k * kTileBytes;
    const int64_t steps = (int64_t)gridDim.x * blockDim.x;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < codes; i += steps) {
        const int64_t tile = i / kTileBytes;
        const int in = (int)(i % kTileBytes), lane = in / 16, step = in % 16 / 4, byte = in % 4;
        const int64_t g = tile / (z.tiles_n * z.blocks_k), t = tile % (z.tiles_n * z.blocks_k);
        const int64_t n = t / z.blocks_k * kTileN + lane % 16;
        const int64_t k0 = t % z.blocks_k * kBlockK + step * 32 + lane / 16 * 8;
        uint32_t v = 0;
        for (int h = 0; h < 2; ++h) {
            const int nibble = 2 * byte + h;
            const int64_t k = k0 + 2 * (nibble & 3) + (nibble >> 2);
            uint32_t c = 8;
            if (n < N && k < K) c = (q[(g * N + n) * (K / 2) + k / 2] >> (4 * (k & 1))) & 15;
            v |= c << (4 * h);
        }
        out[i] = (uint8_t)v;
    }
    const int per = scales_of_block(group_k);
    const int64_t many = G * z.tiles_n * z.scales_k * kTileN;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < many; i += steps) {
        // scale s of block (or group) b of column i / per % 16
        const int64_t b = i / per / kTileN % (z.scales_k / per), t = i / kTileN / z.scales_k;
        const int64_t g = t / z.tiles_n, n = t % z.tiles_n * kTileN + i / per % kTileN, s = b * per + i % per;
        const bool there = n < N && s < K / group_k;
        const int64_t from = (g * N + n) * (K / group_k) + s;
        reinterpret_cast<uint16_t*>(out + z.scales_at)[i] = there ? scales[from] : 0;
        if (zeros) (out + z.zeros_at)[i] = there ? zero[from] : 8;
    }
}

// What a wavefront needs of the weights of a block of 128 values: codes of NT tiles and their scales.
template <typename T, int STEPS, int NT, bool ZEROS>
struct W4Block {
    static constexpr int kPer = 4 / STEPS;
    // as they lie in memory: taken apart where they are used, which is what the registers are enough for
    typedef std::conditional_t<kPer == 4, uint64_t, std::conditional_t<kPer == 2, uint32_t, uint16_t>> scales_t;
    typedef std::conditional_t<kPer == 4, uint32_t, std::conditional_t<kPer == 2, uint16_t, uint8_t>> zeros_t;
    uint4 w[NT];
    scales_t scale[NT];
    zeros_t zero[NT];
    __device__ __forceinline__ float scale_of(int nt, int s) const
    {
        const uint16_t bits = (uint16_t)(scale[nt] >> (16 * s));
        return (float)__builtin_bit_cast(T, bits);
    }
    __device__ __forceinline__ float zero_of(int nt, int s) const { return (float)(uint8_t)(zero[nt] >> (8 * s)); }
};

constexpr int kMostWaves = 8;

// NT tiles of columns and MT tiles of 16 rows to a wavefront; STEPS matrix instructions (32 values each) to a scale, or,
// with STEPS = 4, any whole number of blocks of 128.  The wavefronts of the workgroup share the inner dimension; a block's
// loads are on their way while the block before is multiplied.
// STAGED: the rows of X go through LDS, 256 bytes of a row to sixteen lanes, piece p of row r at place p ^ r.  The matrix
// unit wants neighbouring lanes to have different rows, and loads like that take the cache a turn for every lane: with 48
// rows of 8,192 values by 8,192 columns 34 us, 53,000 of a compute unit's 74,000 clocks, where the rows' loads through LDS
// take 16 lanes to one turn.  For rows at addresses that are multiples of 16 bytes; others load as the unit wants them.
template <typename T, int STEPS, int NT, int MT, bool ZEROS, bool STAGED>
__global__ __launch_bounds__(64 * kMostWaves) void grouped_w4_kernel(GroupedW4Args a, W4Sizes z, int64_t column_items,
                                                                              int64_t blocks, bool tail, int64_t block0)
{
    using Block = W4Block<T, STEPS, NT, ZEROS>;
    constexpr int kPer = Block::kPer, kRowBytes = 2 * kBlockK, kStaged = MT * 16 * kRowBytes;
    extern __shared__ __align__(16) char lds[];  // the rows of X, and at the end the sums of all wavefronts
    f32x4(*const part)[64] = reinterpret_cast<f32x4(*)[64]>(lds);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int waves = blockDim.x >> 6, row = lane & 15, piece = lane >> 4;
    const int64_t at0 = block0 + blockIdx.x, g = at0 / column_items, item = at0 - g * column_items;
    const int64_t tile0 = item * NT;
    const uint8_t* __restrict__ tiles = a.weights + g * z.tiles_n * z.blocks_k * kTileBytes;
    const T* __restrict__ scales = reinterpret_cast<const T*>(a.weights + z.scales_at) + g * z.tiles_n * z.scales_k * kTileN;
    const uint8_t* __restrict__ zeros = a.weights + z.zeros_at + g * z.tiles_n * z.scales_k * kTileN;
    const GroupRows gr = group_rows(a.offsets, g, a.R);
    const T* __restrict__ X = static_cast<const T*>(a.X);
    T* __restrict__ Y = static_cast<T*>(a.Y);
    const int64_t scale_groups = z.scales_k / kPer;
    const uint32_t staged = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds + wave * kStaged;
    piece_t<T> ones;
#pragma unroll
    for (int i = 0; i < 8; ++i) ones[i] = (T)1.0f;
    for (int64_t m0 = gr.first + (int64_t)blockIdx.y * 16 * MT; m0 < gr.end; m0 += (int64_t)gridDim.y * 16 * MT) {
        // Lanes behind the last row read it once more, and their results are not stored; a row that does not exist is read
        // from row 0, and zeros are stored.  A lane has MT rows, or, STAGED, four of each MT times sixteen.
        constexpr int kRows = STAGED ? 4 * MT : MT;
        const T* __restrict__ x[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int64_t r = a.from.row(min(m0 + (STAGED ? 4 * i + piece : 16 * i + row), gr.end - 1));
            x[i] = X + (r < 0 ? 0 : r) * a.ldx + (STAGED ? 0 : piece * 8);
        }
        f32x4 acc[NT][MT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) acc[nt][mt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        piece_t<T> xf[MT][4], coming[STAGED ? 1 : MT][4];
        // Offsets of a block are the wavefront's; made anew each time (or the compiler keeps a pointer for every load, and
        // runs out of registers).
        const auto fetch = [&](int64_t kb, Block& b) {
            asm volatile("" : "+s"(kb));
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const int64_t t = min(tile0 + nt, z.tiles_n - 1);  // a tile behind the last is not stored
                b.w[nt] = *reinterpret_cast<const uint4*>(tiles + (t * z.blocks_k + kb) * kTileBytes + lane * 16);
                const int64_t at = (t * scale_groups + (STEPS == 4 && a.group_k > kBlockK ? kb * kBlockK / a.group_k : kb)) * (kTileN * kPer);
                b.scale[nt] = *reinterpret_cast<const typename Block::scales_t*>(scales + at + row * kPer);
                if (ZEROS) b.zero[nt] = *reinterpret_cast<const typename Block::zeros_t*>(zeros + at + row * kPer);
            }
        };
        // Rows of X of a block; STAGED: into LDS.  A step of 32 values that the last block does not have reads the block's
        // first once more: the scales there are zeros, and a row with values that are not finite is computed again below in
        // any case.
        const auto fetch_rows = [&](int64_t kb, bool whole) {
            asm volatile("" : "+s"(kb));
            const int left = whole ? kBlockK : (int)(a.K - kb * kBlockK);
            if constexpr (STAGED) {
#pragma unroll
                for (int i = 0; i < kRows; ++i) {
                    int k = (row ^ ((4 * i + piece) & 15)) * 8;
                    if (k >= left) k &= 31;
                    const T* from = x[i] + kb * kBlockK + k;
                    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                                 :
                                 : "s"(staged + i * 1024), "v"(from)
                                 : "m0", "memory");
                }
            } else {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) coming[mt][i] = load_piece(x[mt] + kb * kBlockK + (i * 32 < left ? i * 32 : 0));
            }
        };
        // STAGED: the rows that have arrived, out of LDS, which is then free for the next
        const auto take_rows = [&] {
            if constexpr (STAGED) {
                typedef __attribute__((address_space(3))) piece_t<T> lds_piece;
                wait_loads();
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        xf[mt][i] = *(const lds_piece*)(uintptr_t)(staged + (mt * 16 + row) * kRowBytes + (((i * 4 + piece) ^ row) << 4));
                asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
            } else {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) xf[mt][i] = coming[mt][i];
            }
        };
        const auto multiply = [&](const Block& b) {
#pragma unroll
            for (int s = 0; s < kPer; ++s) {
                f32x4 sum[MT];
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    sum[mt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int i = 0; i < STEPS; ++i) sum[mt] = mma16(xf[mt][s * STEPS + i], ones, sum[mt]);
                    if (!ZEROS) {
#pragma unroll
                        for (int r = 0; r < 4; ++r) sum[mt][r] *= -24.0f;  // the same zero point for all: 16 + 8
                    }
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const float scale = b.scale_of(nt, s);
                    const float zero = ZEROS ? -16.0f - b.zero_of(nt, s) : 0.0f;
                    const uint32_t d[4] = {b.w[nt].x, b.w[nt].y, b.w[nt].z, b.w[nt].w};
                    f32x4 dot[MT];
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) {  // the sums begin with what the zero point takes away
                        dot[mt] = sum[mt];
                        if (ZEROS) {
#pragma unroll
                            for (int r = 0; r < 4; ++r) dot[mt][r] *= zero;
                        }
                    }
#pragma unroll
                    for (int i = 0; i < STEPS; ++i) {
                        const piece_t<T> wf = decode<T>(d[s * STEPS + i]);
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) dot[mt] = mma16(xf[mt][s * STEPS + i], wf, dot[mt]);
                    }
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            acc[nt][mt][r] = __builtin_fmaf(scale, dot[mt][r], acc[nt][mt][r]);
                    // (or the compiler decodes everything first and runs out of registers)
                    if constexpr (NT * MT > 1) __builtin_amdgcn_sched_barrier(0);
                }
            }
        };
        // blocks wave, wave + waves, .. of the whole ones; the one that is not whole goes to the wavefront whose turn it is
        const int64_t all = blocks + (STEPS < 4 && tail ? 1 : 0);
        if (wave < all) {
            const auto ask = [&](int64_t kb, Block& b) {
                if (kb >= all) return;
                fetch(kb, b);
                fetch_rows(kb, STEPS == 4 || kb < blocks);
            };
            Block one, two;
            int64_t kb = wave;
            ask(kb, one);
            for (;;) {
                take_rows();
                ask(kb + waves, two);
                multiply(one);
                if ((kb += waves) >= all) break;
                take_rows();
                ask(kb + waves, one);
                multiply(two);
                if ((kb += waves) >= all) break;
            }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                __syncthreads();
                part[wave][lane] = acc[nt][mt];
                __syncthreads();
                const int64_t n0 = (tile0 + nt) * kTileN;
                for (int i = threadIdx.x; i < 256; i += blockDim.x) {
                    // element i: row i / 16 of the tile (rows 4 l + r lie with lane part l), column i % 16
                    const int m = i >> 4, n = i & 15, from = (m >> 2) * 16 + n, r = m & 3;
                    float v = 0.0f;
                    for (int w = 0; w < waves; ++w) v += reinterpret_cast<const float*>(&part[w][from])[r];
                    const int64_t at = m0 + mt * 16 + m;
                    if (at >= gr.end || n0 + n >= a.N) continue;
                    const int64_t xr = a.from.src || !__builtin_isfinite(v) ? a.from.row(at) : 0;
                    if (xr < 0) {
                        v = 0.0f;
                    } else if (!__builtin_isfinite(v)) {
                        v = 0.0f;
                        for (int64_t k = 0; k < a.K; ++k) {
                            const int64_t s = k / a.group_k;
                            const int64_t sc = (((tile0 + nt) * scale_groups + s / kPer) * kTileN + n) * kPer + s % kPer;
                            const float zero = ZEROS ? (float)zeros[sc] : 8.0f;
                            const float wv = ((float)code_at(tiles, z.blocks_k, n0 + n, k) - zero) * (float)scales[sc];
                            v = __builtin_fmaf(wv, (float)X[xr * a.ldx + k], v);
                        }
                    }
                    Y[at * a.ldy + n0 + n] = (T)v;
                }
            }
        if constexpr (STAGED) __syncthreads();  // the sums have been read: their place is the next rows'
    }
    // rows behind the last group
    if (a.offsets && g == a.G - 1) {
        const int columns = (int)min((int64_t)NT * kTileN, a.N - tile0 * kTileN);
        for (int64_t r = gr.end + blockIdx.y; r < a.R; r += gridDim.y)
            for (int n = threadIdx.x; n < columns; n += blockDim.x) Y[r * a.ldy + tile0 * kTileN + n] = (T)0.0f;
    }
}

template <typename T, int STEPS, int NT, int MT, bool ZEROS, bool STAGED>
hipError_t launch_as(const GroupedW4Args& a, const W4Sizes& z, int waves, int row_items, hipStream_t s)
{
    const int64_t items = (z.tiles_n + NT - 1) / NT;
    // whole blocks, and one that is not; without a row of X there is nothing to read
    const int64_t blocks = a.from.rows > 0 ? a.K / kBlockK : 0;
    const bool tail = a.from.rows > 0 && a.K % kBlockK;
    static uint64_t allowed = 0;
    constexpr int kEach = STAGED ? MT * 4096 : 1024;
    if (const hipError_t err = allow_lds(grouped_w4_kernel<T, STEPS, NT, MT, ZEROS, STAGED>, kMostWaves * kEach, allowed)) return err;
    return launch_parts(a.G * items, 64 * waves, [&](unsigned grid, int64_t block0) {
        grouped_w4_kernel<T, STEPS, NT, MT, ZEROS, STAGED><<<dim3(grid, (unsigned)row_items), 64 * waves, waves * kEach, s>>>(
            a, z, items, blocks, tail, block0);
    });
}

template <typename T, int STEPS, int NT, int MT>
hipError_t run_w4(const GroupedW4Args& a, const W4Sizes& z, int waves, int row_items, bool staged, hipStream_t s)
{
    if constexpr (MT != 2) {  // two times sixteen rows: staged only
        if (!staged)
            return a.zeros ? launch_as<T, STEPS, NT, MT, true, false>(a, z, waves, row_items, s)
                           : launch_as<T, STEPS, NT, MT, false, false>(a, z, waves, row_items, s);
    }
    return a.zeros ? launch_as<T, STEPS, NT, MT, true, true>(a, z, waves, row_items, s)
                   : launch_as<T, STEPS, NT, MT, false, true>(a, z, waves, row_items, s);
}

template <typename T, int STEPS>
hipError_t by_rows(const GroupedW4Args& a, const W4Sizes& z, hipStream_t s)
{
    const int64_t mean = (a.R + a.G - 1) / a.G;
    const int64_t most = a.G == 1 ? mean : 2 * mean;  // rows that a group has, or has often
    const auto items = [&](int rows) {
        const int64_t n = (most + rows - 1) / rows;
        return (int)(n < 1 ? 1 : n > 64 ? 64 : n);
    };
    // Wavefronts that share the inner dimension: eight where the workgroups alone would not fill the chip, two where they
    // do several times over, so that a wavefront's start is spread over more blocks.  8 groups of 32 rows by 4,096 x 4,096
    // (2,048 workgroups): 8 60 us, 4 41.6, 2 35.6; one row by 8,192 x 8,192 (512): 16 14.7, 8 12.6, 4 14.3; 128 rows by
    // 8,192 x 8,192 (768): 8 55, 4 45, 2 48; 8 experts of 64 (704 that have rows): 4 12.1, 2 15.3.
    const int64_t used = a.G < a.R ? a.G : a.R;  // groups that may have rows
    const auto waves = [&](int columns, int rows) {
        const int64_t groups = used * ((z.tiles_n * kTileN + columns - 1) / columns) * items(rows);
        int w = groups <= 512 ? 8 : groups <= 1024 ? 4 : 2;
        while (w > 1 && w / 2 >= z.blocks_k) w /= 2;
        return w;
    };
    const bool staged = a.ldx % 8 == 0 && (reinterpret_cast<uintptr_t>(a.X) & 15) == 0;
    // One row or two: sixteen lanes of a load share a row, and the way through LDS would only be longer.  Two tiles of
    // columns to a wavefront where that leaves workgroups enough: 64 experts for 64 rows 24.0 us with one, 20.5 with two;
    // 8 groups of 2 rows by 4,096 x 4,096 21.8 and 17.5; 4,096 columns for one row: 4.7 with one.
    if (most <= 16 && used * z.tiles_n < 512) return run_w4<T, STEPS, 1, 1>(a, z, waves(16, 16), items(16), staged && most > 2, s);
    if (most <= 16) return run_w4<T, STEPS, 2, 1>(a, z, waves(32, 16), items(16), staged && most > 2, s);
    if (most <= 32 && staged) return run_w4<T, STEPS, 2, 2>(a, z, waves(32, 32), items(32), staged, s);
    return run_w4<T, STEPS, 2, 3>(a, z, waves(32, 48), items(48), staged, s);
}

template <typename T>
hipError_t by_scale(const GroupedW4Args& a, const W4Sizes& z, hipStream_t s)
{
    if (a.group_k == 32) return by_rows<T, 1>(a, z, s);
    if (a.group_k == 64) return by_rows<T, 2>(a, z, s);
    return by_rows<T, 4>(a, z, s);
}

int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

}  // namespace

W4Sizes w4_sizes(int64_t G, int64_t K, int64_t N, int group_k, bool zeros)
{
    W4Sizes z;
    z.tiles_n = (N + kTileN - 1) / kTileN;
    z.blocks_k = (K + kBlockK - 1) / kBlockK;
    z.scales_k = group_k >= 128 ? K / group_k : z.blocks_k * scales_of_block(group_k);  // whole blocks of them
    const int64_t codes = G * z.tiles_n * z.blocks_k * kTileBytes, many = G * z.tiles_n * z.scales_k * kTileN;
    z.scales_at = up(codes, 256);
    z.zeros_at = z.scales_at + up(2 * many, 256);
    z.bytes = zeros ? z.zeros_at + up(many, 256) : z.zeros_at;
    return z;
}

hipError_t launch_w4_layout(int64_t G, int64_t K, int64_t N, int group_k, const uint8_t* q, const void* scales,
                            const uint8_t* zeros, uint8_t* out, hipStream_t s)
{
    const W4Sizes z = w4_sizes(G, K, N, group_k, zeros != nullptr);
    const int64_t blocks = (z.bytes + 255) / 256;
    w4_layout_kernel<<<(unsigned)(blocks < 65536 ? blocks : 65536), 256, 0, s>>>(
        G, K, N, group_k, zeros != nullptr, z, q, static_cast<const uint16_t*>(scales), zeros, out);
    return hipGetLastError();
}

hipError_t launch_grouped_w4(const GroupedW4Args& args, int dtype, hipStream_t s)
{
    GroupedW4Args a = args;
    // nothing to multiply: zeros, whatever the groups are (they take no memory here, and might be more than can be launched)
    if (a.K == 0) a.G = 1, a.offsets = nullptr;
    const W4Sizes z = w4_sizes(a.G, a.K, a.N, a.group_k, a.zeros);
    return dtype == 1 ? by_scale<half_t>(a, z, s) : by_scale<bf16_t>(a, z, s);
}

}  // namespace sgap
