// Products over ragged groups of numbers of 8 bits with a scale for each block of 128:
//   Y[r, n] = sum over blocks b of xs[src(r), b] * ws[g, n / 128, b] * sum over k in b of X[src(r), k] W[g, n, k]
// Codes lie in rows of whole blocks, zeros behind the last value, so that no step along the inner dimension is cut off.
//
// A block's sum, times the two scales' product, is added to the result: one multiply-add for each result and block.  The sum
// itself is made in one of two ways.
//   codes    the matrix instruction for numbers of 8 bits, a whole block at a time.  It adds eight neighbouring products with 13
//            bits behind the largest one's exponent, cut off, and those sums with 24: with normally distributed codes a result is
//            1.4e-5 of its size off (root mean square), an eightieth of what rounding to bfloat16 is and a tenth of float16's.
//            Every instruction for these codes on this chip does so.  For results of 16 bits of many rows: half of the time (8,192
//            rows, 4,096 x 8,192 256 us, by numbers 504).  What it does to them: of that product bfloat16 is 1.65857e-3 off 64 bits
//            in place of 1.65851e-3, 1.2 % are another number than sums in 32 bits round to, a step away unless a sum comes to little;
//            of 3,001 rows, 1,000 x 1,531, float16 is 2.078e-4 off in place of 2.073e-4, 7 % are another number.  At its worst it
//            cuts off 7 * 2^-13 of each eight's largest product, beside a rounding of 2^-8 (bfloat16) or 2^-11 (float16) of the result.
//   numbers  the codes as bfloat16, which holds them all, and its matrix instruction: exact products, added in 32 bits, at 3.5
//            times the matrix unit's time.  For results of floats, and for few rows, where the weights' bytes are the bound.
//            (So a row may round otherwise in a call of few rows than in one of many.  Two calls alike give the same bits.)
//
// Few rows are bound by the weights' bytes (64 rows over 64 groups, 2,048 x 1,408: 119 MB in 24.1 us, 4.9 TB/s) or, where these are few too,
// by a block's way through the wavefront; many rows by the tiles' loads beside the products: 256 x 256 tiles take 1.46 to 1.83 us a block
// from one run to the next, 1.3 without the products and 1.3 without the loads, and some 9 us to start and to store.  8,192 rows, 4,096 x
// 8,192, 16 bits: 256 to 261 us in a row of passes of it alone, 2.1 PFLOP/s, where the library's product of such numbers with one scale
// reaches 2.5; under the profiler, among other kernels, 270 to 295.  Results of floats: 504 to 514 us, where the product of 16-bit values takes 446.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "sgap_grouped_tiles.hpp"
#include "sgap_tokens.hpp"

namespace sgap {

namespace {

typedef int Codes __attribute__((ext_vector_type(8)));  // 32 codes of a row or column: a lane's share of a block

// A * B over a block on a 16 x 16 tile; lanes and results as mma16's.  (Without scales of the instruction's own.)
__device__ __forceinline__ f32x4 mma_block(Codes a, Codes b)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, f32x4{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0, 0, 0, 0);
}

typedef int HalfCodes __attribute__((ext_vector_type(4)));
__device__ __forceinline__ Codes join(HalfCodes lo, HalfCodes hi) { return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7); }

// The same out of exact products added in 32 bits: the codes as bfloat16, eight to a piece.
struct Numbers {
    piece_t<bf16_t> piece[4];
};
__device__ __forceinline__ Numbers numbers(Codes c)
{
    typedef bf16_t two_t __attribute__((ext_vector_type(2)));
    Numbers n;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const two_t lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)c[i], 1.0f, false);
        const two_t hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)c[i], 1.0f, true);
        n.piece[i >> 1][4 * (i & 1) + 0] = lo[0];
        n.piece[i >> 1][4 * (i & 1) + 1] = lo[1];
        n.piece[i >> 1][4 * (i & 1) + 2] = hi[0];
        n.piece[i >> 1][4 * (i & 1) + 3] = hi[1];
    }
    return n;
}
__device__ __forceinline__ f32x4 mma_block(const Numbers& a, const Numbers& b)
{
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 4; ++i) acc = mma16(a.piece[i], b.piece[i], acc);
    return acc;
}

// what results of type T are made of
template <typename T>
using operand_t = std::conditional_t<std::is_same<T, float>::value, Numbers, Codes>;
template <typename T>
__device__ __forceinline__ operand_t<T> operand(Codes c)
{
    if constexpr (std::is_same<T, float>::value) return numbers(c);
    else return c;
}

template <typename T>
__device__ __forceinline__ void store4(T* __restrict__ y, int64_t n, int64_t N, bool wide, f32x4 v)
{
    typedef T out4 __attribute__((ext_vector_type(4)));
    if (wide && n + 4 <= N) {
        out4 o;
#pragma unroll
        for (int r = 0; r < 4; ++r) o[r] = (T)v[r];
        *reinterpret_cast<out4*>(y + n) = o;
        return;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
        if (n + r < N) y[n + r] = (T)v[r];
}

// Few rows: a workgroup has NT * 16 columns and MT * 16 rows at a time, its wavefronts share the blocks of the inner dimension,
// U of them on their way while U are multiplied; shares are summed up through LDS.
template <typename T, int NT, int MT, int U>
__global__ __launch_bounds__(512) void grouped_f8_few_kernel(GroupedF8Args a, int64_t column_items, bool wide, int64_t block0)
{
    __shared__ f32x4 part[8][NT * MT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int waves = blockDim.x >> 6, row = lane & 15, piece = lane >> 4;
    const int64_t item = block0 + blockIdx.x, g = item / column_items, n0 = (item - g * column_items) * (NT * 16);
    const GroupRows gr = group_rows(a.offsets, g, a.R);
    T* __restrict__ Y = static_cast<T*>(a.Y);
    const int64_t blocks = f8_blocks(a.K), pitch = blocks * kF8Block;
    const uint8_t* __restrict__ w[NT];
    const float* __restrict__ ws[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        // columns and rows past the last are read from the last, and not stored; a row of X that does not exist is read
        // from row 0, and zeros are stored
        w[nt] = a.W + (g * a.N + min(n0 + nt * 16 + row, a.N - 1)) * pitch + piece * 16;
        ws[nt] = a.w_scales + (g * f8_blocks(a.N) + min(n0 + nt * 16, a.N - 1) / kF8Block) * blocks;
    }
    for (int64_t m0 = gr.first + (int64_t)blockIdx.y * 16 * MT; m0 < gr.end; m0 += (int64_t)gridDim.y * 16 * MT) {
        const uint8_t* __restrict__ x[MT];
        const float* __restrict__ xs[MT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            const int64_t r = a.from.row(min(m0 + mt * 16 + row, gr.end - 1));
            x[mt] = a.X + (r < 0 ? 0 : r) * pitch + piece * 16;
            xs[mt] = a.x_scales + (r < 0 ? 0 : r) * blocks;
        }
        f32x4 acc[NT][MT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) acc[nt][mt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        for (int64_t b0 = (int64_t)wave * U; b0 < blocks; b0 += waves * U) {
            Codes wc[U][NT], xc[U][MT];
            float sw[U][NT], sx[U][MT];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                // (in place of a block behind the last, that one, times 0)
                const int64_t b = min(b0 + u, blocks - 1), at = b * kF8Block;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    wc[u][nt] = join(*reinterpret_cast<const HalfCodes*>(w[nt] + at), *reinterpret_cast<const HalfCodes*>(w[nt] + at + 64));
                    sw[u][nt] = ws[nt][b];
                }
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    xc[u][mt] = join(*reinterpret_cast<const HalfCodes*>(x[mt] + at), *reinterpret_cast<const HalfCodes*>(x[mt] + at + 64));
                    sx[u][mt] = xs[mt][b];
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) {
                        const f32x4 p = mma_block(numbers(wc[u][nt]), numbers(xc[u][mt]));
                        const float s = b0 + u < blocks ? sw[u][nt] * sx[u][mt] : 0.0f;
#pragma unroll
                        for (int r = 0; r < 4; ++r) acc[nt][mt][r] = __builtin_fmaf(p[r], s, acc[nt][mt][r]);
                    }
        }
        __syncthreads();  // of the rows before, everything is read
#pragma unroll
        for (int i = 0; i < NT * MT; ++i) part[wave][i][lane] = acc[i / MT][i % MT];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NT * MT; ++i) {
            if (i % waves != wave) continue;
            // lane: row lane % 16, columns 4 * (lane / 16) + 0 .. 3
            f32x4 v = part[0][i][lane];
#pragma unroll
            for (int s = 1; s < 8; ++s)
                if (s < waves) v += part[s][i][lane];
            const int64_t at = m0 + (i % MT) * 16 + row, n = n0 + (i / MT) * 16 + 4 * piece;
            if (at >= gr.end || n >= a.N) continue;
            if (a.from.src && a.from.row(at) < 0) v = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            store4(Y + at * a.ldy, n, a.N, wide, v);
        }
    }
    // rows behind the last group
    if (a.offsets && g == a.G - 1) {
        const int columns = (int)min((int64_t)NT * 16, a.N - n0);
        for (int64_t r = gr.end + blockIdx.y; r < a.R; r += gridDim.y)
            for (int n = threadIdx.x; n < columns; n += blockDim.x) Y[r * a.ldy + n0 + n] = (T)0.0f;
    }
}

// Work items are dealt to the eight dies (workgroup b runs on die b % 8) in runs of neighbours, which share rows of X and weights
// in the die's L2: bands of eight rows of tiles, and down and up in a band by columns, so that a run is a patch of 8 x 4.
constexpr int kRun = 32, kBand = 8;
__device__ __forceinline__ int64_t dealt(uint32_t b)
{
    const uint32_t die = b & 7, at = b >> 3;
    return (int64_t)((at / kRun) * 8 + die) * kRun + at % kRun;
}

// The rows' scales of a block, put into LDS beside the tiles, a float to a lane.
__device__ __forceinline__ void load_scale(uint32_t lds, const void* base, uint32_t offset)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" : : "s"(lds), "v"(offset), "s"(base) : "m0", "memory");
}
__device__ __forceinline__ void load_scale(uint32_t lds, const void* from)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" : : "s"(lds), "v"(from) : "m0", "memory");
}

// What comes before it in the program is done before what comes after it, where these are made or used.
__device__ __forceinline__ void tie(f32x4& made, f32x4& added, Codes& next) { asm volatile("" : "+v"(made), "+v"(added), "+v"(next) : : "memory"); }
__device__ __forceinline__ void tie(f32x4& made, f32x4& added, Numbers& next)
{
    asm volatile("" : "+v"(made), "+v"(added), "+v"(next.piece[0]), "+v"(next.piece[1]), "+v"(next.piece[2]), "+v"(next.piece[3]) : : "memory");
}

// Until no more than N of this wavefront's loads are on their way.
template <int N>
__device__ __forceinline__ void wait_but()
{
    asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}

// acc += the products of `blocks` blocks.  STAGES of a block's tiles; the loads of a block have the STAGES - 1 before it to
// arrive in, its fragments the products before them, and a product is added to the result while the next ones are made.
// A block has two halves.  In the first the columns' fragments stay and half of the rows' pass, while those of the other half are
// read; then one barrier says that everyone has read the stage, which is filled next, and that the other one is full; in the
// second half the rows' fragments stay, and each of the columns' makes place for the next block's as soon as it has been used:
// so there are always products to make while the next block's first fragments are read, which all wavefronts do at a time.
//   load(t, stage, i)   starts load i of LOADS of block t; every wavefront has so many
//   ACTIVE: this wavefront has products to make
//   real: blocks of them that count, the others (of the last team) are multiplied by 0
template <typename T, int MI, int NJ, int STAGES, int LOADS, bool ACTIVE, typename F>
__device__ __forceinline__ void multiply_blocks(uint32_t lds, uint32_t stage_bytes, int blocks, int real, F&& load, const float* w_scales, uint32_t wbase,
                                                uint32_t xbase, uint32_t sbase, f32x4 (&acc)[MI][NJ])
{
    constexpr int H = NJ / 2;
    static_assert(NJ % 2 == 0, "");
    // (the same in every lane, and nobody writes them)
    const __attribute__((address_space(4))) float* const w_scale = (const __attribute__((address_space(4))) float*)w_scales;
    typedef __attribute__((address_space(3))) HalfCodes lds_piece;
    typedef __attribute__((address_space(3))) float lds_float;
    const auto fragment = [](uint32_t base, int i) {
        return operand<T>(join(*(const lds_piece*)(uintptr_t)(base + i * 2048), *(const lds_piece*)(uintptr_t)((base ^ 64) + i * 2048)));
    };
    const auto scale = [](uint32_t base, int j) { return *(const lds_float*)(uintptr_t)(base + j * 64); };
    operand_t<T> w[MI], x[2], held[H];
    f32x4 p[H];  // of the columns before, made and not yet added
    float s[H], held_s[H];
#pragma unroll
    for (int i = 0; i < H; ++i) p[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < H; ++j) held_s[j] = 0.0f;
#pragma unroll
    for (int b = 0; b < STAGES; ++b) {
        if (b >= blocks) break;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) load(b, lds + b * stage_bytes, i);
    }
    float sw = real > 0 ? w_scale[0] : 0.0f;
    // (also until the compiler's own loads have arrived)
    if (blocks >= STAGES) wait_but<(STAGES - 1) * LOADS>();
    else wait_loads();
    __syncthreads();
    if constexpr (ACTIVE) {
#pragma unroll
        for (int i = 0; i < MI; ++i) w[i] = fragment(wbase, i);
        x[0] = fragment(xbase, 0);
        s[0] = scale(sbase, 0);
    }
    const auto add = [&](f32x4& to, const f32x4& made, float by) {
#pragma unroll
        for (int r = 0; r < 4; ++r) to[r] = __builtin_fmaf(made[r], by, to[r]);
    };
    uint32_t other = 0;
    for (int t = 0; t < blocks; ++t) {
        const uint32_t stage = other;
        other = other == (STAGES - 1) * stage_bytes ? 0 : other + stage_bytes;
        uint32_t xb = xbase + stage, sb = sbase + stage;
        asm volatile("" : "+v"(xb), "+v"(sb));  // made anew each time, not kept in registers
        const float sw_next = t + 1 < real ? w_scale[t + 1] : 0.0f;
        f32x4 q[MI];
#pragma unroll
        for (int j = 0; j < H; ++j) {
            if constexpr (ACTIVE) {
                if (j + 1 < H) {
                    x[(j + 1) & 1] = fragment(xb, j + 1);
                    s[j + 1] = scale(sb, j + 1);
                }
                held[j] = fragment(xb, H + j);
                s[j] *= sw;
#pragma unroll
                for (int i = 0; i < MI; ++i) {
                    const f32x4 made = mma_block(w[i], x[j & 1]);
                    // the last columns of the block before, then the rows before
                    f32x4& to = j == 0 ? acc[MI - 1][H + i % H] : acc[i][j - 1];
                    if (j == 0 && i < H) add(to, p[i], held_s[i]);
                    if (j > 0) add(to, q[i], s[j - 1]);
                    q[i] = made;
                    tie(q[i], to, w[(i + 1) % MI]);
                }
            }
        }
        if constexpr (ACTIVE) {
#pragma unroll
            for (int j = 0; j < H; ++j) held_s[j] = scale(sb, H + j) * sw;
        }
        if (STAGES > 2 && t + STAGES <= blocks) wait_but<(STAGES - 2) * LOADS>();
        else wait_loads();
        __syncthreads();
        uint32_t wn = wbase + other, xn = xbase + other;
        asm volatile("" : "+v"(wn), "+v"(xn));
#pragma unroll
        for (int i = 0; i < MI; ++i) {
#pragma unroll
            for (int j = 0; j < H; ++j) {
                constexpr int kSteps = MI * H;
                if (t + STAGES < blocks) {
#pragma unroll
                    for (int l = (i * H + j) * LOADS / kSteps; l < (i * H + j + 1) * LOADS / kSteps; ++l) load(t + STAGES, lds + stage, l);
                }
                if constexpr (ACTIVE) {
                    const f32x4 made = mma_block(w[i], held[j]);
                    // the last rows of the first half, then the columns before
                    f32x4& to = i == 0 ? acc[j % MI][H - 1] : acc[i - 1][H + j];
                    if (i == 0) add(to, q[j % MI], s[H - 1]);
                    else add(to, p[j], held_s[j]);
                    p[j] = made;
                    tie(p[j], to, held[(j + 1) % H]);
                }
            }
            if constexpr (ACTIVE) {
                if (i == 0) {
                    // (where there are more columns than rows to a half)
#pragma unroll
                    for (int r = H; r < MI; ++r) add(acc[r][H - 1], q[r], s[H - 1]);
                }
                w[i] = fragment(wn, i);  // behind the last block: not used
                if (i == (MI > 1 ? MI - 2 : 0)) {
                    x[0] = fragment(xn, 0);
                    s[0] = scale(sbase + other, 0);
                }
            }
        }
        sw = sw_next;
    }
    if constexpr (ACTIVE) {
#pragma unroll
        for (int j = 0; j < H; ++j) add(acc[MI - 1][H + j], p[j], held_s[j]);
    }
}

// Many rows: tiles of BM rows by BN columns, a block of the inner dimension at a time, by loads straight into LDS.
// FAR: rows are gathered that lie further than 32 bits of bytes from X's first.  Results of floats go by numbers, others by codes.
// TEAMS: 2 where a tile is all that a compute unit has: each team has half of the blocks, stages of its own, and the shares are added
// through LDS.  (A block's chain of fragments, products and a barrier takes 0.55 us however few wavefronts there are: 256 rows, 4,096
// by 4,096 25.6 us, 16.1 by teams with three stages each, 20.2 with three stages and one team.)
// (Two wavefronts to a SIMD: with more registers than that leaves, the compiler has the matrix unit write to those that no vector
// instruction reads, and waits for each product: 64 x 128 tiles took 0.68 us a block.)
template <typename T, int BM, int BN, int STAGES, bool FAR, int THREADS, int TEAMS>
__global__ __launch_bounds__(THREADS * TEAMS, 2) void grouped_f8_tiles_kernel(GroupedF8Args a, int64_t column_tiles, int64_t items, int64_t block0)
{
    using Wt = Tile<uint8_t, BN, true, THREADS, TEAMS>;
    using Xt = Tile<uint8_t, BM, true, THREADS, TEAMS>;
    constexpr int kWaves = THREADS / 64, WN = kWaves / 2, WM = 2;
    constexpr int MI = BN / WN / 16, NJ = BM / WM / 16;
    constexpr uint32_t kStage = Wt::kBytes + Xt::kBytes + BM * 4;
    extern __shared__ __align__(16) char lds_bytes[];
    const int64_t item = block0 + dealt(blockIdx.x);
    if (item >= items) return;
    const int64_t band = item / (kBand * column_tiles), in = item - band * (kBand * column_tiles);
    const int64_t tile = band * kBand + in % kBand, n0 = in / kBand * BN;
    const RowTile rows = find_row_tile<BM>(a.offsets, a.G, a.R, tile);
    if (rows.rows <= 0) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(Wt::thread() >> 6);
    const int team = TEAMS == 1 ? 0 : __builtin_amdgcn_readfirstlane((int)threadIdx.x / THREADS);
    const int wn = (wave % WN) * (BN / WN), wm = (wave / WN) * (BM / WM);
    const int64_t blocks = f8_blocks(a.K), pitch = blocks * kF8Block;
    f32x4 acc[MI][NJ];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (rows.g < a.G) {
        // columns and rows past the last are read from the last, and not stored; a row of X that does not exist is read
        // from row 0, and zeros are stored
        const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds_bytes + team * (STAGES * kStage);
        // a team has so many blocks of the inner dimension, from this one on; behind the last one it loads that again
        const int share = ((int)blocks + TEAMS - 1) / TEAMS, block_first = team * share, last = (int)blocks - 1;
        const uint8_t* const W = uniform(a.W + (rows.g * a.N + n0) * pitch);
        // of X a byte's place, or, FAR, the row
        uint32_t wo[Wt::kRounds], xo[Xt::kRounds];
#pragma unroll
        for (int i = 0; i < Wt::kRounds; ++i) wo[i] = (uint32_t)(min((int64_t)Wt::major(i), a.N - 1 - n0) * pitch + Wt::minor(i) * 16);
        // rows of X from the first of the tile on, or, gathered, from X's
        const int64_t x_first = a.from.src ? 0 : rows.first;
        const uint8_t* const X = uniform(a.X + x_first * pitch);
        const float* const xs = uniform(a.x_scales + x_first * blocks);
        const auto row = [&](int i) {
            const int64_t r = a.from.src ? a.from.row(rows.first + min(i, rows.rows - 1)) : min(i, rows.rows - 1);
            return r < 0 ? 0 : r;
        };
#pragma unroll
        for (int i = 0; i < Xt::kRounds; ++i) {
            const int64_t r = row(Xt::major(i));
            xo[i] = FAR ? (uint32_t)r : (uint32_t)(r * pitch + Xt::minor(i) * 16);
        }
        // a wavefront loads the scales of 64 rows (where there are more wavefronts than that, some the same ones)
        const int scales0 = wave * 64 % BM;
        const int64_t scale_row = row(scales0 + lane);
        const uint32_t so = FAR ? (uint32_t)scale_row : (uint32_t)(scale_row * blocks * 4);
        const float* const sw = uniform(a.w_scales + (rows.g * f8_blocks(a.N) + min(n0 + wn, a.N - 1) / kF8Block) * blocks + block_first);
        constexpr int kLoads = Wt::kRounds + Xt::kRounds + 1;
        const auto load = [&](int t, uint32_t to, int i) {
            const int r = i - Wt::kRounds;
            if constexpr (TEAMS > 1) t = min(block_first + t, last);
            if (i < Wt::kRounds) {
                Wt::load(to, i, uniform(W + (int64_t)t * kF8Block), wo[i]);
            } else if (r < Xt::kRounds) {
                if constexpr (FAR) Xt::load(to + Wt::kBytes, r, X + (int64_t)xo[r] * pitch + Xt::minor(r) * 16 + (int64_t)t * kF8Block);
                else Xt::load(to + Wt::kBytes, r, uniform(X + (int64_t)t * kF8Block), xo[r]);
            } else {
                const uint32_t at = __builtin_amdgcn_readfirstlane(to + Wt::kBytes + Xt::kBytes + scales0 * 4);
                if constexpr (FAR) load_scale(at, xs + (int64_t)so * blocks + t);
                else load_scale(at, uniform(xs + t), so);
            }
        };
        const uint32_t wbase = lds + Wt::lane_base(wn), xbase = lds + Wt::kBytes + Xt::lane_base(wm);
        const uint32_t sbase = lds + Wt::kBytes + Xt::kBytes + (wm + (lane & 15)) * 4;
        if (wm < rows.rows) multiply_blocks<T, MI, NJ, STAGES, kLoads, true>(lds, kStage, share, min(share, last + 1 - block_first), load, sw, wbase, xbase, sbase, acc);
        else multiply_blocks<T, MI, NJ, STAGES, kLoads, false>(lds, kStage, share, min(share, last + 1 - block_first), load, sw, wbase, xbase, sbase, acc);
    }
    // Through LDS, each wavefront its own part, so that rows leave in whole lines: 16-byte chunk c of row r at place c ^ (r & 7).
    constexpr int kColumns = BN / WN, kRows = BM / WM, P = Piece<T>::kCount, kChunks = kColumns / P;
    static_assert(kRows * kColumns * (int)sizeof(T) * kWaves <= STAGES * (int)kStage && kChunks >= 8, "");
    typedef __attribute__((address_space(3))) char lds_char;
    typedef T out4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) out4 lds_out4;
    typedef __attribute__((address_space(3))) piece_t<T> lds_piece;
    lds_char* const part = (lds_char*)lds_bytes + wave * (kRows * kColumns * (int)sizeof(T));
    __syncthreads();  // everyone has read what lies there
    if constexpr (TEAMS > 1) {
        // the second team's share, by way of its own part of LDS
        static_assert(TEAMS == 2 && MI * NJ * THREADS * 16 <= STAGES * (int)kStage, "");
        typedef __attribute__((address_space(3))) f32x4 lds_f32x4;
        lds_f32x4* const shares = (lds_f32x4*)((lds_char*)lds_bytes + STAGES * kStage) + Wt::thread();
        if (team == 1) {
#pragma unroll
            for (int i = 0; i < MI * NJ; ++i) shares[i * THREADS] = acc[i / NJ][i % NJ];
        }
        __syncthreads();
        if (team == 1) return;
#pragma unroll
        for (int i = 0; i < MI * NJ; ++i) acc[i / NJ][i % NJ] += shares[i * THREADS];
    }
    const int real_rows = min(rows.rows - wm, kRows);
    if (real_rows <= 0) return;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
        const int m = 16 * j + (lane & 15);
        const bool real = rows.g < a.G && m < real_rows && (!a.from.src || a.from.row(rows.first + wm + m) >= 0);
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const int n = 16 * i + 4 * (lane >> 4);
            out4 o;
#pragma unroll
            for (int r = 0; r < 4; ++r) o[r] = (T)(real ? acc[i][j][r] : 0.0f);
            *(lds_out4*)(part + m * (kColumns * (int)sizeof(T)) + (((n / P) ^ (m & 7)) * P + n % P) * (int)sizeof(T)) = o;
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    constexpr int kAtOnce = 64 / kChunks;  // rows
    const int chunk = lane % kChunks;
    const int64_t n = n0 + wn + chunk * P;
    T* __restrict__ y = static_cast<T*>(a.Y) + (rows.first + wm) * a.ldy + n;
    for (int m = lane / kChunks; m < real_rows; m += kAtOnce) {
        const piece_t<T> v = *(const lds_piece*)(part + m * (kColumns * (int)sizeof(T)) + (chunk ^ (m & 7)) * 16);
        if (n + P <= a.N) {
            store_piece(y + m * a.ldy, v);
        } else {
#pragma unroll
            for (int i = 0; i < P; ++i)
                if (n + i < a.N) y[m * a.ldy + i] = v[i];
        }
    }
}

template <typename T, int NT, int MT, int U>
hipError_t run_few(const GroupedF8Args& a, bool wide, hipStream_t s)
{
    const int64_t columns = (a.N + NT * 16 - 1) / (NT * 16), blocks = f8_blocks(a.K);
    const int waves = (int)std::min<int64_t>(8, std::max<int64_t>(1, (blocks + U - 1) / U));
    // (groups differ in length: most of the longer ones pass at a time too)
    const int64_t rows = a.offsets ? std::max<int64_t>(1, a.R * 8 / (a.G * 5)) : a.R;
    const unsigned down = (unsigned)std::min<int64_t>(64, (rows + 16 * MT - 1) / (16 * MT));
    return launch_parts(a.G * columns, 512 * (int)down, [&](unsigned grid, int64_t block0) {
        grouped_f8_few_kernel<T, NT, MT, U><<<dim3(grid, down), waves * 64, 0, s>>>(a, columns, wide, block0);
    });
}

template <typename T, int BM, int BN, int STAGES, bool FAR, int THREADS, int TEAMS = 1>
hipError_t run_tiles(const GroupedF8Args& a, hipStream_t s)
{
    const int64_t columns = (a.N + BN - 1) / BN, bands = (most_row_tiles(a.G, a.R, BM, a.offsets != nullptr) + kBand - 1) / kBand;
    const int64_t items = columns * bands * kBand;
    constexpr int kLds = TEAMS * STAGES * (128 * (BM + BN) + BM * 4);
    static uint64_t allowed = 0;
    if (const hipError_t err = allow_lds(grouped_f8_tiles_kernel<T, BM, BN, STAGES, FAR, THREADS, TEAMS>, kLds, allowed)) return err;
    return launch_parts((items + 255) / 256 * 256, THREADS * TEAMS, [&](unsigned grid, int64_t block0) {
        grouped_f8_tiles_kernel<T, BM, BN, STAGES, FAR, THREADS, TEAMS><<<grid, THREADS * TEAMS, kLds, s>>>(a, columns, items, block0);
    });
}

template <typename T>
hipError_t grouped_f8(const GroupedF8Args& a, const GroupedF8Plan& p, hipStream_t s)
{
    // (the address and the row's length that stores of four results ask for)
    const bool wide = a.ldy % 4 == 0 && (reinterpret_cast<uintptr_t>(a.Y) & (4 * sizeof(T) - 1)) == 0;
    if (p.teams == 0) {
        if (p.rows == 32) return run_few<T, 2, 2, 2>(a, wide, s);
        return p.deep ? run_few<T, 1, 1, 8>(a, wide, s) : run_few<T, 1, 1, 4>(a, wide, s);
    }
    if constexpr (sizeof(T) == 2) {
        if (p.rows == 256) return run_tiles<T, 256, 256, 2, false, 512>(a, s);
    }
    if (p.far) return run_tiles<T, 128, 128, 2, true, 256>(a, s);
    if (p.teams == 2) {
        // (results of floats are bound by the conversion of the codes: a third stage gains them nothing)
        if (p.rows == 128) return run_tiles<T, 128, 128, 2, false, 256, 2>(a, s);
        return run_tiles<T, 64, 128, sizeof(T) == 2 ? 3 : 2, false, 256, 2>(a, s);
    }
    return p.rows == 128 ? run_tiles<T, 128, 128, 2, false, 256>(a, s) : run_tiles<T, 64, 128, 2, false, 256>(a, s);
}

}  // namespace

// The least of what the kernels are reckoned to take, in us.  Few rows: a compute unit has n workgroups one after the other, each so
// much and so much a block of the inner dimension (less where the 16 rows are not as many), and not less than the weights' bytes.
// Tiles: n of them, each so much a block and so much besides; where n is 1 two teams share the blocks, unless these are fewer than
// eight.  A group has a last tile that is not full: half a tile more than its rows in the mean; and groups differ in length, so that
// some unit has a fifth more than the mean.
// Measured (us; few rows 16, 32; tiles of 64, 64 by teams, 128, 128 by teams, 256 rows), inner dimension by columns, 16-bit results,
// groups of very different length:
//   1 row, 4,096 x 4,096                      6.2   8.6  19.1  14.0  25.3  20.3  39.9
//   32 rows, 8,192 x 8,192                   40.0  26.6  51.8  26.3  59.2  37.5  75.1
//   64 groups, 64 rows, 2,048 x 1,408        24.9  31.9  23.8  26.4  26.2  33.0  29.6
//   256 rows, 4,096 x 4,096                  79.8  40.0  25.6  16.1  30.5  24.8  51.9
//   1,024 rows, 4,096 x 4,096                 301   147  29.4  31.8  33.3  27.1  54.1
//   2,048 rows, 4,096 x 4,096                 568   288  61.1  61.1  42.8  51.3  63.8
//   64 groups, 8,192 rows, 2,048 x 1,408      409   258  73.1  86.6  79.1  92.3  75.5
//   16 groups, 16,384 rows, 2,048 x 4,096       -     -   249   366   219   309   193
// Over 140 calls of such sizes and sizes between them the choice took 3% more than the best.
GroupedF8Plan plan_grouped_f8(const GroupedF8Args& a, int dtype)
{
    const bool half = dtype != 0, groups = a.offsets != nullptr;
    const double blocks = (double)f8_blocks(a.K), used = groups ? (double)std::min(a.G, std::max<int64_t>(a.R, 1)) : 1.0;
    const double rows = (double)a.R / used, bytes = used * (double)a.K * (double)a.N / 5.7e6;  // the weights', once
    GroupedF8Plan p = {0, 16, 16, false, false};
    p.far = a.from.src && a.from.rows * f8_blocks(a.K) * kF8Block > 1ll << 32;
    const auto down = [&](int size) { return used == 1.0 ? std::ceil(rows / size) : std::max(1.0, rows / size + 0.5); };
    const auto few = [&](int size, double besides, double block, double& n) {
        n = used * down(size) * std::ceil((double)a.N / size) / a.compute_units;
        return 3.0 + std::max(bytes * down(size) * 0.9, (besides + block * blocks) * std::max(std::ceil(n), 1.0));
    };
    double n16, n32;
    const double few16 = few(16, 0.57, 0.06 + 0.06 * std::min(1.0, rows / 8), n16), few32 = few(32, 1.46, 0.242, n32);
    if (few32 < few16) p.rows = p.columns = 32;
    // eight blocks on their way in place of four where that leaves wavefronts enough (7 groups, 18 rows, 3,021 x 1,902: 10.5 us, 12.7)
    p.deep = p.rows == 16 && n16 >= 3.0 && blocks >= 16;
    // 128 lines of an operand have to lie within 32 bits of bytes
    constexpr int64_t kLongest = 1 << 22;
    if (a.K == 0 || a.K > kLongest) return p;
    double least = std::min(few16, few32);
    // a tile costs `block` a block, `only` the only one of a compute unit, and `team` shared by two teams (0: not with them)
    const auto tiles = [&](int size, int columns, double block, double only, double team, double besides) {
        const double all = used == 1.0 ? std::ceil((double)a.R / size) : (double)a.R / size + 0.6 * used;
        const double n = std::ceil(all * std::ceil((double)a.N / columns) / a.compute_units);
        const int teams = n == 1.0 && blocks >= 8 && team > 0.0 ? 2 : 1;
        const double work = n > 1.0 ? n * (block * blocks + besides) : (teams == 2 ? team : only) * blocks + 4.0;
        const double time = (used > 1.0 ? 1.2 : 1.0) * std::max(work, bytes + 2.5);
        if (time >= least) return;
        least = time;
        p.teams = teams;
        p.rows = size;
        p.columns = columns;
        p.deep = false;
    };
    if (!p.far) tiles(64, 128, half ? 0.48 : 0.6, half ? 0.58 : 0.8, half ? 0.4 : 0.61, 0.4);
    tiles(128, 128, half ? 0.72 : 1.02, half ? 0.88 : 1.25, p.far ? 0.0 : half ? 0.66 : 1.02, 1.4);
    if (half && !p.far) tiles(256, 256, 1.67, 1.67, 0.0, 9.0);
    return p;
}

hipError_t launch_grouped_f8(GroupedF8Args a, int dtype, hipStream_t s)
{
    if (a.from.rows == 0) a.K = 0;  // no row of X: zeros, and nothing is read
    const GroupedF8Plan p = plan_grouped_f8(a, dtype);
    switch (dtype) {
        case 0: return grouped_f8<float>(a, p, s);
        case 1: return grouped_f8<half_t>(a, p, s);
        default: return grouped_f8<bf16_t>(a, p, s);
    }
}

}  // namespace sgap
