// Products over ragged groups where rows are multiples of 16 bytes at 16-byte addresses:
//   Y[r, :]  = X[src(r), :] * op(W[g])              r in group g; W[g] is N x K or K x N
//   dW[g]    = sum over the rows r of g of dY[r, :] (x) X[src(r), :]
//
// A workgroup has a tile of the result and goes along the inner dimension 128 bytes at a time; both operands' pieces go
// from memory straight into LDS, the next ones while the present are multiplied.  Bound by the matrix instructions where
// rows are many: what is lost to them is the reads of LDS between them, a tile's first wait and its store, and the part of
// every group's last tile that has no rows.  16 groups, 16,384 rows, 4,096 by 2,048, bf16 (275 GF each): the product 315 us
// (870 TF/s), the gradient of X 313 us, of W 350 us; one group of 8,192 rows, 4,096 by 8,192: 1,310 TF/s, where the library's
// product reaches 1,540.  Floats, 4,096 rows in 8 groups, 1,024 by 1,024, in parts of 16 bits: 90, 91 and 75 us, 8.6 GF each.
// Bound by the weights' bytes where rows are few: 16 experts for 32 rows, 2,048 by 4,096, bf16: 47.6 us, 5.0 TB/s.
#include <algorithm>
#include <type_traits>

#include "sgap_grouped_tiles.hpp"

namespace sgap {

namespace {

// Work items are dealt to the eight dies (workgroup b runs on die b % 8) in runs of RUN neighbours, which share rows of X
// or weights in the die's L2.  Runs in turn, so that the items that turn out not to exist, all at the end, leave no die idle.
template <int RUN>
__device__ __forceinline__ int64_t dealt_item(uint32_t b)
{
    const uint32_t die = b & 7, at = b >> 3;
    return (int64_t)((at / RUN) * 8 + die) * RUN + at % RUN;
}
// so many of a product's tiles, and so many of a gradient's: its groups' tiles differ in length, so that every die should
// have some of each (16 groups of 128 tiles)
constexpr int kRun = 32, kGradientRun = 16;

// Floats in parts, left to the compiler, have 262 registers and half the wavefronts: 565 us in place of 425 for 32,768 rows in 8
// groups, 1,024 by 1,024.
template <typename T>
constexpr int kWavesToSimd = sizeof(T) == 4 ? 2 : 1;

// WIDE: rows of X lie further than 32 bits of bytes from its first.
template <typename T, int BM, int BN, bool KN, bool WIDE, int THREADS>
__global__ __launch_bounds__(THREADS, kWavesToSimd<T>) void grouped_fast_kernel(GroupedArgs a, int64_t column_tiles, int64_t items, bool apart, int64_t block0)
{
    using Wt = Tile<T, BN, !KN, THREADS>;
    using Xt = Tile<T, BM, true, THREADS>;
    constexpr int kWaves = THREADS / 64, WN = kWaves / 2, WM = 2;
    constexpr int MI = BN / WN / 16, NJ = BM / WM / 16;
    extern __shared__ __align__(16) char lds[];
    const int64_t item = block0 + dealt_item<kRun>(blockIdx.x);
    if (item >= items) return;
    const int64_t tile = item / column_tiles, n0 = (item - tile * column_tiles) * BN;
    const RowTile rows = find_row_tile<BM>(a.offsets, a.G, a.R, tile);
    if (rows.rows <= 0) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wn = (wave % WN) * (BN / WN), wm = (wave / WN) * (BM / WM);
    const bool active = rows.g < a.G && wm < rows.rows;
    f32x4 acc[MI][NJ];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (rows.g < a.G) {
        // columns and rows past the last are read from the last, and not stored; a row of X that does not exist is read
        // from row 0, and zeros are stored
        const char* const W = uniform(reinterpret_cast<const char*>(static_cast<const T*>(a.W) + rows.g * a.N * a.K + (KN ? n0 : n0 * a.K)));
        const char* const X = static_cast<const char*>(a.X);
        uint32_t wo[Wt::kRounds];
        uint32_t xo[Xt::kRounds];
        const char* xp[Xt::kRounds];
#pragma unroll
        for (int i = 0; i < Wt::kRounds; ++i) {
            if constexpr (!KN) wo[i] = (uint32_t)((min((int64_t)Wt::major(i), a.N - 1 - n0) * a.K + Wt::minor(i) * Wt::P) * sizeof(T));
            else wo[i] = (uint32_t)((Wt::major(i) * a.N + min((int64_t)Wt::minor(i) * Wt::P, a.N - Wt::P - n0)) * sizeof(T));
        }
#pragma unroll
        for (int i = 0; i < Xt::kRounds; ++i) {
            int64_t r = a.from.row(rows.first + min(Xt::major(i), rows.rows - 1));
            r = ((r < 0 ? 0 : r) * a.ldx + Xt::minor(i) * Xt::P) * (int64_t)sizeof(T);
            if constexpr (WIDE) xp[i] = X + r;
            else xo[i] = (uint32_t)r;
        }
        const int tiles = (int)((a.K + Wt::kInner - 1) / Wt::kInner);
        // APART: where the weights pass once, workgroups begin at different tiles of the inner dimension.  Rows of weights a
        // power of two apart lie in the same memory channels, and all workgroups would ask for the same ones at a time.
        const int begin = apart ? __builtin_amdgcn_readfirstlane((int)(item % tiles)) : 0;
        const auto start_of = [&](int t) { return (int64_t)(t + begin < tiles ? t + begin : t + begin - tiles) * Wt::kInner; };
        // inner values that tile t has
        const auto left = [&](int t) { return (int)min((int64_t)Wt::kInner, a.K - start_of(t)); };
        const auto load = [&](int t, uint32_t to, int i) {
            const int64_t k0 = start_of(t);
            if (i < Wt::kRounds) {
                const char* const w = uniform(W + (KN ? k0 * a.N : k0) * (int64_t)sizeof(T));
                const bool there = (KN ? Wt::major(i) : Wt::minor(i) * Wt::P) < left(t);
                // the tile's first inner values are there
                const uint32_t first = KN ? wo[i] - Wt::major(i) * (uint32_t)(a.N * sizeof(T)) : wo[i] - Wt::minor(i) * 16u;
                Wt::load(to, i, w, there ? wo[i] : first);
            } else {
                const int r = i - Wt::kRounds;
                const int64_t x = k0 * (int64_t)sizeof(T);
                const uint32_t back = Xt::minor(r) * Xt::P < left(t) ? 0u : Xt::minor(r) * 16u;
                if constexpr (WIDE) Xt::load(to + Wt::kBytes, r, xp[r] + x - back);
                else Xt::load(to + Wt::kBytes, r, uniform(X + x), xo[r] - back);
            }
        };
        const auto mend = [&](int t, uint32_t to) {
            const int there = left(t);
            if (there == Wt::kInner) return;
#pragma unroll
            for (int i = 0; i < Wt::kRounds; ++i)
                if ((KN ? Wt::major(i) : Wt::minor(i) * Wt::P) >= there) Wt::clear(to, i);
#pragma unroll
            for (int i = 0; i < Xt::kRounds; ++i)
                if (Xt::minor(i) * Xt::P >= there) Xt::clear(to + Wt::kBytes, i);
        };
        bool done = false;
        if constexpr (sizeof(T) == 4) {
            multiply_tiles_split<Wt, Xt, MI, NJ>(lds, tiles, load, mend, wn, wm, active, acc);
            done = !start_over(acc);
        }
        if (!done) multiply_tiles<Wt, Xt, MI, NJ>(lds, tiles, load, mend, wn, wm, active, acc);
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
        const int m = wm + 16 * j + (lane & 15);
        if (m >= rows.rows) continue;
        const bool real = rows.g < a.G && (!a.from.src || a.from.row(rows.first + m) >= 0);
        T* __restrict__ y = static_cast<T*>(a.Y) + (rows.first + m) * a.ldy;
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const int64_t n = n0 + wn + 16 * i + 4 * (lane >> 4);
            typedef T out4 __attribute__((ext_vector_type(4)));
            if (n < a.N) {
                out4 o;
#pragma unroll
                for (int r = 0; r < 4; ++r) o[r] = (T)(real ? acc[i][j][r] : 0.0f);
                *reinterpret_cast<out4*>(y + n) = o;
            }
        }
    }
}

// The gradient of the weights.  The inner dimension is the group's rows; both operands have their lines contiguous, and
// the first has the result's contiguous dimension.
template <typename T, int BM, int BN, bool KN, bool WIDE, int THREADS>
__global__ __launch_bounds__(THREADS, kWavesToSimd<T>) void grouped_wgrad_fast_kernel(GroupedArgs a, int64_t tiles_m, int64_t tiles_n, int64_t items,
                                                                       int64_t block0)
{
    using Lt = Tile<T, BN, false, THREADS>;
    using Rt = Tile<T, BM, false, THREADS>;
    using Xt = std::conditional_t<KN, Rt, Lt>;
    using Yt = std::conditional_t<KN, Lt, Rt>;
    constexpr int kWaves = THREADS / 64, WN = kWaves / 2, WM = 2;
    constexpr int MI = BN / WN / 16, NJ = BM / WM / 16;
    constexpr int kXAt = KN ? Lt::kBytes : 0, kYAt = KN ? 0 : Lt::kBytes;
    extern __shared__ __align__(16) char lds[];
    const int64_t item = block0 + dealt_item<kGradientRun>(blockIdx.x);
    if (item >= items) return;
    const int64_t per = tiles_m * tiles_n, g = item / per, in = item - g * per;
    const int64_t lines = KN ? a.K : a.N, columns = KN ? a.N : a.K;  // of the result
    const int64_t m0 = in / tiles_n * BM, n0 = in % tiles_n * BN;
    const int64_t x0 = KN ? m0 : n0, y0 = KN ? n0 : m0;
    const GroupRows gr = group_rows(a.offsets, g, a.R);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wn = (wave % WN) * (BN / WN), wm = (wave / WN) * (BM / WM);
    f32x4 acc[MI][NJ];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const char* const X = uniform(reinterpret_cast<const char*>(static_cast<const T*>(a.X) + x0));
    const char* const dY = reinterpret_cast<const char*>(static_cast<const T*>(a.Y) + gr.first * a.ldy + y0);
    // The rounds of a load are so many rows apart, and rows 16 apart have their pieces in the same places: one offset of
    // the lines serves all rounds, or two those of floats, which are 8 rows apart.
    constexpr int kRowsApart = THREADS / Yt::kAcross, kXRowsApart = THREADS / Xt::kAcross;
    constexpr int kYKinds = kRowsApart % 16 ? 2 : 1, kXKinds = kXRowsApart % 16 ? 2 : 1;
    static_assert(kRowsApart % 8 == 0 && kXRowsApart % 8 == 0, "");
    uint32_t yo[kYKinds], xc[kXKinds];
#pragma unroll
    for (int i = 0; i < kYKinds; ++i)
        yo[i] = (uint32_t)((Yt::major(0) * a.ldy + min((int64_t)Yt::minor(i) * Yt::P, a.N - Yt::P - y0)) * sizeof(T));
#pragma unroll
    for (int i = 0; i < kXKinds; ++i) xc[i] = (uint32_t)(min((int64_t)Xt::minor(i) * Xt::P, a.K - Xt::P - x0) * sizeof(T));
    const int first = __builtin_amdgcn_readfirstlane((int)gr.first), end = __builtin_amdgcn_readfirstlane((int)gr.end);
    // What the list says of the rows of the tile that is loaded next (asked for while the tile before is on its way, and
    // looked at when it has arrived: the loads come back in their order); which rounds had no row of X in the last tile and
    // the first, a bit each.
    int32_t entry[Xt::kRounds];
    uint32_t none[2] = {0, 0};
    int next;
    const auto find = [&] {
#pragma unroll
        for (int i = 0; i < Xt::kRounds; ++i) {
            const int r = next + i * kXRowsApart;
            entry[i] = -1;
            if (r < end) entry[i] = a.from.entry(r);
        }
        next += Xt::kInner;
    };
    const auto load = [&](int t, uint32_t to, int i) {
        if (i < Yt::kRounds) {
            const int r = i * kRowsApart, r0 = t * Yt::kInner + r;
            // in place of a row past the last, the one that is the first of the tile
            const bool there = first + r0 + Yt::major(0) < end;
            const char* const y = uniform(dY + (int64_t)(t * Yt::kInner) * a.ldy * (int64_t)sizeof(T));
            const uint32_t down = (uint32_t)(a.ldy * sizeof(T));
            Yt::load(to + kYAt, i, y, there ? yo[i % kYKinds] + r * down : yo[i % kYKinds] - Yt::major(0) * down);
        } else {
            const int x = i - Yt::kRounds;
            const int32_t found = a.from.row_of(entry[x]), r = max(found, 0);
            none[1] = x == 0 ? 0 : none[1];
            none[1] |= found < 0 ? 1u << x : 0u;
            if constexpr (WIDE) Xt::load(to + kXAt, x, X + r * a.ldx * (int64_t)sizeof(T) + xc[x % kXKinds]);
            else Xt::load(to + kXAt, x, X, (uint32_t)r * (uint32_t)(a.ldx * sizeof(T)) + xc[x % kXKinds]);
            if (x == Xt::kRounds - 1) find();
        }
    };
    const auto mend = [&](int t, uint32_t to) {
        const int left = end - first - t * Yt::kInner;
        if (left < Yt::kInner) {
#pragma unroll
            for (int i = 0; i < Yt::kRounds; ++i)
                if (Yt::major(0) + i * kRowsApart >= left) Yt::clear(to + kYAt, i);
        }
        const uint32_t missing = t == 0 ? none[0] : none[1];
        if (__any(missing != 0)) {
#pragma unroll
            for (int i = 0; i < Xt::kRounds; ++i)
                if (missing >> i & 1) Xt::clear(to + kXAt, i);
        }
    };
    const int tiles = (end - first + Lt::kInner - 1) / Lt::kInner;
    const auto start = [&] {
        next = first + Xt::major(0);
        find();
        none[0] = 0;
#pragma unroll
        for (int i = 0; i < Xt::kRounds; ++i) none[0] |= a.from.row_of(entry[i]) < 0 ? 1u << i : 0u;
    };
    bool done = false;
    if constexpr (sizeof(T) == 4) {
        start();
        multiply_tiles_split<Lt, Rt, MI, NJ>(lds, tiles, load, mend, wn, wm, true, acc);
        done = !start_over(acc);
    }
    if (!done) {
        start();
        multiply_tiles<Lt, Rt, MI, NJ>(lds, tiles, load, mend, wn, wm, true, acc);
    }
    T* __restrict__ dW = static_cast<T*>(const_cast<void*>(a.W)) + g * a.N * a.K;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
        const int64_t m = m0 + wm + 16 * j + (lane & 15);
        if (m >= lines) continue;
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const int64_t n = n0 + wn + 16 * i + 4 * (lane >> 4);
            typedef T out4 __attribute__((ext_vector_type(4)));
            if (n < columns) {
                out4 o;
#pragma unroll
                for (int r = 0; r < 4; ++r) o[r] = (T)acc[i][j][r];
                *reinterpret_cast<out4*>(dW + m * columns + n) = o;
            }
        }
    }
}

// whole turns of the dies' runs
int64_t dealt_grid(int64_t items) { return (items + 255) / 256 * 256; }

template <typename T, int BM, int BN, bool KN, bool WIDE, int THREADS>
hipError_t run_fast(const GroupedArgs& a, bool apart, hipStream_t s)
{
    const int64_t columns = (a.N + BN - 1) / BN, items = columns * most_row_tiles(a.G, a.R, BM, a.offsets != nullptr);
    constexpr int kLds = 2 * 128 * (BM + BN);
    static uint64_t allowed = 0;
    if (const hipError_t err = allow_lds(grouped_fast_kernel<T, BM, BN, KN, WIDE, THREADS>, kLds, allowed)) return err;
    return launch_parts(dealt_grid(items), THREADS, [&](unsigned grid, int64_t block0) {
        grouped_fast_kernel<T, BM, BN, KN, WIDE, THREADS><<<grid, THREADS, kLds, s>>>(a, columns, items, apart, block0);
    });
}

template <typename T, int BM, int BN, bool KN, bool WIDE, int THREADS>
hipError_t run_wgrad_fast(const GroupedArgs& a, hipStream_t s)
{
    const int64_t tm = ((KN ? a.K : a.N) + BM - 1) / BM, tn = ((KN ? a.N : a.K) + BN - 1) / BN, items = a.G * tm * tn;
    constexpr int kLds = 2 * 128 * (BM + BN);
    static uint64_t allowed = 0;
    if (const hipError_t err = allow_lds(grouped_wgrad_fast_kernel<T, BM, BN, KN, WIDE, THREADS>, kLds, allowed)) return err;
    return launch_parts(dealt_grid(items), THREADS, [&](unsigned grid, int64_t block0) {
        grouped_wgrad_fast_kernel<T, BM, BN, KN, WIDE, THREADS><<<grid, THREADS, kLds, s>>>(a, tm, tn, items, block0);
    });
}

// Tiles that a compute unit gets, times what one costs: BM x BN products, dearer in small tiles, whose operands are fetched
// and read more often (`rate`: the products a clock of such a tile next to the largest one's).
double turns(int64_t tiles, int compute_units, int BM, int BN, double rate)
{
    return (double)((tiles + compute_units - 1) / compute_units) * BM * BN / rate;
}

template <typename T, bool KN, bool WIDE>
hipError_t by_size(const GroupedArgs& a, bool gradient, const GroupedPlan& p, hipStream_t s)
{
    if constexpr (sizeof(T) == 2) {
        if (p.rows == 256) return gradient ? run_wgrad_fast<T, 256, 256, KN, WIDE, 512>(a, s) : run_fast<T, 256, 256, KN, WIDE, 512>(a, p.apart, s);
    }
    if (gradient) return run_wgrad_fast<T, 128, 128, KN, WIDE, 256>(a, s);
    return p.rows == 128 ? run_fast<T, 128, 128, KN, WIDE, 256>(a, p.apart, s) : run_fast<T, 64, 128, KN, WIDE, 256>(a, p.apart, s);
}

template <typename T>
hipError_t by_layout(const GroupedArgs& a, bool gradient, const GroupedPlan& p, hipStream_t s)
{
    if (p.wide) return a.weights_kn ? by_size<T, true, true>(a, gradient, p, s) : by_size<T, false, true>(a, gradient, p, s);
    return a.weights_kn ? by_size<T, true, false>(a, gradient, p, s) : by_size<T, false, false>(a, gradient, p, s);
}

bool aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

}  // namespace

bool grouped_fast_applies(const GroupedArgs& a, int dtype)
{
    const int64_t piece = dtype == 0 ? 4 : 8;
    // 256 lines of an operand have to lie within 32 bits of bytes
    constexpr int64_t kLongest = 1 << 22;
    return a.K > 0 && a.K <= kLongest && a.N <= kLongest && a.ldx <= kLongest && a.ldy <= kLongest && a.K % piece == 0 && a.N % piece == 0 && a.ldx % piece == 0 && a.ldy % piece == 0 && a.from.rows > 0 &&
           aligned(a.X) && aligned(a.W) && aligned(a.Y);
}

// 256 x 256, 128 x 128 or 64 x 128, whichever leaves the least to the unit that has most.  A group has a last tile that
// is not full: 0.6 of a tile more than its rows in the mean.  16 groups, 16,384 rows, 4,096 x 2,048 bf16: 317 us with
// 256 x 256, 372 with 128 x 128; 64 groups, 8,192 rows, 1,024 x 2,048: 101 and 86.  Floats have the two
// small ones: the instruction's six products of parts leave no registers for the large.
GroupedPlan plan_grouped_fast(const GroupedArgs& a, int dtype, bool gradient)
{
    const bool half = dtype != 0;
    const int64_t size = half ? 2 : 4;
    GroupedPlan p = {GroupedPlan::kTiles, 128, 128, false, false, false};
    // bytes of X from its first row to the end of its last
    p.wide = a.from.rows * a.ldx * size > 0xffffffffLL;
    if (gradient) {
        if (half && a.G * ((a.N + 255) / 256) * ((a.K + 255) / 256) >= 192) p.rows = p.columns = 256;
        return p;
    }
    const auto tiles = [&](int BM, int BN) {
        const double down = a.G == 1 ? (double)((a.R + BM - 1) / BM) : (double)a.R / BM + 0.6 * (double)a.G;
        return (int64_t)(down * (double)((a.N + BN - 1) / BN));
    };
    const double large = turns(tiles(256, 256), a.compute_units, 256, 256, 1.0);
    const double middle = turns(tiles(128, 128), a.compute_units, 128, 128, half ? 0.7 : 1.0);
    const double small = turns(tiles(64, 128), a.compute_units, 64, 128, half ? 0.55 : 0.8);
    if (half && large <= std::min(middle, small)) p.rows = p.columns = 256;
    else if (middle > small) p.rows = 64;
    // (16 experts for 32 rows, 4,096 columns, bf16, together and apart: rows of 4,096 bytes 66.4 us, 54.1, 8,192 122.6, 88.3,
    // 12,288 146.8, 133.3, 16,384 189.0, 176.0; floats, 8,192 columns, 150, 127, 241, 237, 359, 342, 462, 456.  Rows of 512 to 2,560
    // bytes, 4,112, 5,120, 6,144, 8,208 and 10,240: within 6 % of one another, either way.)
    p.apart = !a.weights_kn && a.R <= p.rows * a.G && a.K * size % 4096 == 0;
    return p;
}

hipError_t launch_grouped_fast(const GroupedArgs& a, int dtype, bool gradient, const GroupedPlan& p, hipStream_t s)
{
    switch (dtype) {
        case 0: return by_layout<float>(a, gradient, p, s);
        case 1: return by_layout<half_t>(a, gradient, p, s);
        default: return by_layout<bf16_t>(a, gradient, p, s);
    }
}

}  // namespace sgap
