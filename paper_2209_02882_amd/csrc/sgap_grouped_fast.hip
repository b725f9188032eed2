// Products over ragged groups where rows are multiples of 16 bytes at 16-byte addresses.
#include "sgap_grouped_tiles.hpp"

namespace sgap {

namespace {

// Work items are dealt to the eight dies (workgroup b runs on die b % 8) in runs of 32 neighbours, which share rows of X
// or weights in the die's L2.  Runs in turn, so that the items that turn out not to exist, all at the end, leave no die idle.
__device__ __forceinline__ int64_t dealt_item(uint32_t b)
{
    const uint32_t die = b & 7, at = b >> 3;
    return (int64_t)((at >> 5) * 8 + die) * 32 + (at & 31);
}

template <typename T, int BM, int BN, bool KN, int THREADS>
__global__ __launch_bounds__(THREADS) void grouped_fast_kernel(GroupedArgs a, int64_t column_tiles, int64_t items)
{
    using Wt = Tile<T, BN, !KN, THREADS>;
    using Xt = Tile<T, BM, true, THREADS>;
    constexpr int kWaves = THREADS / 64, WN = kWaves / 2, WM = 2;
    constexpr int MI = BN / WN / 16, NJ = BM / WM / 16;
    extern __shared__ __align__(16) char lds[];
    constexpr int kStage = Wt::kBytes + Xt::kBytes;
    const int64_t item = dealt_item(blockIdx.x);
    if (item >= items) return;
    const int64_t tile = item / column_tiles, n0 = (item - tile * column_tiles) * BN;
    const RowTile rows = find_row_tile<BM>(a.offsets, a.G, a.R, tile);
    if (rows.rows <= 0) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wn = (wave % WN) * (BN / WN), wm = (wave / WN) * (BM / WM);
    f32x4 acc[MI][NJ];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const T* const zero = reinterpret_cast<const T*>(g_zero_piece);
    if (rows.g < a.G) {
        const T* const W = static_cast<const T*>(a.W) + rows.g * a.N * a.K;
        const T* wp[Wt::kRounds];
        const T* xp[Xt::kRounds];
#pragma unroll
        for (int i = 0; i < Wt::kRounds; ++i) {
            if constexpr (!KN) {
                const int64_t n = min(n0 + Wt::major(i), a.N - 1);  // columns past the last are not stored
                wp[i] = W + n * a.K + Wt::minor(i) * Wt::P;
            } else {
                wp[i] = W + (int64_t)Wt::major(i) * a.N + min(n0 + Wt::minor(i) * Wt::P, a.N - Wt::P);
            }
        }
#pragma unroll
        for (int i = 0; i < Xt::kRounds; ++i) {
            const int m = Xt::major(i);
            const int64_t r = m < rows.rows ? a.from.row(rows.first + m) : -1;
            xp[i] = r >= 0 ? static_cast<const T*>(a.X) + r * a.ldx + Xt::minor(i) * Xt::P : nullptr;
        }
        const int tiles = (int)((a.K + Wt::kInner - 1) / Wt::kInner);
        const auto load = [&](int t, char* to) {
            const int64_t k0 = (int64_t)t * Wt::kInner;
#pragma unroll
            for (int i = 0; i < Wt::kRounds; ++i) {
                if constexpr (!KN) Wt::load(to, i, k0 + Wt::minor(i) * Wt::P < a.K ? wp[i] + k0 : zero);
                else Wt::load(to, i, k0 + Wt::major(i) < a.K ? wp[i] + k0 * a.N : zero);
            }
#pragma unroll
            for (int i = 0; i < Xt::kRounds; ++i)
                Xt::load(to + Wt::kBytes, i, xp[i] && k0 + Xt::minor(i) * Xt::P < a.K ? xp[i] + k0 : zero);
        };
        load(0, lds);
        for (int t = 0; t < tiles; ++t) {
            const char* const at = lds + (t & 1) * kStage;
            wait_loads<0>();
            __syncthreads();
            if (t + 1 < tiles) load(t + 1, lds + ((t + 1) & 1) * kStage);
#pragma unroll
            for (int kc = 0; kc < 2; ++kc) {
                piece_t<T> fw[MI], fx[NJ];
#pragma unroll
                for (int i = 0; i < MI; ++i) fw[i] = Wt::fragment(at, wn + 16 * i, kc);
#pragma unroll
                for (int j = 0; j < NJ; ++j) fx[j] = Xt::fragment(at + Wt::kBytes, wm + 16 * j, kc);
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int i = 0; i < MI; ++i) acc[i][j] = mma16(fw[i], fx[j], acc[i][j]);
            }
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
            typedef T out4 __attribute__((ext_vector_type(4)));
            if (n < a.N) {
                out4 o;
#pragma unroll
                for (int r = 0; r < 4; ++r) o[r] = (T)acc[i][j][r];
                *reinterpret_cast<out4*>(y + n) = o;
            }
        }
    }
}

// The gradient of the weights.  The inner dimension is the group's rows; both operands have their lines contiguous.
// lines of the first: the result's contiguous dimension.
template <typename T, int BM, int BN, bool KN, int THREADS>
__global__ __launch_bounds__(THREADS) void grouped_wgrad_fast_kernel(GroupedArgs a, int64_t tiles_m, int64_t tiles_n, int64_t items)
{
    using Lt = Tile<T, BN, false, THREADS>;
    using Rt = Tile<T, BM, false, THREADS>;
    constexpr int kWaves = THREADS / 64, WN = kWaves / 2, WM = 2;
    constexpr int MI = BN / WN / 16, NJ = BM / WM / 16;
    extern __shared__ __align__(16) char lds[];
    constexpr int kStage = Lt::kBytes + Rt::kBytes;
    const int64_t item = dealt_item(blockIdx.x);
    if (item >= items) return;
    const int64_t per = tiles_m * tiles_n, g = item / per, in = item - g * per;
    const int64_t lines = KN ? a.K : a.N, columns = KN ? a.N : a.K;  // of the result
    const int64_t m0 = in / tiles_n * BM, n0 = in % tiles_n * BN;
    const GroupRows gr = group_rows(a.offsets, g, a.R);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wn = (wave % WN) * (BN / WN), wm = (wave / WN) * (BM / WM);
    f32x4 acc[MI][NJ];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const T* const zero = reinterpret_cast<const T*>(g_zero_piece);
    const T* const X = static_cast<const T*>(a.X);
    const T* const dY = static_cast<const T*>(a.Y);
    const auto piece = [&](bool of_x, int64_t r, int64_t line) -> const T* {
        if (r >= gr.end) return zero;
        if (!of_x) return dY + r * a.ldy + min(line, a.N - Lt::P);
        const int64_t s = a.from.row(r);
        return s < 0 ? zero : X + s * a.ldx + min(line, a.K - Lt::P);
    };
    const auto load = [&](int64_t r0, char* to) {
#pragma unroll
        for (int i = 0; i < Lt::kRounds; ++i) Lt::load(to, i, piece(!KN, r0 + Lt::major(i), n0 + Lt::minor(i) * Lt::P));
#pragma unroll
        for (int i = 0; i < Rt::kRounds; ++i)
            Rt::load(to + Lt::kBytes, i, piece(KN, r0 + Rt::major(i), m0 + Rt::minor(i) * Rt::P));
    };
    const int tiles = (int)((gr.end - gr.first + Lt::kInner - 1) / Lt::kInner);
    if (tiles) load(gr.first, lds);
    for (int t = 0; t < tiles; ++t) {
        const char* const at = lds + (t & 1) * kStage;
        wait_loads<0>();
        __syncthreads();
        if (t + 1 < tiles) load(gr.first + (int64_t)(t + 1) * Lt::kInner, lds + ((t + 1) & 1) * kStage);
#pragma unroll
        for (int kc = 0; kc < 2; ++kc) {
            piece_t<T> fl[MI], fr[NJ];
#pragma unroll
            for (int i = 0; i < MI; ++i) fl[i] = Lt::fragment(at, wn + 16 * i, kc);
#pragma unroll
            for (int j = 0; j < NJ; ++j) fr[j] = Rt::fragment(at + Lt::kBytes, wm + 16 * j, kc);
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int i = 0; i < MI; ++i) acc[i][j] = mma16(fl[i], fr[j], acc[i][j]);
        }
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

// More LDS than a launch gets unasked; `allowed` has a bit for each device on which that has been asked for.
template <typename K>
hipError_t allow_lds(K kernel, int bytes, uint64_t& allowed)
{
    int device = 0;
    if (const hipError_t err = hipGetDevice(&device)) return err;
    if (device < 64 && (allowed >> device & 1)) return hipSuccess;
    const hipError_t err = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (err == hipSuccess && device < 64) allowed |= 1ull << device;
    return err;
}

unsigned dealt_grid(int64_t items) { return (unsigned)((items + 255) / 256 * 256); }

template <typename T, int BM, int BN, bool KN, int THREADS>
hipError_t run_fast(const GroupedArgs& a, hipStream_t s)
{
    const int64_t columns = (a.N + BN - 1) / BN, items = columns * most_row_tiles(a.G, a.R, BM, a.offsets != nullptr);
    if (items > 0x7fffff00LL) return hipErrorInvalidConfiguration;
    constexpr int kLds = 2 * 128 * (BM + BN);
    static uint64_t allowed = 0;
    if (const hipError_t err = allow_lds(grouped_fast_kernel<T, BM, BN, KN, THREADS>, kLds, allowed)) return err;
    grouped_fast_kernel<T, BM, BN, KN, THREADS><<<dealt_grid(items), THREADS, kLds, s>>>(a, columns, items);
    return hipGetLastError();
}

template <typename T, int BM, int BN, bool KN, int THREADS>
hipError_t run_wgrad_fast(const GroupedArgs& a, hipStream_t s)
{
    const int64_t tm = ((KN ? a.K : a.N) + BM - 1) / BM, tn = ((KN ? a.N : a.K) + BN - 1) / BN, items = a.G * tm * tn;
    if (items > 0x7fffff00LL) return hipErrorInvalidConfiguration;
    constexpr int kLds = 2 * 128 * (BM + BN);
    static uint64_t allowed = 0;
    if (const hipError_t err = allow_lds(grouped_wgrad_fast_kernel<T, BM, BN, KN, THREADS>, kLds, allowed)) return err;
    grouped_wgrad_fast_kernel<T, BM, BN, KN, THREADS><<<dealt_grid(items), THREADS, kLds, s>>>(a, tm, tn, items);
    return hipGetLastError();
}

template <typename T, bool KN>
hipError_t by_size(const GroupedArgs& a, hipStream_t s)
{
    if (a.R >= 192 * a.G) return run_fast<T, 256, 256, KN, 512>(a, s);
    return run_fast<T, 128, 128, KN, 256>(a, s);
}

template <typename T, bool KN>
hipError_t wgrad_by_size(const GroupedArgs& a, hipStream_t s)
{
    if (a.G * ((a.N + 255) / 256) * ((a.K + 255) / 256) >= 128) return run_wgrad_fast<T, 256, 256, KN, 512>(a, s);
    return run_wgrad_fast<T, 128, 128, KN, 256>(a, s);
}

bool aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

}  // namespace

bool grouped_fast_applies(const GroupedArgs& a, int dtype)
{
    const int64_t piece = dtype == 0 ? 4 : 8;
    return a.K > 0 && a.K % piece == 0 && a.N % piece == 0 && a.ldx % piece == 0 && a.ldy % piece == 0 && a.from.rows > 0 &&
           aligned(a.X) && aligned(a.W) && aligned(a.Y);
}

hipError_t launch_grouped_fast(const GroupedArgs& a, int dtype, hipStream_t s)
{
    switch (dtype) {
        case 0: return a.weights_kn ? by_size<float, true>(a, s) : by_size<float, false>(a, s);
        case 1: return a.weights_kn ? by_size<half_t, true>(a, s) : by_size<half_t, false>(a, s);
        default: return a.weights_kn ? by_size<bf16_t, true>(a, s) : by_size<bf16_t, false>(a, s);
    }
}

hipError_t launch_grouped_wgrad_fast(const GroupedArgs& a, int dtype, hipStream_t s)
{
    switch (dtype) {
        case 0: return a.weights_kn ? wgrad_by_size<float, true>(a, s) : wgrad_by_size<float, false>(a, s);
        case 1: return a.weights_kn ? wgrad_by_size<half_t, true>(a, s) : wgrad_by_size<half_t, false>(a, s);
        default: return a.weights_kn ? wgrad_by_size<bf16_t, true>(a, s) : wgrad_by_size<bf16_t, false>(a, s);
    }
}

}  // namespace sgap
