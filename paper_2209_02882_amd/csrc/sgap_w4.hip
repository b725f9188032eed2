// Products over ragged groups with weights of 4 bits: W[n, k] = (q[n, k] - z[n, k / group]) * s[n, k / group].
//
// Made for few rows a group, where every weight is read for one row or a handful and the bytes of the weights are the
// bound.  A wavefront takes tiles of 16 columns and its share of the inner dimension; the codes of 16 columns by 128
// values lie in 1,024 consecutive bytes (launch_w4_layout puts them there once), 16 bytes to a lane, in the order in
// which the matrix instruction wants them.  No weight is ever rounded: a code goes into the top of the mantissa of the
// number 16 (16 + q, exact in both 16-bit types, one shift and one and-or for two codes), the matrix unit sums
// (16 + q) x and, against ones, x itself over a scale's values in 32 bits, and then
//     acc += s * (sum of (16 + q) x - (16 + z) * sum of x).
// The wavefronts of a workgroup have shares of the inner dimension and are summed up through LDS at the end.
//
// Where x is infinite or so large that the sums overflow, that difference is no number although the definition may be
// one: an element that comes out not finite is computed again value by value.
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

// One byte of the laid-out codes, scales and zero points per thread.
__global__ __launch_bounds__(256) void w4_layout_kernel(int64_t G, int64_t K, int64_t N, int64_t blocks_scale, bool zeros, W4Sizes z,
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
    const int64_t many = G * z.tiles_n * blocks_scale * kTileN;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < many; i += steps) {
        const int64_t b = i / kTileN % blocks_scale, t = i / kTileN / blocks_scale;
        const int64_t g = t / z.tiles_n, n = t % z.tiles_n * kTileN + i % kTileN;
        const int64_t from = (g * N + n) * blocks_scale + b;
        reinterpret_cast<uint16_t*>(out + z.scales_at)[i] = n < N ? scales[from] : 0;
        if (zeros) (out + z.zeros_at)[i] = n < N ? zero[from] : 8;
    }
}

// NT tiles of columns and MT tiles of 16 rows to a wavefront; STEPS matrix instructions (32 values each) to a scale, or,
// with STEPS = 4, any whole number of blocks of 128.  The wavefronts of the workgroup share the inner dimension.
template <typename T, int STEPS, int NT, int MT, bool ZEROS>
__global__ __launch_bounds__(NT * MT > 1 ? 512 : 1024) void grouped_w4_kernel(GroupedW4Args a, W4Sizes z, int64_t column_items)
{
    __shared__ f32x4 part[16][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int waves = blockDim.x >> 6, row = lane & 15, piece = lane >> 4;
    const int64_t g = blockIdx.x / column_items, item = blockIdx.x - g * column_items;
    const int64_t tile0 = item * NT;
    const uint8_t* __restrict__ tiles = a.weights + g * z.tiles_n * z.blocks_k * kTileBytes;
    const T* __restrict__ scales = reinterpret_cast<const T*>(a.weights + z.scales_at) + g * z.tiles_n * z.scales_k * kTileN;
    const uint8_t* __restrict__ zeros = a.weights + z.zeros_at + g * z.tiles_n * z.scales_k * kTileN;
    GroupRows gr = {0, 0};
    if (g < a.G) gr = group_rows(a.offsets, g, a.R);
    const T* __restrict__ X = static_cast<const T*>(a.X);
    T* __restrict__ Y = static_cast<T*>(a.Y);
    piece_t<T> ones;
#pragma unroll
    for (int i = 0; i < 8; ++i) ones[i] = (T)1.0f;
    for (int64_t m0 = gr.first + (int64_t)blockIdx.y * 16 * MT; m0 < gr.end; m0 += (int64_t)gridDim.y * 16 * MT) {
        const T* __restrict__ x[MT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            const int64_t m = m0 + mt * 16 + row;
            const int64_t r = m < gr.end ? a.from.row(m) : -1;
            x[mt] = r >= 0 ? X + r * a.ldx + piece * 8 : nullptr;
        }
        f32x4 acc[NT][MT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) acc[nt][mt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        for (int64_t kb = wave; kb < z.blocks_k; kb += waves) {
            uint4 w[NT];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const int64_t t = min(tile0 + nt, z.tiles_n - 1);  // a tile behind the last is not stored
                w[nt] = *reinterpret_cast<const uint4*>(tiles + (t * z.blocks_k + kb) * kTileBytes + lane * 16);
            }
            const int steps = (int)min((int64_t)4, (a.K - kb * kBlockK) / 32);
#pragma unroll
            for (int s0 = 0; s0 < 4; s0 += STEPS) {
                if (s0 >= steps) break;
                piece_t<T> xf[MT][STEPS];
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int i = 0; i < STEPS; ++i) {
                        xf[mt][i] = piece_t<T>{};
                        if (x[mt] && s0 + i < steps) xf[mt][i] = load_piece(x[mt] + kb * kBlockK + (s0 + i) * 32);
                    }
                f32x4 sum[MT];
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    sum[mt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int i = 0; i < STEPS; ++i) sum[mt] = mma16(xf[mt][i], ones, sum[mt]);
                }
                const int64_t sb = (kb * kBlockK + s0 * 32) / a.group_k;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const int64_t t = min(tile0 + nt, z.tiles_n - 1);
                    const float scale = (float)scales[(t * z.scales_k + sb) * kTileN + row];
                    const float zero = ZEROS ? 16.0f + (float)zeros[(t * z.scales_k + sb) * kTileN + row] : 24.0f;
                    const uint32_t d[4] = {w[nt].x, w[nt].y, w[nt].z, w[nt].w};
                    f32x4 dot[MT];
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) dot[mt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int i = 0; i < STEPS; ++i) {
                        const piece_t<T> wf = decode<T>(d[s0 + i]);
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) dot[mt] = mma16(xf[mt][i], wf, dot[mt]);
                    }
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            acc[nt][mt][r] = __builtin_fmaf(scale, __builtin_fmaf(-zero, sum[mt][r], dot[mt][r]), acc[nt][mt][r]);
                }
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
                    if (!__builtin_isfinite(v)) {
                        const int64_t xr = a.from.row(at);
                        v = 0.0f;
                        for (int64_t k = 0; xr >= 0 && k < a.K; ++k) {
                            const int64_t sc = ((tile0 + nt) * z.scales_k + k / a.group_k) * kTileN + n;
                            const float zero = ZEROS ? (float)zeros[sc] : 8.0f;
                            const float wv = ((float)code_at(tiles, z.blocks_k, n0 + n, k) - zero) * (float)scales[sc];
                            v = __builtin_fmaf(wv, (float)X[xr * a.ldx + k], v);
                        }
                    }
                    Y[at * a.ldy + n0 + n] = (T)v;
                }
            }
    }
    // rows behind the last group
    if (a.offsets && g == a.G - 1) {
        const int columns = (int)min((int64_t)NT * kTileN, a.N - tile0 * kTileN);
        for (int64_t r = gr.end + blockIdx.y; r < a.R; r += gridDim.y)
            for (int n = threadIdx.x; n < columns; n += blockDim.x) Y[r * a.ldy + tile0 * kTileN + n] = (T)0.0f;
    }
}

template <typename T, int STEPS, int NT, int MT>
hipError_t run_w4(const GroupedW4Args& a, const W4Sizes& z, int waves, int row_items, hipStream_t s)
{
    const int64_t items = (z.tiles_n + NT - 1) / NT;
    if (a.G * items > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)(a.G * items), (unsigned)row_items);
    if (a.zeros) grouped_w4_kernel<T, STEPS, NT, MT, true><<<grid, 64 * waves, 0, s>>>(a, z, items);
    else grouped_w4_kernel<T, STEPS, NT, MT, false><<<grid, 64 * waves, 0, s>>>(a, z, items);
    return hipGetLastError();
}

template <typename T, int STEPS>
hipError_t by_rows(const GroupedW4Args& a, const W4Sizes& z, hipStream_t s)
{
    // a wavefront for four blocks of 128 values, 4 to 16 of them
    const int64_t w = (z.blocks_k + 3) / 4;
    const int waves = w <= 4 ? 4 : w <= 8 ? 8 : 16;
    const int64_t mean = (a.R + a.G - 1) / a.G;
    const auto items = [&](int rows) { const int64_t n = (2 * mean + rows - 1) / rows; return (int)(n < 1 ? 1 : n > 64 ? 64 : n); };
    if (mean <= 8 || (a.G == 1 && mean <= 16)) return run_w4<T, STEPS, 1, 1>(a, z, waves, a.G == 1 ? 1 : items(16), s);
    return run_w4<T, STEPS, 2, 3>(a, z, waves < 8 ? waves : 8, a.G == 1 ? (items(48) + 1) / 2 : items(48), s);
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
    z.scales_k = K / group_k;
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
        G, K, N, z.scales_k, zeros != nullptr, z, q, static_cast<const uint16_t*>(scales), zeros, out);
    return hipGetLastError();
}

hipError_t launch_grouped_w4(const GroupedW4Args& a, int dtype, hipStream_t s)
{
    const W4Sizes z = w4_sizes(a.G, a.K, a.N, a.group_k, a.zeros);
    return dtype == 1 ? by_scale<half_t>(a, z, s) : by_scale<bf16_t>(a, z, s);
}

}  // namespace sgap
