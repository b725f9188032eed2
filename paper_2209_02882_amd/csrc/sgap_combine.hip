// The experts' rows back to their tokens: out[t] = sum over j of gates[t, j] * Z[slot[t, j]], and its gradients
// dZ[slot[t, j]] = gates[t, j] * dout[t] and dgates[t, j] = <Z[slot[t, j]], dout[t]>.
//
// Bound by memory: every row of Z and of the result passes once.  A wavefront has a token and takes its columns 16 bytes
// to a lane, all k rows of Z in flight together; the gradient reads a piece of dout once for all of them.  The last
// columns of a row whose length no piece divides are taken by pieces that reach back into the columns before.
//
// 8,192 tokens of 4 rows of 2,048 columns, bf16: 26.3 us, 6.4 TB/s of the 168 MB that the call names (part of Z comes out of
// the last-level cache); the gradient 57 us, 5.3 TB/s of its 302 MB.  A copy reaches 5.6 TB/s.
#include "sgap_experts.hpp"

namespace sgap {

namespace {

constexpr int kCombineThreads = 256;

// the first column of the piece that starts at column c < D of a row of at least a piece's columns
template <int VEC>
__device__ __forceinline__ int64_t piece_first(int64_t c, int64_t D)
{
    return VEC == 1 || c + VEC <= D ? c : D - VEC;
}

template <typename T, int VEC>
struct Columns {
    float v[VEC];
    __device__ __forceinline__ void load(const T* p)
    {
        if constexpr (VEC == 1) {
            v[0] = (float)*p;
        } else {
            const piece_t<T> x = load_piece(p);
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[i] = (float)x[i];
        }
    }
    __device__ __forceinline__ void store(T* p) const
    {
        if constexpr (VEC == 1) {
            *p = (T)v[0];
        } else {
            piece_t<T> x;
#pragma unroll
            for (int i = 0; i < VEC; ++i) x[i] = (T)v[i];
            store_piece(p, x);
        }
    }
};

// A work item: a token and 64 * VEC of its columns.  Sums in 32 bits, rounded once.
template <typename T, int VEC, int KMAX>
__global__ __launch_bounds__(kCombineThreads) void combine_kernel(CombineArgs a, uint32_t column_items, int64_t block0)
{
    const int lane = threadIdx.x & 63;
    const int64_t item = (block0 + blockIdx.x) * (kCombineThreads / 64) + (threadIdx.x >> 6);
    const int64_t t = item / column_items;
    const int64_t c = ((item - t * column_items) * 64 + lane) * VEC;
    if (t >= a.T || c >= a.D) return;
    const int64_t first = piece_first<VEC>(c, a.D), rows = a.T * a.k;
    const T* __restrict__ Z = static_cast<const T*>(a.Z) + first;
    Columns<T, VEC> z[KMAX], sum;
    float gate[KMAX];
#pragma unroll
    for (int j = 0; j < KMAX; ++j) {
        gate[j] = 0.0f;
        const int64_t r = j < a.k ? a.slot[t * a.k + j] : -1;
        const bool there = r >= 0 && r < rows;
        if (there) {
            z[j].load(Z + r * a.D);
            gate[j] = a.gates ? a.gates[t * a.k + j] : 1.0f;
        } else {
#pragma unroll
            for (int i = 0; i < VEC; ++i) z[j].v[i] = 0.0f;
        }
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < KMAX; ++j) s = __builtin_fmaf(gate[j], z[j].v[i], s);
        sum.v[i] = s;
    }
    sum.store(static_cast<T*>(a.out) + t * a.D + first);
}

// WAVES wavefronts share a token's columns.  Behind the tokens' workgroups come those that clear the rows of dZ that
// no token has.
template <typename T, int VEC, int KMAX, int WAVES>
__global__ __launch_bounds__(kCombineThreads) void combine_grad_kernel(CombineArgs a, int64_t token_blocks, int64_t block0)
{
    constexpr int kTokens = kCombineThreads / 64 / WAVES;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t rows = a.T * a.k, block = block0 + blockIdx.x;
    if (block >= token_blocks) {
        const int64_t r0 = (block - token_blocks) * kCombineThreads + wave * 64;
        uint64_t clear = __ballot(r0 + lane < rows && a.order[r0 + lane] < 0);
        for (; clear; clear &= clear - 1) {
            T* __restrict__ row = static_cast<T*>(a.out) + (r0 + __builtin_ctzll(clear)) * a.D;
            for (int64_t c = lane; c < a.D; c += 64) row[c] = (T)0.0f;
        }
        return;
    }
    const int64_t t = block * kTokens + wave / WAVES;
    float dot[KMAX], gate[KMAX];
    int64_t slot[KMAX];
    const bool token = t < a.T;
#pragma unroll
    for (int j = 0; j < KMAX; ++j) {
        dot[j] = 0.0f;
        const int64_t r = token && j < a.k ? a.slot[t * a.k + j] : -1;
        slot[j] = r >= 0 && r < rows ? r : -1;
        gate[j] = slot[j] >= 0 ? a.gates[t * a.k + j] : 0.0f;
    }
    if (token) {
        const T* __restrict__ dout = static_cast<const T*>(a.dout) + t * a.D;
        for (int64_t c = ((wave % WAVES) * 64 + lane) * VEC; c < a.D; c += 64 * VEC * WAVES) {
            const int64_t first = piece_first<VEC>(c, a.D);
            const int shared = (int)(c - first);  // columns that the lane in front has as well: not summed twice
            Columns<T, VEC> d, z[KMAX];
            d.load(dout + first);
#pragma unroll
            for (int j = 0; j < KMAX; ++j)
                if (slot[j] >= 0) z[j].load(static_cast<const T*>(a.Z) + slot[j] * a.D + first);
#pragma unroll
            for (int j = 0; j < KMAX; ++j) {
                if (slot[j] < 0) continue;
                Columns<T, VEC> g;
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    g.v[i] = gate[j] * d.v[i];
                    dot[j] = i >= shared ? __builtin_fmaf(z[j].v[i], d.v[i], dot[j]) : dot[j];
                }
                g.store(static_cast<T*>(a.out) + slot[j] * a.D + first);
            }
        }
    }
    __shared__ float part[kCombineThreads / 64][KMAX];
#pragma unroll
    for (int j = 0; j < KMAX; ++j) {
        float s = dot[j];
#pragma unroll
        for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
        if (WAVES > 1) {
            if (lane == 0) part[wave][j] = s;
        } else if (lane == j && token && j < a.k) {
            a.dgates[t * a.k + j] = slot[j] >= 0 ? s : 0.0f;
        }
    }
    if constexpr (WAVES > 1) {
        __syncthreads();
        if (wave % WAVES == 0 && token && lane < a.k) {
            float s = 0.0f;
            for (int w = 0; w < WAVES; ++w) s += part[wave + w][lane];
            a.dgates[t * a.k + lane] = s;
        }
    }
}

template <typename T, int VEC, int KMAX>
hipError_t combine(const CombineArgs& a, hipStream_t s)
{
    const int64_t columns = (a.D + 64 * VEC - 1) / (64 * VEC), items = a.T * columns;
    return launch_parts((items + kCombineThreads / 64 - 1) / (kCombineThreads / 64), kCombineThreads, [&](unsigned grid, int64_t block0) {
        combine_kernel<T, VEC, KMAX><<<grid, kCombineThreads, 0, s>>>(a, (uint32_t)columns, block0);
    });
}

template <typename T, int VEC, int KMAX>
hipError_t combine_grad(const CombineArgs& a, hipStream_t s)
{
    const int64_t clearing = (a.T * a.k + kCombineThreads - 1) / kCombineThreads;
    // a token's columns go to four wavefronts where tokens are fewer than fill the chip and there are columns for all
    if (a.T < 4096 && a.D >= 2 * 64 * VEC) {
        combine_grad_kernel<T, VEC, KMAX, 4><<<(unsigned)(a.T + clearing), kCombineThreads, 0, s>>>(a, a.T, 0);
        return hipGetLastError();
    }
    const int64_t blocks = (a.T + 3) / 4;
    return launch_parts(blocks + clearing, kCombineThreads, [&](unsigned grid, int64_t block0) {
        combine_grad_kernel<T, VEC, KMAX, 1><<<grid, kCombineThreads, 0, s>>>(a, blocks, block0);
    });
}

template <typename T, int VEC>
hipError_t by_k(const CombineArgs& a, bool grad, hipStream_t s)
{
    if (a.k <= 1) return grad ? combine_grad<T, VEC, 1>(a, s) : combine<T, VEC, 1>(a, s);
    if (a.k <= 2) return grad ? combine_grad<T, VEC, 2>(a, s) : combine<T, VEC, 2>(a, s);
    if (a.k <= 4) return grad ? combine_grad<T, VEC, 4>(a, s) : combine<T, VEC, 4>(a, s);
    if (a.k <= 8) return grad ? combine_grad<T, VEC, 8>(a, s) : combine<T, VEC, 8>(a, s);
    return grad ? combine_grad<T, VEC, 16>(a, s) : combine<T, VEC, 16>(a, s);
}

template <typename T>
hipError_t by_width(const CombineArgs& a, bool grad, hipStream_t s)
{
    return a.D >= Piece<T>::kCount ? by_k<T, Piece<T>::kCount>(a, grad, s) : by_k<T, 1>(a, grad, s);
}

hipError_t by_type(const CombineArgs& a, bool grad, hipStream_t s)
{
    switch (a.dtype) {
        case 0: return by_width<float>(a, grad, s);
        case 1: return by_width<half_t>(a, grad, s);
        default: return by_width<bf16_t>(a, grad, s);
    }
}

}  // namespace

hipError_t launch_combine(const CombineArgs& a, hipStream_t s) { return by_type(a, false, s); }
hipError_t launch_combine_grad(const CombineArgs& a, hipStream_t s) { return by_type(a, true, s); }

}  // namespace sgap
