// The router's balance loss and its gradient.  Sequence s has n_s tokens that chose an expert and c_se pairs of expert e; with
// p_t = softmax of token t's logits over all experts, f_se = E c_se / (k n_s) and P_se = the mean of p_te over its tokens,
//     loss = mean over the sequences that have a token of sum over e of f_se P_se,
//     dl_te = dloss / (sequences * n_s) * p_te * (f_se - sum over i of f_si p_ti);
// the counts are constants.  A token's p sum up to 1, so f - 1 = (E c - k n) / (k n) serves as well as f does, and it is a whole
// number until it is divided: near an even load, which the loss is for, f would lose what counts in the difference.
//
// A row is held by 16 lanes (up to 256 experts) or by a wavefront, some neighbouring experts to a lane, which keeps the sums of
// its own experts over the rows that it sees.  Tiles of rows never cross a sequence; a second launch sums up a sequence's tiles,
// a third the sequences where there is more than one.  The logits are read once each way (4 MB for 16,384 tokens and 128 experts
// in bf16, which no launch waits for): what is left is the launches.  Sums of floats in a fixed order; the only atomics count
// whole numbers in LDS.
#include "sgap_grouped.hpp"
#include "sgap_tokens.hpp"

namespace sgap {

namespace {

constexpr int kThreads = 256;
constexpr int kRows = 64;           // of a tile
constexpr int kJoinThreads = 1024;  // of a sequence's sum
constexpr int kMostExperts = 1024;

template <int LANES>
__device__ __forceinline__ float over_lanes_max(float v)
{
#pragma unroll
    for (int d = LANES / 2; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
    return v;
}
template <int LANES>
__device__ __forceinline__ float over_lanes_sum(float v)
{
#pragma unroll
    for (int d = LANES / 2; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// V neighbouring experts' numbers of a row from e0 on, as they lie in memory.  FULL: E is a multiple of V, so that a lane has all of
// them or none.  Either way without a branch, so that all that a row needs is on its way together; what is behind the last expert is
// the row's first or last.
template <typename T, int V, bool FULL>
struct Experts {
    typedef T loose __attribute__((ext_vector_type(V), aligned(sizeof(T))));
    T v[V];
    __device__ __forceinline__ void load(const T* __restrict__ row, int e0, int E)
    {
        if constexpr (FULL && V > 1) {
            const loose x = *reinterpret_cast<const loose*>(row + (e0 < E ? e0 : 0));
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = x[i];
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = row[min(e0 + i, E - 1)];
        }
    }
    // logits: -infinity behind the last
    __device__ __forceinline__ void numbers(float (&x)[V], int e0, int E) const
    {
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = e0 + i < E ? (float)v[i] : -__builtin_inff();
    }
    static __device__ __forceinline__ void store(T* __restrict__ row, int e0, int E, const float (&x)[V])
    {
        if constexpr (FULL && V > 1) {
            loose o;
#pragma unroll
            for (int i = 0; i < V; ++i) o[i] = (T)x[i];
            if (e0 < E) *reinterpret_cast<loose*>(row + e0) = o;
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (e0 + i < E) row[e0 + i] = (T)x[i];
        }
    }
};

// x becomes the softmax of the row that LANES lanes hold; a row of which nothing is left becomes zeros, one with NaN or
// +infinity NaN (of a maximum that passes NaN by, the exponentials still are).
template <int LANES, int V>
__device__ __forceinline__ void softmax(float (&x)[V])
{
    float m = x[0];
#pragma unroll
    for (int v = 1; v < V; ++v) m = fmaxf(m, x[v]);
    m = over_lanes_max<LANES>(m);
    m = m == -__builtin_inff() ? 0.0f : m;
    float total = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) total += x[v] = expf(x[v] - m);
    total = over_lanes_sum<LANES>(total);
    const float scale = total == 0.0f ? 0.0f : 1.0f / total;
#pragma unroll
    for (int v = 0; v < V; ++v) x[v] *= scale;
}

// Whether a row chose an expert: lane j of the row's lanes has choice j (k <= 16 <= LANES), -1 where it is none
template <int LANES>
__device__ __forceinline__ bool any_choice(int32_t mine)
{
    const int lane = threadIdx.x & 63;
    const uint64_t who = __ballot(mine >= 0);
    return LANES == 64 ? who != 0 : (who >> (lane & 48) & 0xffff) != 0;
}
template <int LANES>
__device__ __forceinline__ int32_t choice_of(const int32_t* __restrict__ experts, int64_t t, int k, int E)
{
    const int sub = threadIdx.x & (LANES - 1);
    const int32_t e = experts[t * k + min(sub, k - 1)];
    return (int)(sub < k) & (int)(e < E) ? e : -1;  // (&&: a branch, and a wait for each row's)
}

// f - 1 of an expert of a sequence with n > 0 tokens
// (whole numbers below 2^42, which 64-bit floats hold; even: k n, by: one over it)
__device__ __forceinline__ float over_even(int32_t count, double even, float by, int E)
{
    return (float)__builtin_fma((double)count, (double)E, -even) * by;
}

// What the tiles leave for the second launch: p's sums, pairs by expert, rows that chose.
struct Partial {
    float* sums;       // tiles x E
    int32_t* counts;   // tiles x E
    int32_t* rows;     // tiles
    float* losses;     // sequences
    int64_t tiles, bytes;
};
Partial partial_view(char* workspace, int64_t T, int64_t E, int64_t S)
{
    const auto up = [](int64_t n) { return (n + 255) / 256 * 256; };
    Partial p;
    p.tiles = most_row_tiles(S, T, kRows, true);
    int64_t at = 0;
    const auto take = [&](int64_t bytes) {
        char* q = workspace + at;
        at += up(bytes);
        return q;
    };
    p.sums = reinterpret_cast<float*>(take(p.tiles * E * 4));
    p.counts = reinterpret_cast<int32_t*>(take(p.tiles * E * 4));
    p.rows = reinterpret_cast<int32_t*>(take(p.tiles * 4));
    p.losses = reinterpret_cast<float*>(take(S * 4));
    p.bytes = at;
    return p;
}

template <typename T, int LANES, int V, bool FULL>
__global__ __launch_bounds__(kThreads) void balance_tiles_kernel(BalanceArgs a, Partial p, int64_t block0)
{
    constexpr int kGroups = kThreads / LANES;
    __shared__ float sums[kGroups][LANES * V];
    __shared__ int32_t counts[kMostExperts], rows;
    const int sub = threadIdx.x & (LANES - 1), group = threadIdx.x / LANES;
    const int64_t index = block0 + blockIdx.x;
    const RowTile tile = find_row_tile<kRows>(a.segments, a.S, a.T, index);
    if (tile.rows <= 0 || tile.g >= a.S) return;
    for (int e = threadIdx.x; e < a.E; e += kThreads) counts[e] = 0;
    if (threadIdx.x == 0) rows = 0;
    __syncthreads();
    float sum[V];
#pragma unroll
    for (int v = 0; v < V; ++v) sum[v] = 0.0f;
    constexpr int kTurns = kRows / kGroups, kAtOnce = V * kTurns > 64 ? 64 / V : kTurns;  // a group's rows; on their way together
    static_assert(kTurns % kAtOnce == 0, "");
#pragma unroll 1
    for (int i0 = 0; i0 < kTurns; i0 += kAtOnce) {
        int32_t e[kAtOnce];
        Experts<T, V, FULL> x[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            // (in place of a row past the last, that one; it is not counted)
            const int r = (i0 + i) * kGroups + group;
            const int64_t t = tile.first + min(r, tile.rows - 1);
            e[i] = choice_of<LANES>(a.experts, t, a.k, a.E);
            if (r >= tile.rows) e[i] = -1;
            x[i].load(static_cast<const T*>(a.logits) + t * a.ld, sub * V, a.E);
        }
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            if (e[i] >= 0) atomicAdd(&counts[e[i]], 1);
            if (!any_choice<LANES>(e[i])) continue;
            if (sub == 0) atomicAdd(&rows, 1);
            float p[V];
            x[i].numbers(p, sub * V, a.E);
            softmax<LANES, V>(p);
#pragma unroll
            for (int v = 0; v < V; ++v) sum[v] += p[v];
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) sums[group][sub * V + v] = sum[v];
    __syncthreads();
    for (int e = threadIdx.x; e < a.E; e += kThreads) {
        float s = 0.0f;
#pragma unroll
        for (int g = 0; g < kGroups; ++g) s += sums[g][e];
        p.sums[index * a.E + e] = s;
        p.counts[index * a.E + e] = counts[e];
    }
    if (threadIdx.x == 0) p.rows[index] = rows;
}

// A sequence's tiles, by one workgroup: LINES of E threads each take every LINES-th tile.
__global__ __launch_bounds__(kJoinThreads) void balance_join_kernel(BalanceArgs a, Partial p, int64_t block0)
{
    __shared__ float sums[kJoinThreads], wave_loss[kJoinThreads / 64];
    __shared__ int32_t counts[kJoinThreads], wave_rows[kJoinThreads / 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t seq = block0 + blockIdx.x;
    // the sequence's first tile: those of the sequences before it
    int64_t first = 0;
    if (a.segments) {
        for (int64_t g0 = 0; g0 < seq; g0 += 64) {
            GroupRows r = {0, 0};
            if (g0 + lane < seq) r = group_rows(a.segments, g0 + lane, a.T);
            int t = (int)((r.end - r.first + kRows - 1) / kRows);
#pragma unroll
            for (int d = 32; d; d >>= 1) t += __shfl_xor(t, d);
            first += t;
        }
    }
    const GroupRows own = group_rows(a.segments, seq, a.T);
    // (offsets that are not in order may name more tiles than there are)
    const int64_t end = min(first + (own.end - own.first + kRows - 1) / kRows, p.tiles);
    int n = 0;
    for (int64_t t = first + threadIdx.x; t < end; t += kJoinThreads) n += p.rows[t];
#pragma unroll
    for (int d = 32; d; d >>= 1) n += __shfl_xor(n, d);
    if (lane == 0) wave_rows[wave] = n;
    const int lines = kJoinThreads / a.E, line = threadIdx.x / a.E, e = threadIdx.x - line * a.E;
    float s = 0.0f;
    int32_t c = 0;
    if (line < lines) {
        int64_t t = first + line;
        constexpr int kAtOnce = 16;
        for (; t + (kAtOnce - 1) * lines < end; t += kAtOnce * lines) {
            float more[kAtOnce];
            int32_t pairs[kAtOnce];
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
                more[i] = p.sums[(t + i * lines) * a.E + e];
                pairs[i] = p.counts[(t + i * lines) * a.E + e];
            }
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
                s += more[i];
                c += pairs[i];
            }
        }
        for (; t < end; t += lines) {
            s += p.sums[t * a.E + e];
            c += p.counts[t * a.E + e];
        }
    }
    sums[threadIdx.x] = s;
    counts[threadIdx.x] = c;
    __syncthreads();
    n = 0;
#pragma unroll
    for (int w = 0; w < kJoinThreads / 64; ++w) n += wave_rows[w];
    float loss = 0.0f;
    if (threadIdx.x < a.E) {
        for (int i = 1; i < lines; ++i) {
            s += sums[i * a.E + e];
            c += counts[i * a.E + e];
        }
        a.counts[seq * a.E + e] = c;
        const double even = (double)a.k * n;
        if (n > 0) loss = (1.0f + over_even(c, even, 1.0f / (float)even, a.E)) * (s / (float)n);
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) loss += __shfl_xor(loss, d);
    if (lane == 0) wave_loss[wave] = loss;
    __syncthreads();
    if (threadIdx.x == 0) {
        loss = 0.0f;
        for (int w = 0; w < kJoinThreads / 64; ++w) loss += wave_loss[w];
        a.rows[seq] = n;
        (a.S == 1 ? a.loss : p.losses + seq)[0] = loss;
    }
}

// Sequences that have a token, by a whole workgroup
template <int THREADS>
__device__ __forceinline__ int sequences_used(const int32_t* __restrict__ rows, int64_t S)
{
    __shared__ int32_t part[THREADS / 64];
    int n = 0;
    for (int64_t i = threadIdx.x; i < S; i += THREADS) n += rows[i] > 0;
#pragma unroll
    for (int d = 32; d; d >>= 1) n += __shfl_xor(n, d);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = n;
    __syncthreads();
    n = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) n += part[w];
    return n;
}

__global__ __launch_bounds__(kThreads) void balance_mean_kernel(BalanceArgs a, Partial p)
{
    __shared__ float part[kThreads / 64];
    const int used = sequences_used<kThreads>(a.rows, a.S);
    float s = 0.0f;
    for (int64_t i = threadIdx.x; i < a.S; i += kThreads) s += p.losses[i];
#pragma unroll
    for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = 0.0f;
        for (int w = 0; w < kThreads / 64; ++w) s += part[w];
        a.loss[0] = used > 0 ? s / (float)used : 0.0f;
    }
}

// SEQUENCES: there are segments.
template <typename T, int LANES, int V, bool FULL, bool SEQUENCES>
__global__ __launch_bounds__(kThreads) void balance_grad_kernel(BalanceGradArgs a, int64_t row_blocks)
{
    constexpr int kGroups = kThreads / LANES;
    const int sub = threadIdx.x & (LANES - 1), group = threadIdx.x / LANES, e0 = sub * V;
    Experts<int32_t, V, FULL> count;
    int32_t n = 0;
    if (!SEQUENCES) {
        count.load(a.counts, e0, a.E);
        n = a.rows[0];
    }
    const float dloss = a.dloss[0];
    const int used = SEQUENCES ? sequences_used<kThreads>(a.rows, a.S) : 1;
    int64_t of = -1;  // the sequence whose f are held
    float f[V], scale = 0.0f;
    for (int64_t b = blockIdx.x; b < row_blocks; b += gridDim.x) {
        const int64_t t = b * kGroups + group;
        if (t >= a.T) continue;
        Experts<T, V, FULL> held, was;
        held.load(static_cast<const T*>(a.logits) + t * a.ld, e0, a.E);
        const int32_t e = choice_of<LANES>(a.experts, t, a.k, a.E);
        T* const out = static_cast<T*>(a.dlogits) + t * a.ldd;
        if (a.accumulate) was.load(out, e0, a.E);
        int64_t seq = 0;
        bool there = true;
        if (SEQUENCES) {
            // the last sequence that begins at t or before it
            int64_t lo = 0, hi = a.S;
            while (lo < hi) {
                const int64_t mid = (lo + hi) >> 1;
                if (a.segments[mid] <= t) lo = mid + 1;
                else hi = mid;
            }
            there = lo > 0 && t < a.segments[lo];
            seq = lo > 0 ? lo - 1 : 0;
        }
        if (seq != of) {
            of = seq;
            if (SEQUENCES) {
                count.load(a.counts + seq * a.E, e0, a.E);
                n = a.rows[seq];
            }
            const double even = (double)a.k * n;
            const float by = n > 0 ? 1.0f / (float)even : 0.0f;
            scale = n > 0 && used > 0 ? dloss / ((float)used * (float)n) : 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v) f[v] = e0 + v < a.E ? over_even(count.v[v], even, by, a.E) : 0.0f;
        }
        there = any_choice<LANES>(e) && there && n > 0 && used > 0;
        if (!there && a.accumulate) continue;
        float x[V];
        if (there) {
            held.numbers(x, e0, a.E);
            softmax<LANES, V>(x);
            float inner = 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v) inner = __builtin_fmaf(f[v], x[v], inner);
            inner = over_lanes_sum<LANES>(inner);
#pragma unroll
            for (int v = 0; v < V; ++v) x[v] = scale * x[v] * (f[v] - inner) + (a.accumulate ? (float)was.v[v] : 0.0f);
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) x[v] = 0.0f;
        }
        held.store(out, e0, a.E, x);
    }
}

// F(lanes, experts to a lane)
template <typename F>
hipError_t by_experts(int E, F&& f)
{
    using std::integral_constant;
    if (E <= 16) return f(integral_constant<int, 16>{}, integral_constant<int, 1>{});
    if (E <= 32) return f(integral_constant<int, 16>{}, integral_constant<int, 2>{});
    if (E <= 64) return f(integral_constant<int, 16>{}, integral_constant<int, 4>{});
    if (E <= 128) return f(integral_constant<int, 16>{}, integral_constant<int, 8>{});
    if (E <= 256) return f(integral_constant<int, 16>{}, integral_constant<int, 16>{});
    if (E <= 512) return f(integral_constant<int, 64>{}, integral_constant<int, 8>{});
    return f(integral_constant<int, 64>{}, integral_constant<int, 16>{});
}

template <typename T>
hipError_t balance(const BalanceArgs& a, hipStream_t s)
{
    const Partial p = partial_view(a.workspace, a.T, a.E, a.S);
    hipError_t err = by_experts(a.E, [&](auto lanes, auto v) {
        constexpr int L = decltype(lanes)::value, V = decltype(v)::value;
        return launch_parts(most_row_tiles(a.S, a.T, kRows, a.segments != nullptr), kThreads, [&](unsigned grid, int64_t block0) {
            if (a.E % V == 0) balance_tiles_kernel<T, L, V, true><<<grid, kThreads, 0, s>>>(a, p, block0);
            else balance_tiles_kernel<T, L, V, false><<<grid, kThreads, 0, s>>>(a, p, block0);
        });
    });
    if (err != hipSuccess) return err;
    err = launch_parts(a.S, kJoinThreads, [&](unsigned grid, int64_t block0) {
        balance_join_kernel<<<grid, kJoinThreads, 0, s>>>(a, p, block0);
    });
    if (err != hipSuccess || a.S == 1) return err;
    balance_mean_kernel<<<1, kThreads, 0, s>>>(a, p);
    return hipGetLastError();
}

template <typename T>
hipError_t balance_grad(const BalanceGradArgs& a, hipStream_t s)
{
    return by_experts(a.E, [&](auto lanes, auto v) {
        constexpr int kGroups = kThreads / decltype(lanes)::value;
        const int64_t row_blocks = (a.T + kGroups - 1) / kGroups;
        const unsigned grid = (unsigned)(row_blocks < 2048 ? row_blocks : 2048);
        constexpr int L = decltype(lanes)::value, V = decltype(v)::value;
        if (a.E % V == 0) {
            if (a.segments) balance_grad_kernel<T, L, V, true, true><<<grid, kThreads, 0, s>>>(a, row_blocks);
            else balance_grad_kernel<T, L, V, true, false><<<grid, kThreads, 0, s>>>(a, row_blocks);
        } else {
            if (a.segments) balance_grad_kernel<T, L, V, false, true><<<grid, kThreads, 0, s>>>(a, row_blocks);
            else balance_grad_kernel<T, L, V, false, false><<<grid, kThreads, 0, s>>>(a, row_blocks);
        }
        return hipGetLastError();
    });
}

}  // namespace

int64_t balance_workspace_bytes(int64_t T, int64_t E, int64_t S) { return partial_view(nullptr, T, E, S).bytes; }

hipError_t launch_balance(const BalanceArgs& a, hipStream_t s)
{
    switch (a.dtype) {
        case 0: return balance<float>(a, s);
        case 1: return balance<half_t>(a, s);
        default: return balance<bf16_t>(a, s);
    }
}

hipError_t launch_balance_grad(const BalanceGradArgs& a, hipStream_t s)
{
    switch (a.dtype) {
        case 0: return balance_grad<float>(a, s);
        case 1: return balance_grad<half_t>(a, s);
        default: return balance_grad<bf16_t>(a, s);
    }
}

}  // namespace sgap
