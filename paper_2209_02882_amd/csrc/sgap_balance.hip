// The router's balance loss and its gradient.  Sequence s has n_s tokens that chose an expert and c_se pairs of expert e; with
// p_t = softmax of token t's logits over all experts, f_se = E c_se / (k n_s) and P_se = the mean of p_te over its tokens,
//     loss = mean over the sequences that have a token of sum over e of f_se P_se,
//     dl_te = dloss / (sequences * n_s) * p_te * (f_se - sum over i of f_si p_ti);
// the counts are constants.  A token's p sum up to 1, so f - 1 = (E c - k n) / (k n) serves as well as f does, and it is a whole
// number until it is divided: near an even load, which the loss is for, f would lose what counts in the difference.
//
// A row is held by 16 lanes (up to 256 experts) or by a wavefront, some neighbouring experts to a lane, which keeps the sums of
// its own experts over the rows that it sees.  Tiles of rows never cross a sequence; a second launch sums up a sequence's tiles,
// a third the sequences, or a sequence's parts, where there is more than one.  The logits are read once each way (4 MB for 16,384 tokens and 128 experts
// in bf16, which no launch waits for): what is left is the launches, 15.2 us both ways in a row of passes, where three empty ones
// take 10.  From about 300 experts on it is the exponentials and sums of the vector unit and the bytes: 65,536 rows of 512 in bf16,
// 67 MB, 23 us forth and 28 us for the gradient, 201 MB in all at 3.9 TB/s.  Sums of floats in a fixed order; the only atomics count
// whole numbers in LDS.
#include "sgap_grouped.hpp"
#include "sgap_tokens.hpp"

namespace sgap {

namespace {

constexpr int kThreads = 256;
constexpr int kRows = 64;           // of a tile
constexpr int kJoinThreads = 1024, kManyThreads = 256;  // of a sequence's sum, and of one of many sequences'
constexpr int kMostExperts = 1024;

// op over 16 lanes or all 64, the same bits in each: 16 lanes by turning them, then the two halves of each 32 and of the 64 changing
// places.  (By way of LDS, as a shuffle goes, each step takes as long as a row's exponentials.)
template <int LANES, typename F>
__device__ __forceinline__ float over_lanes(float v, F&& op)
{
    const auto bits = [](float x) { return __builtin_bit_cast(int, x); };
    const auto number = [](int x) { return __builtin_bit_cast(float, x); };
    v = op(v, number(__builtin_amdgcn_update_dpp(0, bits(v), 0x128, 0xf, 0xf, true)));
    v = op(v, number(__builtin_amdgcn_update_dpp(0, bits(v), 0x124, 0xf, 0xf, true)));
    v = op(v, number(__builtin_amdgcn_update_dpp(0, bits(v), 0x122, 0xf, 0xf, true)));
    v = op(v, number(__builtin_amdgcn_update_dpp(0, bits(v), 0x121, 0xf, 0xf, true)));
    if constexpr (LANES == 64) {
        const auto a = __builtin_amdgcn_permlane16_swap(bits(v), bits(v), false, false);
        v = op(number(a[0]), number(a[1]));
        const auto b = __builtin_amdgcn_permlane32_swap(bits(v), bits(v), false, false);
        v = op(number(b[0]), number(b[1]));
    }
    return v;
}
template <int LANES>
__device__ __forceinline__ float over_lanes_max(float v)
{
    return over_lanes<LANES>(v, [](float a, float b) { return fmaxf(a, b); });
}
template <int LANES>
__device__ __forceinline__ float over_lanes_sum(float v)
{
    return over_lanes<LANES>(v, [](float a, float b) { return a + b; });
}

// A lane's experts of a row: pieces of P neighbouring ones, as they lie in memory, a piece of every lane and then the next of
// every lane.  The last piece of a row whose length P does not divide reaches back into the one before, so that every load is
// whole and in the row, without a branch: all that a row needs is on its way together.  What it has in common with the one before,
// and what pieces behind the last expert hold (the row's first), is not this lane's own: it is neither summed nor counted.
// (E is at least P.)  By elements, 17,403 rows of 184 took 46 us both ways in place of 18.
constexpr int kMostPiece = 8;
template <int LANES, int V>
struct Held {
    static constexpr int P = V < kMostPiece ? V : kMostPiece, kPieces = V / P;
    int first[kPieces];  // expert that the piece begins with
    int own[kPieces];    // its first element that is this lane's, P: none
    __device__ __forceinline__ Held(int E)
    {
        const int sub = threadIdx.x & (LANES - 1);
#pragma unroll
        for (int h = 0; h < kPieces; ++h) {
            const int e = (h * LANES + sub) * P, f = min(e, E - P);
            own[h] = e < E ? e - f : P;
            first[h] = e < E ? f : 0;
        }
    }
    __device__ __forceinline__ bool has(int v) const { return v % P >= own[v / P]; }
    __device__ __forceinline__ int expert(int v) const { return first[v / P] + v % P; }
};
template <typename T, int LANES, int V>
struct Experts {
    using H = Held<LANES, V>;
    typedef T loose __attribute__((ext_vector_type(H::P), aligned(sizeof(T))));
    loose piece[H::kPieces];
    __device__ __forceinline__ void load(const T* __restrict__ row, const H& held)
    {
#pragma unroll
        for (int h = 0; h < H::kPieces; ++h) piece[h] = *reinterpret_cast<const loose*>(row + held.first[h]);
    }
    __device__ __forceinline__ T operator[](int v) const
    {
        if constexpr (H::P == 1) return reinterpret_cast<const T&>(piece[v]);
        else return piece[v / H::P][v % H::P];
    }
    // (two lanes that have an element both store the same)
    static __device__ __forceinline__ void store(T* __restrict__ row, const H& held, const float (&x)[V])
    {
#pragma unroll
        for (int h = 0; h < H::kPieces; ++h) {
            loose o;
            if constexpr (H::P == 1) reinterpret_cast<T&>(o) = (T)x[h];
            else {
#pragma unroll
                for (int i = 0; i < H::P; ++i) o[i] = (T)x[h * H::P + i];
            }
            if (held.own[h] < H::P) *reinterpret_cast<loose*>(row + held.first[h]) = o;
        }
    }
};

// x: the softmax of the row that LANES lanes hold; a row of which nothing is left becomes zeros, one with NaN or
// +infinity NaN (of a maximum that passes NaN by, the exponentials still are).
template <typename T, int LANES, int V>
__device__ __forceinline__ void softmax(const Experts<T, LANES, V>& logits, const Held<LANES, V>& held, float (&x)[V])
{
    float m = -__builtin_inff();
#pragma unroll
    for (int v = 0; v < V; ++v) {
        x[v] = (float)logits[v];
        m = fmaxf(m, x[v]);
    }
    m = over_lanes_max<LANES>(m);
    m = m == -__builtin_inff() ? 0.0f : m;
    float total = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        // (2^ by the instruction for it: the factor's rounding is another |x - m| 2^-24 of the result, as the difference's is, and what
        // is below 2^-126 becomes 0.  With a function that does more, 65,536 rows of 512 in bf16 take 30 us in place of 23.)
        x[v] = __builtin_amdgcn_exp2f((x[v] - m) * 1.44269504f);
        total += held.has(v) ? x[v] : 0.0f;
    }
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
    float* losses;     // sequences x parts
    int64_t tiles, bytes;
    int parts, part;   // workgroups that share a sequence's experts, and experts of each
    int threads;       // of those
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
    // one workgroup for a sequence, or one for 64 of its experts where it has much to read (us of the join, one and several:
    // 35,906 rows of 353 26, 10; 65,536 rows of 512 46, 12; the mean's launch comes to 2)
    // (Many sequences share the compute units: 1,000 of 16,384 tokens, 128 experts, loss alone with workgroups of 1,024 threads 21.6 us,
    // of 256 14.3; 20,000 sequences 246, 99; one long one and 999 of a token each 25.3, 20.0; of 65,536 tokens, 256 experts 29.9, 22.8 and 58, 71)
    p.threads = S >= 512 ? kManyThreads : kJoinThreads;
    p.part = p.tiles / S * E >= 65536 ? 64 : (int)(E < p.threads ? E : p.threads);
    p.parts = (int)((E + p.part - 1) / p.part);
    p.losses = reinterpret_cast<float*>(take(S * p.parts * 4));
    p.bytes = at;
    return p;
}

// The first tile of sequence `seq`, which begins at token `first`: the sequences before it have first tokens, so that no more than
// min(seq, first) of them have any, and each has one tile at most that is not full.  Some tiles are of no sequence, but nobody has to count
// those of all sequences before (which took 31 us of 41 with 1,000 sequences, and 5 ms with 20,000).
__device__ __forceinline__ int64_t first_tile(int64_t first, int64_t seq) { return first / kRows + min(seq, first); }

// Tile number `index`, of no rows if no sequence has it.  By one wavefront, whose lanes look for the last sequence that begins at this tile or
// before it in 64 places at a time; every lane gets the answer.
__device__ __forceinline__ RowTile find_tile(const int32_t* __restrict__ segments, int S, int64_t T, int64_t index)
{
    if (!segments) return {0, index * kRows, (int)min((int64_t)kRows, T - index * kRows)};
    const int lane = threadIdx.x & 63;
    int lo = 0, n = S;
    for (;;) {
        const int step = (n + 63) / 64, seq = lo + min(lane * step, n - 1);
        const GroupRows rows = group_rows(segments, seq, T);
        const int64_t tile = first_tile(rows.first, seq);
        const uint64_t upto = __ballot(lane * step < n && tile <= index);
        if (!upto) return {S, 0, 0};
        const int who = 63 - __builtin_clzll(upto);
        if (step == 1) {
            const int64_t first = __builtin_amdgcn_readlane((int)rows.first, who), end = __builtin_amdgcn_readlane((int)rows.end, who);
            const int64_t at = first + (index - first_tile(first, lo + who)) * kRows;
            return {lo + who, at, at < end ? (int)min((int64_t)kRows, end - at) : 0};
        }
        lo += who * step;
        n = min(step, n - who * step);
    }
}

template <typename T, int LANES, int V>
__global__ __launch_bounds__(kThreads) void balance_tiles_kernel(BalanceArgs a, Partial p, int64_t block0)
{
    constexpr int kGroups = kThreads / LANES;
    __shared__ float sums[kGroups][LANES * V];
    __shared__ int32_t counts[kMostExperts], rows;
    const int sub = threadIdx.x & (LANES - 1), group = threadIdx.x / LANES;
    const int64_t index = block0 + blockIdx.x;
    const RowTile tile = find_tile(a.segments, (int)a.S, a.T, index);
    if (tile.rows <= 0) {
        // (read only where offsets in no order give it to a sequence all the same)
        for (int e = threadIdx.x; e < a.E; e += kThreads) {
            p.sums[index * a.E + e] = 0.0f;
            p.counts[index * a.E + e] = 0;
        }
        if (threadIdx.x == 0) p.rows[index] = 0;
        return;
    }
    for (int e = threadIdx.x; e < a.E; e += kThreads) counts[e] = 0;
    if (threadIdx.x == 0) rows = 0;
    __syncthreads();
    const Held<LANES, V> held(a.E);
    float sum[V];
#pragma unroll
    for (int v = 0; v < V; ++v) sum[v] = 0.0f;
    constexpr int kTurns = kRows / kGroups, kAtOnce = V * kTurns > 64 ? 64 / V : kTurns;  // a group's rows; on their way together
    static_assert(kTurns % kAtOnce == 0, "");
#pragma unroll 1
    for (int i0 = 0; i0 < kTurns; i0 += kAtOnce) {
        int32_t e[kAtOnce];
        Experts<T, LANES, V> x[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            // (in place of a row past the last, that one; it is not counted)
            const int r = (i0 + i) * kGroups + group;
            const int64_t t = tile.first + min(r, tile.rows - 1);
            e[i] = choice_of<LANES>(a.experts, t, a.k, a.E);
            if (r >= tile.rows) e[i] = -1;
            x[i].load(static_cast<const T*>(a.logits) + t * a.ld, held);
        }
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            if (e[i] >= 0) atomicAdd(&counts[e[i]], 1);
            if (!any_choice<LANES>(e[i])) continue;
            if (sub == 0) atomicAdd(&rows, 1);
            float p[V];
            softmax(x[i], held, p);
#pragma unroll
            for (int v = 0; v < V; ++v) sum[v] += p[v];
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v)
        if (held.has(v)) sums[group][held.expert(v)] = sum[v];
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

// A sequence's tiles, or of a part of its experts: lines of E threads each take every `lines`th tile.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void balance_join_kernel(BalanceArgs a, Partial p, int64_t block0)
{
    __shared__ float sums[THREADS], wave_loss[THREADS / 64];
    __shared__ int32_t counts[THREADS], wave_rows[THREADS / 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t item = block0 + blockIdx.x, seq = item / p.parts;
    const int part = (int)(item - seq * p.parts), e0 = part * p.part, experts = min(p.part, a.E - e0);
    const GroupRows own = group_rows(a.segments, seq, a.T);
    const int64_t first = first_tile(own.first, seq);
    // (offsets that are not in order may name more tiles than there are)
    const int64_t end = min(first + (own.end - own.first + kRows - 1) / kRows, p.tiles);
    int n = 0;
    for (int64_t t = first + threadIdx.x; t < end; t += THREADS) n += p.rows[t];
#pragma unroll
    for (int d = 32; d; d >>= 1) n += __shfl_xor(n, d);
    if (lane == 0) wave_rows[wave] = n;
    // (no more lines than a line has loads on their way: they are added up one after the other)
    constexpr int kAtOnce = 16;
    const int lines = min(THREADS / experts, 2 * kAtOnce), line = threadIdx.x / experts, e = threadIdx.x - line * experts;
    float s = 0.0f;
    int32_t c = 0;
    if (line < lines) {
        for (int64_t t = first + line; t < end; t += kAtOnce * lines) {
            float more[kAtOnce];
            int32_t pairs[kAtOnce];
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
                const int64_t at = min(t + i * lines, end - 1) * a.E + e0 + e;
                more[i] = p.sums[at];
                pairs[i] = p.counts[at];
            }
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
                s += t + i * lines < end ? more[i] : 0.0f;
                c += t + i * lines < end ? pairs[i] : 0;
            }
        }
    }
    sums[threadIdx.x] = s;
    counts[threadIdx.x] = c;
    __syncthreads();
    n = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) n += wave_rows[w];
    float loss = 0.0f;
    if ((int)threadIdx.x < experts) {
        for (int i = 1; i < lines; ++i) {
            s += sums[i * experts + e];
            c += counts[i * experts + e];
        }
        a.counts[seq * a.E + e0 + e] = c;
        const double even = (double)a.k * n;
        if (n > 0) loss = (1.0f + over_even(c, even, 1.0f / (float)even, a.E)) * (s / (float)n);
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) loss += __shfl_xor(loss, d);
    if (lane == 0) wave_loss[wave] = loss;
    __syncthreads();
    if (threadIdx.x == 0) {
        loss = 0.0f;
        for (int w = 0; w < THREADS / 64; ++w) loss += wave_loss[w];
        if (part == 0) a.rows[seq] = n;
        (a.S * p.parts == 1 ? a.loss : p.losses + item)[0] = loss;
    }
}

// Sequences that have a token, by a whole workgroup
template <int THREADS>
__device__ __forceinline__ int sequences_used(const int32_t* __restrict__ rows, int64_t S)
{
    __shared__ int32_t part[THREADS / 64];
    int n = 0;
#pragma unroll 8
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
#pragma unroll 8
    for (int64_t i = threadIdx.x; i < a.S * p.parts; i += kThreads) s += p.losses[i];
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

// SEQUENCES: there are segments.  Each workgroup counts those that have a token, which takes longer the more there are (us, 128
// experts, bf16, 1 / 1,000 / 20,000 / 65,536 sequences: 16,384 tokens 4.6, 6.5, 9.8, 15.2; 65,536 tokens 8.8, 15.2, 24.3, 36.5).
template <typename T, int LANES, int V, bool SEQUENCES>
__global__ __launch_bounds__(kThreads) void balance_grad_kernel(BalanceGradArgs a, int64_t row_blocks)
{
    constexpr int kGroups = kThreads / LANES;
    const int group = threadIdx.x / LANES;
    const Held<LANES, V> held(a.E);
    Experts<int32_t, LANES, V> count;
    int32_t n = 0;
    if (!SEQUENCES) {
        count.load(a.counts, held);
        n = a.rows[0];
    }
    const float dloss = a.dloss[0];
    const int used = SEQUENCES ? sequences_used<kThreads>(a.rows, a.S) : 1;
    int64_t of = -1;  // the sequence whose f are held
    float f[V], scale = 0.0f;
    for (int64_t b = blockIdx.x; b < row_blocks; b += gridDim.x) {
        const int64_t t = b * kGroups + group;
        if (t >= a.T) continue;
        Experts<T, LANES, V> logits, was;
        logits.load(static_cast<const T*>(a.logits) + t * a.ld, held);
        const int32_t e = choice_of<LANES>(a.experts, t, a.k, a.E);
        T* const out = static_cast<T*>(a.dlogits) + t * a.ldd;
        if (a.accumulate) was.load(out, held);
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
                count.load(a.counts + seq * a.E, held);
                n = a.rows[seq];
            }
            const double even = (double)a.k * n;
            const float by = n > 0 ? 1.0f / (float)even : 0.0f;
            scale = n > 0 && used > 0 ? dloss / ((float)used * (float)n) : 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v) f[v] = over_even(count[v], even, by, a.E);
        }
        there = any_choice<LANES>(e) && there && n > 0 && used > 0;
        if (!there && a.accumulate) continue;
        float x[V];
        if (there) {
            softmax(logits, held, x);
            float inner = 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v) inner = held.has(v) ? __builtin_fmaf(f[v], x[v], inner) : inner;
            inner = over_lanes_sum<LANES>(inner);
#pragma unroll
            for (int v = 0; v < V; ++v) x[v] = scale * x[v] * (f[v] - inner) + (a.accumulate ? (float)was[v] : 0.0f);
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) x[v] = 0.0f;
        }
        logits.store(out, held, x);
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
            balance_tiles_kernel<T, L, V><<<grid, kThreads, 0, s>>>(a, p, block0);
        });
    });
    if (err != hipSuccess) return err;
    err = launch_parts(a.S * p.parts, p.threads, [&](unsigned grid, int64_t block0) {
        if (p.threads == kManyThreads) balance_join_kernel<kManyThreads><<<grid, kManyThreads, 0, s>>>(a, p, block0);
        else balance_join_kernel<kJoinThreads><<<grid, kJoinThreads, 0, s>>>(a, p, block0);
    });
    if (err != hipSuccess || a.S * p.parts == 1) return err;
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
        if (a.segments) balance_grad_kernel<T, L, V, true><<<grid, kThreads, 0, s>>>(a, row_blocks);
        else balance_grad_kernel<T, L, V, false><<<grid, kThreads, 0, s>>>(a, row_blocks);
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
