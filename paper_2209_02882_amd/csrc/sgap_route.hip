// The router: the k largest of E logits for each of T tokens, their gates, and the pairs (token, expert) grouped by
// expert; and the gradient of the logits.
//
// gates: p = exp(l - m) / sum over all experts, or over the chosen ones where they are renormalised; m, the largest logit,
// is the first that is chosen, so one pass over a row that lies in registers has everything.
//
// A row is held by a group of 16 lanes (up to 256 experts) or by a wavefront, some consecutive experts to a lane.  Choosing
// goes by k rounds of "largest of the lanes' largest": the values as ordered integers, a maximum by row rotations, the
// lowest lane that holds it.  What bounds it is those rounds' instructions, so four rows to a wavefront.
//
// Grouping is a counting sort that keeps the pairs' order: every block counts its pairs by expert and ranks them among
// themselves (pairs of one expert found by comparing the bits of 64 experts at a time), the counts are summed up over
// the blocks, and every pair is put in its place.  No atomics, so that the lists are the same on every run.
#include "sgap_experts.hpp"

namespace sgap {

namespace {

constexpr int kRouteThreads = 256;
constexpr int kMaxExperts = 1024;
constexpr int kMaxChosen = 16;
constexpr int kBlockPairs = 1024;  // pairs of a block at most
constexpr int kWaves = kRouteThreads / 64;

// Ordered like the floats: NaN above everything (as a sort has it), -infinity, which is never chosen, 0.  -0 is +0.
__device__ __forceinline__ uint32_t order_key(float x)
{
    if (x != x) return 0xffffffffu;
    if (x == -__builtin_inff()) return 0u;
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b ^ ((int32_t)b < 0 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k)
{
    return __uint_as_float(k == 0xffffffffu ? 0x7fc00000u : k ^ ((int32_t)k < 0 ? 0x80000000u : 0xffffffffu));
}

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
constexpr int kRor1 = 0x121, kRor2 = 0x122, kRor4 = 0x124, kRor8 = 0x128;

// over the 16 or 64 lanes that hold a row; all of them get it
template <int LANES>
__device__ __forceinline__ uint32_t lanes_max(uint32_t v)
{
    v = max(v, dpp<kRor8>(v));
    v = max(v, dpp<kRor4>(v));
    v = max(v, dpp<kRor2>(v));
    v = max(v, dpp<kRor1>(v));
    if constexpr (LANES == 64) {
        v = max(v, (uint32_t)__shfl_xor((int)v, 16));
        v = max(v, (uint32_t)__shfl_xor((int)v, 32));
    }
    return v;
}
template <int LANES>
__device__ __forceinline__ float lanes_sum(float v)
{
    v += __uint_as_float(dpp<kRor8>(__float_as_uint(v)));
    v += __uint_as_float(dpp<kRor4>(__float_as_uint(v)));
    v += __uint_as_float(dpp<kRor2>(__float_as_uint(v)));
    v += __uint_as_float(dpp<kRor1>(__float_as_uint(v)));
    if constexpr (LANES == 64) {
        v += __shfl_xor(v, 16);
        v += __shfl_xor(v, 32);
    }
    return v;
}

template <typename T, int V>
__device__ __forceinline__ void load_row(const T* __restrict__ row, int e0, int E, float (&x)[V])
{
#pragma unroll
    for (int v = 0; v < V; ++v) x[v] = e0 + v < E ? (float)row[e0 + v] : -__builtin_inff();
}

// The k largest of a row that LANES lanes hold, V experts each (expert sub * V + v).  Lane j of them gets choice j.
template <int LANES, int V>
__device__ __forceinline__ void choose(const float (&x)[V], int k, bool renormalise, float& gate, int& expert)
{
    const int lane = threadIdx.x & 63, sub = lane & (LANES - 1);
    uint32_t key[V];
#pragma unroll
    for (int v = 0; v < V; ++v) key[v] = order_key(x[v]);
    uint32_t own = 0;
    expert = -1;
    uint32_t first = 0;
    for (int j = 0; j < k; ++j) {
        uint32_t top = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) top = max(top, key[v]);
        const uint32_t most = lanes_max<LANES>(top);
        if (j == 0) first = most;
        const uint64_t who = __ballot(top == most);
        const uint64_t mine = LANES == 64 ? who : (who >> (lane & 48)) & 0xffffu;
        const int winner = __builtin_ctzll(mine);
        // the winner's first value of that size leaves; every lane learns which it was
        int at = 0;
#pragma unroll
        for (int v = V - 1; v >= 0; --v) at = key[v] == most ? v : at;
        const int e = __shfl(sub * V + at, winner, LANES);
#pragma unroll
        for (int v = 0; v < V; ++v) key[v] = sub == winner && v == at ? 0u : key[v];
        if (sub == j && most != 0) { own = most; expert = e; }
    }
    // first = 0: a row of which nothing is left, and all gates are zero
    const float m = first ? key_value(first) : 0.0f;
    const float mine = expert >= 0 ? expf(key_value(own) - m) : 0.0f;
    float part = mine;
    if (!renormalise) {
        part = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) part += expf(x[v] - m);  // of -infinity: 0
    }
    const float total = lanes_sum<LANES>(part);
    gate = expert >= 0 ? mine / total : 0.0f;
}

struct RouteShared {
    int32_t expert[kBlockPairs];
    int32_t count[kWaves][kMaxExperts];  // pairs of each expert in a wavefront's share of the pairs
};

// Ranks the pairs of a block among those of the same expert, in their order.  In: s.expert (-1: none).  Out: per pair
// the rank among the earlier pairs of the wavefront's share, in `rank` for the pairs this lane looks at, and s.count.
// A wavefront's share: pairs_per_wave consecutive ones, 64 at a time.
template <typename F>
__device__ __forceinline__ void rank_pairs(RouteShared& s, int E, int pairs, int pairs_per_wave, F&& put)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int e = lane; e < E; e += 64) s.count[wave][e] = 0;
    const uint64_t below = (1ull << lane) - 1;
    const int bits = 32 - __builtin_clz(E);
    const int end = min(pairs, (wave + 1) * pairs_per_wave);
    for (int p0 = wave * pairs_per_wave; p0 < end; p0 += 64) {
        const int p = p0 + lane;
        const int e = p < end ? s.expert[p] : -1;
        uint64_t same = __ballot(e >= 0);
        for (int b = 0; b < bits; ++b) {
            const uint64_t set = __ballot((e >> b) & 1);
            same &= (e >> b) & 1 ? set : ~set;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (e >= 0) {
            const int before = s.count[wave][e];
            put(p, before + __popcll(same & below));
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if ((same & below) == 0) s.count[wave][e] = before + __popcll(same);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

// Rows of the block are chosen for, their experts left in s.expert.
template <typename T, int LANES, int V>
__device__ __forceinline__ void choose_rows(const RouteArgs& a, RouteShared& s, int64_t row0, int rows)
{
    constexpr int kGroups = kRouteThreads / LANES;
    const int sub = threadIdx.x & (LANES - 1), group = threadIdx.x / LANES;
    for (int i = group; i < rows; i += kGroups) {
        const int64_t t = row0 + i;
        float x[V], gate;
        int expert;
        load_row<T, V>(static_cast<const T*>(a.logits) + t * a.ld, sub * V, a.E, x);
        choose<LANES, V>(x, a.k, a.renormalise, gate, expert);
        if (sub < a.k) {
            a.gates[t * a.k + sub] = gate;
            a.experts[t * a.k + sub] = expert;
            s.expert[i * a.k + sub] = expert;
        }
    }
}

// inclusive sum over the 64 lanes
__device__ __forceinline__ int wave_scan(int v)
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
    return v;
}

// out[e] = sum of in[0 .. e) for e <= n, by the whole workgroup, through shared memory
__device__ __forceinline__ void block_offsets(const int32_t* in, int32_t* out, int n, int32_t* wave_total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int carry = 0;
    for (int e0 = 0; e0 < n; e0 += kRouteThreads) {
        const int e = e0 + threadIdx.x;
        const int v = e < n ? in[e] : 0;
        const int inc = wave_scan(v);
        if (lane == 63) wave_total[wave] = inc;
        __syncthreads();
        int base = carry;
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) base += wave_total[w];
            carry += wave_total[w];
        }
        if (e < n) out[e] = base + inc - v;
        __syncthreads();
    }
    if (threadIdx.x == 0) out[n] = carry;
    __syncthreads();
}

// All tokens in one workgroup: one launch, which is what a few tokens cost.
template <typename T, int LANES, int V>
__global__ __launch_bounds__(kRouteThreads) void route_few_kernel(RouteArgs a)
{
    __shared__ RouteShared s;
    __shared__ int32_t total[kMaxExperts], start[kMaxExperts + 1], wave_total[kWaves];
    const int pairs = (int)a.T * a.k;
    choose_rows<T, LANES, V>(a, s, 0, (int)a.T);
    __syncthreads();
    const int per_wave = (pairs + 64 * kWaves - 1) / (64 * kWaves) * 64;
    // the ranks wait in registers: a lane looks at kBlockPairs / 256 pairs at most
    int rank[kBlockPairs / kRouteThreads];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int i = 0; i < kBlockPairs / kRouteThreads; ++i) rank[i] = 0;
    rank_pairs(s, a.E, pairs, per_wave, [&](int p, int r) {
        const int at = (p - wave * per_wave) >> 6;
#pragma unroll
        for (int i = 0; i < kBlockPairs / kRouteThreads; ++i) rank[i] = at == i ? r : rank[i];
    });
    __syncthreads();
    for (int e = threadIdx.x; e < a.E; e += kRouteThreads) {
        int sum = 0;
        for (int w = 0; w < kWaves; ++w) {
            const int c = s.count[w][e];
            s.count[w][e] = sum;
            sum += c;
        }
        total[e] = sum;
    }
    __syncthreads();
    block_offsets(total, start, a.E, wave_total);
    for (int e = threadIdx.x; e <= a.E; e += kRouteThreads) a.offsets[e] = start[e];
#pragma unroll
    for (int i = 0; i < kBlockPairs / kRouteThreads; ++i) {
        const int p = wave * per_wave + i * 64 + lane;
        if (i * 64 < per_wave && p < pairs) {
            const int e = s.expert[p];
            const int at = e >= 0 ? start[e] + s.count[wave][e] + rank[i] : -1;
            a.slot[p] = at;
            if (e >= 0) a.order[at] = p;
        }
    }
    for (int p = start[a.E] + threadIdx.x; p < pairs; p += kRouteThreads) a.order[p] = -1;
}

// Three launches for more: the choice, with the blocks' counts by expert (count[e * blocks + b]) and the pairs' ranks
// within their block (in slot) ...
template <typename T, int LANES, int V>
__global__ __launch_bounds__(kRouteThreads) void route_choose_kernel(RouteArgs a, int rows_per_block, int32_t* count, int blocks)
{
    __shared__ RouteShared s;
    const int64_t row0 = (int64_t)blockIdx.x * rows_per_block;
    const int rows = (int)min((int64_t)rows_per_block, a.T - row0);
    const int pairs = rows * a.k;
    choose_rows<T, LANES, V>(a, s, row0, rows);
    __syncthreads();
    const int per_wave = (pairs + 64 * kWaves - 1) / (64 * kWaves) * 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int rank[kBlockPairs / kRouteThreads];
#pragma unroll
    for (int i = 0; i < kBlockPairs / kRouteThreads; ++i) rank[i] = 0;
    rank_pairs(s, a.E, pairs, per_wave, [&](int p, int r) {
        const int at = (p - wave * per_wave) >> 6;
#pragma unroll
        for (int i = 0; i < kBlockPairs / kRouteThreads; ++i) rank[i] = at == i ? r : rank[i];
    });
    __syncthreads();
    for (int e = threadIdx.x; e < a.E; e += kRouteThreads) {
        int sum = 0;
        for (int w = 0; w < kWaves; ++w) {
            const int c = s.count[w][e];
            s.count[w][e] = sum;
            sum += c;
        }
        count[(int64_t)e * blocks + blockIdx.x] = sum;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kBlockPairs / kRouteThreads; ++i) {
        const int p = wave * per_wave + i * 64 + lane;
        if (i * 64 < per_wave && p < pairs) {
            const int e = s.expert[p];
            a.slot[row0 * a.k + p] = e >= 0 ? s.count[wave][e] + rank[i] : -1;
        }
    }
}

// ... the counts of one expert summed up over the blocks (a wavefront per expert) ...
__global__ __launch_bounds__(kRouteThreads) void route_scan_kernel(int32_t* count, int32_t* total, int blocks, int E)
{
    const int e = blockIdx.x * kWaves + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (e >= E) return;
    int32_t* row = count + (int64_t)e * blocks;
    int carry = 0;
    for (int b0 = 0; b0 < blocks; b0 += 64) {
        const int b = b0 + lane;
        const int v = b < blocks ? row[b] : 0;
        const int inc = wave_scan(v);
        if (b < blocks) row[b] = carry + inc - v;
        carry += __shfl(inc, 63);
    }
    if (lane == 0) total[e] = carry;
}

// ... and every pair into its place.
__global__ __launch_bounds__(kRouteThreads) void route_place_kernel(RouteArgs a, int rows_per_block, const int32_t* count,
                                                                    const int32_t* total, int blocks)
{
    __shared__ int32_t start[kMaxExperts + 1], wave_total[kWaves];
    block_offsets(total, start, a.E, wave_total);
    if (blockIdx.x == 0)
        for (int e = threadIdx.x; e <= a.E; e += kRouteThreads) a.offsets[e] = start[e];
    const int64_t first = (int64_t)blockIdx.x * rows_per_block * a.k;
    const int64_t end = min(first + (int64_t)rows_per_block * a.k, a.T * a.k);
    for (int64_t p = first + threadIdx.x; p < end; p += kRouteThreads) {
        const int e = a.experts[p];
        if (e >= 0) {
            const int at = start[e] + count[(int64_t)e * blocks + blockIdx.x] + a.slot[p];
            a.slot[p] = at;
            a.order[at] = (int32_t)p;
        }
        if (p >= start[a.E]) a.order[p] = -1;  // places that no pair has
    }
}

// dl_e = p_e ([e chosen] dg_e - sum of g dg) with p over all experts, or, renormalised, the same over the chosen ones alone.
template <typename T, int LANES, int V>
__global__ __launch_bounds__(kRouteThreads) void route_grad_kernel(RouteGradArgs a)
{
    constexpr int kGroups = kRouteThreads / LANES;
    const int sub = threadIdx.x & (LANES - 1);
    const int64_t t = (int64_t)blockIdx.x * kGroups + threadIdx.x / LANES;
    if (t >= a.T) return;
    int expert = -1;
    float gate = 0.0f, dgate = 0.0f;
    if (sub < a.k) {
        expert = a.experts[t * a.k + sub];
        if (expert >= 0) {
            gate = a.gates[t * a.k + sub];
            dgate = a.dgates[t * a.k + sub];
        }
    }
    const float inner = lanes_sum<LANES>(gate * dgate);
    float d[V];
    if (a.renormalise) {
#pragma unroll
        for (int v = 0; v < V; ++v) d[v] = 0.0f;
    } else {
        float x[V], m = -__builtin_inff();
        load_row<T, V>(static_cast<const T*>(a.logits) + t * a.ld, sub * V, a.E, x);
        uint32_t top = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) top = max(top, order_key(x[v]));
        top = lanes_max<LANES>(top);
        m = top ? key_value(top) : 0.0f;
        float part = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            d[v] = expf(x[v] - m);
            part += d[v];
        }
        const float total = lanes_sum<LANES>(part);
        const float scale = top ? -inner / total : 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) d[v] *= scale;
    }
    const float own = a.renormalise ? gate * (dgate - inner) : gate * dgate;
    for (int j = 0; j < a.k; ++j) {
        const int e = __shfl(expert, j, LANES) - sub * V;
        const float g = __shfl(own, j, LANES);
#pragma unroll
        for (int v = 0; v < V; ++v) d[v] += e == v ? g : 0.0f;
    }
    T* __restrict__ out = static_cast<T*>(a.dlogits) + t * a.ldd;
#pragma unroll
    for (int v = 0; v < V; ++v)
        if (sub * V + v < a.E) out[sub * V + v] = (T)d[v];
}

template <typename F, typename T>
bool by_experts(int E, F&& f, T)
{
    if (E <= 16) f.template operator()<T, 16, 1>();
    else if (E <= 32) f.template operator()<T, 16, 2>();
    else if (E <= 64) f.template operator()<T, 16, 4>();
    else if (E <= 128) f.template operator()<T, 16, 8>();
    else if (E <= 256) f.template operator()<T, 16, 16>();
    else if (E <= 512) f.template operator()<T, 64, 8>();
    else f.template operator()<T, 64, 16>();
    return true;
}
template <typename F>
bool by_type(int dtype, int E, F&& f)
{
    switch (dtype) {
        case 0: return by_experts(E, f, 0.0f);
        case 1: return by_experts(E, f, half_t(0));
        default: return by_experts(E, f, bf16_t(0));
    }
}

// Rows of a block: up to kBlockPairs pairs; 64 rows unless there are so many tokens that the blocks' counts would be long.
int rows_per_block(int64_t T, int k)
{
    const int most = kBlockPairs / k;
    return most < 64 ? most : 64;
}

struct RouteFew {
    const RouteArgs& a;
    hipStream_t s;
    template <typename T, int LANES, int V>
    void operator()() const { route_few_kernel<T, LANES, V><<<1, kRouteThreads, 0, s>>>(a); }
};
struct RouteChoose {
    const RouteArgs& a;
    hipStream_t s;
    int rows, blocks;
    int32_t* count;
    template <typename T, int LANES, int V>
    void operator()() const { route_choose_kernel<T, LANES, V><<<blocks, kRouteThreads, 0, s>>>(a, rows, count, blocks); }
};
struct RouteGrad {
    const RouteGradArgs& a;
    hipStream_t s;
    template <typename T, int LANES, int V>
    void operator()() const
    {
        constexpr int kGroups = kRouteThreads / LANES;
        route_grad_kernel<T, LANES, V><<<(unsigned)((a.T + kGroups - 1) / kGroups), kRouteThreads, 0, s>>>(a);
    }
};

// One workgroup for all tokens: up to 64 rows, four passes of its sixteen groups of lanes.
bool route_in_one(int64_t T, int k) { return T <= 64 && T * k <= kBlockPairs; }

}  // namespace

int64_t route_workspace_bytes(int64_t T, int64_t E, int64_t k)
{
    if (route_in_one(T, (int)k)) return 0;
    const int64_t rows = rows_per_block(T, (int)k), blocks = (T + rows - 1) / rows;
    return 4 * E * (blocks + 1);
}

hipError_t launch_route(const RouteArgs& a, hipStream_t s)
{
    if (route_in_one(a.T, a.k)) {
        by_type(a.dtype, a.E, RouteFew{a, s});
        return hipGetLastError();
    }
    const int rows = rows_per_block(a.T, a.k), blocks = (int)((a.T + rows - 1) / rows);
    int32_t *count = static_cast<int32_t*>(a.workspace), *total = count + (int64_t)a.E * blocks;
    by_type(a.dtype, a.E, RouteChoose{a, s, rows, blocks, count});
    route_scan_kernel<<<(a.E + kWaves - 1) / kWaves, kRouteThreads, 0, s>>>(count, total, blocks, a.E);
    route_place_kernel<<<blocks, kRouteThreads, 0, s>>>(a, rows, count, total, blocks);
    return hipGetLastError();
}

hipError_t launch_route_grad(const RouteGradArgs& a, hipStream_t s)
{
    by_type(a.dtype, a.E, RouteGrad{a, s});
    return hipGetLastError();
}

}  // namespace sgap
