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
// the blocks, and every pair is put in its place.  No atomics, so that the lists are the same on every run.  One launch
// for the tokens of one block, otherwise two: the second one's blocks each sum up the counts for themselves, as long as
// those are few; with many a kernel between them does it once.
//
// 16,384 tokens, 8 of 128 experts, bf16: choosing 8.1 us, placing 6.4 (11 MB, 2 us at the rate of a copy: instructions of
// the rounds, the barriers and the second launch), the gradient 4.8; 4 tokens, 4 of 64: 3.4 us, a launch.
#include "sgap_experts.hpp"

namespace sgap {

namespace {

constexpr int kRouteThreads = 1024;  // sixteen wavefronts: what hides the rounds' latency
constexpr int kFewThreads = 256;     // a few tokens: a start and barriers that cost less
constexpr int kGradThreads = 256;
constexpr int kMaxExperts = 1024;
constexpr int kMaxChosen = 16;
constexpr int kBlockRows = 64;     // tokens of a block: a pass of its groups of sixteen lanes
constexpr int kBlockPairs = 1024;  // pairs of a block at most, one to a thread
static_assert(kBlockRows * kMaxChosen <= kBlockPairs && kBlockPairs <= kRouteThreads, "");

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
__device__ __forceinline__ int lanes_sum16(int v)
{
    v += (int)dpp<kRor8>((uint32_t)v);
    v += (int)dpp<kRor4>((uint32_t)v);
    v += (int)dpp<kRor2>((uint32_t)v);
    v += (int)dpp<kRor1>((uint32_t)v);
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

// V consecutive experts of a row, as one access where all of them are there
template <typename T, int V>
struct Experts {
    typedef T loose __attribute__((ext_vector_type(V), aligned(sizeof(T))));
};

template <typename T, int V>
__device__ __forceinline__ void load_row(const T* __restrict__ row, int e0, int E, float (&x)[V])
{
    if (V > 1 && e0 + V <= E) {
        const typename Experts<T, V>::loose v = *reinterpret_cast<const typename Experts<T, V>::loose*>(row + e0);
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = (float)v[i];
        return;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) x[v] = e0 + v < E ? (float)row[e0 + v] : -__builtin_inff();
}

template <typename T, int V>
__device__ __forceinline__ void store_row(T* __restrict__ row, int e0, int E, const float (&x)[V])
{
    if (V > 1 && e0 + V <= E) {
        typename Experts<T, V>::loose v;
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = (T)x[i];
        *reinterpret_cast<typename Experts<T, V>::loose*>(row + e0) = v;
        return;
    }
#pragma unroll
    for (int v = 0; v < V; ++v)
        if (e0 + v < E) row[e0 + v] = (T)x[v];
}

// The k largest of a row that LANES lanes hold, V experts each (expert sub * V + v), largest first, left in chosen[0 .. k)
// (-1: nothing left); lane j of them gets choice j's gate.
template <int LANES, int V>
__device__ __forceinline__ float choose(const float (&x)[V], int k, bool renormalise, int32_t* chosen)
{
    const int lane = threadIdx.x & 63, sub = lane & (LANES - 1);
    // the row's lanes below this one
    const uint64_t below = ((1ull << lane) - 1) & (LANES == 64 ? ~0ull : 0xffffull << (lane & 48));
    uint32_t key[V];
#pragma unroll
    for (int v = 0; v < V; ++v) key[v] = order_key(x[v]);
    uint32_t own = 0, first = 0;
    for (int j = 0; j < k; ++j) {
        uint32_t top = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) top = max(top, key[v]);
        const uint32_t most = lanes_max<LANES>(top);
        if (j == 0) first = most;
        if (sub == j) own = most;
        // the lowest lane that holds it: its first value of that size leaves
        const uint64_t who = __ballot(top == most);
        if (top == most && (who & below) == 0) {
            int at = 0;
#pragma unroll
            for (int v = V - 1; v >= 0; --v) at = key[v] == most ? v : at;
            chosen[j] = most ? sub * V + at : -1;
#pragma unroll
            for (int v = 0; v < V; ++v) key[v] = v == at ? 0u : key[v];
        }
    }
    // first = 0: a row of which nothing is left, and all gates are zero
    const float m = first ? key_value(first) : 0.0f;
    const float mine = own ? expf(key_value(own) - m) : 0.0f;
    float part = mine;
    if (!renormalise) {
        part = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) part += expf(x[v] - m);  // of -infinity: 0
    }
    const float total = lanes_sum<LANES>(part);
    return own ? mine / total : 0.0f;
}

// In shared memory, behind one another: the block's experts by pair, and the pairs of each expert in each wavefront's
// share of them.
struct RouteShared {
    int32_t* expert;  // kBlockPairs
    uint16_t* count;  // wavefronts x E
};
__device__ __forceinline__ RouteShared route_shared(char* lds)
{
    return {reinterpret_cast<int32_t*>(lds), reinterpret_cast<uint16_t*>(lds + kBlockPairs * 4)};
}
int route_shared_bytes(int threads, int E) { return kBlockPairs * 4 + threads / 64 * E * 2; }

// A wavefront's share of the block's pairs: 64 of them, or a part.
__device__ __forceinline__ int my_pair() { return threadIdx.x; }

// Ranks the pairs of a block among those of the same expert, in their order: each thread gets its pair's (-1: a missing
// choice), and s.count what every wavefront's share has of each expert.
__device__ __forceinline__ int rank_pair(const RouteShared& s, int E, int pairs)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, p = my_pair();
    uint16_t* const count = s.count + wave * E;
    for (int e = lane; e < E; e += 64) count[e] = 0;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const int e = p < pairs ? s.expert[p] : -1;
    uint64_t same = __ballot(e >= 0);
    const int bits = 32 - __builtin_clz(E);
    for (int b = 0; b < bits; ++b) {
        const uint64_t set = __ballot((e >> b) & 1);
        same &= (e >> b) & 1 ? set : ~set;
    }
    if (e < 0) return -1;
    const uint64_t before = same & ((1ull << lane) - 1);
    if (before == 0) count[e] = (uint16_t)__popcll(same);
    return __popcll(before);
}

// count[w][e] becomes the pairs of e in the shares before w; the sum of all of them
template <int THREADS>
__device__ __forceinline__ int sum_shares(const RouteShared& s, int E, int e)
{
    int sum = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        const int c = s.count[w * E + e];
        s.count[w * E + e] = (uint16_t)sum;
        sum += c;
    }
    return sum;
}

// Rows of the block are chosen for, their experts left in s.expert.
template <typename T, int LANES, int V, int THREADS>
__device__ __forceinline__ void choose_rows(const RouteArgs& a, const RouteShared& s, int64_t row0, int rows)
{
    constexpr int kGroups = THREADS / LANES;
    const int sub = threadIdx.x & (LANES - 1), group = threadIdx.x / LANES;
    for (int i = group; i < rows; i += kGroups) {
        const int64_t t = row0 + i;
        float x[V];
        load_row<T, V>(static_cast<const T*>(a.logits) + t * a.ld, sub * V, a.E, x);
        const float gate = choose<LANES, V>(x, a.k, a.renormalise, s.expert + i * a.k);
        if (sub < a.k) a.gates[t * a.k + sub] = gate;
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
template <int THREADS>
__device__ __forceinline__ void block_offsets(const int32_t* in, int32_t* out, int n, int32_t* wave_total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int carry = 0;
    for (int e0 = 0; e0 < n; e0 += THREADS) {
        const int e = e0 + threadIdx.x;
        const int v = e < n ? in[e] : 0;
        const int inc = wave_scan(v);
        if (lane == 63) wave_total[wave] = inc;
        __syncthreads();
        int base = carry;
        for (int w = 0; w < THREADS / 64; ++w) {
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
template <typename T, int LANES, int V, int THREADS>
__global__ __launch_bounds__(THREADS) void route_few_kernel(RouteArgs a)
{
    extern __shared__ __align__(16) char lds[];
    __shared__ int32_t total[kMaxExperts], start[kMaxExperts + 1], wave_total[THREADS / 64];
    const RouteShared s = route_shared(lds);
    const int pairs = (int)a.T * a.k, p = my_pair();
    choose_rows<T, LANES, V, THREADS>(a, s, 0, (int)a.T);
    __syncthreads();
    const int rank = rank_pair(s, a.E, pairs);
    __syncthreads();
    for (int e = threadIdx.x; e < a.E; e += THREADS) total[e] = sum_shares<THREADS>(s, a.E, e);
    __syncthreads();
    block_offsets<THREADS>(total, start, a.E, wave_total);
    for (int e = threadIdx.x; e <= a.E; e += THREADS) a.offsets[e] = start[e];
    if (p >= pairs) return;
    const int e = s.expert[p];
    const int at = e >= 0 ? start[e] + s.count[(threadIdx.x >> 6) * a.E + e] + rank : -1;
    a.experts[p] = e;
    a.slot[p] = at;
    if (e >= 0) a.order[at] = p;
    if (p >= start[a.E]) a.order[p] = -1;  // places that no pair has
}

// More tokens: the choice, with the blocks' counts by expert (count[e * stride + b]) and the pairs' ranks within their
// block (in slot) ...
template <typename T, int LANES, int V>
__global__ __launch_bounds__(kRouteThreads) void route_choose_kernel(RouteArgs a, uint16_t* count, int stride, int64_t block0)
{
    extern __shared__ __align__(16) char lds[];
    const RouteShared s = route_shared(lds);
    const int64_t block = block0 + blockIdx.x, row0 = block * kBlockRows;
    const int rows = (int)min((int64_t)kBlockRows, a.T - row0);
    const int pairs = rows * a.k, p = my_pair();
    choose_rows<T, LANES, V, kRouteThreads>(a, s, row0, rows);
    __syncthreads();
    const int rank = rank_pair(s, a.E, pairs);
    __syncthreads();
    for (int e = threadIdx.x; e < a.E; e += kRouteThreads)
        count[(int64_t)e * stride + block] = (uint16_t)sum_shares<kRouteThreads>(s, a.E, e);
    __syncthreads();
    if (p >= pairs) return;
    const int e = s.expert[p];
    a.experts[row0 * a.k + p] = e;
    a.slot[row0 * a.k + p] = e >= 0 ? s.count[(threadIdx.x >> 6) * a.E + e] + rank : -1;
}

// ... the counts of one expert summed up over the blocks (a wavefront per expert), where there are many of them ...
__global__ __launch_bounds__(256) void route_scan_kernel(const uint16_t* count, int32_t* before, int32_t* total, int blocks, int stride, int E)
{
    const int e = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (e >= E) return;
    int carry = 0;
    for (int b0 = 0; b0 < blocks; b0 += 64) {
        const int b = b0 + lane;
        const int v = b < blocks ? count[(int64_t)e * stride + b] : 0;
        const int inc = wave_scan(v);
        if (b < blocks) before[(int64_t)e * stride + b] = carry + inc - v;
        carry += __shfl(inc, 63);
    }
    if (lane == 0) total[e] = carry;
}

// ... and every pair into its place.  SUM: sixteen lanes sum up the counts of an expert, eight to a load: those of the
// blocks before this one, and all of them.
template <bool SUM>
__global__ __launch_bounds__(kRouteThreads) void route_place_kernel(RouteArgs a, const uint16_t* count,
                                                                    const int32_t* summed, const int32_t* total, int blocks, int stride,
                                                                    int64_t block0)
{
    __shared__ int32_t all[kMaxExperts], before[kMaxExperts], start[kMaxExperts + 1], wave_total[kRouteThreads / 64];
    const int mine = (int)(block0 + blockIdx.x);
    if constexpr (SUM) {
        const int sub = threadIdx.x & 15;
        for (int e = threadIdx.x >> 4; e < a.E; e += kRouteThreads / 16) {
            int sum = 0, earlier = 0;
#pragma unroll 2
            for (int b = sub * 8; b < blocks; b += 128) {
                const uint4 v = *reinterpret_cast<const uint4*>(count + (int64_t)e * stride + b);
                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int c = (int)(i & 1 ? w[i >> 1] >> 16 : w[i >> 1] & 0xffffu);
                    sum += b + i < blocks ? c : 0;
                    earlier += b + i < mine ? c : 0;
                }
            }
            sum = lanes_sum16(sum);
            earlier = lanes_sum16(earlier);
            if (sub == 0) {
                all[e] = sum;
                before[e] = earlier;
            }
        }
    } else {
        for (int e = threadIdx.x; e < a.E; e += kRouteThreads) {
            all[e] = total[e];
            before[e] = summed[(int64_t)e * stride + mine];
        }
    }
    __syncthreads();
    block_offsets<kRouteThreads>(all, start, a.E, wave_total);
    if (mine == 0)
        for (int e = threadIdx.x; e <= a.E; e += kRouteThreads) a.offsets[e] = start[e];
    const int64_t p = (int64_t)mine * kBlockRows * a.k + threadIdx.x;
    if ((int)threadIdx.x >= kBlockRows * a.k || p >= a.T * a.k) return;
    const int e = a.experts[p];
    if (e >= 0) {
        const int at = start[e] + before[e] + a.slot[p];
        a.slot[p] = at;
        a.order[at] = (int32_t)p;
    }
    if (p >= start[a.E]) a.order[p] = -1;
}

// dl_e = p_e ([e chosen] dg_e - sum of g dg) with p over all experts, or, renormalised, the same over the chosen ones alone.
template <typename T, int LANES, int V>
__global__ __launch_bounds__(kGradThreads) void route_grad_kernel(RouteGradArgs a, int64_t block0)
{
    constexpr int kGroups = kGradThreads / LANES;
    const int sub = threadIdx.x & (LANES - 1);
    const int64_t t = (block0 + blockIdx.x) * kGroups + threadIdx.x / LANES;
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
    store_row<T, V>(static_cast<T*>(a.dlogits) + t * a.ldd, sub * V, a.E, d);
}

template <typename F, typename T>
hipError_t by_experts(int E, F&& f, T)
{
    if (E <= 16) return f.template operator()<T, 16, 1>();
    if (E <= 32) return f.template operator()<T, 16, 2>();
    if (E <= 64) return f.template operator()<T, 16, 4>();
    if (E <= 128) return f.template operator()<T, 16, 8>();
    if (E <= 256) return f.template operator()<T, 16, 16>();
    if (E <= 512) return f.template operator()<T, 64, 8>();
    return f.template operator()<T, 64, 16>();
}
template <typename F>
hipError_t by_type(int dtype, int E, F&& f)
{
    switch (dtype) {
        case 0: return by_experts(E, f, 0.0f);
        case 1: return by_experts(E, f, half_t(0));
        default: return by_experts(E, f, bf16_t(0));
    }
}

struct RouteFew {
    const RouteArgs& a;
    hipStream_t s;
    template <typename T, int LANES, int V>
    hipError_t operator()() const
    {
        // a pass of the small block's groups of lanes: their pairs are one to a thread, as k is no more than LANES
        static_assert(LANES >= kMaxChosen, "");
        if (a.T <= kFewThreads / LANES)
            route_few_kernel<T, LANES, V, kFewThreads><<<1, kFewThreads, route_shared_bytes(kFewThreads, a.E), s>>>(a);
        else
            route_few_kernel<T, LANES, V, kRouteThreads><<<1, kRouteThreads, route_shared_bytes(kRouteThreads, a.E), s>>>(a);
        return hipGetLastError();
    }
};

// Where the counts lie in the workspace.
struct RouteCounts {
    int blocks, stride;              // blocks, and as many in whole loads
    int64_t summed_at, total_at, bytes;
    bool each;                       // each block sums them up for itself: no more than 128 KB of them
};
RouteCounts route_counts(int64_t T, int64_t E)
{
    RouteCounts c;
    c.blocks = (int)((T + kBlockRows - 1) / kBlockRows);
    c.stride = (c.blocks + 7) / 8 * 8;
    c.each = E * c.stride <= 65536;
    c.summed_at = (E * c.stride * 2 + 15) / 16 * 16;
    c.total_at = c.summed_at + (c.each ? 0 : E * c.stride * 4);
    c.bytes = c.total_at + (c.each ? 0 : E * 4);
    return c;
}

struct RouteChoose {
    const RouteArgs& a;
    const RouteCounts& c;
    hipStream_t s;
    template <typename T, int LANES, int V>
    hipError_t operator()() const
    {
        return launch_parts(c.blocks, kRouteThreads, [&](unsigned grid, int64_t block0) {
            route_choose_kernel<T, LANES, V><<<grid, kRouteThreads, route_shared_bytes(kRouteThreads, a.E), s>>>(
                a, static_cast<uint16_t*>(a.workspace), c.stride, block0);
        });
    }
};
struct RouteGrad {
    const RouteGradArgs& a;
    hipStream_t s;
    template <typename T, int LANES, int V>
    hipError_t operator()() const
    {
        constexpr int kGroups = kGradThreads / LANES;
        return launch_parts((a.T + kGroups - 1) / kGroups, kGradThreads, [&](unsigned grid, int64_t block0) {
            route_grad_kernel<T, LANES, V><<<grid, kGradThreads, 0, s>>>(a, block0);
        });
    }
};

// One workgroup for all tokens: as many as a block of more has.
bool route_in_one(int64_t T) { return T <= kBlockRows; }

}  // namespace

int64_t route_workspace_bytes(int64_t T, int64_t E)
{
    return route_in_one(T) ? 0 : route_counts(T, E).bytes;
}

hipError_t launch_route(const RouteArgs& a, hipStream_t s)
{
    if (route_in_one(a.T)) return by_type(a.dtype, a.E, RouteFew{a, s});
    const RouteCounts c = route_counts(a.T, a.E);
    char* const at = static_cast<char*>(a.workspace);
    const uint16_t* const count = reinterpret_cast<const uint16_t*>(at);
    int32_t *summed = reinterpret_cast<int32_t*>(at + c.summed_at), *total = reinterpret_cast<int32_t*>(at + c.total_at);
    if (const hipError_t err = by_type(a.dtype, a.E, RouteChoose{a, c, s})) return err;
    if (!c.each) route_scan_kernel<<<(a.E + 3) / 4, 256, 0, s>>>(count, summed, total, c.blocks, c.stride, a.E);
    return launch_parts(c.blocks, kRouteThreads, [&](unsigned grid, int64_t block0) {
        if (c.each) route_place_kernel<true><<<grid, kRouteThreads, 0, s>>>(a, count, nullptr, nullptr, c.blocks, c.stride, block0);
        else route_place_kernel<false><<<grid, kRouteThreads, 0, s>>>(a, count, summed, total, c.blocks, c.stride, block0);
    });
}

hipError_t launch_route_grad(const RouteGradArgs& a, hipStream_t s)
{
    return by_type(a.dtype, a.E, RouteGrad{a, s});
}

}  // namespace sgap
