// Rows of a table by token, out[t] = scale * W[id[t]], and the gradient of the table,
// dW[v] = scale * sum of dout[t] over the tokens t with id[t] = v.
//
// A lookup is the product with a sparse matrix that has one entry a row; the gradient is the product with its transpose, a
// sum by segments of very different length: most rows of a table no token has, and one token may be a tenth of a batch.
//
// The gradient in three steps.  1. The tokens by their id, in their order within one: a workgroup has a range of ids and
// looks at all tokens, so that it knows by itself how many come before its range, and no workgroup waits for another.
// 2. Tiles of that order, each an equal number of tokens whatever ids they have; a run of one id that lies in a tile is
// summed up and stored, what crosses a tile's ends goes to the workspace; rows without a token are cleared beside it.
// 3. The parts of the runs that cross tiles are added, in their order.  Sums in 32 bits, rounded once; no atomics on floats.
#include <algorithm>
#include <type_traits>

#include "sgap_columns.hpp"
#include "sgap_tokens.hpp"

namespace sgap {

namespace {

constexpr int kThreads = 256;
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kMostIds = 512;  // of a workgroup's range
constexpr int kClearRows = 16;  // rows that a group of lanes looks at, whether they have a token

// Groups of `lanes` (a power of two, 64 at most) have an item each: a row, or a tile, and lanes * VEC of its columns.
struct Spread {
    int lanes;
    int64_t column_items;
};
template <int VEC>
Spread spread(int64_t D)
{
    const int64_t pieces = (D + VEC - 1) / VEC;
    int lanes = 1;
    while (lanes < 64 && lanes < pieces) lanes *= 2;
    return {lanes, (pieces + lanes - 1) / lanes};
}
int64_t blocks_of(const Spread& sp, int64_t items) { return (items * sp.column_items * sp.lanes + kThreads - 1) / kThreads; }

struct Place {
    int64_t item, c;
};
template <int VEC>
__device__ __forceinline__ Place place_of(int lanes, int64_t column_items, int64_t block)
{
    const int64_t group = block * (kThreads / lanes) + threadIdx.x / lanes, item = group / column_items;
    return {item, ((group - item * column_items) * lanes + (threadIdx.x & (lanes - 1))) * VEC};
}

template <typename T, int VEC>
__global__ __launch_bounds__(kThreads) void embed_kernel(EmbedArgs a, int lanes, int64_t column_items, int64_t block0)
{
    const Place at = place_of<VEC>(lanes, column_items, block0 + blockIdx.x);
    if (at.item >= a.T || at.c >= a.D) return;
    const int64_t first = piece_first<VEC>(at.c, a.D);
    const int32_t id = a.ids[at.item];
    Columns<T, VEC> x;
    if (id >= 0 && id < a.V) {
        x.load(static_cast<const T*>(a.weights) + id * a.ldw + first);
#pragma unroll
        for (int i = 0; i < VEC; ++i) x.v[i] *= a.scale;
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) x.v[i] = 0.0f;
    }
    x.store(static_cast<T*>(a.out) + at.item * a.ldo + first);
}

// What the gradient keeps in its workspace.  Place p of the order has token order[p], of id key[p]; id v has the places
// start[v] .. start[v + 1].
struct Sorted {
    int32_t *start, *key, *order;
    float* parts;  // tiles x 2 x D: of the run that a tile begins in the middle of, and of the one that goes on behind it
    int64_t tile, tiles, bytes;
};
Sorted sorted_view(char* workspace, int64_t T, int64_t V, int64_t D)
{
    const auto up = [](int64_t n) { return (n + 255) / 256 * 256; };
    Sorted s;
    // tokens of a tile: 32, or what makes 1,024 tiles at most
    s.tile = 32;
    while (s.tile * 1024 < T) s.tile *= 2;
    s.tiles = (T + s.tile - 1) / s.tile;
    int64_t at = 0;
    const auto take = [&](int64_t bytes) {
        char* p = workspace + at;
        at += up(bytes);
        return p;
    };
    s.start = reinterpret_cast<int32_t*>(take((V + 1) * 4));
    s.key = reinterpret_cast<int32_t*>(take(T * 4));
    s.order = reinterpret_cast<int32_t*>(take(T * 4));
    s.parts = reinterpret_cast<float*>(take(s.tiles * 2 * D * 4));
    s.bytes = at;
    return s;
}

// ids range .. range + ids_of of a workgroup.  Every wavefront has a run of the tokens: it counts its own by id, the counts
// are summed up over the wavefronts and the ids, and every wavefront puts its tokens in their places, in order.
__global__ __launch_bounds__(kSortThreads) void embed_sort_kernel(const int32_t* __restrict__ ids, int64_t T, int64_t V, int ids_of,
                                                                  int32_t* __restrict__ start, int32_t* __restrict__ key,
                                                                  int32_t* __restrict__ order, int64_t block0)
{
    extern __shared__ int32_t count[];  // wavefronts x ids_of: tokens of an id, then the next place
    __shared__ int32_t before[kSortWaves], wave_total[kSortWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int64_t range = (block0 + blockIdx.x) * ids_of;
    const uint32_t lo = (uint32_t)range, n = (uint32_t)min((int64_t)ids_of, V - range);
    const int64_t share = ((T + kSortWaves - 1) / kSortWaves + 63) / 64 * 64;
    const int64_t first = min((int64_t)wave * share, T), end = min(first + share, T);
    int32_t* const own = count + wave * ids_of;
    for (int i = lane; i < ids_of; i += 64) own[i] = 0;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    int below = 0;
    for (int64_t t0 = first; t0 < end; t0 += 256) {
        uint32_t id[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t t = t0 + u * 64 + lane;
            id[u] = t < end ? (uint32_t)ids[t] : 0xffffffffu;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            below += __popcll(__ballot(id[u] < lo));
            if (id[u] - lo < n) atomicAdd(&own[id[u] - lo], 1);  // (counts: whole numbers)
        }
    }
    if (lane == 0) before[wave] = below;
    __syncthreads();
    int base = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) base += before[w];
    // thread i: id i of the range (kMostIds <= kSortThreads)
    const int i = threadIdx.x;
    int total = 0;
    if (i < ids_of) {
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) {
            const int c = count[w * ids_of + i];
            count[w * ids_of + i] = total;
            total += c;
        }
    }
    int upto = total;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(upto, d);
        if (lane >= d) upto += o;
    }
    if (lane == 63) wave_total[wave] = upto;
    __syncthreads();
    for (int w = 0; w < wave; ++w) base += wave_total[w];
    const int place = base + upto - total;
    if (i < ids_of) {
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) count[w * ids_of + i] += place;
        if (i < (int)n) {
            start[range + i] = place;
            if (range + i == V - 1) start[V] = place + total;
        }
    }
    __syncthreads();
    for (int64_t t0 = first; t0 < end; t0 += 256) {
        uint32_t id[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t t = t0 + u * 64 + lane;
            id[u] = t < end ? (uint32_t)ids[t] : 0xffffffffu;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const uint32_t in = id[u] - lo;
            uint64_t left = __ballot(in < n);
            while (left) {
                // the tokens of the id that the lowest lane left has
                const uint32_t which = (uint32_t)__builtin_amdgcn_readlane((int)in, __builtin_ctzll(left));
                const uint64_t same = __ballot(in == which);
                const int at = own[which];
                if (in == which) {
                    const int p = at + __popcll(same & ((1ull << lane) - 1));
                    key[p] = (int32_t)id[u];
                    order[p] = (int32_t)(t0 + u * 64 + lane);
                }
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                if (lane == 0) own[which] = at + __popcll(same);
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                left &= ~same;
            }
        }
    }
}

template <typename G, int VEC>
__device__ __forceinline__ void store_row(const EmbedGradArgs& a, int64_t v, int64_t first, int shared, const float (&sum)[VEC])
{
    G* const to = static_cast<G*>(a.dweights) + v * a.ldw + first;
    if (a.accumulate && shared > 0) {
        // columns that the lane in front has as well are added by it alone
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (i >= shared) to[i] = (G)((float)to[i] + a.scale * sum[i]);
        return;
    }
#pragma unroll
    for (int h = 0; h < (VEC + Piece<G>::kCount - 1) / Piece<G>::kCount; ++h) {
        constexpr int kPart = VEC < Piece<G>::kCount ? 1 : Piece<G>::kCount;
        Columns<G, kPart> x;
        if (a.accumulate) x.load(to + h * kPart);
#pragma unroll
        for (int i = 0; i < kPart; ++i) x.v[i] = (a.accumulate ? x.v[i] : 0.0f) + a.scale * sum[h * kPart + i];
        x.store(to + h * kPart);
    }
}

// Behind the tiles' workgroups come those that clear the rows that no token has.
template <typename T, typename G, int VEC>
__global__ __launch_bounds__(kThreads) void embed_sum_kernel(EmbedGradArgs a, Sorted s, int lanes, int64_t column_items, int64_t tile_blocks,
                                                             int64_t block0)
{
    constexpr int kAhead = 8;
    const int64_t block = block0 + blockIdx.x;
    if (block >= tile_blocks) {
        const Place at = place_of<VEC>(lanes, column_items, block - tile_blocks);
        if (at.c >= a.D) return;
        const int64_t first = piece_first<VEC>(at.c, a.D), v0 = at.item * kClearRows;
        const float none[VEC] = {};
#pragma unroll 4
        for (int i = 0; i < kClearRows; ++i) {
            const int64_t v = v0 + i;
            if (v < a.V && s.start[v] == s.start[v + 1]) store_row<G, VEC>(a, v, first, 0, none);
        }
        return;
    }
    const Place at = place_of<VEC>(lanes, column_items, block);
    const int64_t p0 = at.item * s.tile, used = s.start[a.V];
    if (p0 >= used || at.c >= a.D) return;
    const int64_t p1 = min(p0 + s.tile, used), first = piece_first<VEC>(at.c, a.D);
    const int shared = (int)(at.c - first);
    const T* __restrict__ dout = static_cast<const T*>(a.dout) + first;
    float* __restrict__ part = s.parts + at.item * 2 * a.D + first;
    float sum[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) sum[i] = 0.0f;
    int32_t run = s.key[p0];
    bool open = s.start[run] < p0;  // the run began in front of the tile
    const auto keep = [&](int which) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) part[which * a.D + i] = sum[i];
    };
    for (int64_t p = p0; p < p1; p += kAhead) {
        int32_t id[kAhead];
        Columns<T, VEC> x[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int64_t q = min(p + u, p1 - 1);
            id[u] = s.key[q];
            x[u].load(dout + s.order[q] * a.ldd);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (p + u >= p1) break;
            if (id[u] != run) {
                if (open) keep(0);
                else store_row<G, VEC>(a, run, first, shared, sum);
                open = false;
                run = id[u];
#pragma unroll
                for (int i = 0; i < VEC; ++i) sum[i] = 0.0f;
            }
#pragma unroll
            for (int i = 0; i < VEC; ++i) sum[i] += x[u].v[i];
        }
    }
    if (open) keep(0);
    else if (s.start[run + 1] > p1) keep(1);
    else store_row<G, VEC>(a, run, first, shared, sum);
}

// The runs that begin in a tile and go on behind it.
template <typename G, int VEC>
__global__ __launch_bounds__(kThreads) void embed_join_kernel(EmbedGradArgs a, Sorted s, int lanes, int64_t column_items, int64_t block0)
{
    const Place at = place_of<VEC>(lanes, column_items, block0 + blockIdx.x);
    const int64_t p0 = at.item * s.tile, p1 = p0 + s.tile, used = s.start[a.V];
    if (p1 >= used || at.c >= a.D) return;
    const int32_t run = s.key[p1 - 1];
    if (s.start[run] < p0 || s.start[run + 1] <= p1) return;
    const int64_t first = piece_first<VEC>(at.c, a.D), last = (s.start[run + 1] - 1) / s.tile;
    const float* __restrict__ part = s.parts + at.item * 2 * a.D + first;
    float sum[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) sum[i] = part[a.D + i];
#pragma unroll 4
    for (int64_t t = at.item + 1; t <= last; ++t) {
        const float* __restrict__ more = s.parts + t * 2 * a.D + first;
#pragma unroll
        for (int i = 0; i < VEC; ++i) sum[i] += more[i];
    }
    store_row<G, VEC>(a, run, first, (int)(at.c - first), sum);
}

template <typename T, int VEC>
hipError_t embed(const EmbedArgs& a, hipStream_t s)
{
    const Spread sp = spread<VEC>(a.D);
    return launch_parts(blocks_of(sp, a.T), kThreads, [&](unsigned grid, int64_t block0) {
        embed_kernel<T, VEC><<<grid, kThreads, 0, s>>>(a, sp.lanes, sp.column_items, block0);
    });
}

template <typename T, typename G, int VEC>
hipError_t embed_grad(const EmbedGradArgs& a, hipStream_t s)
{
    const Sorted st = sorted_view(a.workspace, a.T, a.V, a.D);
    int ids_of = 1;
    while (ids_of < kMostIds && (int64_t)ids_of * 512 < a.V) ids_of *= 2;
    hipError_t err = launch_parts((a.V + ids_of - 1) / ids_of, kSortThreads, [&](unsigned grid, int64_t block0) {
        embed_sort_kernel<<<grid, kSortThreads, kSortWaves * ids_of * 4, s>>>(a.ids, a.T, a.V, ids_of, st.start, st.key, st.order, block0);
    });
    if (err != hipSuccess) return err;
    const Spread sp = spread<VEC>(a.D);
    const int64_t tile_blocks = blocks_of(sp, st.tiles);
    const int64_t clearing = a.accumulate ? 0 : blocks_of(sp, (a.V + kClearRows - 1) / kClearRows);
    err = launch_parts(tile_blocks + clearing, kThreads, [&](unsigned grid, int64_t block0) {
        embed_sum_kernel<T, G, VEC><<<grid, kThreads, 0, s>>>(a, st, sp.lanes, sp.column_items, tile_blocks, block0);
    });
    if (err != hipSuccess || st.tiles < 2) return err;
    return launch_parts(blocks_of(sp, st.tiles - 1), kThreads, [&](unsigned grid, int64_t block0) {
        embed_join_kernel<G, VEC><<<grid, kThreads, 0, s>>>(a, st, sp.lanes, sp.column_items, block0);
    });
}

template <typename T>
hipError_t embed_by_width(const EmbedArgs& a, hipStream_t s)
{
    return a.D >= Piece<T>::kCount ? embed<T, Piece<T>::kCount>(a, s) : embed<T, 1>(a, s);
}

template <typename T>
hipError_t grad_by_type(const EmbedGradArgs& a, hipStream_t s)
{
    constexpr int kVec = Piece<T>::kCount;
    if (a.grad_dtype == a.dtype) return a.D >= kVec ? embed_grad<T, T, kVec>(a, s) : embed_grad<T, T, 1>(a, s);
    return a.D >= kVec ? embed_grad<T, float, kVec>(a, s) : embed_grad<T, float, 1>(a, s);
}

}  // namespace

int64_t embed_grad_workspace_bytes(int64_t T, int64_t V, int64_t D) { return sorted_view(nullptr, T, V, D).bytes; }

hipError_t launch_embed(const EmbedArgs& a, hipStream_t s)
{
    switch (a.dtype) {
        case 0: return embed_by_width<float>(a, s);
        case 1: return embed_by_width<half_t>(a, s);
        default: return embed_by_width<bf16_t>(a, s);
    }
}

hipError_t launch_embed_grad(const EmbedGradArgs& a, hipStream_t s)
{
    switch (a.dtype) {
        case 0: return grad_by_type<float>(a, s);
        case 1: return grad_by_type<half_t>(a, s);
        default: return grad_by_type<bf16_t>(a, s);
    }
}

}  // namespace sgap
