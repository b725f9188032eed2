// Rows of a table by token, out[t] = scale * W[id[t]], and the gradient of the table,
// dW[v] = scale * sum of dout[t] over the tokens t with id[t] = v.
//
// A lookup is the product with a sparse matrix that has one entry a row; the gradient is the product with its transpose, a
// sum by segments of very different length: most rows of a table no token has, and one token may be a tenth of a batch.
//
// The gradient of many tokens in three steps.  1. The tokens by their id, those of one always in the same order: a workgroup has a range
// of ids and looks at all tokens, so that it knows by itself how many come before its range, and no workgroup waits for another.
// 2. Tiles of that order, each an equal number of tokens whatever ids they have; a run of one id that lies in a tile is
// summed up and stored, what crosses a tile's ends goes to the workspace.
// 3. The parts of the runs that cross tiles are added, always in the same order, and rows without a token are cleared.  Sums in 32
// bits, rounded once; no atomics on floats.  Of a few tokens it is one launch, in which every workgroup looks at all tokens for those of
// its rows.
//
// Bound by memory where there are many: 16,384 tokens (a tenth of them one), 65,536 rows of 2,048, bf16: the lookup 16.4 us, 106 MB at
// 6.5 TB/s; the gradient 72 us: sorting 28, which clears 134 MB, sums 21, which read 67 MB, joins 23, which clear the other half: 339 MB
// at 4.7 TB/s.  Of few the launches are: 8 rows of 4,096 3.4 us, and 1,498 tokens' gradient in 551 rows of 256 7.6.
#include <algorithm>
#include <type_traits>

#include "sgap_columns.hpp"
#include "sgap_tokens.hpp"

namespace sgap {

namespace {

constexpr int kThreads = 256;
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kMostIds = 256;  // of a workgroup's range
constexpr int kList = 416;     // tokens of it that a wavefront collects, 256 at a time
constexpr int kClearRows = 128;  // rows that a workgroup looks at and clears where they have no token

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

// A group of lanes has TOKENS neighbouring tokens, all of their rows on the way together.
template <typename T, int VEC, int TOKENS>
__global__ __launch_bounds__(kThreads) void embed_kernel(EmbedArgs a, int lanes, int64_t column_items, int64_t block0)
{
    const Place at = place_of<VEC>(lanes, column_items, block0 + blockIdx.x);
    const int64_t t0 = at.item * TOKENS;
    if (t0 >= a.T || at.c >= a.D) return;
    const int64_t first = piece_first<VEC>(at.c, a.D);
    const T* __restrict__ W = static_cast<const T*>(a.weights) + first;
    Columns<T, VEC> x[TOKENS];
#pragma unroll
    for (int u = 0; u < TOKENS; ++u) {
        const int32_t id = t0 + u < a.T ? a.ids[t0 + u] : -1;
        if (id >= 0 && id < a.V) {
            x[u].load(W + id * a.ldw);
#pragma unroll
            for (int i = 0; i < VEC; ++i) x[u].v[i] *= a.scale;
        } else {
#pragma unroll
            for (int i = 0; i < VEC; ++i) x[u].v[i] = 0.0f;
        }
    }
#pragma unroll
    for (int u = 0; u < TOKENS; ++u) {
        if (t0 + u >= a.T) break;
        T* const out = static_cast<T*>(a.out) + (t0 + u) * a.ldo + first;
        // many rows are written past the caches, which keep the table's frequent rows (16,384 by 2,048, bf16: 16.4 us, 22.5 without)
        if constexpr (TOKENS > 1) x[u].stream_store(out);
        else x[u].store(out);
    }
}

// What the gradient keeps in its workspace.  Place p of the order has token order[p], of id key[p]; id v has the places
// start[v] .. start[v + 1].
struct Sorted {
    int32_t *start, *key, *order;
    float* parts;  // tiles x 2 x D: of the run that a tile begins in the middle of, and of the one that goes on behind it
    int64_t part, tile, tiles, bytes;  // places of a group of lanes, and of a workgroup of them
};
// groups: of lanes to a workgroup, four at least
Sorted sorted_view(char* workspace, int64_t T, int64_t V, int64_t D, int groups)
{
    const auto up = [](int64_t n) { return (n + 255) / 256 * 256; };
    Sorted s;
    // tokens of a part: 8, or what makes 1,024 parts at most, or more where rows are so short that 4,096 wavefronts have more
    s.part = 8;
    const int64_t most = std::max<int64_t>(1024, (1 << 21) / std::max<int64_t>(D, 1));
    while (s.part * most < T) s.part *= 2;
    s.tile = s.part * groups;
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

// Rows of the gradient that no token has, as 16-bit halves of zeros, whatever type they have.  Neighbouring ones are cleared as one
// piece of memory where nothing lies between them: by rows, their ends write parts of lines, and short ones use few lanes (100 tokens,
// by rows and so: 262,144 rows of 64 in 16 bits 25 us, 12; 66,727 of 2,280 floats 188, 124).
struct Clearing {
    uint16_t* __restrict__ rows;  // null: nothing is cleared
    int64_t halves, pitch;
};
// PAST: past the caches, which keep what other kernels read (65,536 rows of 2,048, bf16, lookup and gradient: 99.9 us, 90.7; one launch of few
// tokens has nothing to keep: 66,727 rows of 2,280 floats 124 us, 145)
template <bool PAST>
__device__ __forceinline__ void clear_halves(uint16_t* to, int64_t n)
{
    typedef uint16_t loose __attribute__((ext_vector_type(8), aligned(2)));
    const int lane = threadIdx.x & 63;
    if (n < 8) {
        if (lane < n) to[lane] = 0;
        return;
    }
    for (int64_t i = lane * 8; i < n; i += 512) {
        loose* const at = reinterpret_cast<loose*>(to + min(i, n - 8));
        if constexpr (PAST) __builtin_nontemporal_store(loose{0, 0, 0, 0, 0, 0, 0, 0}, at);
        else *at = loose{0, 0, 0, 0, 0, 0, 0, 0};
    }
}
// rows v0 + i for the bits i of `which`, by a wavefront
template <bool PAST>
__device__ __forceinline__ void clear_rows(const Clearing& c, int64_t v0, uint64_t which)
{
    while (which) {
        const int i = __builtin_ctzll(which);
        const uint64_t others = ~(which >> i);
        const int run = c.pitch != c.halves ? 1 : others ? __builtin_ctzll(others) : 64;
        clear_halves<PAST>(c.rows + (v0 + i) * c.pitch, run * c.halves);
        which &= run == 64 ? 0 : ~(((1ull << run) - 1) << i);
    }
}
// With many tokens half of the rows are cleared beside the sorting and half beside the joins, which both wait more than they work (all
// of them beside the joins: 83 us in place of 76 for 65,536 rows of 2,048, bf16): blocks of kClearBlock in turn (of 1, 4 and 8 rows: these 100.0,
// 100.4, 102.7 us with their lookup, 50,001 of 1,001 floats 95.7, 92.3, 89.0, not past the caches).
constexpr int kClearBlock = 4;
__device__ __forceinline__ bool cleared_early(int64_t v) { return (v / kClearBlock & 1) == 0; }

// ids range .. range + ids_of of a workgroup.  Every wavefront has a run of the tokens and collects those of the range, so that it
// deals with 64 of them at a time; it counts them by id, the counts are summed up over the wavefronts and the ids, and every wavefront
// puts its tokens in their places, always in the same order.  Where they are more than its list holds, it looks at the tokens again.
// unseen: every other workgroup clears in place of the next one, whatever tokens there are; the later steps write the rows in use.
__global__ __launch_bounds__(kSortThreads) void embed_sort_kernel(const int32_t* __restrict__ ids, int64_t T, int64_t V, int ids_of,
                                                                  int32_t* __restrict__ start, int32_t* __restrict__ key,
                                                                  int32_t* __restrict__ order, Clearing clearing, bool unseen, int64_t block0)
{
    extern __shared__ int32_t count[];  // wavefronts x ids_of: tokens of an id, then the next place
    __shared__ int32_t found[kSortWaves][kList];  // tokens of the range ...
    __shared__ uint16_t found_id[kSortWaves][kList];  // ... and their ids in it
    __shared__ bool none[kMostIds];
    __shared__ int32_t before[kSortWaves], wave_total[kSortWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int64_t block = block0 + blockIdx.x, range = (unseen ? block / 2 : block) * ids_of;
    const uint32_t lo = (uint32_t)range, n = (uint32_t)min((int64_t)ids_of, V - range);
    const int mine = (ids_of + kSortWaves - 1) / kSortWaves, r = wave * mine + lane;  // a wavefront's rows to be cleared, neighbouring ones
    static_assert(kMostIds <= 64 * kSortWaves, "");
    if (unseen && block % 2 == 0) {
        clear_rows<true>(clearing, range + wave * mine, __ballot(lane < mine && r < (int)n && cleared_early(range + r)));
        return;
    }
    const int64_t share = ((T + kSortWaves - 1) / kSortWaves + 63) / 64 * 64;
    const int64_t first = min((int64_t)wave * share, T), end = min(first + share, T);
    int32_t* const own = count + wave * ids_of;
    int32_t* const list = found[wave];
    uint16_t* const list_id = found_id[wave];
    for (int i = lane; i < ids_of; i += 64) own[i] = 0;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    // Collects the tokens of the range; `deal` has the list when it is full.  A lane has four neighbouring tokens, the next ones are on
    // their way.  (id 2^32 - 1, which no range has, behind the last)
    int fill = 0, below = 0;
    const auto scan = [&](auto&& deal) {
        if (first >= end) return;  // (no tokens at all: nothing to read in place of one past the last)
        typedef int32_t loose __attribute__((ext_vector_type(4), aligned(4)));
        constexpr int kAhead = 4;
        loose next[kAhead];
        const auto ask = [&](int64_t t0) {
            if (t0 + 256 <= end) return *reinterpret_cast<const loose*>(ids + t0 + lane * 4);
            loose v;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int64_t t = t0 + lane * 4 + u;
                v[u] = ids[min(t, T - 1)];
                v[u] = t < end ? v[u] : -1;
            }
            return v;
        };
#pragma unroll
        for (int h = 0; h < kAhead; ++h) next[h] = ask(first + h * 256);
#pragma unroll 1
        for (int64_t t0 = first; t0 < end; t0 += 256) {
            const loose id = next[0];
#pragma unroll
            for (int h = 0; h + 1 < kAhead; ++h) next[h] = next[h + 1];
            next[kAhead - 1] = ask(t0 + kAhead * 256);
            if (fill > kList - 256) {
                deal();
                fill = 0;
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const uint32_t in = (uint32_t)id[u] - lo;
                below += (uint32_t)id[u] < lo ? 1 : 0;
                const uint64_t hit = __ballot(in < n);
                if (in < n) {
                    const int at = fill + __popcll(hit & ((1ull << lane) - 1));
                    list[at] = (int32_t)(t0 + lane * 4 + u);
                    list_id[at] = (uint16_t)in;
                }
                fill += __popcll(hit);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    };
    bool whole = true;  // the list has all of the wavefront's
    const auto counted = [&] {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        for (int i = lane; i < fill; i += 64) atomicAdd(&own[list_id[i]], 1);  // (counts: whole numbers)
    };
    scan([&] {
        counted();
        whole = false;
    });
    counted();
#pragma unroll
    for (int d = 32; d; d >>= 1) below += __shfl_xor(below, d);
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
        none[i] = i < (int)n && total == 0;
        if (i < (int)n) {
            start[range + i] = place;
            if (range + i == V - 1) start[V] = place + total;
        }
    }
    __syncthreads();
    const auto placed = [&] {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        for (int l = 0; l < fill; l += 64) {
            const int e = l + lane;
            const bool mine = e < fill;
            const int32_t token = mine ? list[e] : 0;
            const uint32_t in = mine ? list_id[e] : 0;
            // the lanes whose tokens have this one's id, a bit of it at a time (one id after the other, which is slow where a workgroup
            // has many tokens of many ids: 65,536 tokens, ids' frequency one over their rank, 65,536 rows of 1,024 with their lookup 400 us, 129)
            uint64_t same = __ballot(mine);
            for (uint32_t bit = 1; bit < (uint32_t)ids_of; bit <<= 1) {
                const uint64_t has = __ballot((in & bit) != 0);
                same &= (in & bit) != 0 ? has : ~has;
            }
            const int rank = __popcll(same & ((1ull << lane) - 1));
            int at = 0;
            if (mine && rank == 0) at = atomicAdd(&own[in], __popcll(same));  // (this wavefront's alone)
            at = __shfl(at, mine ? __builtin_ctzll(same) : lane) + rank;
            if (mine) {
                key[at] = (int32_t)(lo + in);
                order[at] = token;
            }
        }
    };
    if (!whole) {
        fill = 0;
        scan(placed);
    }
    placed();
    if (unseen || !clearing.rows) return;
    clear_rows<true>(clearing, range + wave * mine, __ballot(lane < mine && r < (int)n && none[min(r, kMostIds - 1)] && cleared_early(range + r)));
}

// A piece of a row of the gradient, in accesses of 16 bytes at most.
template <typename G, int VEC>
struct GradPiece {
    static constexpr int kPart = VEC < Piece<G>::kCount ? 1 : Piece<G>::kCount, kParts = VEC / kPart;
    Columns<G, kPart> part[kParts];
    __device__ __forceinline__ void load(const G* p)
    {
#pragma unroll
        for (int h = 0; h < kParts; ++h) part[h].load(p + h * kPart);
    }
    // = scale * sum (and +0 of nothing)
    __device__ __forceinline__ void set(float scale, const float (&sum)[VEC])
    {
#pragma unroll
        for (int i = 0; i < VEC; ++i) part[i / kPart].v[i % kPart] = 0.0f + scale * sum[i];
    }
    __device__ __forceinline__ void add(float scale, const float (&sum)[VEC])
    {
#pragma unroll
        for (int i = 0; i < VEC; ++i) part[i / kPart].v[i % kPart] += scale * sum[i];
    }
    __device__ __forceinline__ void store(G* p) const
    {
#pragma unroll
        for (int h = 0; h < kParts; ++h) part[h].store(p + h * kPart);
    }
};

// A row's piece out of its sum; ADD: added to `was`, by each lane to its own columns alone (the first `shared` of a row's last
// piece are the lane's in front).
template <bool ADD, typename G, int VEC>
__device__ __forceinline__ void store_row(const EmbedGradArgs& a, int64_t v, int64_t first, int shared, const float (&sum)[VEC],
                                          GradPiece<G, VEC>& was)
{
    G* const to = static_cast<G*>(a.dweights) + v * a.ldw + first;
    if constexpr (ADD) {
        was.add(a.scale, sum);
        if (shared > 0) {
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (i >= shared) to[i] = (G)was.part[i / was.kPart].v[i % was.kPart];
            return;
        }
    } else {
        was.set(a.scale, sum);
    }
    was.store(to);
}

// A group of lanes has a part of the workgroup's tile, s.part places, and lanes * VEC columns.  A run within a part is stored; what
// crosses parts is put together in LDS, and what crosses the tile's ends goes to the workspace.
template <typename T, typename G, int VEC, bool ADD>
__global__ __launch_bounds__(kThreads) void embed_sum_kernel(EmbedGradArgs a, Sorted s, int lanes, int64_t column_items, int64_t block0)
{
    constexpr int kAhead = 8;
    enum { kHead = 1, kThrough = 2, kTail = 4 };  // of a part: a run that began before it, which goes on behind it; one that begins in it and goes on
    __shared__ float heads[VEC * kThreads], tails[VEC * kThreads];
    __shared__ int marks[kThreads];
    const int sub = threadIdx.x & (lanes - 1), group = threadIdx.x / lanes, groups = kThreads / lanes;
    const int64_t block = block0 + blockIdx.x, tile = block / column_items;
    const int64_t c = ((block - tile * column_items) * lanes + sub) * VEC;
    const int64_t p0 = tile * s.tile + group * s.part, used = s.start[a.V];
    const bool there = c < a.D;
    const int64_t first = there ? piece_first<VEC>(c, a.D) : 0, p1 = min(p0 + s.part, used);
    const int shared = (int)(c - first);
    const T* __restrict__ dout = static_cast<const T*>(a.dout) + first;
    int mark = 0;
    int32_t last_run = 0;
    if (p0 < used) {
        float sum[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) sum[i] = 0.0f;
        bool open = p0 > 0 && s.key[p0 - 1] == s.key[p0];
        for (int64_t p = p0; p < p1; p += kAhead) {
            // the tokens of the places, and whether their runs go on behind them
            int32_t id[kAhead + 1];
            Columns<T, VEC> x[kAhead];
            GradPiece<G, VEC> was[kAhead];
#pragma unroll
            for (int u = 0; u <= kAhead; ++u) id[u] = s.key[min(p + u, used - 1)];
            if (p + kAhead >= used) {
#pragma unroll
                for (int u = 0; u <= kAhead; ++u) id[u] = p + u < used ? id[u] : -1;
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                x[u].stream_load(dout + s.order[min(p + u, p1 - 1)] * a.ldd);
                // (not only where a run ends: a branch would wait for each)
                if (ADD) was[u].load(static_cast<const G*>(a.dweights) + (id[u] >= 0 ? id[u] : id[0]) * a.ldw + first);
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (p + u >= p1) break;
#pragma unroll
                for (int i = 0; i < VEC; ++i) sum[i] += x[u].v[i];
                const bool ends = id[u] != id[u + 1];
                if (!ends && p + u + 1 < p1) continue;
                last_run = id[u];
                if (open || !ends) {
                    float* const to = open ? heads : tails;
                    mark |= open ? (ends ? kHead : kHead | kThrough) : kTail;
#pragma unroll
                    for (int i = 0; i < VEC; ++i) to[i * kThreads + threadIdx.x] = sum[i];
                } else if (there) {
                    store_row<ADD>(a, id[u], first, shared, sum, was[u]);
                }
                open = false;
#pragma unroll
                for (int i = 0; i < VEC; ++i) sum[i] = 0.0f;
            }
        }
    }
    if (sub == 0) marks[group] = mark;
    __syncthreads();
    // the run that goes on behind this part, or, in the first, that began before the tile
    const bool before = group == 0 && (mark & kHead);
    for (int which = before ? 0 : 1; which < 2; ++which) {
        if (which == 1 && !(mark & kTail)) break;
        float sum[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) sum[i] = (which ? tails : heads)[i * kThreads + threadIdx.x];
        bool goes_on = which == 1 || (mark & kThrough);
        for (int g = group + 1; goes_on && g < groups; ++g) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) sum[i] += heads[i * kThreads + g * lanes + sub];
            goes_on = marks[g] & kThrough;
        }
        if (!there) continue;
        GradPiece<G, VEC> piece;
        if (which == 0 || goes_on) {
            GradPiece<float, VEC> part;
            part.set(1.0f, sum);
            part.store(s.parts + (tile * 2 + which) * a.D + first);
        } else {
            if (ADD) piece.load(static_cast<const G*>(a.dweights) + last_run * a.ldw + first);
            store_row<ADD>(a, last_run, first, shared, sum, piece);
        }
    }
}

constexpr int kJoinThreads = 1024, kFewTiles = 8;

// The runs that begin in a tile and go on behind it: a group of lanes has one, and lanes * VEC of its columns, and a whole workgroup,
// whose groups share the tiles, each of its longer ones (a token that is half of a batch).  Behind these workgroups, which wait more
// than they work, come those that clear the rows that no token has.
template <typename G, int VEC, bool ADD>
__global__ __launch_bounds__(kJoinThreads) void embed_join_kernel(EmbedGradArgs a, Sorted s, Clearing clearing, int lanes, int64_t column_items,
                                                                  int64_t join_blocks, int64_t block0)
{
    __shared__ float shares[kJoinThreads * VEC];
    __shared__ int32_t longer[kJoinThreads];
    __shared__ int many;
    const int64_t block = block0 + blockIdx.x;
    if (block >= join_blocks) {
        constexpr int kMine = kClearRows / (kJoinThreads / 64);  // a wavefront's rows, of which half are cleared late
        const int lane = threadIdx.x & 63;
        const int64_t v0 = (block - join_blocks) * kClearRows + (threadIdx.x >> 6) * kMine, v = v0 + lane;
        clear_rows<true>(clearing, v0, __ballot(lane < kMine && v < a.V && !cleared_early(v) && s.start[min(v, a.V - 1)] == s.start[min(v, a.V - 1) + 1]));
        return;
    }
    const int sub = threadIdx.x & (lanes - 1), group = threadIdx.x / lanes, groups = kJoinThreads / lanes;
    const int64_t used = s.start[a.V];
    if (threadIdx.x == 0) many = 0;
    __syncthreads();
    // what group g of the workgroup has: a tile and columns; the run and the last tile it is in, -1 for none
    struct Item {
        int64_t tile, c, last;
        int32_t run;
    };
    const auto item_of = [&](int g) {
        // (a long run's columns are different workgroups')
        const int64_t item = block * groups + g, columns = item / (s.tiles - 1);
        Item it;
        it.tile = item - columns * (s.tiles - 1);
        it.c = (columns * lanes + sub) * VEC;
        it.last = -1;
        it.run = 0;
        const int64_t p0 = it.tile * s.tile, p1 = p0 + s.tile;
        if (p1 >= used) return it;
        const int32_t next = s.key[p1], before = s.key[p0 > 0 ? p0 - 1 : 0];
        it.run = s.key[p1 - 1];
        if (next != it.run || (p0 > 0 && before == it.run)) return it;
        it.last = ((int64_t)s.start[it.run + 1] - 1) / s.tile;
        return it;
    };
    // the part that the run's first tile ends with, then those that the others begin with: every `step`th from the `from`th
    const auto add_parts = [&](const Item& it, int64_t first, int from, int step, float (&sum)[VEC]) {
#pragma unroll 8
        for (int64_t t = it.tile + from; t <= it.last; t += step) {
            GradPiece<float, VEC> more;
            more.load(s.parts + (t * 2 + (t == it.tile ? 1 : 0)) * a.D + first);
#pragma unroll
            for (int i = 0; i < VEC; ++i) sum[i] += more.part[i / more.kPart].v[i % more.kPart];
        }
    };
    const auto finish = [&](const Item& it, int64_t first, const float (&sum)[VEC]) {
        GradPiece<G, VEC> was;
        if (ADD) was.load(static_cast<const G*>(a.dweights) + it.run * a.ldw + first);
        store_row<ADD>(a, it.run, first, (int)(it.c - first), sum, was);
    };
    const Item own = item_of(group);
    if (own.last >= own.tile + kFewTiles) {
        if (sub == 0) longer[atomicAdd(&many, 1)] = group;  // (in any order: each is summed up by itself)
    } else if (own.last >= 0 && own.c < a.D) {
        const int64_t first = piece_first<VEC>(own.c, a.D);
        float sum[VEC] = {};
        add_parts(own, first, 0, 1, sum);
        finish(own, first, sum);
    }
    __syncthreads();
    for (int l = 0; l < many; ++l) {
        const Item it = item_of(longer[l]);
        const bool there = it.c < a.D;
        const int64_t first = there ? piece_first<VEC>(it.c, a.D) : 0;
        float sum[VEC] = {};
        if (there) add_parts(it, first, group, groups, sum);
#pragma unroll
        for (int i = 0; i < VEC; ++i) shares[i * kJoinThreads + threadIdx.x] = sum[i];
        __syncthreads();
        // halves of the groups are added until one is left
        for (int half = groups / 2; half > 0; half /= 2) {
            if (group < half) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) shares[i * kJoinThreads + threadIdx.x] += shares[i * kJoinThreads + threadIdx.x + half * lanes];
            }
            __syncthreads();
        }
        if (group == 0 && there) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) sum[i] = shares[i * kJoinThreads + threadIdx.x];
            finish(it, first, sum);
        }
        __syncthreads();
    }
}

constexpr int kFewTokens = 8192, kFewThreads = 1024, kFewWaves = kFewThreads / 64, kFewRows = 1024;

// The gradient of a few tokens in one launch: workgroup b has the rows b, b + 2^shift, .. (so that frequent ids, which vocabularies have
// first, are different workgroups'), looks at all tokens and lists those of its rows.  A wavefront has a row and lanes * VEC columns and
// adds up the tokens that the list has for the row; a row of many tokens is the whole workgroup's, whose wavefronts share the list.
// The rows that a workgroup clears are others, neighbouring ones.
template <typename T, typename G, int VEC, bool ADD>
__global__ __launch_bounds__(kFewThreads) void embed_few_kernel(EmbedGradArgs a, Clearing clearing, int shift)
{
    constexpr int kAhead = 8, kMany = 32;  // tokens on their way; more of them are a row of many
    __shared__ uint16_t tokens[kFewTokens];
    __shared__ uint16_t rows_of[kFewTokens];
    __shared__ int count[kFewRows], found[kFewWaves];
    __shared__ bool busy[ADD ? 1 : kFewRows];  // of the rows to be cleared
    __shared__ float shares[kFewWaves][VEC][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int64_t b = blockIdx.x, step = 1ll << shift;
    const int rows = (int)((a.V - b + step - 1) >> shift);  // kFewRows at most
    static_assert(kFewRows == kFewThreads && kFewRows == 64 * kFewWaves && kFewTokens <= 65536, "");
    count[threadIdx.x] = 0;
    const int clear_each = (int)((a.V + (int64_t)gridDim.x * gridDim.y - 1) / ((int64_t)gridDim.x * gridDim.y));  // kFewRows at most
    const int64_t clear0 = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (clear_each);
    if (!ADD) busy[threadIdx.x] = false;
    // a wavefront has a run of the tokens
    constexpr int kEach = kFewTokens / kFewThreads;
    int32_t id[kEach];
    uint64_t hits[kEach];
    int fill = 0;
    const int share = ((int)a.T + kFewThreads - 1) / kFewThreads * 64;  // kEach * 64 at most
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int at = wave * share + i * 64 + lane;
        id[i] = a.ids[min(at, (int)a.T - 1)];
        id[i] = (int)(i * 64 < share) & (int)(at < a.T) ? id[i] : -1;
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        hits[i] = __ballot(id[i] >= 0 && id[i] < a.V && (id[i] & (step - 1)) == b);
        fill += __popcll(hits[i]);
    }
    if (lane == 0) found[wave] = fill;
    __syncthreads();
    if (!ADD) {
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (id[i] >= clear0 && id[i] < clear0 + clear_each && id[i] < a.V) busy[id[i] - clear0] = true;
    }
    int at = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) {
        at += w < wave ? found[w] : 0;
        all += found[w];
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        if (hits[i] >> lane & 1) {
            const int to = at + __popcll(hits[i] & ((1ull << lane) - 1)), row = id[i] >> shift;
            tokens[to] = (uint16_t)(wave * share + i * 64 + lane);
            rows_of[to] = (uint16_t)row;
            atomicAdd(&count[row], 1);  // (whole numbers)
        }
        at += __popcll(hits[i]);
    }
    __syncthreads();
    // sum += the rows of dout of the list's entries from .. to that are row r's, in their order
    const auto add_tokens = [&](int r, int from, int to, int64_t first, float (&sum)[VEC]) {
        const T* __restrict__ dout = static_cast<const T*>(a.dout) + first;
        for (int e0 = from; e0 < to; e0 += 64) {
            const int e = e0 + lane;
            const bool mine = e < to && rows_of[e] == r;
            const int token = e < to ? tokens[e] : 0;
            uint64_t left = __ballot(mine);
            while (__popcll(left) >= kAhead) {
                Columns<T, VEC> x[kAhead];
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    x[u].load(dout + (int64_t)__builtin_amdgcn_readlane(token, __builtin_ctzll(left)) * a.ldd);
                    left &= left - 1;
                }
#pragma unroll
                for (int u = 0; u < kAhead; ++u)
#pragma unroll
                    for (int i = 0; i < VEC; ++i) sum[i] += x[u].v[i];
            }
            if (left) {
                // (in place of one that is not there, the last, and not added)
                const int n = __popcll(left);
                Columns<T, VEC> x[kAhead];
#pragma unroll
                for (int u = 0; u + 1 < kAhead; ++u) {
                    x[u].load(dout + (int64_t)__builtin_amdgcn_readlane(token, __builtin_ctzll(left)) * a.ldd);
                    left = left & (left - 1) ? left & (left - 1) : left;
                }
#pragma unroll
                for (int u = 0; u + 1 < kAhead; ++u)
#pragma unroll
                    for (int i = 0; i < VEC; ++i) sum[i] += u < n ? x[u].v[i] : 0.0f;
            }
        }
    };
    const int pieces = (int)((a.D + 64 * VEC - 1) / (64 * VEC));
    const auto row_of = [&](int r) { return b + ((int64_t)r << shift); };
    // a wavefront's rows, as many as lanes at most
    const int own = lane * kFewWaves + wave, n = own < rows ? count[own] : -1;
    if constexpr (!ADD) {
        const int mine = (clear_each + kFewWaves - 1) / kFewWaves, r = wave * mine + lane;  // a wavefront's rows, neighbouring ones
        clear_rows<false>(clearing, clear0 + wave * mine,
                   __ballot(lane < mine && r < clear_each && clear0 + r < a.V && !busy[min(r, kFewRows - 1)]));
    }
    for (uint64_t left = __ballot(n > 0 && n <= kMany); left; left &= left - 1) {
        const int r = __builtin_ctzll(left) * kFewWaves + wave;
        const int64_t v = row_of(r);
        for (int piece = blockIdx.y; piece < pieces; piece += gridDim.y) {
            const int64_t c = ((int64_t)piece * 64 + lane) * VEC;
            const bool there = c < a.D;
            const int64_t first = there ? piece_first<VEC>(c, a.D) : 0;
            float sum[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) sum[i] = 0.0f;
            GradPiece<G, VEC> was;
            if (ADD) was.load(static_cast<const G*>(a.dweights) + v * a.ldw + first);
            add_tokens(r, 0, all, first, sum);
            if (there) store_row<ADD>(a, v, first, (int)(c - first), sum, was);
        }
    }
    for (int g = 0; g < rows; g += 64)
    for (uint64_t left = __ballot(g + lane < rows && count[min(g + lane, rows - 1)] > kMany); left; left &= left - 1) {
        const int r = g + __builtin_ctzll(left), each = (all + kFewWaves - 1) / kFewWaves, from = min(wave * each, all);
        const int64_t v = row_of(r);
        for (int piece = blockIdx.y; piece < pieces; piece += gridDim.y) {
            const int64_t c = ((int64_t)piece * 64 + lane) * VEC;
            const bool there = c < a.D;
            const int64_t first = there ? piece_first<VEC>(c, a.D) : 0;
            float sum[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) sum[i] = 0.0f;
            add_tokens(r, from, min(from + each, all), first, sum);
            __syncthreads();  // the shares before are read
#pragma unroll
            for (int i = 0; i < VEC; ++i) shares[wave][i][lane] = sum[i];
            __syncthreads();
            if (wave != piece % kFewWaves || !there) continue;
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                sum[i] = 0.0f;
#pragma unroll
                for (int w = 0; w < kFewWaves; ++w) sum[i] += shares[w][i][lane];
            }
            GradPiece<G, VEC> was;
            if (ADD) was.load(static_cast<const G*>(a.dweights) + v * a.ldw + first);
            store_row<ADD>(a, v, first, (int)(c - first), sum, was);
        }
    }
}

template <typename T, int VEC, int TOKENS>
hipError_t embed_tokens(const EmbedArgs& a, const Spread& sp, hipStream_t s)
{
    return launch_parts(blocks_of(sp, (a.T + TOKENS - 1) / TOKENS), kThreads, [&](unsigned grid, int64_t block0) {
        embed_kernel<T, VEC, TOKENS><<<grid, kThreads, 0, s>>>(a, sp.lanes, sp.column_items, block0);
    });
}

template <typename T, int VEC>
hipError_t embed(const EmbedArgs& a, hipStream_t s)
{
    const Spread sp = spread<VEC>(a.D);
    // two tokens to a group where that leaves wavefronts enough for the chip, and many rows are written (16,384 by 2,048, bf16: 23.9 us
    // with one, 16.4, 16.8 with four)
    return blocks_of(sp, a.T) >= 2048 ? embed_tokens<T, VEC, 2>(a, sp, s) : embed_tokens<T, VEC, 1>(a, sp, s);
}

template <typename T, typename G, int VEC, bool ADD>
hipError_t embed_grad(const EmbedGradArgs& a, hipStream_t s)
{
    const int64_t halves = sizeof(G) / 2;
    const Clearing clearing = {ADD ? nullptr : static_cast<uint16_t*>(a.dweights), a.D * halves, a.ldw * halves};
    // One launch for a few tokens.  It reads a frequent token's rows by one compute unit, and where a large table is cleared that comes on
    // top.  (us, three launches and one, ids' frequency one over their rank, 16 bits: 92 tokens, 496 rows of 557 15.4, 5.0; 1,498, 551 of
    // 256 19.0, 7.6; 4,096, 32,000 of 1,024 41.2, 20.5; 8,192, 8,000 of 512 35.0, 19.0; 8,192, 65,536 of 2,048 82.9, 88.2, and added up
    // 64.6, 36.1.)  It is the slower one where one id has a large part of the tokens, since a row's columns are four workgroups' at most with
    // 64 rows or more: all of 4,096 tokens of 1,024 34.5, 53.7; three launches with 8,193 tokens, one with 8,192 added to 8,000 rows in 16 bits, all / half /
    // frequency one over rank: of 1,024 42.5, 90.3 / 35.7, 51.2 / 32.5, 21.9; of 4,096 48.6, 176 / 47.1, 142 / 46.5, 46.7; of 8,192 58.5, 328 /
    // 67.0, 277 / 64.7, 104.  And where the ids have few residues of the number of workgroups across rows, whose list each wavefront looks through for
    // each row: 8,192 tokens of 1,024, 32,768 rows, ids multiples of 1 / 64 / 256 / 4,096 23.1, 21.2 / 20.3, 537 / 20.6, 929 / 24.1, 153.
    // The ids are on the device: the host's rule cannot tell.
    if (a.T > 0 && a.T <= kFewTokens && a.V <= 1 << 22 && (ADD || a.T <= 1024 || a.V * a.D * (int64_t)sizeof(G) <= 128 << 20)) {
        // 256 workgroups, by rows first; columns are shared by four of them where there are so many, so that a frequent token's are
        const int64_t pieces = (a.D + 64 * VEC - 1) / (64 * VEC), four = std::min<int64_t>(pieces, 4);
        int shift = 0;
        while ((int64_t)kFewRows << shift < a.V || (four << shift < 256 && 2ll << shift <= a.V)) ++shift;
        const int64_t across = std::min(pieces, std::max<int64_t>(four, 256 >> shift));
        embed_few_kernel<T, G, VEC, ADD><<<dim3(1u << shift, (unsigned)across), kFewThreads, 0, s>>>(a, clearing, shift);
        return hipGetLastError();
    }
    const Spread sp = spread<VEC>(a.D);
    const Sorted st = sorted_view(a.workspace, a.T, a.V, a.D, kThreads / sp.lanes);
    // A workgroup of the sort looks at all tokens, so that its time grows with tokens times rows: even ids, floats, 262,144 tokens and rows of 64
    // 113 us, 1,048,576 of 16 969, 4,194,304 tokens of those 3,597.
    // 256 ranges, one for each compute unit (us of lookup and gradient, 512 and 256: 16,384 tokens, 65,536 rows of 2,048 95.7, 95.0; 16,384
    // rows 62.3, 57.8; 12,000 tokens, 50,001 rows of 64 26.1, 22.1)
    constexpr int64_t ranges = 256;
    // Few of many long rows are in use: cleared without waiting for the tokens, which writes the rows in use twice.  (us of lookup and
    // gradient after the tokens are known and before, ids' frequencies even / one over their rank: 9,000 tokens, 262,144 rows of 512
    // floats 123, 113 / 121, 111; 16,384, 65,536 of 1,024 in 16 bits 56.8, 51.4 / 57.6, 53.0; 16,384, 65,536 of 2,048 95.8, 96.4 / 88.1, 84.1;
    // shorter rows: 9,000, 131,072 of 256 floats 45.5, 48.5 / 45.7, 49.4; more tokens: 10,000, 30,000 of 1,000 39.7, 41.4 / 46.3, 47.7)
    const bool unseen = !ADD && a.T <= a.V / 4 && a.D * (int64_t)sizeof(G) >= 2048;
    int ids_of = 1;
    while (ids_of < kMostIds && ids_of * ranges < a.V) ids_of *= 2;
    hipError_t err = launch_parts((a.V + ids_of - 1) / ids_of * (unseen ? 2 : 1), kSortThreads, [&](unsigned grid, int64_t block0) {
        embed_sort_kernel<<<grid, kSortThreads, kSortWaves * ids_of * 4, s>>>(a.ids, a.T, a.V, ids_of, st.start, st.key, st.order, clearing, unseen, block0);
    });
    if (err != hipSuccess) return err;
    err = launch_parts(st.tiles * sp.column_items, kThreads, [&](unsigned grid, int64_t block0) {
        embed_sum_kernel<T, G, VEC, ADD><<<grid, kThreads, 0, s>>>(a, st, sp.lanes, sp.column_items, block0);
    });
    if (err != hipSuccess) return err;
    const int64_t groups = kJoinThreads / sp.lanes, joins = st.tiles > 1 ? ((st.tiles - 1) * sp.column_items + groups - 1) / groups : 0;
    return launch_parts(joins + (ADD ? 0 : (a.V + kClearRows - 1) / kClearRows), kJoinThreads, [&](unsigned grid, int64_t block0) {
        embed_join_kernel<G, VEC, ADD><<<grid, kJoinThreads, 0, s>>>(a, st, clearing, sp.lanes, sp.column_items, joins, block0);
    });
}

template <typename T>
hipError_t embed_by_width(const EmbedArgs& a, hipStream_t s)
{
    return a.D >= Piece<T>::kCount ? embed<T, Piece<T>::kCount>(a, s) : embed<T, 1>(a, s);
}

template <typename T, typename G>
hipError_t grad_by_width(const EmbedGradArgs& a, hipStream_t s)
{
    constexpr int kVec = Piece<T>::kCount;
    if (a.accumulate) return a.D >= kVec ? embed_grad<T, G, kVec, true>(a, s) : embed_grad<T, G, 1, true>(a, s);
    return a.D >= kVec ? embed_grad<T, G, kVec, false>(a, s) : embed_grad<T, G, 1, false>(a, s);
}

template <typename T>
hipError_t grad_by_type(const EmbedGradArgs& a, hipStream_t s)
{
    return a.grad_dtype == a.dtype ? grad_by_width<T, T>(a, s) : grad_by_width<T, float>(a, s);
}

}  // namespace

int64_t embed_grad_workspace_bytes(int64_t T, int64_t V, int64_t D) { return sorted_view(nullptr, T, V, D, 4).bytes; }

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
