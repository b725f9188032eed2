// How the products over groups find their work: tiles of rows that never cross a group, found from the offsets on the
// device, so that the host needs no group's size.
#pragma once
#include "sgap_experts.hpp"

namespace sgap {

// The rows of one tile: up to BM rows from `first`, of group g; g = G: rows behind the last group, whose results are zero.
struct RowTile {
    int64_t g, first;
    int rows;  // 0: no such tile
};

__device__ __forceinline__ int wave_scan_int(int v)
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
    return v;
}

// Tile number `index` of the tiles of BM rows of all groups, in their order, and of the rows behind them.  By one
// wavefront, whose lanes look at 64 groups at a time; every lane gets the answer.
template <int BM>
__device__ __forceinline__ RowTile find_row_tile(const int32_t* __restrict__ offsets, int64_t G, int64_t R, int64_t index)
{
    if (!offsets) {
        const int64_t first = index * BM;
        return {0, first, first < R ? (int)min((int64_t)BM, R - first) : 0};
    }
    const int lane = threadIdx.x & 63;
    int64_t passed = 0;  // tiles of the groups looked at
    for (int64_t g0 = 0; g0 < G; g0 += 64) {
        const int64_t g = g0 + lane;
        GroupRows rows = {0, 0};
        if (g < G) rows = group_rows(offsets, g, R);
        const int tiles = (int)((rows.end - rows.first + BM - 1) / BM);
        const int upto = wave_scan_int(tiles);
        const uint64_t behind = __ballot(passed + upto > index);
        if (behind) {
            const int who = __builtin_ctzll(behind);
            const int before = __builtin_amdgcn_readlane(upto - tiles, who);
            const int first = __builtin_amdgcn_readlane((int)rows.first, who), end = __builtin_amdgcn_readlane((int)rows.end, who);
            const int64_t at = first + (index - passed - before) * BM;
            return {g0 + who, at, (int)min((int64_t)BM, end - at)};
        }
        passed += __builtin_amdgcn_readlane(upto, 63);
    }
    const int64_t last = group_rows(offsets, G - 1, R).end;
    const int64_t at = last + (index - passed) * BM;
    return {G, at, at < R ? (int)min((int64_t)BM, R - at) : 0};
}

// tiles of BM rows at most: every group may have a last tile that is not full, and the rows behind the groups too
inline int64_t most_row_tiles(int64_t G, int64_t R, int BM, bool offsets)
{
    return offsets ? (R + BM - 1) / BM + (G < R ? G : R) + 1 : (R + BM - 1) / BM;
}

// More LDS than a launch gets unasked; `allowed` has a bit for each device on which that has been asked for.
template <typename K>
inline hipError_t allow_lds(K kernel, int bytes, uint64_t& allowed)
{
    int device = 0;
    if (const hipError_t err = hipGetDevice(&device)) return err;
    if (device < 64 && (allowed >> device & 1)) return hipSuccess;
    const hipError_t err = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (err == hipSuccess && device < 64) allowed |= 1ull << device;
    return err;
}

// Until none of this wavefront's loads is on its way; to the compiler, nothing moves across.  (The builtin tells it that
// its own loads have arrived as well: vmcnt 0, the other counters as they are.)
__device__ __forceinline__ void wait_loads()
{
    asm volatile("" : : : "memory");
    __builtin_amdgcn_s_waitcnt(0x0f70);
    asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
}

// Sums of floats over a long inner dimension: what a run of tiles sums up is added to the total of the runs before, so that a
// sum's error grows with the length of a run (512 values) and the number of runs, not with their product.  Root mean square
// of the result's error, with and without: 3,384 values through registers 4.0e-7, 1.0e-6; 262,144 rows of a gradient shared by
// eight wavefronts 4.3e-7, 3.2e-6 (4.8e-6 in a library's product), where 1,024 x 1,024 weights then take 5.5 ms, 5.0 without.
// TILES: tiles of the inner dimension to a run.  ASIDE: the totals wait in scratch memory, for kernels whose registers the sums
// and what is multiplied fill; they are read and written once a run.
template <bool LONG, int MI, int NJ, int TILES, bool ASIDE = false>
struct Runs {
    typedef __attribute__((address_space(5))) f32x4 aside_t;
    f32x4 total[LONG ? MI : 1][LONG ? NJ : 1];
    bool any = false;
    __device__ __forceinline__ Runs()
    {
        if constexpr (LONG && !ASIDE) {
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NJ; ++j) total[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
    }
    // total i, j from where the compiler cannot see that it might be a register
    __device__ __forceinline__ aside_t* aside()
    {
        aside_t* p = (aside_t*)&total[0][0];
        asm volatile("" : "+s"(p));
        return p;
    }
    // after tile t
    __device__ __forceinline__ void end_of(int t, f32x4 (&acc)[MI][NJ])
    {
        if constexpr (LONG) {
            if ((t + 1) % TILES) return;
            aside_t* const kept = ASIDE ? aside() : nullptr;
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NJ; ++j) {
                    if (ASIDE) kept[i * NJ + j] = any ? kept[i * NJ + j] + acc[i][j] : acc[i][j];
                    else total[i][j] += acc[i][j];
                    acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                }
            any = true;
        }
    }
    __device__ __forceinline__ void finish(f32x4 (&acc)[MI][NJ])
    {
        if constexpr (LONG) {
            if (ASIDE && !any) return;
            aside_t* const kept = ASIDE ? aside() : nullptr;
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NJ; ++j) acc[i][j] += ASIDE ? kept[i * NJ + j] : total[i][j];
        }
    }
};

}  // namespace sgap
