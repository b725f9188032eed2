// Tiles of an operand in LDS, put there by loads that go past the registers, and their fragments for the matrix unit.
//
// An operand has LINES lines (columns or rows of the result) and 128 bytes of the inner dimension in a tile.
//   inner contiguous  a line is 128 bytes, its 16-byte piece p at place p ^ (line & 7): sixteen lanes that read one piece of
//                     sixteen lines meet in no bank
//   lines contiguous  an inner value has a row of LINES elements, in chunks of 32 bytes (16-bit types) or 64 (floats) whose
//                     places are rotated by the row's number, so that the rows that lanes read together lie apart.  16-bit
//                     values are turned by the LDS itself on the way out (four inner values of sixteen lines at a time),
//                     floats are read one by one.
// The loads write LDS in the order of the lanes, so it is the addresses they read from that are rotated.  In place of a
// piece that does not exist (inner values past the end, rows that are not there) a lane reads one that does, and writes
// zeros over it when it has arrived.
#pragma once
#include "sgap_grouped.hpp"

namespace sgap {

// The same in every lane of the wavefront, in scalar registers.
template <typename P>
__device__ __forceinline__ const P* uniform(const P* p)
{
    const uint64_t v = (uint64_t)(uintptr_t)p;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
    return (const P*)(uintptr_t)((uint64_t)hi << 32 | lo);
}

template <typename T, int LINES, bool INNER, int THREADS>
struct Tile {
    static constexpr int P = Piece<T>::kCount;
    static constexpr int kInner = 128 / (int)sizeof(T);  // inner values of a tile
    static constexpr int kBytes = LINES * 128;
    static constexpr int kRounds = kBytes / 16 / THREADS;
    static constexpr int kAcross = LINES / P;  // pieces of a row (lines contiguous)
    static_assert(kBytes % (16 * THREADS) == 0 && (INNER || LINES >= 128), "");

    // the rotation of row k's chunks
    static __device__ __forceinline__ int turn(int k) { return sizeof(T) == 2 ? (k & 3) | ((k >> 3) & 1) << 2 : (k >> 2) & 3; }

    // What the piece at place `round * THREADS + thread` holds: a line and an inner piece, or an inner value and a piece
    // of the lines.
    static __device__ __forceinline__ int major(int round) { return (round * THREADS + (int)threadIdx.x) / (INNER ? 8 : kAcross); }
    static __device__ __forceinline__ int minor(int round)
    {
        const int place = (round * THREADS + (int)threadIdx.x) % (INNER ? 8 : kAcross), m = major(round);
        if (INNER) return place ^ (m & 7);
        if (sizeof(T) == 2) return place ^ (turn(m) << 1);
        return place ^ (turn(m) << 2);
    }

    // In the assembler's words, because the compiler, which cannot tell the stage that is being filled from the one that is
    // read, would wait for every load before the next read.  They count as vector memory loads: wait_loads().
    // `lds`: the tile's LDS address; the wavefront's lanes fill 1,024 consecutive bytes of it a round.
    static __device__ __forceinline__ uint32_t place(uint32_t lds, int round)
    {
        const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        return lds + (round * THREADS + wave * 64) * 16;
    }
    static __device__ __forceinline__ void load(uint32_t lds, int round, const void* base, uint32_t offset)  // base: the wavefront's
    {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                     :
                     : "s"(place(lds, round)), "v"(offset), "s"(base)
                     : "m0", "memory");
    }
    static __device__ __forceinline__ void load(uint32_t lds, int round, const void* from)
    {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                     :
                     : "s"(place(lds, round)), "v"(from)
                     : "m0", "memory");
    }
    // into the place that this lane's load would fill
    static __device__ __forceinline__ void put(uint32_t lds, int round, piece_t<T> v)
    {
        typedef __attribute__((address_space(3))) piece_t<T> lds_piece;
        *(lds_piece*)(uintptr_t)(lds + (round * THREADS + threadIdx.x) * 16) = v;
    }
    static __device__ __forceinline__ void clear(uint32_t lds, int round) { put(lds, round, piece_t<T>{}); }

    // Where in a tile this lane's fragments begin, for the lines from line0 on: a multiple of sixteen times the power of two that
    // the wavefront's fragments are.
    static __device__ __forceinline__ uint32_t lane_base(int line0)
    {
        const int lane = threadIdx.x & 63, row = lane & 15, part = lane >> 4;
        if constexpr (INNER) return (uint32_t)((line0 + row) * 128 + ((part ^ (row & 7)) << 4));
        const int chunk = line0 >> 4;
        if constexpr (sizeof(T) == 2) {
            const int k = part * 8 + (row >> 2);  // this lane's row of the four that are turned together; four rows on: the same turn
            return (uint32_t)(k * (LINES * 2) + (chunk >> 3) * 256 + (((chunk & 7) ^ turn(k)) << 5) + (row & 3) * 8);
        }
        const int k = part * 4;
        return (uint32_t)(k * (LINES * 4) + (chunk >> 2) * 256 + (((chunk & 3) ^ turn(k)) << 6) + row * 4);
    }

    // Lanes' pieces of the sixteen lines number i behind lane_base's, inner values of step kc of 2.  `base`: the LDS address.
    static __device__ __forceinline__ piece_t<T> fragment(uint32_t base, int i, int kc)
    {
        typedef __attribute__((address_space(3))) piece_t<T> lds_piece;
        if constexpr (INNER) {
            return *(const lds_piece*)(uintptr_t)((base ^ (kc << 6)) + i * 2048);
        } else if constexpr (sizeof(T) == 2) {
            typedef short short4_t __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) short4_t lds_short4;
            union {
                short4_t h[2];
                piece_t<T> v;
            } r;
            const uint32_t at = (base ^ ((i & 7) << 5)) + (i >> 3) * 256 + kc * (32 * LINES * 2);
#pragma unroll
            for (int h = 0; h < 2; ++h)
                r.h[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4*)(uintptr_t)(at + h * (4 * LINES * 2)));
            return r.v;
        } else {
            typedef __attribute__((address_space(3))) float lds_float;
            piece_t<T> v;
            const uint32_t at = (base ^ ((i & 3) << 6)) + (i >> 2) * 256 + kc * (16 * LINES * 4);
#pragma unroll
            for (int h = 0; h < 4; ++h) v[h] = *(const lds_float*)(uintptr_t)(at + h * (LINES * 4));
            return v;
        }
    }
};

// acc += first x second over `tiles` tiles of the inner dimension.  Two stages: the loads of a tile have the whole of the
// one before to arrive in, the fragments of a half tile the products of the half before, so that the matrix unit waits for
// neither; one barrier a tile, in its middle, says that everyone has read the stage that is filled next and that the other
// stage is full.  Loads, fragments and products are dealt out evenly (the compiler by itself puts all fragments behind the
// products, and then waits).
//   load(t, stage, i)   starts load i of LOADS of tile t; every lane reads something that is there
//   mend(t, stage)      after tile t's loads have arrived: zeros where a lane had nothing to read
// ACTIVE: this wavefront has products to make.
template <typename L, typename R, int MI, int NJ, bool ACTIVE, typename F, typename M>
__device__ __forceinline__ void multiply_tiles_as(uint32_t lds, int tiles, F&& load, M&& mend, int l0, int r0, f32x4 (&acc)[MI][NJ])
{
    constexpr uint32_t kStage = L::kBytes + R::kBytes;
    constexpr int kLoads = L::kRounds + R::kRounds;
    using frag = decltype(L::fragment(0u, 0, 0));
    frag fl[2][MI], fr[2][NJ];
    Runs<L::P == 4, MI, NJ, 512 / L::kInner, true> runs;  // floats: only where sums are not finite, and time counts less
    const uint32_t lbase = lds + L::lane_base(l0), rbase = lds + L::kBytes + R::lane_base(r0);
    uint32_t lb, rb;
    const auto at = [&](uint32_t stage) {
        lb = lbase + stage, rb = rbase + stage;
        asm volatile("" : "+v"(lb), "+v"(rb));  // the fragments' addresses are made anew each time, not kept in registers
    };
    const auto read = [&](int kc, int i) {
        if (i < MI) fl[kc][i] = L::fragment(lb, i, kc);
        else fr[kc][i - MI] = R::fragment(rb, i - MI, kc);
    };
    // the products of one half, with the reads of the next and, if any, the loads of a tile between them
    const auto half = [&](int kc, auto&& between) {
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            between(j);
            if constexpr (ACTIVE) {
#pragma unroll
                for (int i = j * (MI + NJ) / NJ; i < (j + 1) * (MI + NJ) / NJ; ++i) read(1 - kc, i);
#pragma unroll
                for (int i = 0; i < MI; ++i) acc[i][j] = mma16(fl[kc][i], fr[kc][j], acc[i][j]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    const auto meet = [&](int t) {
        wait_loads();
        if (t < tiles) mend(t, lds + (t & 1) * kStage);
        __syncthreads();
    };
#pragma unroll
    for (int i = 0; i < kLoads; ++i) load(0, lds, i);
    if (tiles > 1) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) load(1, lds + kStage, i);
    }
    wait_loads();
    mend(0, lds);
    __syncthreads();
    at(0);
    if constexpr (ACTIVE) {
#pragma unroll
        for (int i = 0; i < MI + NJ; ++i) read(0, i);
    }
    int t = 0;
    for (; t + 2 < tiles; ++t) {
        const uint32_t stage = (t & 1) * kStage;
        at(stage);
        half(0, [](int) {});
        meet(t + 1);
        at(kStage - stage);
        half(1, [&](int j) {
#pragma unroll
            for (int i = j * kLoads / NJ; i < (j + 1) * kLoads / NJ; ++i) load(t + 2, lds + stage, i);
        });
        runs.end_of(t, acc);
    }
    for (; t < tiles; ++t) {
        const uint32_t stage = (t & 1) * kStage;
        at(stage);
        half(0, [](int) {});
        meet(t + 1);
        at(kStage - stage);
        half(1, [](int) {});  // behind the last tile the fragments that are read are not used
        runs.end_of(t, acc);
    }
    runs.finish(acc);
}
template <typename L, typename R, int MI, int NJ, typename F, typename M>
__device__ __forceinline__ void multiply_tiles(char* shared, int tiles, F&& load, M&& mend, int l0, int r0, bool active,
                                               f32x4 (&acc)[MI][NJ])
{
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)shared;
    if (tiles == 0) return;
    if (active) multiply_tiles_as<L, R, MI, NJ, true>(lds, tiles, load, mend, l0, r0, acc);
    else multiply_tiles_as<L, R, MI, NJ, false>(lds, tiles, load, mend, l0, r0, acc);
}

// Eight floats as three times eight 16-bit ones, x = high + middle + low: eight bits of x's 24 each, rounded to nearest, so
// that the middle one is at most 2^-8 of x and the low one 2^-17.
struct Split {
    piece_t<bf16_t> high, middle, low;
};
// Two floats rounded to 16 bits, and in `rest` what that leaves of them (exact): an instruction for both, and four.
__device__ __forceinline__ uint32_t round_two(float x, float y, float (&rest)[2])
{
    typedef float float2_t __attribute__((ext_vector_type(2)));
    typedef bf16_t bf2_t __attribute__((ext_vector_type(2)));
    const uint32_t both = __builtin_bit_cast(uint32_t, __builtin_convertvector(float2_t{x, y}, bf2_t));
    rest[0] = x - __uint_as_float(both << 16);
    rest[1] = y - __uint_as_float(both & 0xffff0000u);
    return both;
}
__device__ __forceinline__ Split split(piece_t<float> x, piece_t<float> y)
{
    uint32_t high[4], middle[4], low[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float r[2], q[2], none[2];
        high[i] = round_two(i < 2 ? x[2 * i] : y[2 * i - 4], i < 2 ? x[2 * i + 1] : y[2 * i - 3], r);
        middle[i] = round_two(r[0], r[1], q);
        low[i] = round_two(q[0], q[1], none);
    }
    Split s;
    __builtin_memcpy(&s.high, high, 16);
    __builtin_memcpy(&s.middle, middle, 16);
    __builtin_memcpy(&s.low, low, 16);
    return s;
}

// Products of floats on the 16-bit matrix instruction, which makes sixteen times as many in the same time as the one for
// floats: of the nine products of the parts the six that count, and what is left out (middle x low twice and low x low) is
// 2^-24 of a product at most, no more than the rounding of a float.  The two half tiles are the instruction's 32 inner values.
// The six products of 32 inner values are summed up by themselves and then added: one rounding of the sum for 32 values, where
// the matrix instruction's own additions to it would be six.  Root mean square of the result's
// error over 1,024, 16,384 and 65,536 values: 1.2e-7, 4.3e-7 and 8.5e-7 (six additions: 4.8e-7, 2.1e-6 and 4.5e-6; a library's
// product 2.9e-7, 1.1e-6 and 2.8e-6).
// Where a value is infinite, no number or rounds up to infinity, every result that it has a part in comes out not finite,
// and the caller computes the tile again with the instruction for floats.
template <typename L, typename R, int MI, int NJ, typename F, typename M>
__device__ __forceinline__ void multiply_tiles_split(char* shared, int tiles, F&& load, M&& mend, int l0, int r0, bool active,
                                                     f32x4 (&acc)[MI][NJ])
{
    constexpr uint32_t kStage = L::kBytes + R::kBytes;
    constexpr int kLoads = L::kRounds + R::kRounds;
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)shared;
    const uint32_t lbase = lds + L::lane_base(l0), rbase = lds + L::kBytes + R::lane_base(r0);
    if (tiles == 0) return;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) load(0, lds, i);
    for (int t = 0; t < tiles; ++t) {
        const uint32_t stage = (t & 1) * kStage;
        wait_loads();
        mend(t, lds + stage);
        __syncthreads();
        if (t + 1 < tiles) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) load(t + 1, lds + kStage - stage, i);
        }
        if (!active) continue;
        uint32_t lb = lbase + stage, rb = rbase + stage;
        asm volatile("" : "+v"(lb), "+v"(rb));
        // Taking a value apart is five and a half vector instructions, an eighth of what its products cost the matrix unit;
        // they are dealt out between the products of the columns before.
        Split l[MI], r = split(R::fragment(rb, 0, 0), R::fragment(rb, 0, 1));
#pragma unroll
        for (int i = 0; i < MI; ++i) l[i] = split(L::fragment(lb, i, 0), L::fragment(lb, i, 1));
        __builtin_amdgcn_sched_barrier(0);
        f32x4 sum[MI];  // of the column before, added when the matrix unit has it
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            const Split now = r;
            if (j + 1 < NJ) r = split(R::fragment(rb, j + 1, 0), R::fragment(rb, j + 1, 1));
            // the smallest first
            f32x4 fresh[MI];
#pragma unroll
            for (int i = 0; i < MI; ++i) fresh[i] = mma16(l[i].low, now.high, f32x4{0.0f, 0.0f, 0.0f, 0.0f});
#pragma unroll
            for (int i = 0; i < MI; ++i) fresh[i] = mma16(l[i].high, now.low, fresh[i]);
#pragma unroll
            for (int i = 0; i < MI; ++i) fresh[i] = mma16(l[i].middle, now.middle, fresh[i]);
#pragma unroll
            for (int i = 0; i < MI; ++i) fresh[i] = mma16(l[i].middle, now.high, fresh[i]);
#pragma unroll
            for (int i = 0; i < MI; ++i) fresh[i] = mma16(l[i].high, now.middle, fresh[i]);
#pragma unroll
            for (int i = 0; i < MI; ++i) fresh[i] = mma16(l[i].high, now.high, fresh[i]);
            if (j > 0) {
#pragma unroll
                for (int i = 0; i < MI; ++i) acc[i][j - 1] += sum[i];
            }
#pragma unroll
            for (int i = 0; i < MI; ++i) sum[i] = fresh[i];
            __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);  // the reads
#pragma unroll
            for (int i = 0; i < 6 * MI; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // a matrix instruction
                __builtin_amdgcn_sched_group_barrier(0x002, 2, 0);  // two vector ones
            }
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int i = 0; i < MI; ++i) acc[i][NJ - 1] += sum[i];
    }
}

// Whether some wavefront of the workgroup has a sum that is not finite; clears the sums if so.
template <int MI, int NJ>
__device__ __forceinline__ bool start_over(f32x4 (&acc)[MI][NJ])
{
    bool finite = true;
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) finite = finite && __builtin_isfinite(acc[i][j][r]);
    if (!__syncthreads_or(!finite)) return false;
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    return true;
}

// multiply_tiles where the loads cannot go past the registers (rows at addresses that are no multiples of 16 bytes): a tile's
// pieces wait in registers from the middle of one tile to the middle of the next and are then put into LDS.
//   fetch(t, i)    piece i of LOADS of tile t as it lies in memory; called for one tile after the other
//   mend(t, i, v)  what of it belongs there, looked at when it has arrived
template <typename L, typename R, int MI, int NJ, typename T, typename F, typename M>
__device__ __forceinline__ void multiply_tiles_staged(char* shared, int tiles, F&& fetch, M&& mend, int l0, int r0, f32x4 (&acc)[MI][NJ])
{
    constexpr uint32_t kStage = L::kBytes + R::kBytes;
    constexpr int kLoads = L::kRounds + R::kRounds;
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)shared;
    if (tiles == 0) return;
    piece_t<T> fl[2][MI], fr[2][NJ], coming[kLoads];
    Runs<sizeof(T) == 4, MI, NJ, 512 / L::kInner> runs;
    const uint32_t lbase = lds + L::lane_base(l0), rbase = lds + L::kBytes + R::lane_base(r0);
    uint32_t lb, rb;
    const auto at = [&](uint32_t stage) {
        lb = lbase + stage, rb = rbase + stage;
        asm volatile("" : "+v"(lb), "+v"(rb));
    };
    const auto read = [&](int kc, int i) {
        if (i < MI) fl[kc][i] = L::fragment(lb, i, kc);
        else fr[kc][i - MI] = R::fragment(rb, i - MI, kc);
    };
    const auto half = [&](int kc) {
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
#pragma unroll
            for (int i = j * (MI + NJ) / NJ; i < (j + 1) * (MI + NJ) / NJ; ++i) read(1 - kc, i);
#pragma unroll
            for (int i = 0; i < MI; ++i) acc[i][j] = mma16(fl[kc][i], fr[kc][j], acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    const auto get = [&](int t) {
        if (t >= tiles) return;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) coming[i] = fetch(t, i);
    };
    const auto put = [&](int t, uint32_t stage) {
#pragma unroll
        for (int i = 0; i < L::kRounds; ++i) L::put(lds + stage, i, mend(t, i, coming[i]));
#pragma unroll
        for (int i = 0; i < R::kRounds; ++i) R::put(lds + stage + L::kBytes, i, mend(t, L::kRounds + i, coming[L::kRounds + i]));
    };
    get(0);
    put(0, 0);
    get(1);
    __syncthreads();
    at(0);
#pragma unroll
    for (int i = 0; i < MI + NJ; ++i) read(0, i);
    for (int t = 0; t < tiles; ++t) {
        const uint32_t stage = (t & 1) * kStage;
        at(stage);
        half(0);
        if (t + 1 < tiles) put(t + 1, kStage - stage);
        __syncthreads();
        get(t + 2);
        at(kStage - stage);
        half(1);
        runs.end_of(t, acc);
    }
    runs.finish(acc);
}

}  // namespace sgap
