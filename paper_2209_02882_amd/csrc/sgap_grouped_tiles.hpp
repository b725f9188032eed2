// Tiles of an operand in LDS, put there by loads that go past the registers, and their fragments for the matrix unit.
//
// An operand has LINES lines (columns or rows of the result) and 128 bytes of the inner dimension in a tile.
//   inner contiguous  a line is 128 bytes, its 16-byte piece p at place p ^ (line & 7): sixteen lanes that read one piece of
//                     sixteen lines meet in no bank
//   lines contiguous  an inner value has a row of LINES elements, in chunks of 32 bytes (16-bit types) or 64 (floats) whose
//                     places are rotated by the row's number, so that the rows that lanes read together lie apart.  16-bit
//                     values are turned by the LDS itself on the way out (four inner values of sixteen lines at a time),
//                     floats are read one by one.
// The loads write LDS in the order of the lanes, so it is the addresses they read from that are rotated.  A piece that
// does not exist (inner values past the end, rows that are not there) is read from 16 bytes of zeros.
#pragma once
#include "sgap_grouped.hpp"

namespace sgap {

// what pieces that do not exist are read from
static __device__ __align__(16) const uint32_t g_zero_piece[4] = {0, 0, 0, 0};

// Until at most LEFT of this wavefront's loads are still on their way; to the compiler, nothing moves across.
template <int LEFT>
__device__ __forceinline__ void wait_loads()
{
    asm volatile("s_waitcnt vmcnt(%0)" : : "n"(LEFT) : "memory");
}

template <typename T, int LINES, bool INNER, int THREADS>
struct Tile {
    static constexpr int P = Piece<T>::kCount;
    static constexpr int kInner = 128 / (int)sizeof(T);  // inner values of a tile
    static constexpr int kBytes = LINES * 128;
    static constexpr int kRounds = kBytes / 16 / THREADS;
    static constexpr int kAcross = LINES / P;  // pieces of a row (lines contiguous)
    static_assert(kRounds >= 1 && (INNER || LINES >= 128), "");

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
    static __device__ __forceinline__ void load(char* lds, int round, const T* from)
    {
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
        const uint32_t to = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)(lds + (round * THREADS + wave * 64) * 16);
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                     :
                     : "s"(__builtin_amdgcn_readfirstlane(to)), "v"(from)
                     : "m0", "memory");
    }

    // lanes' pieces of lines line0 .. line0 + 16, inner values of step kc of 2
    static __device__ __forceinline__ piece_t<T> fragment(const char* lds, int line0, int kc)
    {
        const int lane = threadIdx.x & 63, row = lane & 15, part = lane >> 4;
        if constexpr (INNER) {
            const int line = line0 + row;
            return *reinterpret_cast<const piece_t<T>*>(lds + line * 128 + (((kc * 4 + part) ^ (line & 7)) << 4));
        } else if constexpr (sizeof(T) == 2) {
            typedef short short4_t __attribute__((ext_vector_type(4)));
            union {
                short4_t h[2];
                piece_t<T> v;
            } r;
            const int k = kc * 32 + part * 8 + (row >> 2);  // this lane's row of four, and four rows on
            const int chunk = line0 >> 4, within = (row & 3) * 8;
#pragma unroll
            for (int i = 0; i < 2; ++i)
                r.h[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4_t*)(
                    lds + (k + 4 * i) * (LINES * 2) + ((chunk ^ turn(k + 4 * i)) << 5) + within));
            return r.v;
        } else {
            piece_t<T> v;
            const int k = kc * 16 + part * 4, chunk = line0 >> 4;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                v[i] = *reinterpret_cast<const float*>(lds + (k + i) * (LINES * 4) + ((chunk ^ turn(k)) << 6) + row * 4);
            return v;
        }
    }
};

}  // namespace sgap
