// A lane's share of a row: VEC neighbouring columns as 32-bit floats, read and written as one access.
#pragma once
#include "sgap_experts.hpp"

namespace sgap {

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
    // what nobody reads again soon
    __device__ __forceinline__ void stream_load(const T* p)
    {
        if constexpr (VEC == 1) {
            v[0] = (float)__builtin_nontemporal_load(p);
        } else {
            const piece_t<T> x = __builtin_nontemporal_load(reinterpret_cast<const typename Piece<T>::loose*>(p));
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[i] = (float)x[i];
        }
    }
    __device__ __forceinline__ void stream_store(T* p) const
    {
        if constexpr (VEC == 1) {
            __builtin_nontemporal_store((T)v[0], p);
        } else {
            piece_t<T> x;
#pragma unroll
            for (int i = 0; i < VEC; ++i) x[i] = (T)v[i];
            __builtin_nontemporal_store((typename Piece<T>::loose)x, reinterpret_cast<typename Piece<T>::loose*>(p));
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

}  // namespace sgap
