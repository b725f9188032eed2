// Shared by the operators of a mixture of experts: element types, 16-byte pieces of rows, the matrix instruction, and
// the host-side launch entry points.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sgap {

typedef _Float16 half_t;
typedef __bf16 bf16_t;

// 16 bytes as the memory path takes them, asking for no more alignment than an element has: this chip reads and writes
// such addresses in one instruction.
template <typename T>
struct Piece {
    static constexpr int kCount = 16 / (int)sizeof(T);
    typedef T vec __attribute__((ext_vector_type(16 / sizeof(T))));
    typedef T loose __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
};
template <typename T>
using piece_t = typename Piece<T>::vec;

template <typename T>
__device__ __forceinline__ piece_t<T> load_piece(const T* p)
{
    return *reinterpret_cast<const typename Piece<T>::loose*>(p);
}
template <typename T>
__device__ __forceinline__ void store_piece(T* p, piece_t<T> v)
{
    *reinterpret_cast<typename Piece<T>::loose*>(p) = v;
}

typedef float f32x4 __attribute__((ext_vector_type(4)));

// acc += A * B on a 16 x 16 tile.  A lane has 16 bytes of one row of A (row lane % 16) and of one column of B (column
// lane % 16), the piece lane / 16 of four: 32 values of the inner dimension with 16-bit types, 16 with floats, where one
// instruction takes one value of each lane.  Which lane holds which value of the inner dimension does not matter as long
// as A and B agree.  Result: lane l has rows 4 * (l / 16) + 0 .. 3 of column l % 16.
__device__ __forceinline__ f32x4 mma16(piece_t<half_t> a, piece_t<half_t> b, f32x4 acc)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, acc, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma16(piece_t<bf16_t> a, piece_t<bf16_t> b, f32x4 acc)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, acc, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma16(piece_t<float> a, piece_t<float> b, f32x4 acc)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], acc, 0, 0, 0);
    return acc;
}

// The rows that a product takes: row r is row src[r] / div of X, or row r itself without a list.
struct RowSource {
    const int32_t* __restrict__ src;
    uint32_t mul;  // n / div = n * mul >> shift for every n < 2^31 (shift = 31 + log2 of div, rounded up)
    int shift;
    int64_t rows;  // rows of X; a row that lies outside counts as zeros
    RowSource(const int32_t* src_, int64_t div, int64_t rows_) : src(src_), shift(31), rows(rows_)
    {
        while ((1ll << (shift - 31)) < div) ++shift;
        // 2^shift / div, rounded up; shift is 62 at most
        mul = (uint32_t)(((1ull << shift) + (uint64_t)div - 1) / (uint64_t)div);
    }
    // what the list says for row r, and what row of X that is (-1: none): in two steps, for who wants the first to be on
    // its way for a while
    __device__ __forceinline__ int32_t entry(int64_t r) const { return src ? src[r] : (int32_t)r; }
    __device__ __forceinline__ int32_t row_of(int32_t e) const
    {
        const int32_t t = src ? (int32_t)(((uint64_t)(uint32_t)e * mul) >> shift) : e;
        return e < 0 || t >= rows ? -1 : t;
    }
    __device__ __forceinline__ int64_t row(int64_t r) const { return row_of(entry(r)); }
};

// Rows first .. end of group g; nothing outside 0 .. rows whatever the offsets hold.  Without offsets: one group of all rows.
struct GroupRows {
    int64_t first, end;
};
__device__ __forceinline__ GroupRows group_rows(const int32_t* __restrict__ offsets, int64_t g, int64_t rows)
{
    if (!offsets) return {0, rows};
    const int64_t a = offsets[g], b = offsets[g + 1];
    const int64_t first = a < 0 ? 0 : a, end = b > rows ? rows : b;
    return {first, end < first ? first : end};
}

// What a product over groups has to know.  K: inner dimension of the product, N: its columns.  For the weights' gradient Y
// holds the gradient of the product's result (read), W the gradient of the weights (written).
struct GroupedArgs {
    int64_t G, R, K, N;
    const int32_t* __restrict__ offsets;
    RowSource from;
    const void* __restrict__ X;
    int64_t ldx;
    const void* __restrict__ W;  // G matrices, N x K or K x N
    void* __restrict__ Y;
    int64_t ldy;
    bool weights_kn;  // K x N
    int compute_units;
};

struct GroupedW4Args {
    int64_t G, R, K, N;
    const int32_t* __restrict__ offsets;
    RowSource from;
    const void* __restrict__ X;
    int64_t ldx;
    const uint8_t* __restrict__ weights;  // as launch_w4_layout leaves them
    int group_k;
    bool zeros;
    void* __restrict__ Y;
    int64_t ldy;
};

struct RouteArgs {
    int64_t T;
    int E, k, dtype;
    bool renormalise;
    const void* __restrict__ logits;
    int64_t ld;
    float* __restrict__ gates;
    int32_t *__restrict__ experts, *__restrict__ slot, *__restrict__ order, *__restrict__ offsets;
    void* workspace;
};

struct RouteGradArgs {
    int64_t T;
    int E, k, dtype;
    bool renormalise;
    const void* __restrict__ logits;
    int64_t ld;
    const float* __restrict__ gates;
    const int32_t* __restrict__ experts;
    const float* __restrict__ dgates;
    void* __restrict__ dlogits;
    int64_t ldd;
};

struct CombineArgs {
    int64_t T, D;
    int k, dtype;
    const void* __restrict__ Z;
    const int32_t* __restrict__ slot;
    const int32_t* __restrict__ order;
    const float* __restrict__ gates;
    const void* __restrict__ dout;
    void* __restrict__ out;  // the sum, or the gradient of Z
    float* __restrict__ dgates;
};

// A launch has fewer than 2^32 threads (a larger grid is cut off to what is left over 2^32, mostly without an error): more
// workgroups go out as several launches, launch(workgroups, block0), in which workgroup b is number block0 + b of all.  (Parts are multiples of 256 workgroups, so that eight dies have whole turns.)
template <typename F>
inline hipError_t launch_parts(int64_t workgroups, int threads, F&& launch)
{
    const int64_t most = (0xffffffffLL / threads) & ~255LL;
    for (int64_t block0 = 0; block0 < workgroups; block0 += most) {
        const int64_t left = workgroups - block0;
        launch((unsigned)(left < most ? left : most), block0);
        if (const hipError_t err = hipGetLastError()) return err;
    }
    return hipSuccess;
}

int64_t route_workspace_bytes(int64_t T, int64_t E);
hipError_t launch_route(const RouteArgs& a, hipStream_t s);
hipError_t launch_route_grad(const RouteGradArgs& a, hipStream_t s);
hipError_t launch_combine(const CombineArgs& a, hipStream_t s);
hipError_t launch_combine_grad(const CombineArgs& a, hipStream_t s);
// dtype as in sgap.h
// Which kernel a product over groups, or the gradient of its weights, takes.
struct GroupedPlan {
    enum Way {
        kTiles,     // rows that are multiples of 16 bytes at 16-byte addresses: sgap_grouped_fast.hip
        kFew,       // of those, too few rows, columns or weights for tiles to fill the chip: sgap_grouped_few.hip
        kRegisters  // every other call: sgap_grouped_general.hip
    } way;
    int rows, columns;  // of a workgroup's part of the result
    bool wide;          // kTiles: X is longer than 4 GiB
    bool apart;         // kTiles: workgroups begin at different places of the inner dimension
    bool short_rows;    // kRegisters: rows of fewer elements than 16 bytes hold
};
GroupedPlan plan_grouped(const GroupedArgs& a, int dtype, bool gradient);
// the parts of that
bool grouped_fast_applies(const GroupedArgs& a, int dtype);
GroupedPlan plan_grouped_fast(const GroupedArgs& a, int dtype, bool gradient);
hipError_t launch_grouped_fast(const GroupedArgs& a, int dtype, bool gradient, const GroupedPlan& p, hipStream_t s);
bool grouped_few_applies(const GroupedArgs& a, int dtype, bool gradient);
GroupedPlan plan_grouped_few(const GroupedArgs& a, int dtype, bool gradient);
hipError_t launch_grouped_few(const GroupedArgs& a, int dtype, bool gradient, const GroupedPlan& p, hipStream_t s);
hipError_t launch_grouped_mm(const GroupedArgs& a, int dtype, hipStream_t s);
hipError_t launch_grouped_wgrad(const GroupedArgs& a, int dtype, hipStream_t s);
struct W4Sizes {
    int64_t tiles_n, blocks_k, scales_k;   // per group: tiles of 16 columns, blocks of 128 weights, scales along K
    int64_t scales_at, zeros_at, bytes;    // byte offsets in the laid-out weights
};
W4Sizes w4_sizes(int64_t G, int64_t K, int64_t N, int group_k, bool zeros);
hipError_t launch_w4_layout(int64_t G, int64_t K, int64_t N, int group_k, const uint8_t* q, const void* scales,
                            const uint8_t* zeros, uint8_t* out, hipStream_t s);
hipError_t launch_grouped_w4(const GroupedW4Args& a, int dtype, hipStream_t s);

}  // namespace sgap
