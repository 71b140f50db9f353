// What the kernels of mg_experts.h share: their problems as the host hands them on, loads and stores of the three element types at any
// alignment, 8-bit rounding, and the search for the expert whose rows a work-group takes.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/mg_experts.h"

namespace mg {

constexpr int SCALE_BLOCK = 128;          // elements along a row (and rows, of square blocks) that share a scale

// Where the rows of a call belong: all of them to one matrix (offsets null), or rows offsets[e] .. offsets[e+1]-1 to expert e.
struct Groups {
    const int32_t *offsets;
    int count;
    int64_t rows;                         // upper bound of offsets[count]
    const int32_t *source;                // row r comes from row source[r] / fan; null: from row r
    int fan;
};

struct QuantizeProblem {
    int dtype;                            // of X
    bool square;
    int64_t rows, cols, batch;
    const void *X;
    int64_t ldx, stride_x;
    uint8_t *Q;
    int64_t ldq, stride_q;
    float *S;
    int64_t lds, stride_s;
    uint8_t *T;
    int64_t ldt, stride_t;
    float *ST;
    int64_t ldst, stride_st;
    Groups groups;
    hipStream_t stream;
};
hipError_t launch_quantize(const QuantizeProblem &p);

// Canonical product: C row-major, C(i, j) = alpha * sum A(i, l) B(j, l) + beta * C(i, j).  MODE says what `groups` does.
enum BlockMode {
    BLOCK_DENSE = 0,
    BLOCK_ROWS = 1,                       // rows of A and C belong to experts, each with a B of its own
    BLOCK_SUM = 2                         // the summed index runs over an expert's rows, each expert has a C of its own
};
struct BlockProblem {
    int mode;
    int64_t m, n, k;                      // BLOCK_ROWS: m = rows; BLOCK_SUM: k = rows
    float alpha, beta;
    bool pow2, fp32_sums;
    bool a_square, b_square;
    const uint8_t *A;
    int64_t lda;
    const float *SA;
    int64_t ldsa;
    const uint8_t *B;
    int64_t ldb, stride_b;
    const float *SB;
    int64_t ldsb, stride_sb;
    int c_type;
    void *C;
    int64_t ldc, stride_c;
    Groups groups;
    void *workspace;
    size_t workspace_bytes;
    hipStream_t stream;
};
hipError_t launch_block_gemm(const BlockProblem &p);
// bytes with which the product runs its preferred number of slices, whatever its operands' alignment
size_t block_gemm_workspace(int mode, int groups, int64_t m, int64_t n, int64_t k);

hipError_t launch_expert_sort(int64_t tokens, int fan, int experts, const int32_t *ids, int32_t *offsets, int32_t *position, int32_t *source,
                              void *workspace, hipStream_t stream);
size_t expert_sort_workspace(int64_t tokens, int fan, int experts);
hipError_t launch_expert_gather(int dtype, int64_t tokens, int fan, int64_t cols, const void *X, int64_t ldx, const int32_t *source,
                                const float *weights, void *Y, int64_t ldy, hipStream_t stream);
hipError_t launch_expert_combine(int dtype, int64_t tokens, int fan, int64_t cols, const void *Y, int64_t ldy, const int32_t *position,
                                 const float *weights, void *O, int64_t ldo, hipStream_t stream);
hipError_t launch_expert_combine_grad(int dtype, int64_t tokens, int fan, int64_t cols, const void *dO, int64_t lddo, const void *Y, int64_t ldy,
                                      const int32_t *position, const float *weights, void *dY, int64_t lddy, float *dweights, hipStream_t stream);

#if defined(__HIPCC__)

typedef __bf16 bfloat;

// n elements of T from an address aligned to T only: one vector access, which the memory pipeline splits as needed
template <typename T, int N> struct __attribute__((packed, aligned(sizeof(T)))) Piece {
    T v[N];
};

// N consecutive elements, those from `valid` on zero and not read
template <typename T, int N> __device__ inline void load_piece(const T *p, int valid, float (&out)[N])
{
    if (valid >= N) {
        const Piece<T, N> x = *reinterpret_cast<const Piece<T, N> *>(p);
#pragma unroll
        for (int i = 0; i < N; ++i) out[i] = static_cast<float>(x.v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) out[i] = i < valid ? static_cast<float>(p[i]) : 0.f;
    }
}
template <typename T, int N> __device__ inline void store_piece(T *p, int valid, const float (&in)[N])
{
    if (valid >= N) {
        Piece<T, N> x;
#pragma unroll
        for (int i = 0; i < N; ++i) x.v[i] = static_cast<T>(in[i]);
        *reinterpret_cast<Piece<T, N> *>(p) = x;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < valid) p[i] = static_cast<T>(in[i]);
    }
}

// Largest value over the 16 lanes of a row, in all of them
__device__ inline uint32_t max_over_16_lanes(uint32_t v)
{
    auto step = [&](auto n) {
        const uint32_t o = __builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x120 + decltype(n)::value, 0xf, 0xf, false);      // rotated by n lanes
        v = v > o ? v : o;
    };
    step(std::integral_constant<int, 8>{});
    step(std::integral_constant<int, 4>{});
    step(std::integral_constant<int, 2>{});
    step(std::integral_constant<int, 1>{});
    return v;
}

// Sum over the lanes up to this one: inside rows of 16 lanes by shifts, then each row's total into those behind it
__device__ inline int sum_up_to_lane(int v)
{
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);       // row_shr 1, 2, 4, 8
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);       // lane 15 of a row into the next, rows 1 and 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);       // lane 31 into rows 2 and 3
    return v;
}

// The scale 2^e of a block whose largest magnitude has the bits `largest`: e is the least with largest / 2^e <= 448 = 1.75 * 2^8, -126 at least.
// Adding 0x1fffff to the bits carries into the exponent exactly where the mantissa is above 1.75.
__device__ inline int scale_exponent(uint32_t largest)
{
    if (largest == 0) return 0;
    const int e = static_cast<int>((largest + 0x1fffffu) >> 23) - 127 - 8;
    return e < -126 ? -126 : e;
}
__device__ inline float power_of_two(int e) { return __builtin_bit_cast(float, static_cast<uint32_t>(e + 127) << 23); }

// A tile of up to 2^LOG rows that belong to one expert
struct RowTile {
    int group;
    int64_t first, end;                  // rows first .. end-1 (end: the expert's)
    int64_t start;                       // the expert's first row
};

// 64 experts' tiles, a lane each: rows lo .. hi-1, and the tiles up to this lane's.  Offsets are held to 0 .. rows, whatever the array says.
struct RowTiles {
    int lo, hi, tiles, sum;
};
template <int LOG> __device__ inline RowTiles row_tiles(const Groups &g, int base)
{
    const int rows = static_cast<int>(g.rows), e = base + static_cast<int>(threadIdx.x % 64);
    auto offset = [&](int i) {
        const int o = g.offsets[i < g.count ? i : g.count];
        return o < 0 ? 0 : o > rows ? rows : o;
    };
    RowTiles t{offset(e), offset(e + 1), 0, 0};
    t.tiles = t.hi > t.lo ? (t.hi - t.lo + (1 << LOG) - 1) >> LOG : 0;
    t.sum = sum_up_to_lane(t.tiles);
    return t;
}

// The `tile`-th of all experts' tiles, counted expert by expert; false behind the last one.  Every wavefront finds it by itself: 64 experts
// at a time, a running sum of their tiles over the lanes.
template <int LOG> __device__ inline bool find_row_tile(const Groups &g, int tile, RowTile *found)
{
    int before = 0;
    for (int base = 0; base < g.count; base += 64) {
        const RowTiles t = row_tiles<LOG>(g, base);
        const int total = __builtin_amdgcn_readlane(t.sum, 63);        // (read by lane: the compiler has to know that all lanes go the same way)
        if (tile < before + total) {
            const uint64_t behind = __ballot(before + t.sum > tile);
            const int at = __ffsll(static_cast<unsigned long long>(behind)) - 1;
            const int first_tile = before + __builtin_amdgcn_readlane(t.sum - t.tiles, at);
            found->group = base + at;
            found->start = __builtin_amdgcn_readlane(t.lo, at);
            found->end = __builtin_amdgcn_readlane(t.hi, at);
            found->first = found->start + (static_cast<int64_t>(tile - first_tile) << LOG);
            return true;
        }
        before += total;
    }
    return false;
}

// How many tiles all experts' rows make
template <int LOG> __device__ inline int count_row_tiles(const Groups &g)
{
    int total = 0;
    for (int base = 0; base < g.count; base += 64) total += __builtin_amdgcn_readlane(row_tiles<LOG>(g, base).sum, 63);
    return total;
}

// Column at which an expert's rows start in a transposed matrix: a block boundary, with at least a block's room for rounding up in front of the next
__device__ inline int64_t group_column(int64_t start, int group) { return ((start + SCALE_BLOCK - 1) / SCALE_BLOCK + group) * SCALE_BLOCK; }

__device__ inline int64_t source_row(const Groups &g, int64_t row)
{
    if (g.source == nullptr) return row;
    const int slot = g.source[row];
    return slot < 0 ? 0 : slot < g.rows ? slot / g.fan : 0;
}
#endif

}  // namespace mg
