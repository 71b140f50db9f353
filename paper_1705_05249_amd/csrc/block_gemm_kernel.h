// Products of two 8-bit (e4m3) matrices whose summed index is contiguous in memory, with an FP32 scale for each block of 128 of it:
//
//     C(i, j) = alpha * sum_b sa(i, b) * sb(j, b) * ( sum_{l in block b} A(i, l) B(j, l) ) + beta * C(i, j)
//
// Two ways of summing.  The FP8 pipes: one v_mfma_f32_16x16x128_f8f6f4 sums a whole block; its result is scaled and added in FP32 (scales of any
// value), or the scales go into the instruction as exponents and it adds to the running sum itself (powers of two).  Inside, the instruction
// adds eight products at a time on a grid of 2^-13 of the largest of them (measured: a product 2^-13 of another in its group of eight bytes counts, one
// of 2^-14 does not, towards zero for either sign; groups and the running sum add up in FP32).  That leaves 1.5e-5 of the result for normal data and
// 5e-5 with outliers, for any length: a fiftieth of bfloat16's rounding, a quarter of FP16's.  Terms of one sign lose on one side: 2.5e-6 of the sum of magnitudes
// for |normal| data, 9.5e-6 for a rectifier's squared output, 6e-5 for exp(2 normal).  Fewer bits than FP32 for twice the rate: these pipes serve results of 16 bits, unless
// a call asks for FP32 sums.
// Results in FP32, and calls that ask for it, take the FP16 or bfloat16 pipes: both operands are widened in registers, which is exact, and
// v_mfma_f32_16x16x32 adds on a grid of 2^-24, at half the rate.
//
// The lanes of the instruction's first operand are rows of B, those of the second rows of A: a lane then holds four consecutive
// columns of one row of C, and with square blocks of B (weights) the scale of B is one number for all of a fragment.
#pragma once

#include "block_plan.h"
#include "experts.h"
#include "mfma_kernel.h"

namespace mg {

typedef int intx8 __attribute__((ext_vector_type(8)));
typedef __bf16 bfloatx8 __attribute__((ext_vector_type(8)));

struct BlockArgs {
    const uint8_t *A, *B;
    const float *SA, *SB;
    void *C;
    float *partial;                   // slices' sums [slice][row of C][n] (BLOCK_SUM: row = group * m + i), or null
    int64_t lda, ldb, ldsa, ldsb, ldc, stride_b, stride_sb, stride_c;
    Groups groups;
    int m, n, k;
    int a_shift, b_shift;             // 7 where a scale belongs to 128 rows
    int c_type;
    float alpha, beta;
    int tiles_m, tiles_n;             // BLOCK_ROWS: tiles_m counts the tiles there can be at most
    int slices;                       // of the summed index
    int each_own_c;                   // BLOCK_SUM: every group has a C
    int64_t partial_rows;             // rows of C in a slice's sums
};

// What a work-group computes: rows m0 .. m_end-1 of A, from n0 on of B, blocks b0 .. b_end-1 of the sum
struct BlockTile {
    int group;
    int64_t m0, m_end;
    int64_t n0;
    int64_t column;                   // of A and B in memory where the sum starts (a block boundary)
    int k;                            // length of the whole sum
    int b0, b_end;
};

// This work-group's tile; false: nothing to do.  The walk of tile_coords: a die takes neighbouring tiles.
template <int MODE, int LOG_BM, int BN> __device__ inline bool block_tile(const BlockArgs &args, BlockTile *t)
{
    constexpr int BM = 1 << LOG_BM;
    int tm, tn, tiles_m = args.tiles_m;
    if constexpr (MODE == BLOCK_ROWS) {
        // The walk goes over the tiles there are: over all there could be, some dies would have few (64 experts, 16384 rows, 2048 x 2048: 159 -> 140 us)
        const int there = count_row_tiles<LOG_BM>(args.groups);
        tiles_m = there < tiles_m ? there : tiles_m;
        if (static_cast<int>(blockIdx.x) >= tiles_m * args.tiles_n) return false;
    }
    tile_coords(blockIdx.x, tiles_m, args.tiles_n, 8, tm, tn);
    t->group = 0;
    t->column = 0;
    t->k = args.k;
    t->m0 = static_cast<int64_t>(tm) * BM;
    t->m_end = args.m;
    if constexpr (MODE == BLOCK_ROWS) {
        RowTile r;
        if (!find_row_tile<LOG_BM>(args.groups, tm, &r)) return false;
        t->group = __builtin_amdgcn_readfirstlane(r.group);
        t->m0 = __builtin_amdgcn_readfirstlane(static_cast<int>(r.first));
        t->m_end = __builtin_amdgcn_readfirstlane(static_cast<int>(r.end));
    }
    if constexpr (MODE == BLOCK_SUM) {
        // With C in 16 bits every die (work-groups go round the eight of them) starts with another expert, so that not all of them write C at the same time: 16 experts of
        // 1024 rows, 4096 x 2048, 215 -> 190 us on the FP8 pipes; with FP32 sums the same, and 332 -> 324 where the experts' rows differ (61 to 2879).  C in FP32 keeps
        // the order: no difference, or 5 % slower where experts differ.
        t->group = args.c_type == MG_F32 ? blockIdx.z : (blockIdx.z + blockIdx.x % 8 * args.groups.count / 8) % args.groups.count;
        const int rows = static_cast<int>(args.groups.rows);
        int lo = args.groups.offsets[t->group], hi = args.groups.offsets[t->group + 1];
        lo = lo < 0 ? 0 : lo > rows ? rows : lo;
        hi = hi < lo ? lo : hi > rows ? rows : hi;
        t->k = args.k == 0 ? 0 : hi - lo;
        t->column = group_column(lo, t->group);
    }
    t->n0 = static_cast<int64_t>(tn) * BN;
    const int blocks = (t->k + SCALE_BLOCK - 1) / SCALE_BLOCK;
    const int each = (blocks + args.slices - 1) / args.slices;
    t->b0 = blockIdx.y * each < blocks ? blockIdx.y * each : blocks;
    t->b_end = t->b0 + each < blocks ? t->b0 + each : blocks;
    return true;
}

hipError_t launch_block_dma_dense(const BlockArgs &args, int sums, int tile, hipStream_t stream);
hipError_t launch_block_dma_rows(const BlockArgs &args, int sums, int tile, hipStream_t stream);
hipError_t launch_block_dma_sum(const BlockArgs &args, int sums, int tile, hipStream_t stream);
// Few rows of A (few_b: of B), 16 * fragments for a work-group: BLOCK_DENSE or (of A) BLOCK_ROWS (block_few.hip)
hipError_t launch_block_few(const BlockArgs &args, int mode, bool few_b, int fragments, bool fp32, hipStream_t stream);

// The scale of a power of two as the matrix instruction takes it: the exponent's eight bits
__device__ inline int scale_bits(float s) { return static_cast<int>(__builtin_bit_cast(uint32_t, s) >> 23); }

// An operand's fragment of a block (16 rows x 128: 32 bytes for each lane), ready for the pipes
struct Fp8Fragment {
    intx8 v;
    __device__ inline void set(const intx8 &x) { v = x; }
};
struct Fp16Fragment {
    halfx8 v[4];
    __device__ inline void set(const intx8 &x)
    {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            using Pair = decltype(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(0, 1.f, false));
            const Pair two[4] = {__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x[2 * q], 1.f, false), __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x[2 * q], 1.f, true),
                                 __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x[2 * q + 1], 1.f, false),
                                 __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x[2 * q + 1], 1.f, true)};
            __builtin_memcpy(&v[q], two, 16);
        }
    }
};
// scaled: the lane's row of the operand has the scale `s`, a power of two
struct Bf16Fragment {
    bfloatx8 v[4];
    template <int Q> __device__ inline void quarter(uint32_t lo, uint32_t hi, float s)
    {
        using Pair = decltype(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(0, 1.f, false));
        const Pair two[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, true),
                             __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, true)};
        __builtin_memcpy(&v[Q], two, 16);
    }
    template <int Q> __device__ inline void quarter(const u32x4 (&x)[2], float s) { quarter<Q>(x[Q / 2][Q % 2 * 2], x[Q / 2][Q % 2 * 2 + 1], s); }
    __device__ inline void set(const u32x4 (&x)[2], float s)
    {
        quarter<0>(x, s);
        quarter<1>(x, s);
        quarter<2>(x, s);
        quarter<3>(x, s);
    }
};
template <int SUMS> struct FragmentOf { using type = Fp8Fragment; };
template <> struct FragmentOf<SUMS_FP32> { using type = Fp16Fragment; };
template <> struct FragmentOf<SUMS_FP32_POW2> { using type = Bf16Fragment; };

// acc += the block's sum times its scales; sb: the scales of the lane's four rows of B
__device__ inline floatx4 block_sum(const Fp8Fragment &b, const Fp8Fragment &a)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b.v, a.v, floatx4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
}
__device__ inline floatx4 block_sum(const Fp16Fragment &b, const Fp16Fragment &a)
{
    floatx4 d{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int q = 0; q < 4; ++q) d = __builtin_amdgcn_mfma_f32_16x16x32_f16(b.v[q], a.v[q], d, 0, 0, 0);
    return d;
}
template <typename F> __device__ inline void add_block(floatx4 &acc, const F &b, const F &a, const floatx4 &sb, float sa)
{
    const floatx4 d = block_sum(b, a);
#pragma unroll
    for (int r = 0; r < 4; ++r) acc[r] = __builtin_fmaf(d[r], sb[r] * sa, acc[r]);
}
// acc += d times the scales, s alone or with the four rows' of B
template <bool ALONE> __device__ inline void scale_add(floatx4 &acc, const floatx4 &d, float s, std::integral_constant<bool, ALONE>, const u32x4 &sb)
{
#pragma unroll
    for (int r = 0; r < 4; ++r) acc[r] = __builtin_fmaf(d[r], ALONE ? s : s * __builtin_bit_cast(floatx4, sb)[r], acc[r]);
}
// the same with exponents, of the lane's row of either operand
__device__ inline void add_block_pow2(floatx4 &acc, const Fp8Fragment &b, const Fp8Fragment &a, int sb, int sa)
{
    acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b.v, a.v, acc, 0, 0, 0, sb, 0, sa);
}

__device__ inline intx8 join(const u32x4 &lo, const u32x4 &hi)
{
    return intx8{static_cast<int>(lo[0]), static_cast<int>(lo[1]), static_cast<int>(lo[2]), static_cast<int>(lo[3]),
                 static_cast<int>(hi[0]), static_cast<int>(hi[1]), static_cast<int>(hi[2]), static_cast<int>(hi[3])};
}

// Four consecutive columns of a row of C, the first `valid` of them
template <typename T> __device__ inline void write_c(T *c, int valid, floatx4 acc, float alpha, float beta)
{
    float v[4], old[4] = {0.f, 0.f, 0.f, 0.f};
    if (beta != 0.f) load_piece<T, 4>(c, valid, old);
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = beta != 0.f ? __builtin_fmaf(beta, old[r], alpha * acc[r]) : alpha * acc[r];
    store_piece<T, 4>(c, valid, v);
}
__device__ inline void write_block(const BlockArgs &args, int group, int64_t row, int64_t col, const floatx4 &acc)
{
    const int valid = static_cast<int>(args.n - col < 4 ? args.n - col : 4);
    if (valid <= 0) return;
    if (args.partial != nullptr) {
        const int64_t at = static_cast<int64_t>(blockIdx.y) * args.partial_rows + (args.each_own_c ? group * static_cast<int64_t>(args.m) : 0) + row;
        const float v[4] = {acc[0], acc[1], acc[2], acc[3]};
        store_piece<float, 4>(args.partial + at * args.n + col, valid, v);
        return;
    }
    const int64_t at = group * args.stride_c + row * args.ldc + col;
    if (args.c_type == MG_F32) write_c(static_cast<float *>(args.C) + at, valid, acc, args.alpha, args.beta);
    else if (args.c_type == MG_F16) write_c(static_cast<_Float16 *>(args.C) + at, valid, acc, args.alpha, args.beta);
    else write_c(static_cast<bfloat *>(args.C) + at, valid, acc, args.alpha, args.beta);
}

// A wavefront's FM x FN fragments to C by way of LDS: as the matrix instructions leave them, a store would reach 32 bytes of 16 rows; from LDS
// every row's WIDTH columns leave together.  16-bit results that need no old C are rounded on the way in, others stay FP32 until they leave.  With 16
// bytes between the rows in LDS no bank is asked twice, in either direction.  `region` is the wavefront's own.  4096 x 4096 in bfloat16 behind
// one K-tile: 29 us stored straight from registers, 18 with FP32 in LDS and every store checked for the ends of C, 11.6 as it is (32 MB alone: 6.9).
template <typename T, bool OLD, int FN> struct StoreRegion {
    using Held = std::conditional_t<sizeof(T) == 2 && !OLD, T, float>;
    static constexpr int WIDTH = FN * 16, PITCH = WIDTH * static_cast<int>(sizeof(Held)) + 16;
    static constexpr int FRAGMENTS = 9216 / (16 * PITCH) >= 4 ? 4 : 9216 / (16 * PITCH) >= 2 ? 2 : 1;        // at a time
};
constexpr int STORE_REGION = 9216;
template <typename T, bool OLD, bool WHOLE, int FM, int FN>
__device__ __forceinline__ void store_fragments(T *c, int64_t ld, const floatx4 (&acc)[FN][FM], char *region, int64_t rows, int64_t cols, float alpha, float beta, int lane)
{
    using R = StoreRegion<T, OLD, FN>;
    using Held = typename R::Held;
    constexpr int STEP = R::FRAGMENTS < FM ? R::FRAGMENTS : FM, ROWS = STEP * 16, N = 16 / sizeof(T), ACROSS = R::WIDTH / N, DOWN = 64 / ACROSS;
    static_assert(FM % STEP == 0 && ROWS % DOWN == 0 && ROWS * R::PITCH <= STORE_REGION, "whole passes");
    const int col = lane % ACROSS * N;
    const int valid = WHOLE ? N : static_cast<int>(cols - col < N ? cols - col : N);
    T *at = c + lane / ACROSS * ld + col;
    const int64_t step = DOWN * ld;
#pragma unroll
    for (int i0 = 0; i0 < FM; i0 += STEP) {
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < STEP; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                Piece<Held, 4> x;
#pragma unroll
                for (int r = 0; r < 4; ++r) x.v[r] = static_cast<Held>(alpha * acc[j][i0 + i][r]);
                __builtin_memcpy(__builtin_assume_aligned(region + (i * 16 + lane % 16) * R::PITCH + (j * 16 + lane / 16 * 4) * sizeof(Held), 4 * sizeof(Held)), &x, sizeof(x));
            }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int r0 = 0; r0 < ROWS; r0 += DOWN, at += step) {
            const int row = r0 + lane / ACROSS;
            if (!WHOLE && (valid <= 0 || i0 * 16 + row >= rows)) continue;
            Piece<Held, N> x;
            __builtin_memcpy(&x, __builtin_assume_aligned(region + row * R::PITCH + col * sizeof(Held), 16), sizeof(x));
            if constexpr (sizeof(T) == sizeof(Held) && !OLD) {
                if (WHOLE || valid >= N) {
                    *reinterpret_cast<Piece<Held, N> *>(at) = x;
                } else {
#pragma unroll
                    for (int q = 0; q < N; ++q)
                        if (q < valid) at[q] = x.v[q];
                }
            } else {
                float v[N], old[N];
                load_piece<T, N>(at, valid, old);
#pragma unroll
                for (int q = 0; q < N; ++q) v[q] = __builtin_fmaf(beta, old[q], x.v[q]);
                store_piece<T, N>(at, valid, v);
            }
        }
    }
}
template <typename T, int FM, int FN>
__device__ __forceinline__ void store_as(T *c, int64_t ld, const floatx4 (&acc)[FN][FM], char *region, int64_t rows, int64_t cols, float alpha, float beta, int lane)
{
    if (beta != 0.f) store_fragments<T, true, false>(c, ld, acc, region, rows, cols, alpha, beta, lane);
    else if (rows >= FM * 16 && cols >= FN * 16) store_fragments<T, false, true>(c, ld, acc, region, rows, cols, alpha, beta, lane);
    else store_fragments<T, false, false>(c, ld, acc, region, rows, cols, alpha, beta, lane);
}
template <int FM, int FN>
__device__ __forceinline__ void store_tile(const BlockArgs &args, const BlockTile &tile, const floatx4 (&acc)[FN][FM], char *region, int64_t row0, int64_t col0, int lane)
{
    const int64_t rows = tile.m_end - row0, cols = args.n - col0;
    if (rows <= 0 || cols <= 0) return;
    if (args.partial != nullptr) {
        const int64_t first = static_cast<int64_t>(blockIdx.y) * args.partial_rows + (args.each_own_c ? tile.group * static_cast<int64_t>(args.m) : 0) + row0;
        store_as(args.partial + first * args.n + col0, args.n, acc, region, rows, cols, 1.f, 0.f, lane);
        return;
    }
    const int64_t at = tile.group * args.stride_c + row0 * args.ldc + col0;
    if (args.c_type == MG_F32) store_as(static_cast<float *>(args.C) + at, args.ldc, acc, region, rows, cols, args.alpha, args.beta, lane);
    else if (args.c_type == MG_F16) store_as(static_cast<_Float16 *>(args.C) + at, args.ldc, acc, region, rows, cols, args.alpha, args.beta, lane);
    else store_as(static_cast<bfloat *>(args.C) + at, args.ldc, acc, region, rows, cols, args.alpha, args.beta, lane);
}

// The first `valid` of 16 bytes, zeros behind them
__device__ inline u32x4 first_bytes(u32x4 x, int valid)
{
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        const int bits = (valid - 4 * d) * 8;                    // of this word, from its low end
        x[d] &= bits <= 0 ? 0u : bits >= 32 ? ~0u : (1u << bits) - 1;
    }
    return x;
}
// 16 bytes of a row at any address, those from `valid` on zero.  A row's last piece is read word by word, each word on four bytes and with a byte of the row in it.
__device__ inline u32x4 load_bytes16(const uint8_t *p, int valid)
{
    if (valid >= 16) return __builtin_bit_cast(u32x4, *reinterpret_cast<const Piece<uint8_t, 16> *>(p));
    if (valid <= 0) return u32x4{0u, 0u, 0u, 0u};
    const int skew = static_cast<int>(reinterpret_cast<uintptr_t>(p) & 3);
    const uint32_t *words = reinterpret_cast<const uint32_t *>(p - skew);
    uint32_t w[5];
#pragma unroll
    for (int d = 0; d < 5; ++d) w[d] = 4 * d < skew + valid ? words[d] : 0u;
    u32x4 r;
#pragma unroll
    for (int d = 0; d < 4; ++d) r[d] = __builtin_amdgcn_alignbyte(w[d + 1], w[d], skew);
    return first_bytes(r, valid);
}
// The same from an address on 16 bytes, where a piece with a byte of the row in it may be read whole
__device__ inline u32x4 load_aligned16(const uint8_t *p, int valid)
{
    if (valid <= 0) return u32x4{0u, 0u, 0u, 0u};
    return first_bytes(*reinterpret_cast<const u32x4 *>(p), valid);
}

}  // namespace mg
