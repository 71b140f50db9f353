// Quantising to e4m3 with a power-of-two scale for each block of 128 elements of a row, or of 128 x 128.
//
//     e = max(-126, least integer with max|x| / 2^e <= 448)      q = round_to_nearest_even_e4m3(x / 2^e)
//
// A power of two because the division is then exact: one rounding, no bit of the 8-bit mantissa's precision lost to the scale (e4m3
// numbers have the same relative precision in every binade; what a scale off by less than two costs is less than one binade at the bottom
// of the range), and the products can hand the scale to the matrix instructions as an exponent.
//
// Bound by memory: z bytes read, one or two written per element (8192 x 4096 of bfloat16 in both orders 33.7 us, 4.0 TB/s, 24.6 with the input in the last-level
// cache; 16 weights of 4096 x 2048 in both orders 108, 5.0 TB/s; 64 x 1024 3.0, a launch and a round trip).
#include "internal.h"
#include "experts.h"

namespace mg {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// Pairs of 16-bit elements are looked at and converted as pairs: three vector instructions for an element and both of its results (as single FP32
// numbers fifteen, which took as long as the memory).
template <typename T> struct Pairs {                    // 16-bit types: eight elements are four words of two
    static constexpr int WORDS = 4;
    static constexpr uint32_t SIGNLESS = 0x7fff7fffu;
    static constexpr uint32_t INFINITE = std::is_same_v<T, bfloat> ? 0x7f80u : 0x7c00u;
};
template <> struct Pairs<float> {
    static constexpr int WORDS = 8;
    static constexpr uint32_t SIGNLESS = 0x7fffffffu;
    static constexpr uint32_t INFINITE = 0x7f800000u;
};

// Eight consecutive elements as they are in memory, those from `valid` on zero and not read
template <typename T> __device__ inline void load_words(const T *p, int valid, uint32_t (&x)[Pairs<T>::WORDS])
{
    Piece<T, 8> v;
    if (valid >= 8) {
        v = *reinterpret_cast<const Piece<T, 8> *>(p);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v.v[i] = i < valid ? p[i] : static_cast<T>(0.f);
    }
    __builtin_memcpy(x, &v, sizeof(v));
}
// The larger of two words of magnitudes, element by element
template <typename T> __device__ inline uint32_t larger(uint32_t a, uint32_t b)
{
    if constexpr (sizeof(T) == 4) return a > b ? a : b;
    else return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
// The largest magnitude of a word, as bits of T
template <typename T> __device__ inline uint32_t largest_of(uint32_t word)
{
    if constexpr (sizeof(T) == 4) return word;
    const uint32_t lo = word & 0xffffu, hi = word >> 16;
    return lo > hi ? lo : hi;
}
// Magnitudes with infinities and NaN left out
template <typename T> __device__ inline uint32_t finite_only(uint32_t word)
{
    word &= Pairs<T>::SIGNLESS;
    if constexpr (sizeof(T) == 4) return word < Pairs<T>::INFINITE ? word : 0u;
    const uint32_t lo = word & 0xffffu, hi = word >> 16;
    return (lo < Pairs<T>::INFINITE ? lo : 0u) | (hi < Pairs<T>::INFINITE ? hi << 16 : 0u);
}
// Bits of a magnitude of T -> bits of the same number in FP32
template <typename T> __device__ inline uint32_t as_fp32(uint32_t bits)
{
    if constexpr (sizeof(T) == 4) return bits;
    else if constexpr (std::is_same_v<T, bfloat>) return bits << 16;
    else return __builtin_bit_cast(uint32_t, static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(bits))));
}
// Four elements, divided by the scale, to four e4m3 numbers
template <typename T> __device__ inline uint32_t four_quantized(uint32_t a, uint32_t b, float scale)
{
    s16x2 q{0, 0};
    if constexpr (std::is_same_v<T, bfloat>) {
        q = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(q, __builtin_bit_cast(bf16x2, a), scale, false);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(q, __builtin_bit_cast(bf16x2, b), scale, true);
    } else {
        q = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(q, __builtin_bit_cast(f16x2, a), scale, false);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(q, __builtin_bit_cast(f16x2, b), scale, true);
    }
    return __builtin_bit_cast(uint32_t, q);
}
__device__ inline uint32_t four_quantized(uint32_t a, uint32_t b, uint32_t c, uint32_t d, float scale)
{
    s16x2 q{0, 0};
    q = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(q, __builtin_bit_cast(float, a), __builtin_bit_cast(float, b), scale, false);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(q, __builtin_bit_cast(float, c), __builtin_bit_cast(float, d), scale, true);
    return __builtin_bit_cast(uint32_t, q);
}
template <typename T> __device__ inline u32x2 eight_quantized(const uint32_t (&x)[Pairs<T>::WORDS], float scale)
{
    if constexpr (sizeof(T) == 4) return u32x2{four_quantized(x[0], x[1], x[2], x[3], scale), four_quantized(x[4], x[5], x[6], x[7], scale)};
    else return u32x2{four_quantized<T>(x[0], x[1], scale), four_quantized<T>(x[2], x[3], scale)};
}

template <int N> __device__ inline void store_bytes(uint8_t *p, int valid, const uint32_t (&x)[N / 4])
{
    if (valid >= N) {
        Piece<uint8_t, N> v;
        __builtin_memcpy(&v, x, N);
        *reinterpret_cast<Piece<uint8_t, N> *>(p) = v;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < valid) p[i] = static_cast<uint8_t>(x[i / 4] >> (8 * (i % 4)));
    }
}

// ---- row blocks, not transposed: 16 lanes hold a block, 8 elements each; a thread takes U blocks, 16 apart, for U loads in flight
template <typename T, int U> __global__ __launch_bounds__(256) void quantize_rows_kernel(const QuantizeProblem p, int64_t blocks_per_row, int64_t blocks)
{
    constexpr int WORDS = Pairs<T>::WORDS;
    const int part = threadIdx.x % 16;
    const int64_t batch = blockIdx.y;
    const int64_t rows = p.groups.offsets != nullptr ? p.groups.offsets[p.groups.count] : p.rows;
    uint32_t x[U][WORDS];
    int64_t row[U], at[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t block = (static_cast<int64_t>(blockIdx.x) * U + u) * 16 + threadIdx.x / 16;
        row[u] = block / blocks_per_row;
        at[u] = block % blocks_per_row;
        const int64_t col = at[u] * SCALE_BLOCK + part * 8;
        const bool here = block < blocks && row[u] < rows;
        const int valid = !here ? 0 : static_cast<int>(p.cols - col < 8 ? p.cols - col : 8);
        if (!here) row[u] = -1;
        load_words<T>(static_cast<const T *>(p.X) + batch * p.stride_x + (here ? source_row(p.groups, row[u]) * p.ldx : 0) + (here ? col : 0), valid, x[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        uint32_t most = 0;
#pragma unroll
        for (int w = 0; w < WORDS; ++w) most = larger<T>(most, x[u][w] & Pairs<T>::SIGNLESS);
        if (largest_of<T>(most) >= Pairs<T>::INFINITE) {
            most = 0;
#pragma unroll
            for (int w = 0; w < WORDS; ++w) most = larger<T>(most, finite_only<T>(x[u][w]));
        }
        const float scale = power_of_two(scale_exponent(as_fp32<T>(max_over_16_lanes(largest_of<T>(most)))));
        if (row[u] < 0) continue;
        const u32x2 q = eight_quantized<T>(x[u], scale);
        const int64_t col = at[u] * SCALE_BLOCK + part * 8;
        store_bytes<8>(p.Q + batch * p.stride_q + row[u] * p.ldq + col, static_cast<int>(p.cols - col < 8 ? p.cols - col : 8), {q[0], q[1]});
        if (part == 0) p.S[batch * p.stride_s + row[u] * p.lds + at[u]] = scale;
    }
}

// ---- 128 x 128 tiles: square blocks, transposed results.  A thread holds 8 rows x 8 columns in registers, so X is read once for both results;
// eight rows of a column are eight consecutive bytes of the transposed tile, which goes through LDS to leave in whole rows of 128 bytes.
// 8-byte slot s of line c sits at slot s ^ (c / 8 % 16): the 16 threads that write the same rows of 16 different lines hit different banks.
template <typename T> __global__ __launch_bounds__(256) void quantize_tiles_kernel(const QuantizeProblem p, uint32_t across)
{
    constexpr int WORDS = Pairs<T>::WORDS, COLUMNS = 8 / WORDS;                          // words of eight elements, elements of a word
    __shared__ uint32_t most_of[4][128 / COLUMNS];
    __shared__ __attribute__((aligned(16))) uint8_t turned[128 * 128];
    const int t = threadIdx.x, wave = t / 64, part = t % 16, rows8 = t / 16;            // rows 8 * rows8 .., columns 8 * part ..
    const uint32_t down = blockIdx.x / across, over = blockIdx.x % across;              // the tile's place
    const int64_t c0 = static_cast<int64_t>(over) * 128, batch = blockIdx.y;
    RowTile tile{0, static_cast<int64_t>(down) * 128, p.rows, 0};
    int64_t turned0 = tile.first;                                                        // the tile's first column of the transposed result
    if (p.groups.offsets != nullptr) {
        if (!find_row_tile<7>(p.groups, static_cast<int>(down), &tile)) return;
        turned0 = group_column(tile.start, tile.group) + (tile.first - tile.start);
    }
    const int rows_here = static_cast<int>(tile.end - tile.first < 128 ? tile.end - tile.first : 128);
    const int cols_here = static_cast<int>(p.cols - c0 < 128 ? p.cols - c0 : 128);
    const int valid = cols_here - 8 * part;                                              // of this thread's 8 columns
    const T *X = static_cast<const T *>(p.X) + batch * p.stride_x + c0;

    uint32_t v[8][WORDS];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = 8 * rows8 + i;
        const bool here = r < rows_here && valid > 0;
        const int64_t from = here ? source_row(p.groups, tile.first + r) : 0;
        load_words<T>(X + from * p.ldx + (here ? 8 * part : 0), here ? valid : 0, v[i]);
    }
    uint32_t row_most[8], col_most[WORDS];
    auto look = [&](auto &&magnitude) {
#pragma unroll
        for (int w = 0; w < WORDS; ++w) col_most[w] = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            row_most[i] = 0;
#pragma unroll
            for (int w = 0; w < WORDS; ++w) {
                const uint32_t u = magnitude(v[i][w]);
                row_most[i] = larger<T>(row_most[i], u);
                col_most[w] = larger<T>(col_most[w], u);
            }
        }
        uint32_t most = 0;
#pragma unroll
        for (int w = 0; w < WORDS; ++w) most = larger<T>(most, col_most[w]);
        return largest_of<T>(most);
    };
    uint32_t most = look([](uint32_t x) { return x & Pairs<T>::SIGNLESS; });
    if (most >= Pairs<T>::INFINITE) most = look([](uint32_t x) { return finite_only<T>(x); });

    float square = 1.f;                                                                  // square blocks: the tile's scale
    if (p.square) {
        most = max_over_16_lanes(most);
        for (int d = 16; d < 64; d <<= 1) {
            const uint32_t o = __shfl_xor(most, d);
            most = most > o ? most : o;
        }
        if (t % 64 == 0) most_of[wave][0] = most;
        __syncthreads();
        for (int w = 0; w < 4; ++w) most = most > most_of[w][0] ? most : most_of[w][0];
        square = power_of_two(scale_exponent(as_fp32<T>(most)));
    } else if (p.T != nullptr) {
#pragma unroll
        for (int w = 0; w < WORDS; ++w) {
            for (int d = 16; d < 64; d <<= 1) col_most[w] = larger<T>(col_most[w], __shfl_xor(col_most[w], d));
            if (t % 64 < 16) most_of[wave][WORDS * part + w] = col_most[w];
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WORDS; ++w)
            for (int o = 0; o < 4; ++o) col_most[w] = larger<T>(col_most[w], most_of[o][WORDS * part + w]);
    }
    if (p.Q != nullptr) {
        uint8_t *to = p.Q + batch * p.stride_q + (tile.first + 8 * rows8) * p.ldq + c0 + 8 * part;
#pragma unroll
        for (int i = 0; i < 8; ++i, to += p.ldq) {
            const int r = 8 * rows8 + i;
            const float scale = p.square ? square : power_of_two(scale_exponent(as_fp32<T>(max_over_16_lanes(largest_of<T>(row_most[i])))));
            const u32x2 q = eight_quantized<T>(v[i], scale);
            if (r < rows_here) {
                store_bytes<8>(to, valid, {q[0], q[1]});
                if (!p.square && part == 0) p.S[batch * p.stride_s + (tile.first + r) * p.lds + over] = scale;
            }
        }
        if (p.square && t == 0) p.S[batch * p.stride_s + static_cast<int64_t>(down) * p.lds + over] = square;
    }
    if (p.T == nullptr) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int w = j / COLUMNS, line = 8 * part + j;
        const uint32_t of_column = sizeof(T) == 4 ? col_most[w] : j % 2 ? col_most[w] >> 16 : col_most[w] & 0xffffu;
        const float scale = p.square ? square : power_of_two(scale_exponent(as_fp32<T>(of_column)));
        u32x2 q;
        if constexpr (sizeof(T) == 4) {
            q = u32x2{four_quantized(v[0][j], v[1][j], v[2][j], v[3][j], scale), four_quantized(v[4][j], v[5][j], v[6][j], v[7][j], scale)};
        } else {
            const uint32_t halves = j % 2 ? 0x07060302u : 0x05040100u;                   // the column's element of two rows
            uint32_t two[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) two[i] = __builtin_amdgcn_perm(v[2 * i + 1][w], v[2 * i][w], halves);
            q = u32x2{four_quantized<T>(two[0], two[1], scale), four_quantized<T>(two[2], two[3], scale)};
        }
        *reinterpret_cast<u32x2 *>(turned + line * 128 + ((rows8 ^ part) << 3)) = q;
        if (!p.square && rows8 == 0 && line < cols_here) p.ST[batch * p.stride_st + (c0 + line) * p.ldst + turned0 / SCALE_BLOCK] = scale;
    }
    if (p.square && t == 0) p.ST[batch * p.stride_st + static_cast<int64_t>(over) * p.ldst + down] = square;
    __syncthreads();
    // whole lines: 8 lanes write the 128 bytes of one; of an expert's last block the bytes behind its rows too (zeros)
    const int wide = p.groups.offsets != nullptr ? 128 : rows_here;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int line = t / 8 + 32 * i, piece = t % 8;
        auto slot = [&](int s) { return *reinterpret_cast<const u32x2 *>(turned + line * 128 + ((s ^ ((line >> 3) & 15)) << 3)); };
        const u32x2 lo = slot(2 * piece), hi = slot(2 * piece + 1);
        if (line < cols_here) store_bytes<16>(p.T + batch * p.stride_t + (c0 + line) * p.ldt + turned0 + 16 * piece, wide - 16 * piece, {lo[0], lo[1], hi[0], hi[1]});
    }
}

template <typename T> hipError_t launch_as(const QuantizeProblem &p)
{
    const int64_t across = ceil_div(p.cols, SCALE_BLOCK);
    if (!p.square && p.T == nullptr) {
        const int64_t blocks = p.rows * across;
        // four blocks a thread where that still leaves eight work-groups for each compute unit
        if (blocks * p.batch >= 16 * 4 * 2048)
            quantize_rows_kernel<T, 4><<<dim3(static_cast<uint32_t>(ceil_div(blocks, 64)), static_cast<uint32_t>(p.batch)), 256, 0, p.stream>>>(p, across, blocks);
        else
            quantize_rows_kernel<T, 1><<<dim3(static_cast<uint32_t>(ceil_div(blocks, 16)), static_cast<uint32_t>(p.batch)), 256, 0, p.stream>>>(p, across, blocks);
    } else {
        const int64_t down = ceil_div(p.rows, SCALE_BLOCK) + (p.groups.offsets != nullptr ? p.groups.count : 0);
        quantize_tiles_kernel<T><<<dim3(static_cast<uint32_t>(across * down), static_cast<uint32_t>(p.batch)), 256, 0, p.stream>>>(p, static_cast<uint32_t>(across));
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize(const QuantizeProblem &p)
{
    if (p.dtype == MG_F32) return launch_as<float>(p);
    if (p.dtype == MG_F16) return launch_as<_Float16>(p);
    return launch_as<bfloat>(p);
}

}  // namespace mg
