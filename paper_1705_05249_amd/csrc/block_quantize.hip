// Quantising to e4m3 with a power-of-two scale for each block of 128 elements of a row, or of 128 x 128.
//
//     e = max(-126, least integer with max|x| / 2^e <= 448)      q = round_to_nearest_even_e4m3(x / 2^e)
//
// A power of two because the division is then exact: one rounding, no bit of the 8-bit mantissa's precision lost to the scale (e4m3
// numbers have the same relative precision in every binade; what a scale off by less than two costs is less than one binade at the bottom
// of the range), and the products can hand the scale to the matrix instructions as an exponent.
//
// Bound by memory: z bytes read, one or two written per element.
#include "internal.h"
#include "experts.h"

namespace mg {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ inline void store_bytes8(uint8_t *p, int valid, uint32_t lo, uint32_t hi)
{
    if (valid >= 8) {
        Piece<uint8_t, 8> x;
        __builtin_memcpy(x.v, &lo, 4);
        __builtin_memcpy(x.v + 4, &hi, 4);
        *reinterpret_cast<Piece<uint8_t, 8> *>(p) = x;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < valid) p[i] = static_cast<uint8_t>((i < 4 ? lo >> (8 * i) : hi >> (8 * i - 32)));
    }
}

// ---- row blocks, not transposed: 16 lanes hold a block, 8 elements each
template <typename T> __global__ __launch_bounds__(256) void quantize_rows_kernel(const QuantizeProblem p, int64_t blocks_per_row, int64_t blocks)
{
    const int64_t block = static_cast<int64_t>(blockIdx.x) * 16 + threadIdx.x / 16;
    const int part = threadIdx.x % 16;
    if (block >= blocks) return;                                  // (whole groups of 16 lanes)
    const int64_t batch = blockIdx.y;
    const int64_t row = block / blocks_per_row, at = block % blocks_per_row;
    if (p.groups.offsets != nullptr && row >= p.groups.offsets[p.groups.count]) return;
    const int64_t col = at * SCALE_BLOCK + part * 8;
    const int valid = static_cast<int>(p.cols - col < 8 ? p.cols - col : 8);
    const T *x = static_cast<const T *>(p.X) + batch * p.stride_x + source_row(p.groups, row) * p.ldx + col;
    float v[8];
    load_piece<T, 8>(x, valid, v);
    uint32_t largest = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t u = finite_magnitude(v[i]);
        largest = largest > u ? largest : u;
    }
    const int e = scale_exponent(max_over_16_lanes(largest));
    const float inverse = power_of_two(-e);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = scaled_or_nan(v[i], inverse);
    store_bytes8(p.Q + batch * p.stride_q + row * p.ldq + col, valid, four_e4m3(v[0], v[1], v[2], v[3]), four_e4m3(v[4], v[5], v[6], v[7]));
    if (part == 0) p.S[batch * p.stride_s + row * p.lds + at] = power_of_two(e);
}

// ---- 128 x 128 tiles: square blocks, transposed results.  A thread holds 8 rows x 8 columns in registers, so X is read once for both results;
// eight rows of a column are eight consecutive bytes of the transposed tile, which goes through LDS to leave in whole rows of 128 bytes.
// 8-byte slot s of line c sits at slot s ^ (c / 8 % 16): the 16 threads that write the same rows of 16 different lines hit different banks.
template <typename T> __global__ __launch_bounds__(256) void quantize_tiles_kernel(const QuantizeProblem p, uint32_t across)
{
    __shared__ uint32_t column_max[4][128];
    __shared__ __attribute__((aligned(16))) uint8_t turned[128 * 128];
    const int t = threadIdx.x, wave = t / 64, part = t % 16, rows8 = t / 16;            // rows 8 * rows8 .., columns 8 * part ..
    const uint32_t down = blockIdx.x / across, over = blockIdx.x % across;                // the tile's place
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
    const T *X = static_cast<const T *>(p.X) + batch * p.stride_x + c0 + 8 * part;

    float v[8][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = 8 * rows8 + i;
        const bool here = r < rows_here;
        const int64_t from = here ? source_row(p.groups, tile.first + r) : 0;
        load_piece<T, 8>(X + from * p.ldx, here ? valid : 0, v[i]);
    }
    uint32_t row_max[8], col_max[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) row_max[i] = col_max[i] = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t u = finite_magnitude(v[i][j]);
            row_max[i] = row_max[i] > u ? row_max[i] : u;
            col_max[j] = col_max[j] > u ? col_max[j] : u;
        }
    int square = 0;                                                                      // square blocks: the tile's exponent
    if (p.square) {
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) most = most > row_max[i] ? most : row_max[i];
        most = max_over_16_lanes(most);
        for (int d = 16; d < 64; d <<= 1) {
            const uint32_t o = __shfl_xor(most, d);
            most = most > o ? most : o;
        }
        if (t % 64 == 0) column_max[wave][0] = most;
        __syncthreads();
        for (int w = 0; w < 4; ++w) most = most > column_max[w][0] ? most : column_max[w][0];
        square = scale_exponent(most);
    } else if (p.T != nullptr) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            for (int d = 16; d < 64; d <<= 1) {
                const uint32_t o = __shfl_xor(col_max[j], d);
                col_max[j] = col_max[j] > o ? col_max[j] : o;
            }
            if (t % 64 < 16) column_max[wave][8 * part + j] = col_max[j];
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 8; ++j)
            for (int w = 0; w < 4; ++w) {
                const uint32_t o = column_max[w][8 * part + j];
                col_max[j] = col_max[j] > o ? col_max[j] : o;
            }
    }
    if (p.Q != nullptr) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = 8 * rows8 + i;
            const int e = p.square ? square : scale_exponent(max_over_16_lanes(row_max[i]));
            const float inverse = power_of_two(-e);
            float q[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) q[j] = scaled_or_nan(v[i][j], inverse);
            if (r < rows_here) {
                const int64_t row = tile.first + r;
                store_bytes8(p.Q + batch * p.stride_q + row * p.ldq + c0 + 8 * part, valid, four_e4m3(q[0], q[1], q[2], q[3]),
                             four_e4m3(q[4], q[5], q[6], q[7]));
                if (!p.square && part == 0) p.S[batch * p.stride_s + row * p.lds + over] = power_of_two(e);
            }
        }
        if (p.square && t == 0) p.S[batch * p.stride_s + static_cast<int64_t>(down) * p.lds + over] = power_of_two(square);
    }
    if (p.T == nullptr) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int e = p.square ? square : scale_exponent(col_max[j]);
        const float inverse = power_of_two(-e);
        const int line = 8 * part + j;
        float q[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = scaled_or_nan(v[i][j], inverse);
        *reinterpret_cast<u32x2 *>(turned + line * 128 + ((rows8 ^ part) << 3)) =
            u32x2{four_e4m3(q[0], q[1], q[2], q[3]), four_e4m3(q[4], q[5], q[6], q[7])};
        if (!p.square && rows8 == 0 && line < cols_here)
            p.ST[batch * p.stride_st + (c0 + line) * p.ldst + turned0 / SCALE_BLOCK] = power_of_two(e);
    }
    if (p.square && t == 0) p.ST[batch * p.stride_st + static_cast<int64_t>(over) * p.ldst + down] = power_of_two(square);
    __syncthreads();
    // whole lines: 16 lanes write the 128 bytes of one; of an expert's last block the bytes behind its rows too (zeros)
    const int wide = p.groups.offsets != nullptr ? 128 : rows_here;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int line = t / 16 + 16 * i, slot = t % 16;
        const u32x2 x = *reinterpret_cast<const u32x2 *>(turned + line * 128 + ((slot ^ ((line >> 3) & 15)) << 3));
        if (line < cols_here) store_bytes8(p.T + batch * p.stride_t + (c0 + line) * p.ldt + turned0 + 8 * slot, wide - 8 * slot, x[0], x[1]);
    }
}

template <typename T> hipError_t launch_as(const QuantizeProblem &p)
{
    const int64_t across = ceil_div(p.cols, SCALE_BLOCK);
    if (!p.square && p.T == nullptr) {
        const int64_t blocks = p.rows * across;
        quantize_rows_kernel<T><<<dim3(static_cast<uint32_t>(ceil_div(blocks, 16)), static_cast<uint32_t>(p.batch)), 256, 0, p.stream>>>(p, across, blocks);
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
