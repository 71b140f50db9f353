// Products of 16-bit matrices: the kernel that the plan takes, copies of operands, sums of slices.
#include "linear_plan.h"
#include "linear_end.h"

namespace mg {
namespace {

// scale[0] = most / (the largest weight of the tokens that count), scale[1] its inverse: what dz is multiplied with while it is an operand in 16 bits, and its products with afterwards.
// Where all weights are alike, as in a mean, dz then is p - [target] itself, whose -1 of an unlikely target is exact (1 / count is not: off by up to half a
// step in every token, where it is the largest part of dz).  FP16: most = 2^13, an eighth of the largest number; probabilities down to 2^-27 stay normal.
__device__ inline void weight_scale(const float *weights, const int64_t *targets, int64_t vocab, int64_t tokens, float most, float *scale)
{
    __shared__ uint32_t parts[4];
    uint32_t largest = weights == nullptr ? 0x3f800000u : 0u;
    if (weights != nullptr) {
        // (eight at a time: a load behind the other would be 0.5 us each)
        for (int64_t t = threadIdx.x; t < tokens; t += 8 * 256) {
            uint32_t w[8];
            int64_t target[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int64_t at = t + 256 * e < tokens ? t + 256 * e : tokens - 1;      // (the last one again)
                w[e] = __builtin_bit_cast(uint32_t, weights[at]) & 0x7fffffffu;
                target[e] = targets[at];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) largest = target[e] >= 0 && target[e] < vocab && w[e] < 0x7f800000u && w[e] > largest ? w[e] : largest;
        }
    }
    for (int d = 32; d > 0; d /= 2) {
        const uint32_t other = __shfl_xor(largest, d);
        largest = other > largest ? other : largest;
    }
    if (threadIdx.x % 64 == 0) parts[threadIdx.x / 64] = largest;
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (int w = 1; w < 4; ++w) largest = parts[w] > largest ? parts[w] : largest;
    // (weights beyond 2^100 either way: the scale and its inverse have to be normal numbers)
    const float w = fminf(fmaxf(__builtin_bit_cast(float, largest), 0x1p-100f), 0x1p100f);
    scale[0] = largest == 0 ? 1.f : most / w;
    scale[1] = largest == 0 ? 1.f : w / most;
}

constexpr uint32_t COPY_GROUPS = uint32_t(1) << 22;           // along x: a launch has fewer than 2^32 threads there, five large matrices more pieces

// A thread moves a piece of eight elements; the work-group behind the last matrix makes the scale.
__global__ __launch_bounds__(256) void copy_kernel(const LinearCopies c)
{
    const uint32_t group = blockIdx.y * gridDim.x + blockIdx.x;
    if (group >= c.begin[c.count]) {
        if (group == c.begin[c.count] && c.scale != nullptr) weight_scale(c.weights, c.targets, c.vocab, c.rows[0], c.most, c.scale);
        return;
    }
    int m = 0;
    while (m + 1 < c.count && group >= c.begin[m + 1]) ++m;
    // (copy_rows: a launch has at most 2^32 of them in a matrix)
    const uint32_t piece = (group - c.begin[m]) * 256 + threadIdx.x;
    const int cols = c.cols[m];
    const uint32_t per_row = static_cast<uint32_t>(padded(cols) / 8), in_column = piece / per_row;
    const int64_t row = in_column;
    if (row >= c.rows[m]) return;
    const int col = static_cast<int>(piece - in_column * per_row) * 8;
    int left = cols - col;
    if (m == 0 && c.targets != nullptr) {
        // nothing times an infinity is no number: a token that does not count must not reach the sums over tokens
        const int64_t target = c.targets[row];
        if (target < 0 || target >= c.vocab || (c.weights != nullptr && c.weights[row] == 0.f)) left = 0;
    }
    const uint16_t *from = static_cast<const uint16_t *>(c.from[m]) + row * c.ld[m] + col;
    Piece<uint16_t, 8> x;
    if (left >= 8) {
        x = *reinterpret_cast<const Piece<uint16_t, 8> *>(from);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x.v[e] = e < left ? from[e] : uint16_t(0);
    }
    *reinterpret_cast<end_floatx4 *>(static_cast<uint16_t *>(c.to[m]) + row * padded(cols) + col) = __builtin_bit_cast(end_floatx4, x);
}

// C = the sum of the slices, in their order (T float: C may be the first of them).  A work-group has 1024 elements of a row.
template <typename T> __global__ __launch_bounds__(256) void linear_sum_kernel(const LinearArgs args, int slices)
{
    int64_t row = blockIdx.x;
    const int col = (blockIdx.y * 256 + threadIdx.x) * 4;
    if (col >= args.cols) return;
    const float *from = args.partial + row * args.partial_ld + col;      // (partial_ld is a multiple of 64)
    T *C = static_cast<T *>(args.C0);
    int64_t ldc = args.ldc0;
    if (args.second > 0) {
        if (row >= args.second) {
            C = static_cast<T *>(args.C1);
            ldc = args.ldc1;
            row -= args.second;
        }
        if (row >= args.rows0 || C == nullptr) return;
    }
    const float scale = args.scale == nullptr ? 1.f : *args.scale;
    end_floatx4 sum = *reinterpret_cast<const end_floatx4 *>(from);
    for (int s = 1; s < slices; ++s) sum += *reinterpret_cast<const end_floatx4 *>(from + s * args.partial_stride);
    float out[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) out[e] = sum[e] * scale;
    store_piece<T, 4>(C + row * ldc + col, args.cols - col, out);
}

}  // namespace

hipError_t launch_linear_copies(LinearCopies c, hipStream_t stream)
{
    if (c.count == 0) return hipSuccess;
    if (c.count == 1 && c.scale == nullptr)
        for (const int64_t most = copy_rows(c.cols[0]); c.rows[0] > most;)
            if (const hipError_t e = launch_linear_copies(take_copy_rows(c, most), stream)) return e;
    for (int m = 0; m < c.count; ++m)
        if (c.rows[m] > copy_rows(c.cols[m])) return hipErrorInvalidValue;
    c.begin[0] = 0;
    for (int m = 0; m < c.count; ++m) c.begin[m + 1] = c.begin[m] + static_cast<uint32_t>(ceil_div(c.rows[m] * (padded(c.cols[m]) / 8), 256));
    const uint32_t groups = c.begin[c.count] + (c.scale != nullptr ? 1 : 0), wide = groups < COPY_GROUPS ? groups : COPY_GROUPS;
    if (groups == 0) return hipSuccess;               // matrices without rows or columns
    copy_kernel<<<dim3(wide, (groups + wide - 1) / wide), 256, 0, stream>>>(c);
    return hipGetLastError();
}

hipError_t launch_linear_sum(int dtype, const LinearArgs &args, int slices, hipStream_t stream)
{
    const dim3 grid(static_cast<uint32_t>(args.rows), static_cast<uint32_t>(ceil_div(args.cols, 1024)));
    if (dtype == MG_F32) linear_sum_kernel<float><<<grid, 256, 0, stream>>>(args, slices);
    else if (dtype == MG_F16) linear_sum_kernel<_Float16><<<grid, 256, 0, stream>>>(args, slices);
    else linear_sum_kernel<bfloat><<<grid, 256, 0, stream>>>(args, slices);
    return hipGetLastError();
}

size_t linear_room(int form, int end, int64_t rows, int64_t cols, int64_t k)
{
    size_t most = 0;
    for (const bool aligned : {true, false}) {
        const int slices = linear_plan(form, end, rows, cols, k, aligned, ~size_t(0)).slices;
        const size_t room = slices > 1 ? static_cast<size_t>(slices) * rows * padded(cols) * sizeof(float) : 0;
        most = room > most ? room : most;
    }
    return most;
}

hipError_t launch_linear(int dtype, int form, int end, LinearArgs args, void *room, size_t room_bytes, hipStream_t stream, int *scores_columns)
{
    const LinearPlan how = linear_plan(form, end, args.rows, args.cols, args.k, linear_aligned(form, end, args), args.partial != nullptr || room == nullptr ? 0 : room_bytes);
    const bool sliced = how.slices > 1;
    if (sliced) {
        args.partial = static_cast<float *>(room);
        args.partial_ld = padded(args.cols);
        args.partial_stride = args.rows * args.partial_ld;
    }
    args.k_per_slice = how.k_per_slice;
    if (scores_columns != nullptr) *scores_columns = how.tile == LINEAR_FEW || how.tile == LINEAR_ANY_FEW ? linear_few_columns(end) : linear_tile_size(how.tile);
    hipError_t e = hipErrorInvalidValue;
    if (how.tile == LINEAR_ANY) e = launch_linear_any(dtype, form, end, args, how.slices, stream);
    else if (how.tile == LINEAR_FEW) e = launch_linear_few_dma(dtype, end, args, stream);
    else if (how.tile == LINEAR_ANY_FEW) e = launch_linear_few_any(dtype, end, args, stream);
    else if (form == FORM_KK && end == END_STORE) e = launch_linear_dma_kk_store(dtype, how.tile, args, how.slices, stream);
    else if (form == FORM_KK && end == END_GATED) e = launch_linear_dma_kk_gated(dtype, how.tile, args, how.slices, stream);
    else if (form == FORM_KK && end == END_SCORES) e = launch_linear_dma_kk_scores(dtype, how.tile, args, how.slices, stream);
    else if (form == FORM_KK && end == END_SCORES_GRAD) e = launch_linear_dma_kk_scores_grad(dtype, how.tile, args, how.slices, stream);
    else if (form == FORM_KN && end == END_STORE) e = launch_linear_dma_kn_store(dtype, how.tile, args, how.slices, stream);
    else if (form == FORM_KN && end == END_GATED_GRAD) e = launch_linear_dma_kn_gated_grad(dtype, how.tile, args, how.slices, stream);
    else if (form == FORM_NN && end == END_STORE) e = launch_linear_dma_nn_store(dtype, how.tile, args, how.slices, stream);
    if (e != hipSuccess || !sliced) return e;
    return launch_linear_sum(dtype, args, how.slices, stream);
}

}  // namespace mg
