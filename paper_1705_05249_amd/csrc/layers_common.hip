// Helpers of the operators of mg_layers.h: adding slices of a sum, clearing.
#include "linear_end.h"
#include "internal.h"

namespace mg {
namespace {

// C = the sum of the slices, in their order.  A work-group has 1024 elements of a row.
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

template <typename U> __global__ __launch_bounds__(256) void zero_rows_kernel(U *X, int64_t cols, int64_t ld)
{
    for (int64_t c = blockIdx.y * 256 + threadIdx.x; c < cols; c += 256 * static_cast<int64_t>(gridDim.y)) X[blockIdx.x * ld + c] = 0;
}

}  // namespace

hipError_t launch_linear_sum(int dtype, const LinearArgs &args, int slices, hipStream_t stream)
{
    const dim3 grid(static_cast<uint32_t>(args.rows), static_cast<uint32_t>(ceil_div(args.cols, 1024)));
    if (dtype == MG_F16) linear_sum_kernel<_Float16><<<grid, 256, 0, stream>>>(args, slices);
    else linear_sum_kernel<bfloat><<<grid, 256, 0, stream>>>(args, slices);
    return hipGetLastError();
}

hipError_t launch_zero_rows(void *X, int64_t rows, int64_t cols, int64_t ld, int size, hipStream_t stream)
{
    if (rows == 0 || cols == 0 || X == nullptr) return hipSuccess;
    const int64_t wide = ceil_div(cols, 256);
    const dim3 grid(static_cast<uint32_t>(rows), static_cast<uint32_t>(wide < 64 ? wide : 64));
    if (size == 4) zero_rows_kernel<<<grid, 256, 0, stream>>>(static_cast<uint32_t *>(X), cols, ld);
    else zero_rows_kernel<<<grid, 256, 0, stream>>>(static_cast<uint16_t *>(X), cols, ld);
    return hipGetLastError();
}

}  // namespace mg
