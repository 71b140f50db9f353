// Helpers of the operators of mg_layers.h: clearing.
#include "layers.h"
#include "internal.h"

namespace mg {
namespace {

template <typename U> __global__ __launch_bounds__(256) void zero_rows_kernel(U *X, int64_t cols, int64_t ld)
{
    for (int64_t c = blockIdx.y * 256 + threadIdx.x; c < cols; c += 256 * static_cast<int64_t>(gridDim.y)) X[blockIdx.x * ld + c] = 0;
}

}  // namespace

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
