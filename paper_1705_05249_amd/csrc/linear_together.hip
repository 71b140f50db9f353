// Products that do not wait for each other, in one launch: the gradients that read dG and dU, or dz.  FORM_KN, END_STORE (a sum that may be sliced) and up to two of
// FORM_NN, END_STORE, on the tiles of linear_dma_kernel.h.
//
// A small product by itself is a launch, a start, a few K-tiles and an end, on part of the compute units; together they fill each other's gaps.  The long sums come first.
#include "linear_dma_kernel.h"
#include "linear_plan.h"

namespace mg {
namespace {

template <typename T, int SIZE, int STAGES> __global__ __launch_bounds__(256) void linear_together_kernel(const LinearTogether all)
{
    const uint32_t group = blockIdx.x;
    if (group < all.begin[1]) {
        const LinearArgs &args = all.of[0];
        const uint32_t tiles = static_cast<uint32_t>(args.tiles_c) * args.tiles_r, slice = group / tiles;
        linear_dma_tile<T, FORM_KN, END_STORE, SIZE, SIZE, 2, 2, STAGES, 1>(args, group - slice * tiles, slice);
    } else {
        const int n = group < all.begin[2] ? 1 : 2;
        linear_dma_tile<T, FORM_NN, END_STORE, SIZE, SIZE, 2, 2, STAGES, 1>(all.of[n], group - all.begin[n], 0);
    }
}

template <typename T, int SIZE, int STAGES> hipError_t launch_as(const LinearTogether &all, hipStream_t stream)
{
    constexpr int LDS = linear_dma_lds<SIZE, SIZE, 2, 2, STAGES>();
    static RaisedLds raised;
    auto kernel = linear_together_kernel<T, SIZE, STAGES>;
    if (const hipError_t e = raised(reinterpret_cast<const void *>(kernel), LDS)) return e;
    kernel<<<all.begin[3], 256, LDS, stream>>>(all);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_linear_together(int dtype, LinearTogether all, void *room, size_t room_bytes, hipStream_t stream)
{
    LinearSize sizes[3] = {};
    bool aligned = true;
    for (int n = 0; n < 3; ++n) {
        const LinearArgs &a = all.of[n];
        sizes[n] = {a.rows, a.cols, a.k};
        aligned = aligned && (a.rows == 0 || linear_aligned(n == 0 ? FORM_KN : FORM_NN, END_STORE, a));
    }
    LinearPlan how{LINEAR_ANY, 1, 0, 0};
    if (aligned && all.of[0].partial == nullptr) how = linear_plan_together(sizes, room == nullptr ? 0 : room_bytes);
    if (how.tile == LINEAR_ANY) {
        for (int n = 0; n < 3; ++n)
            if (all.of[n].rows > 0)
                if (const hipError_t e = launch_linear(dtype, n == 0 ? FORM_KN : FORM_NN, END_STORE, all.of[n], room, room_bytes, stream)) return e;
        return hipSuccess;
    }
    LinearArgs &first = all.of[0];
    first.k_per_slice = how.k_per_slice;
    if (how.slices > 1) {
        first.partial = static_cast<float *>(room);
        first.partial_ld = padded(first.cols);
        first.partial_stride = first.rows * first.partial_ld;
    }
    if (const hipError_t e = launch_linear_together_on(dtype, how.tile, all, how.slices, stream)) return e;
    return how.slices > 1 ? launch_linear_sum(dtype, first, how.slices, stream) : hipSuccess;
}

hipError_t launch_linear_together_on(int dtype, int tile, LinearTogether all, int slices, hipStream_t stream)
{
    const int size = linear_tile_size(tile);
    all.begin[0] = 0;
    for (int n = 0; n < 3; ++n) {
        LinearArgs &a = all.of[n];
        a.tiles_c = static_cast<int>(ceil_div(a.cols, size));
        a.tiles_r = static_cast<int>(ceil_div(a.rows, size));
        if (n > 0) a.k_per_slice = static_cast<int>(padded(a.k));
        all.begin[n + 1] = all.begin[n] + static_cast<uint32_t>(a.tiles_c) * a.tiles_r * (n == 0 ? slices : 1);
    }
    if (tile == LINEAR_128) return dtype == MG_F16 ? launch_as<_Float16, 128, 2>(all, stream) : launch_as<bfloat, 128, 2>(all, stream);
    return dtype == MG_F16 ? launch_as<_Float16, 64, 4>(all, stream) : launch_as<bfloat, 64, 4>(all, stream);
}

}  // namespace mg
