// Products of a few rows of P (the tokens being generated) with weights Q that are read once: Y of a served token, H, logits.
//
// Operands at any address; those on 16 bytes go through LDS (linear_few_dma.hip).  Bound by the weights' bytes.  A work-group has 16 rows of Q (gate and up 16 each; logits 64) and eight wavefronts that share the sum, 32 * U values at a time each;
// fragments go from memory straight into registers, rows of Q at 64 bytes an instruction and 64 U on end; P comes out of the caches.  The wavefronts'
// sums meet in LDS, the first one finishes.  Any address: 16 bytes are read at the alignment of an element.
#include "linear_end.h"
#include "internal.h"

namespace mg {
namespace {

typedef _Float16 few_halfx8 __attribute__((ext_vector_type(8)));
typedef __bf16 few_bfloatx8 __attribute__((ext_vector_type(8)));

constexpr int W = 8;

template <typename T> __device__ inline end_floatx4 multiply(const Piece<T, 8> &q, const Piece<T, 8> &p, end_floatx4 sum)
{
    if constexpr (std::is_same_v<T, _Float16>)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(few_halfx8, q), __builtin_bit_cast(few_halfx8, p), sum, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(few_bfloatx8, q), __builtin_bit_cast(few_bfloatx8, p), sum, 0, 0, 0);
}

// END: LinearEnd; FM, FN: blocks of 16 columns and rows; U: steps of 32 values of the sum that are loaded together
template <typename T, int END, int FM, int FN, int U> __global__ __launch_bounds__(W * 64) void linear_few_kernel(const LinearArgs args)
{
    __shared__ __attribute__((aligned(16))) end_floatx4 sums[(W - 1) * FM * FN * 64];
    __shared__ __attribute__((aligned(16))) char region[end_region<FM * 16>()];
    __shared__ float2 shared[END == END_SCORES ? FN * 16 : 1];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int col0 = blockIdx.x * FM * 16, at = lane / 16 * 8;

    const T *q[FM], *p[FN];
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        // (rows behind the last one read it again; their results are not stored)
        if (END == END_GATED) {
            const int feature = col0 / 2 + i / 2 * 16 + lane % 16, row = feature < args.hidden ? feature : args.hidden - 1;
            q[i] = static_cast<const T *>(i % 2 != 0 ? args.Q1 : args.Q0) + row * (i % 2 != 0 ? args.ldq1 : args.ldq0) + at;
        } else {
            const int col = col0 + 16 * i + lane % 16;
            q[i] = static_cast<const T *>(args.Q0) + (col < args.cols ? col : args.cols - 1) * args.ldq0 + at;
        }
    }
#pragma unroll
    for (int j = 0; j < FN; ++j) {
        const int row = 16 * j + lane % 16;
        p[j] = static_cast<const T *>(args.P) + (row < args.rows ? row : args.rows - 1) * args.ldp + at;
    }
    end_floatx4 acc[FN][FM];
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int i = 0; i < FM; ++i) acc[j][i] = end_floatx4{0.f, 0.f, 0.f, 0.f};

    constexpr int STEP = 32 * U;
    for (int l = wave * STEP; l + STEP <= args.k; l += W * STEP) {
        Piece<T, 8> x[U][FM], y[U][FN];
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int i = 0; i < FM; ++i) x[u][i] = *reinterpret_cast<const Piece<T, 8> *>(q[i] + l + 32 * u);
#pragma unroll
            for (int j = 0; j < FN; ++j) y[u][j] = *reinterpret_cast<const Piece<T, 8> *>(p[j] + l + 32 * u);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int i = 0; i < FM; ++i) acc[j][i] = multiply<T>(x[u][i], y[u][j], acc[j][i]);
    }
    // the sum's end: steps of 32, dealt out to the wavefronts, elements behind it zero
    const int rest = args.k / STEP * STEP;
    for (int l = rest + wave * 32; l < args.k; l += W * 32) {
        const int left = args.k - l - at;
        auto piece = [&](const T *from) {
            if (left >= 8) return *reinterpret_cast<const Piece<T, 8> *>(from);
            Piece<T, 8> v;
#pragma unroll
            for (int e = 0; e < 8; ++e) v.v[e] = e < left ? from[e] : static_cast<T>(0.f);
            return v;
        };
        Piece<T, 8> x[FM], y[FN];
#pragma unroll
        for (int i = 0; i < FM; ++i) x[i] = piece(q[i] + l);
#pragma unroll
        for (int j = 0; j < FN; ++j) y[j] = piece(p[j] + l);
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int i = 0; i < FM; ++i) acc[j][i] = multiply<T>(x[i], y[j], acc[j][i]);
    }
    if (wave > 0) {
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int i = 0; i < FM; ++i) sums[(((wave - 1) * FN + j) * FM + i) * 64 + lane] = acc[j][i];
    }
    __syncthreads();
    if (wave > 0) return;
#pragma unroll 2
    for (int w = 0; w < W - 1; ++w)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int i = 0; i < FM; ++i) acc[j][i] += sums[((w * FN + j) * FM + i) * 64 + lane];
    linear_end<T, END, FM, FN, 1, 1>(args, acc, region, shared, 0, col0, 0, 0, lane);
}

template <typename T> hipError_t launch(int end, const LinearArgs &args, hipStream_t stream)
{
    const uint32_t groups = static_cast<uint32_t>(ceil_div(args.cols, linear_few_columns(end)));
    const bool two = args.rows > 16;
    if (end == END_STORE) {
        if (two) linear_few_kernel<T, END_STORE, 1, 2, 8><<<groups, W * 64, 0, stream>>>(args);
        else linear_few_kernel<T, END_STORE, 1, 1, 8><<<groups, W * 64, 0, stream>>>(args);
    } else if (end == END_GATED) {
        if (two) linear_few_kernel<T, END_GATED, 2, 2, 4><<<groups, W * 64, 0, stream>>>(args);
        else linear_few_kernel<T, END_GATED, 2, 1, 8><<<groups, W * 64, 0, stream>>>(args);
    } else if (end == END_SCORES) {
        if (two) linear_few_kernel<T, END_SCORES, 4, 2, 2><<<groups, W * 64, 0, stream>>>(args);
        else linear_few_kernel<T, END_SCORES, 4, 1, 4><<<groups, W * 64, 0, stream>>>(args);
    } else {
        return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_linear_few_any(int dtype, int end, const LinearArgs &args, hipStream_t stream)
{
    if (args.rows > LINEAR_FEW_ROWS || args.rows < 1 || args.cols < 1) return hipErrorInvalidValue;
    return dtype == MG_F16 ? launch<_Float16>(end, args, stream) : launch<bfloat>(end, args, stream);
}

}  // namespace mg
