// Products of 16-bit matrices whose rows start at any element: 64 x 64 tiles, four wavefronts, staged through registers.  Every element's place is
// checked; nothing outside the operands is read.  Operands that the direct-to-LDS kernels can take do not come here.
#include "linear_end.h"
#include "internal.h"

namespace mg {
namespace {

constexpr int TILE = 64, STEP = 32, LEAD = STEP + 8;          // LDS rows of 80 bytes: 16-byte reads of 16 rows meet in no bank four times

typedef uint32_t any_u32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 any_halfx8 __attribute__((ext_vector_type(8)));
typedef __bf16 any_bfloatx8 __attribute__((ext_vector_type(8)));

template <typename T> __device__ inline end_floatx4 multiply(const T *q, const T *p, end_floatx4 sum)
{
    if constexpr (std::is_same_v<T, _Float16>)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(*reinterpret_cast<const any_halfx8 *>(q), *reinterpret_cast<const any_halfx8 *>(p), sum, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(*reinterpret_cast<const any_bfloatx8 *>(q), *reinterpret_cast<const any_bfloatx8 *>(p), sum, 0, 0, 0);
}

// eight consecutive elements, those from `valid` on zero and not read
template <typename T> __device__ inline Piece<T, 8> eight(const T *at, int valid)
{
    if (valid >= 8) return *reinterpret_cast<const Piece<T, 8> *>(at);
    Piece<T, 8> x;
#pragma unroll
    for (int e = 0; e < 8; ++e) x.v[e] = e < valid ? at[e] : static_cast<T>(0.f);
    return x;
}

// FORM, END: LinearForm, LinearEnd
template <typename T, int FORM, int END> __global__ __launch_bounds__(256) void linear_any_kernel(const LinearArgs args)
{
    __shared__ __attribute__((aligned(16))) T tiles[2 * TILE * LEAD];
    __shared__ __attribute__((aligned(16))) char regions[4][end_region<32>()];
    __shared__ float2 shared[END == END_SCORES ? 2 * TILE : 1];
    const int tile_r = blockIdx.x % args.tiles_r, tile_c = blockIdx.x / args.tiles_r;
    const int row0 = tile_r * TILE, col0 = tile_c * TILE;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, wc = wave % 2, wr = wave / 2;
    const int from = blockIdx.z * args.k_per_slice;
    const int to = from + args.k_per_slice < args.k ? from + args.k_per_slice : args.k;
    constexpr bool P_ALONG = FORM != FORM_NN, Q_ALONG = FORM == FORM_KK;

    // what the sum has of the lines from l on
    auto left_of = [&](int l) {
        if (args.segment == 0) return to - l;
        const int left = args.lines - (l < args.segment ? l : l - args.segment);
        return left < to - l ? left : to - l;
    };
    auto load = [&](bool along, bool of_q, int l0) {
        const int t = threadIdx.x;
        const int place = along ? t / 4 : t % 8 * 8;                          // row (or first of eight rows) inside the tile
        const int l = l0 + (along ? t % 4 * 8 : t / 8);
        const int i = (of_q ? col0 : row0) + place, extent = of_q ? args.cols : args.rows;
        const int left = left_of(l);
        if (!of_q) {
            const T *P = static_cast<const T *>(args.P);
            if (along) return eight(P + i * args.ldp + l, i < extent ? left : 0);
            return eight(P + l * args.ldp + i, left > 0 ? extent - i : 0);
        }
        if (along) {
            if (END == END_GATED) {
                const int feature = i / 32 * 16 + i % 16;
                const bool up = (i / 16) % 2 != 0;
                const T *Q = static_cast<const T *>(up ? args.Q1 : args.Q0);
                return eight(Q + feature * (up ? args.ldq1 : args.ldq0) + l, feature < args.hidden ? left : 0);
            }
            return eight(static_cast<const T *>(args.Q0) + i * args.ldq0 + l, i < extent ? left : 0);
        }
        const bool second = args.segment > 0 && l >= args.segment;
        const T *Q = static_cast<const T *>(second ? args.Q1 : args.Q0);
        return eight(Q + (second ? l - args.segment : l) * (second ? args.ldq1 : args.ldq0) + i, left > 0 ? extent - i : 0);
    };
    auto store = [&](bool along, T *tile, const Piece<T, 8> &x) {
        const int t = threadIdx.x;
        if (along) {
            *reinterpret_cast<any_u32x4 *>(tile + t / 4 * LEAD + t % 4 * 8) = __builtin_bit_cast(any_u32x4, x);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) tile[(t % 8 * 8 + e) * LEAD + t / 8] = x.v[e];
        }
    };

    end_floatx4 acc[2][2];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < 2; ++i) acc[j][i] = end_floatx4{0.f, 0.f, 0.f, 0.f};
    if (from < to) {
        Piece<T, 8> p = load(P_ALONG, false, from), q = load(Q_ALONG, true, from);
        for (int l = from; l < to; l += STEP) {
            store(P_ALONG, tiles, p);
            store(Q_ALONG, tiles + TILE * LEAD, q);
            __syncthreads();
            if (l + STEP < to) {
                p = load(P_ALONG, false, l + STEP);
                q = load(Q_ALONG, true, l + STEP);
            }
            const T *const at_p = tiles + (wr * 32 + lane % 16) * LEAD + lane / 16 * 8, *const at_q = tiles + (TILE + wc * 32 + lane % 16) * LEAD + lane / 16 * 8;
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int i = 0; i < 2; ++i) acc[j][i] = multiply<T>(at_q + 16 * i * LEAD, at_p + 16 * j * LEAD, acc[j][i]);
            __syncthreads();
        }
    }
    linear_end<T, END, 2, 2, 2, 2>(args, acc, regions[wave], shared, row0, col0, wr, wc, lane, blockIdx.z);
}

template <typename T> hipError_t launch(int form, int end, const LinearArgs &args, int slices, hipStream_t stream)
{
    const dim3 grid(static_cast<uint32_t>(args.tiles_r) * args.tiles_c, 1, slices);
    if (form == FORM_KK && end == END_STORE) linear_any_kernel<T, FORM_KK, END_STORE><<<grid, 256, 0, stream>>>(args);
    else if (form == FORM_KK && end == END_GATED) linear_any_kernel<T, FORM_KK, END_GATED><<<grid, 256, 0, stream>>>(args);
    else if (form == FORM_KK && end == END_SCORES) linear_any_kernel<T, FORM_KK, END_SCORES><<<grid, 256, 0, stream>>>(args);
    else if (form == FORM_KK && end == END_SCORES_GRAD) linear_any_kernel<T, FORM_KK, END_SCORES_GRAD><<<grid, 256, 0, stream>>>(args);
    else if (form == FORM_KN && end == END_STORE) linear_any_kernel<T, FORM_KN, END_STORE><<<grid, 256, 0, stream>>>(args);
    else if (form == FORM_KN && end == END_GATED_GRAD) linear_any_kernel<T, FORM_KN, END_GATED_GRAD><<<grid, 256, 0, stream>>>(args);
    else if (form == FORM_NN && end == END_STORE) linear_any_kernel<T, FORM_NN, END_STORE><<<grid, 256, 0, stream>>>(args);
    else return hipErrorInvalidValue;
    return hipGetLastError();
}

}  // namespace

hipError_t launch_linear_any(int dtype, int form, int end, LinearArgs args, int slices, hipStream_t stream)
{
    args.tiles_r = static_cast<int>(ceil_div(args.rows, TILE));
    args.tiles_c = static_cast<int>(ceil_div(args.cols, TILE));
    return dtype == MG_F16 ? launch<_Float16>(form, end, args, slices, stream) : launch<bfloat>(form, end, args, slices, stream);
}

}  // namespace mg
