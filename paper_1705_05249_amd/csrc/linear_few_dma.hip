// Products of a few rows of P (the tokens being generated) with weights Q that are read once: Y of a served token, H, logits.  Rows on 16 bytes.
//
// Bound by the weights' bytes.  A work-group has 16 rows of Q (gate and up 16 each; logits 64); its W wavefronts share the sum, every W-th K-tile of 64 each, and
// meet in LDS at its end.  Each wavefront has a ring of S stages of its own, filled by direct-to-LDS loads of 128 bytes a row, eight rows an instruction: no
// barrier in the loop, and what is in flight costs no registers.  (Fragments loaded straight into registers take 64 bytes of a row an instruction, half a cache
// line: 4096 x 8192 with one row 17 us however many were in flight, 67 MB at 3.9 TB/s.)
#include "linear_dma_kernel.h"
#include "internal.h"

namespace mg {
namespace {

template <int FM, int FN, int W, int S> constexpr int few_lds()
{
    const int ring = W * S * (FM + FN) * 2048, end = (W - 1) * FM * FN * 1024 + end_region<FM * 16>() + FN * 128;
    return ring > end ? ring : end;
}

// END: LinearEnd; FM, FN: blocks of 16 columns and rows; ONCE: Q is not kept in the caches
template <typename T, int END, int FM, int FN, int W, int S, bool ONCE> __global__ __launch_bounds__(W * 64) void linear_few_dma_kernel(const LinearArgs args)
{
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr bool GATED = END == END_GATED;
    using LoadQ = LinearLoader<16 * FM, 64, true, GATED, ONCE>;
    using LoadP = LinearLoader<16 * FN, 64, true>;
    constexpr int Q_BYTES = FM * 2048, STAGE = (FM + FN) * 2048, PIECES = LoadQ::COUNT + LoadP::COUNT;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    lds_char *const lds3 = (lds_char *)lds;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int col0 = blockIdx.x * FM * 16;
    lds_char *const ring = lds3 + wave * (S * STAGE);

    LoadQ lq;
    LoadP lp;
    lq.prepare(args.ldq0, args.ldq1, 0, lane, GATED ? args.hidden - col0 / 2 : args.cols - col0);
    lp.prepare(args.ldp, args.ldp, 0, lane, args.rows);
    const _Float16 *const P = static_cast<const _Float16 *>(args.P), *const Q0 = static_cast<const _Float16 *>(args.Q0), *const Q1 = static_cast<const _Float16 *>(args.Q1);
    const int ktiles = (args.k + 63) / 64, mine = ktiles > wave ? (ktiles - wave + W - 1) / W : 0;
    auto load = [&](int n, int stage) {                 // this wavefront's n-th K-tile; behind its last one zeros, without memory being touched
        const int l0 = n < mine ? (wave + n * W) * 64 : 0, left = n < mine ? args.k - l0 : 0;
        lds_char *const to = ring + stage * STAGE;
        if constexpr (GATED) lq.aim_gated(Q0, args.ldq0, Q1, args.ldq1, col0 / 2, l0, left, args.hidden - col0 / 2);
        else lq.aim(Q0, args.ldq0, col0, l0, left, args.cols - col0);
        lp.aim(P, args.ldp, 0, l0, left, args.rows);
        static_for<LoadQ::COUNT>([&](auto N) { lq.template issue<decltype(N)::value>(to, left); });
        static_for<LoadP::COUNT>([&](auto N) { lp.template issue<decltype(N)::value>(to + Q_BYTES, left); });
    };
    floatx4 acc[FN][FM];
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int i = 0; i < FM; ++i) acc[j][i] = floatx4{0.f, 0.f, 0.f, 0.f};

    constexpr int AHEAD = (S - 2) * PIECES;
    static_assert(S >= 2 && AHEAD < 64, "six bits of the wait count");
    if (mine > 0) {
        static_for<S - 1>([&](auto N) { load(decltype(N)::value, decltype(N)::value); });
        const uint32_t first = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(ring)) + static_cast<uint32_t>(ldsmap::kcontig_base<16>(lane, 0));
        int stage = 0;
        for (int n = 0; n < mine; ++n) {
            __builtin_amdgcn_s_waitcnt(0x0F70 | (AHEAD & 15) | (AHEAD / 16) << 14);      // K-tile n is in LDS; loads return in order
            __builtin_amdgcn_sched_barrier(0);
            const uint32_t at = first + stage * STAGE;
            u32x4 fq[2][FM], fp[2][FN];
            static_for<2>([&](auto N) {
                constexpr int s = decltype(N)::value;
                static_for<FM>([&](auto I) { fq[s][decltype(I)::value] = read_linear<true, 16 * FM, decltype(I)::value, s, 0>(at); });
                static_for<FN>([&](auto J) { fp[s][decltype(J)::value] = read_linear<true, 16 * FN, decltype(J)::value, s, Q_BYTES>(at); });
            });
            __builtin_amdgcn_s_waitcnt(0xC07F);                                          // lgkmcnt(0)
            __builtin_amdgcn_sched_barrier(0);
            load(n + S - 1, stage == 0 ? S - 1 : stage - 1);                             // into the stage of K-tile n - 1, whose fragments have been read
            static_for<2>([&](auto N) {
                constexpr int s = decltype(N)::value;
#pragma unroll
                for (int j = 0; j < FN; ++j)
#pragma unroll
                    for (int i = 0; i < FM; ++i) mma(acc[j][i], fp[s][j], fq[s][i], T{});
            });
            __builtin_amdgcn_sched_barrier(0);
            stage = stage + 1 < S ? stage + 1 : 0;
        }
        __builtin_amdgcn_s_waitcnt(0x0F70);                                              // the loads behind the end
    }
    __syncthreads();
    end_floatx4 *const sums = reinterpret_cast<end_floatx4 *>(lds);
    if (wave > 0) {
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int i = 0; i < FM; ++i) sums[(((wave - 1) * FN + j) * FM + i) * 64 + lane] = acc[j][i];
    }
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int w = 0; w < W - 1; ++w)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int i = 0; i < FM; ++i) acc[j][i] += sums[((w * FN + j) * FM + i) * 64 + lane];
    char *const behind = lds + (W - 1) * FM * FN * 1024;
    linear_end<T, END, FM, FN, 1, 1>(args, acc, behind, reinterpret_cast<float2 *>(behind + end_region<FM * 16>()), 0, col0, 0, 0, lane);
#else
    (void)args;
#endif
}

template <typename T, int END, int FM, int FN, int W, int S, bool ONCE> hipError_t launch_with(const LinearArgs &args, hipStream_t stream)
{
    constexpr int LDS = few_lds<FM, FN, W, S>();
    static_assert(LDS <= 160 * 1024, "LDS of a compute unit");
    static RaisedLds raised;
    auto kernel = linear_few_dma_kernel<T, END, FM, FN, W, S, ONCE>;
    if (const hipError_t e = raised(reinterpret_cast<const void *>(kernel), LDS)) return e;
    kernel<<<static_cast<uint32_t>(ceil_div(args.cols, FM * 16)), W * 64, LDS, stream>>>(args);
    return hipGetLastError();
}

// Weights of 64 MB and more do not stay in the last-level cache (256 MB) until the next call of a model of some layers, and pass it by: 134 MB 28.8 -> 25.5 us.  From
// smaller ones that do stay, a call gets them faster (gate and up weights of 34 MB 8.0 us against 10.4).
template <typename T, int END, int FM, int FN, int W, int S> hipError_t launch_as(const LinearArgs &args, hipStream_t stream)
{
    const bool once = static_cast<int64_t>(args.cols) * args.k >= int64_t(1) << 25;
    return once ? launch_with<T, END, FM, FN, W, S, true>(args, stream) : launch_with<T, END, FM, FN, W, S, false>(args, stream);
}

template <typename T> hipError_t launch(int end, const LinearArgs &args, hipStream_t stream)
{
    const bool two = args.rows > 16;
    if (end == END_STORE) return two ? launch_as<T, END_STORE, 1, 2, 8, 3>(args, stream) : launch_as<T, END_STORE, 1, 1, 8, 4>(args, stream);
    if (end == END_GATED) return two ? launch_as<T, END_GATED, 2, 2, 4, 3>(args, stream) : launch_as<T, END_GATED, 2, 1, 4, 2>(args, stream);
    if (end == END_SCORES) return two ? launch_as<T, END_SCORES, 4, 2, 4, 3>(args, stream) : launch_as<T, END_SCORES, 4, 1, 4, 2>(args, stream);
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_linear_few_dma(int dtype, int end, const LinearArgs &args, hipStream_t stream)
{
    if (args.rows > LINEAR_FEW_ROWS || args.rows < 1 || args.cols < 1) return hipErrorInvalidValue;
    return dtype == MG_F16 ? launch<_Float16>(end, args, stream) : launch<bfloat>(end, args, stream);
}

}  // namespace mg
