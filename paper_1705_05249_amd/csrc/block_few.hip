// Products with few rows in one operand (the tokens that are being generated): the other operand, the weights, is read once and little else counts.
//
// A work-group takes 16 rows of the weights and up to 16 TF of the few; its four or eight wavefronts share the sum, each every fourth or eighth block
// of 128, straight from memory into registers (a fragment of 16 x 128 bytes is 32 bytes for each lane, four lanes to a row's 128): two blocks on
// their way at a time.  The wavefronts' sums meet in LDS and are added in their order.  Bound by the weights' bytes
// (1 x 4096 x 4096: 5.4 us, 3.1 TB/s and the launch; 1 x 16384 x 4096: 14.2, 4.7 TB/s), with more of the few also by what the caches pass on: the few
// are read once for every 16 rows of the weights (32 x 8192 x 8192 took 33 us, 64 x 64 tiles take 18).
#include "internal.h"
#include "block_gemm_kernel.h"

namespace mg {
namespace {

struct FewArgs {
    const uint8_t *many, *few;                // the operands: `rows_many` rows that are streamed, few of the other
    const float *s_many, *s_few;
    void *C;
    int64_t ld_many, ld_few, lds_many, lds_few, stride_many, stride_s_many;
    int64_t c_many, c_few;                    // distance in C from one row of either operand to the next
    Groups groups;                            // of the few
    int rows_many, rows_few, k;
    int shift_many, shift_few;
    int c_type;
    float alpha, beta;
};

template <typename T> __device__ inline void write_one(T *c, float v, float alpha, float beta)
{
    v *= alpha;
    if (beta != 0.f) v = __builtin_fmaf(beta, static_cast<float>(*c), v);
    *c = static_cast<T>(v);
}

template <int MODE, int FEW_WAVES, int TF, typename FRAGMENT> __global__ __launch_bounds__(FEW_WAVES * 64) void block_few_kernel(const FewArgs args)
{
    constexpr int FEW = 16 * TF, PITCH = 20;                              // floats between the rows of a sum in LDS
    static_assert(MODE == BLOCK_DENSE || TF == 1, "tiles of 16 rows of an expert");
    __shared__ __attribute__((aligned(16))) float sums[FEW_WAVES][FEW * PITCH];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    int64_t first = static_cast<int64_t>(blockIdx.y) * FEW, end = args.rows_few, group = 0;
    if constexpr (MODE == BLOCK_ROWS) {
        RowTile tile;
        if (!find_row_tile<4>(args.groups, blockIdx.y, &tile)) return;
        first = __builtin_amdgcn_readfirstlane(static_cast<int>(tile.first));
        end = __builtin_amdgcn_readfirstlane(static_cast<int>(tile.end));
        group = __builtin_amdgcn_readfirstlane(tile.group);
    }
    const int64_t many0 = static_cast<int64_t>(blockIdx.x) * 16;
    const int blocks = (args.k + SCALE_BLOCK - 1) / SCALE_BLOCK;
    // rows that do not exist: the last one again, whose results nobody stores
    const int64_t row_many = many0 + lane % 16 < args.rows_many ? many0 + lane % 16 : args.rows_many - 1;
    const uint8_t *const at_many = args.many + group * args.stride_many + row_many * args.ld_many + lane / 16 * 16;
    const float *s_many[4];                                               // scales of the lane's four rows of the result
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int64_t row = many0 + lane / 16 * 4 + r < args.rows_many ? many0 + lane / 16 * 4 + r : args.rows_many - 1;
        s_many[r] = args.s_many + group * args.stride_s_many + (row >> args.shift_many) * args.lds_many;
    }
    const uint8_t *at_few[TF];
    const float *s_few[TF];
#pragma unroll
    for (int f = 0; f < TF; ++f) {
        const int64_t wanted = first + 16 * f + lane % 16, row = wanted < end ? wanted : end - 1;
        const int64_t from = MODE == BLOCK_ROWS ? source_row(args.groups, row) : row;
        at_few[f] = args.few + from * args.ld_few + lane / 16 * 16;
        s_few[f] = args.s_few + (from >> args.shift_few) * args.lds_few;
    }

    floatx4 acc[TF];
#pragma unroll
    for (int f = 0; f < TF; ++f) acc[f] = floatx4{0.f, 0.f, 0.f, 0.f};
    struct Many {
        u32x4 x[2];
        float s[4];
    };
    struct Few {
        u32x4 x[TF][2];
        float s[TF];
    };
    // block b of either operand; WHOLE: not the end of a sum that is no multiple of 128
    auto fetch_many = [&](int b, Many &m, auto whole) {
        const int64_t at = static_cast<int64_t>(b) * SCALE_BLOCK;
#pragma unroll
        for (int h = 0; h < 2; ++h) m.x[h] = load_bytes16(at_many + at + 64 * h, decltype(whole)::value ? 16 : static_cast<int>(args.k - at) - lane / 16 * 16 - 64 * h);
        m.s[0] = s_many[0][b];
#pragma unroll
        for (int r = 1; r < 4; ++r) m.s[r] = args.shift_many != 0 ? m.s[0] : s_many[r][b];       // (16 rows lie in one square block)
    };
    auto fetch_few = [&](int b, Few &x, auto whole) {
        const int64_t at = static_cast<int64_t>(b) * SCALE_BLOCK;
#pragma unroll
        for (int f = 0; f < TF; ++f) {
#pragma unroll
            for (int h = 0; h < 2; ++h) x.x[f][h] = load_bytes16(at_few[f] + at + 64 * h, decltype(whole)::value ? 16 : static_cast<int>(args.k - at) - lane / 16 * 16 - 64 * h);
            x.s[f] = s_few[f][b];
        }
    };
    auto multiply = [&](const Many &m, const Few &x) {
        FRAGMENT many, few;
        many.set(join(m.x[0], m.x[1]));
        const floatx4 s{m.s[0], m.s[1], m.s[2], m.s[3]};
#pragma unroll
        for (int f = 0; f < TF; ++f) {
            few.set(join(x.x[f][0], x.x[f][1]));
            add_block(acc[f], many, few, s, x.s[f]);
        }
    };
    using Whole = std::true_type;
    constexpr int AHEAD = 2;
    const int whole_blocks = args.k / SCALE_BLOCK;
    Many many[AHEAD];
    Few few[2];
    static_for<AHEAD>([&](auto U) {
        constexpr int u = decltype(U)::value;
        if (wave + u * FEW_WAVES < whole_blocks) fetch_many(wave + u * FEW_WAVES, many[u], Whole{});
    });
    if (wave < whole_blocks) fetch_few(wave, few[0], Whole{});
    for (int b0 = wave; b0 < whole_blocks; b0 += AHEAD * FEW_WAVES)
        static_for<AHEAD>([&](auto U) {
            constexpr int u = decltype(U)::value;
            const int b = b0 + u * FEW_WAVES;
            if (b < whole_blocks) {
                if (b + FEW_WAVES < whole_blocks) fetch_few(b + FEW_WAVES, few[(u + 1) % 2], Whole{});
                multiply(many[u], few[u % 2]);
                if (b + AHEAD * FEW_WAVES < whole_blocks) fetch_many(b + AHEAD * FEW_WAVES, many[u], Whole{});
            }
        });
    if (whole_blocks < blocks && wave == whole_blocks % FEW_WAVES) {
        fetch_many(whole_blocks, many[0], std::false_type{});
        fetch_few(whole_blocks, few[0], std::false_type{});
        multiply(many[0], few[0]);
    }

#pragma unroll
    for (int f = 0; f < TF; ++f) *reinterpret_cast<floatx4 *>(&sums[wave][(16 * f + lane % 16) * PITCH + lane / 16 * 4]) = acc[f];
    __syncthreads();
    for (int i = threadIdx.x; i < FEW * 16; i += FEW_WAVES * 64) {
        const int64_t row = first + i / 16, col = many0 + i % 16;
        if (row >= end || col >= args.rows_many) continue;
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < FEW_WAVES; ++w) v += sums[w][i / 16 * PITCH + i % 16];
        const int64_t at = row * args.c_few + col * args.c_many;
        if (args.c_type == MG_F32) write_one(static_cast<float *>(args.C) + at, v, args.alpha, args.beta);
        else if (args.c_type == MG_F16) write_one(static_cast<_Float16 *>(args.C) + at, v, args.alpha, args.beta);
        else write_one(static_cast<bfloat *>(args.C) + at, v, args.alpha, args.beta);
    }
}

template <int MODE> hipError_t launch_as(const FewArgs &args, int fragments, bool fp32, hipStream_t stream)
{
    const int64_t tiles = ceil_div(args.rows_few, 16 * fragments) + (MODE == BLOCK_ROWS ? args.groups.count : 0);
    const dim3 grid(static_cast<uint32_t>(ceil_div(args.rows_many, 16)), static_cast<uint32_t>(tiles));
    auto launch = [&](auto waves) {
        constexpr int W = decltype(waves)::value;
        auto with = [&](auto count) {
            constexpr int TF = decltype(count)::value;
            if (fp32) block_few_kernel<MODE, W, TF, Fp16Fragment><<<grid, W * 64, 0, stream>>>(args);
            else block_few_kernel<MODE, W, TF, Fp8Fragment><<<grid, W * 64, 0, stream>>>(args);
        };
        if constexpr (MODE == BLOCK_DENSE) {                              // (experts' rows: 16 at a time)
            if (fragments == 2) return with(std::integral_constant<int, 2>{});
        }
        with(std::integral_constant<int, 1>{});
    };
    // Two work-groups and more for each compute unit: four wavefronts each, of which more fit (1024 work-groups: 8 experts with 2 rows, 2048 x 4096, 22.8 -> 15.7 us;
    // 1 x 16384 x 4096 20.8 -> 14.2; 512 work-groups: within 3 % of each other, 1 x 8192 x 4096 7.4 either way); fewer: eight, for the length of the sum
    // (1 x 8192 x 4096 with two wavefronts 10.6)
    const int64_t busy = grid.x * (MODE == BLOCK_ROWS ? (args.rows_few < args.groups.count ? args.rows_few : args.groups.count) : tiles);
    if (busy >= 512) launch(std::integral_constant<int, 4>{});
    else launch(std::integral_constant<int, 8>{});
    return hipGetLastError();
}

}  // namespace

hipError_t launch_block_few(const BlockArgs &a, int mode, bool few_b, int fragments, bool fp32, hipStream_t stream)
{
    FewArgs f{};
    f.groups = a.groups;
    f.k = a.k;
    f.C = a.C;
    f.c_type = a.c_type;
    f.alpha = a.alpha;
    f.beta = a.beta;
    if (few_b) {
        f.many = a.A; f.s_many = a.SA; f.ld_many = a.lda; f.lds_many = a.ldsa; f.shift_many = a.a_shift; f.rows_many = a.m; f.c_many = a.ldc;
        f.few = a.B; f.s_few = a.SB; f.ld_few = a.ldb; f.lds_few = a.ldsb; f.shift_few = a.b_shift; f.rows_few = a.n; f.c_few = 1;
    } else {
        f.many = a.B; f.s_many = a.SB; f.ld_many = a.ldb; f.lds_many = a.ldsb; f.shift_many = a.b_shift; f.rows_many = a.n; f.c_many = 1;
        f.few = a.A; f.s_few = a.SA; f.ld_few = a.lda; f.lds_few = a.ldsa; f.shift_few = a.a_shift; f.rows_few = a.m; f.c_few = a.ldc;
        f.stride_many = a.stride_b; f.stride_s_many = a.stride_sb;
    }
    return mode == BLOCK_DENSE ? launch_as<BLOCK_DENSE>(f, fragments, fp32, stream) : launch_as<BLOCK_ROWS>(f, fragments, fp32, stream);
}

}  // namespace mg
