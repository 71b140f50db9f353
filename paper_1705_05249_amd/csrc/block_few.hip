// Products with few rows in one operand (the tokens that are being generated): the other operand, the weights, is read once and little else counts.
//
// A work-group takes 16 rows of the weights and up to 16 TF of the few; its eight wavefronts share the sum, each every eighth block
// of 128, straight from memory into registers (a fragment of 16 x 128 bytes is 32 bytes for each lane, four lanes to a row's 128), the next block's
// loads in flight during the instructions of this one.  The wavefronts' sums meet in LDS and are added in their order.  Memory leaves the matrix pipes
// nine tenths idle, so the sums are always FP32's (operands widened to FP16).
#include "internal.h"
#include "block_gemm_kernel.h"

namespace mg {
namespace {

constexpr int FEW_WAVES = 8;

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

template <int MODE, int TF> __global__ __launch_bounds__(FEW_WAVES * 64) void block_few_kernel(const FewArgs args)
{
    constexpr int FEW = 16 * TF, PITCH = 20;                              // floats between the rows of a sum in LDS
    __shared__ __attribute__((aligned(16))) float sums[FEW_WAVES][FEW * PITCH];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    int64_t first = static_cast<int64_t>(blockIdx.y) * FEW, end = args.rows_few, group = 0;
    if constexpr (MODE == BLOCK_ROWS) {
        RowTile tile;
        if (!find_row_tile<TF == 1 ? 4 : TF == 2 ? 5 : 6>(args.groups, blockIdx.y, &tile)) return;
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
    struct Block {
        u32x4 many[2], few[TF][2];
        float s_many[4], s_few[TF];
    };
    auto fetch = [&](int b, Block &x) {
        const int64_t at = static_cast<int64_t>(b) * SCALE_BLOCK;
        const int64_t left = args.k - at - lane / 16 * 16;
        if (args.k - at >= SCALE_BLOCK) {                                 // (the same in all lanes)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                x.many[h] = load_bytes16(at_many + at + 64 * h, 16);
#pragma unroll
                for (int f = 0; f < TF; ++f) x.few[f][h] = load_bytes16(at_few[f] + at + 64 * h, 16);
            }
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int valid = static_cast<int>(left - 64 * h < 16 ? left - 64 * h : 16);
                x.many[h] = load_bytes16(at_many + at + 64 * h, valid);
#pragma unroll
                for (int f = 0; f < TF; ++f) x.few[f][h] = load_bytes16(at_few[f] + at + 64 * h, valid);
            }
        }
        x.s_many[0] = s_many[0][b];
#pragma unroll
        for (int r = 1; r < 4; ++r) x.s_many[r] = args.shift_many != 0 ? x.s_many[0] : s_many[r][b];       // (16 rows lie in one square block)
#pragma unroll
        for (int f = 0; f < TF; ++f) x.s_few[f] = s_few[f][b];
    };
    auto multiply = [&](const Block &x) {
        Fp16Fragment many, few;
        many.set(join(x.many[0], x.many[1]));
        const floatx4 s{x.s_many[0], x.s_many[1], x.s_many[2], x.s_many[3]};
#pragma unroll
        for (int f = 0; f < TF; ++f) {
            few.set(join(x.few[f][0], x.few[f][1]));
            add_block(acc[f], many, few, s, x.s_few[f]);
        }
    };
    Block x[2];
    int b = wave;
    if (b < blocks) fetch(b, x[0]);
    for (; b + FEW_WAVES < blocks; b += 2 * FEW_WAVES) {
        fetch(b + FEW_WAVES, x[1]);
        multiply(x[0]);
        if (b + 2 * FEW_WAVES < blocks) fetch(b + 2 * FEW_WAVES, x[0]);
        multiply(x[1]);
    }
    if (b < blocks) multiply(x[0]);

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

template <int MODE> hipError_t launch_as(const FewArgs &args, int fragments, hipStream_t stream)
{
    const int64_t tiles = ceil_div(args.rows_few, 16 * fragments) + (MODE == BLOCK_ROWS ? args.groups.count : 0);
    const dim3 grid(static_cast<uint32_t>(ceil_div(args.rows_many, 16)), static_cast<uint32_t>(tiles));
    if (fragments == 1) block_few_kernel<MODE, 1><<<grid, FEW_WAVES * 64, 0, stream>>>(args);
    else if (fragments == 2) block_few_kernel<MODE, 2><<<grid, FEW_WAVES * 64, 0, stream>>>(args);
    else block_few_kernel<MODE, 4><<<grid, FEW_WAVES * 64, 0, stream>>>(args);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_block_few(const BlockArgs &a, int mode, bool few_b, int fragments, hipStream_t stream)
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
    return mode == BLOCK_DENSE ? launch_as<BLOCK_DENSE>(f, fragments, stream) : launch_as<BLOCK_ROWS>(f, fragments, stream);
}

}  // namespace mg
