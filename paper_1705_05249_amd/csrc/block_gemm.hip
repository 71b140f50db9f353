// Host side of the 8-bit products, the kernel for operands at any address, and the launch that adds slices.
#include "internal.h"
#include "block_gemm_kernel.h"

namespace mg {
namespace {

// ---- operands at any address: SIZE x SIZE tiles (128, or 64 where those would leave compute units idle), staged through registers.  LDS rows of 128 bytes as in lds_layout.h (16-row fragments).
template <int MODE, int SUMS, int SIZE> __global__ __launch_bounds__(256) void block_any_kernel(const BlockArgs args)
{
    constexpr int BM = SIZE, BN = SIZE, HALF = SIZE / 2, FM = HALF / 16, FN = HALF / 16, PIECES = SIZE / 32;
    constexpr int OPERANDS = (BM + BN) * 128, STORES = 4 * STORE_REGION;
    __shared__ __attribute__((aligned(1024))) uint8_t lds_a[OPERANDS > STORES ? OPERANDS : STORES];
    uint8_t *const lds_b = lds_a + BM * 128;
    __shared__ __attribute__((aligned(16))) float scale_a[BM], scale_b[BN];
    BlockTile tile;
    if (!block_tile<MODE, SIZE == 128 ? 7 : 6, BN>(args, &tile)) return;
    const int t = threadIdx.x, lane = t % 64, wave = t / 64, wm = wave % 2, wn = wave / 2;
    const uint8_t *const B = args.B + (MODE == BLOCK_ROWS ? tile.group * args.stride_b : 0);
    const float *const SB = args.SB + (MODE == BLOCK_ROWS ? tile.group * args.stride_sb : 0);

    // this thread's piece of PIECES rows of each operand; rows that do not exist: the tile's first, whose products nobody stores
    const int piece = t % 8;
    const uint8_t *from_a[PIECES], *from_b[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int r = t / 8 + 32 * i;
        const int64_t row = tile.m0 + r < tile.m_end ? tile.m0 + r : tile.m0;
        from_a[i] = args.A + (MODE == BLOCK_ROWS ? source_row(args.groups, row) : row) * args.lda + tile.column + 16 * piece;
        from_b[i] = B + (tile.n0 + r < args.n ? tile.n0 + r : tile.n0) * args.ldb + tile.column + 16 * piece;
    }
    const float *from_s;
    {
        const int r = t % SIZE;                    // (of 64 x 64 tiles the upper two wavefronts repeat the lower ones)
        if (t / SIZE % 2 == 0) {
            const int64_t row = tile.m0 + r < tile.m_end ? tile.m0 + r : tile.m0;
            from_s = args.SA + ((MODE == BLOCK_ROWS ? source_row(args.groups, row) : row) >> args.a_shift) * args.ldsa;
        } else {
            from_s = SB + ((tile.n0 + r < args.n ? tile.n0 + r : tile.n0) >> args.b_shift) * args.ldsb;
        }
        from_s += tile.column / SCALE_BLOCK;
    }

    floatx4 acc[FN][FM];
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int i = 0; i < FM; ++i) acc[j][i] = floatx4{0.f, 0.f, 0.f, 0.f};

    // K-tiles on their way in registers, one more in LDS.  (Two of 128 x 128 take the registers of a second work-group: 57 -> 66 us for 2000 x 3001 x 1999.)
    constexpr int SETS = SIZE == 128 ? 1 : 2;
    struct Fetched {
        u32x4 a[PIECES], b[PIECES];
        float s;
    } fetched[SETS];
    auto fetch = [&](int b, Fetched &next) {
        const int64_t at = static_cast<int64_t>(b) * SCALE_BLOCK;
        const int64_t left = tile.k - at - 16 * piece;
        const int valid = static_cast<int>(left < 16 ? left : 16);
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            next.a[i] = load_bytes16(from_a[i] + at, valid);
            next.b[i] = load_bytes16(from_b[i] + at, valid);
        }
        next.s = from_s[b];
    };
    auto multiply = [&](int b, Fetched &next) {
        __syncthreads();                                   // the block before has been read
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int at = ldsmap::kcontig_slot<16>(t / 8 + 32 * i, piece);
            *reinterpret_cast<u32x4 *>(lds_a + at) = next.a[i];
            *reinterpret_cast<u32x4 *>(lds_b + at) = next.b[i];
        }
        (t / SIZE % 2 == 0 ? scale_a : scale_b)[t % SIZE] = next.s;
        __syncthreads();
        if (b + SETS < tile.b_end) fetch(b + SETS, next);
        typename FragmentOf<SUMS>::type fa[FM], fb;
        float sa[FM];
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            const int row = HALF * wm + 16 * i + lane % 16;
            fa[i].set(join(*reinterpret_cast<const u32x4 *>(lds_a + ldsmap::kcontig_slot<16>(row, lane / 16)),
                           *reinterpret_cast<const u32x4 *>(lds_a + ldsmap::kcontig_slot<16>(row, lane / 16 + 4))));
            sa[i] = scale_a[row];
        }
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const int row = HALF * wn + 16 * j + lane % 16;
            fb.set(join(*reinterpret_cast<const u32x4 *>(lds_b + ldsmap::kcontig_slot<16>(row, lane / 16)),
                        *reinterpret_cast<const u32x4 *>(lds_b + ldsmap::kcontig_slot<16>(row, lane / 16 + 4))));
            if constexpr (SUMS == SUMS_POW2) {
                const int sb = scale_bits(scale_b[row]);
#pragma unroll
                for (int i = 0; i < FM; ++i) add_block_pow2(acc[j][i], fb, fa[i], sb, scale_bits(sa[i]));
            } else {
                const floatx4 sb = *reinterpret_cast<const floatx4 *>(scale_b + HALF * wn + 16 * j + 4 * (lane / 16));
#pragma unroll
                for (int i = 0; i < FM; ++i) add_block(acc[j][i], fb, fa[i], sb, sa[i]);
            }
        }
    };
    static_for<SETS>([&](auto S) {
        if (tile.b0 + decltype(S)::value < tile.b_end) fetch(tile.b0 + decltype(S)::value, fetched[decltype(S)::value]);
    });
    for (int b = tile.b0; b < tile.b_end; b += SETS)
        static_for<SETS>([&](auto S) {
            if (b + decltype(S)::value < tile.b_end) multiply(b + decltype(S)::value, fetched[decltype(S)::value]);
        });
    __syncthreads();
    store_tile(args, tile, acc, reinterpret_cast<char *>(lds_a) + wave * STORE_REGION, tile.m0 + HALF * wm, tile.n0 + HALF * wn, lane);
}

// ---- C = alpha * (sum of the slices) + beta * C
__global__ __launch_bounds__(256) void block_add_slices_kernel(const BlockArgs args)
{
    const int64_t quads = (args.n + 3) / 4;
    const int64_t id = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const int64_t row = id / quads, col = id % quads * 4;
    if (row >= args.partial_rows) return;
    if (!args.each_own_c && args.groups.offsets != nullptr && row >= args.groups.offsets[args.groups.count]) return;      // belongs to no expert
    const int valid = static_cast<int>(args.n - col < 4 ? args.n - col : 4);
    floatx4 sum{0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < args.slices; ++s) {
        float v[4];
        load_piece<float, 4>(args.partial + (s * args.partial_rows + row) * args.n + col, valid, v);
#pragma unroll
        for (int r = 0; r < 4; ++r) sum[r] += v[r];
    }
    BlockArgs whole = args;
    whole.partial = nullptr;
    const bool many = args.each_own_c;
    write_block(whole, many ? static_cast<int>(row / args.m) : 0, many ? row % args.m : row, col, sum);
}

template <int MODE> hipError_t launch_mode(const BlockProblem &p, const BlockArgs &args, int sums, int tile)
{
    if (tile >= 0) {
        if constexpr (MODE == BLOCK_DENSE) return launch_block_dma_dense(args, sums, tile, p.stream);
        else if constexpr (MODE == BLOCK_ROWS) return launch_block_dma_rows(args, sums, tile, p.stream);
        else return launch_block_dma_sum(args, sums, tile, p.stream);
    }
    const dim3 grid(static_cast<uint32_t>(args.tiles_m) * args.tiles_n, args.slices, MODE == BLOCK_SUM ? p.groups.count : 1);
    auto launch = [&](auto size) {
        constexpr int SIZE = decltype(size)::value;
        if (sums_fp32(sums)) block_any_kernel<MODE, SUMS_FP32, SIZE><<<grid, 256, 0, p.stream>>>(args);
        else if (sums == SUMS_POW2) block_any_kernel<MODE, SUMS_POW2, SIZE><<<grid, 256, 0, p.stream>>>(args);
        else block_any_kernel<MODE, SUMS_ANY, SIZE><<<grid, 256, 0, p.stream>>>(args);
    };
    if (tile == TILE_ANY) launch(std::integral_constant<int, 128>{});
    else launch(std::integral_constant<int, 64>{});
    return hipGetLastError();
}

}  // namespace

size_t block_gemm_workspace(int mode, int groups, int64_t m, int64_t n, int64_t k)
{
    int slices = 1;
    for (const int sums : {SUMS_POW2, SUMS_ANY, SUMS_FP32, SUMS_FP32_POW2})
        for (const bool aligned : {false, true}) {
            const Plan p = plan(mode, groups, m, n, k, sums, aligned, SIZE_MAX);
            slices = slices > p.slices ? slices : p.slices;
        }
    return slices > 1 ? static_cast<size_t>(output_rows(mode, groups, m)) * n * 4 * slices : 0;
}

hipError_t launch_block_gemm(const BlockProblem &p)
{
    const int sums = block_sums(p);
    const Plan how = plan(p);
    BlockArgs args{};
    args.A = p.A; args.lda = p.lda; args.SA = p.SA; args.ldsa = p.ldsa; args.a_shift = p.a_square ? 7 : 0;
    args.B = p.B; args.ldb = p.ldb; args.SB = p.SB; args.ldsb = p.ldsb; args.b_shift = p.b_square ? 7 : 0;
    args.stride_b = p.stride_b; args.stride_sb = p.stride_sb;
    args.C = p.C; args.ldc = p.ldc; args.c_type = p.c_type; args.stride_c = p.stride_c; args.each_own_c = p.mode == BLOCK_SUM;
    args.groups = p.groups;
    args.m = static_cast<int>(p.m); args.n = static_cast<int>(p.n); args.k = p.alpha == 0.f ? 0 : static_cast<int>(p.k);
    args.alpha = p.alpha; args.beta = p.beta;
    args.tiles_m = how.tiles_m; args.tiles_n = how.tiles_n; args.slices = how.slices;
    args.partial = how.slices > 1 ? static_cast<float *>(p.workspace) : nullptr;
    args.partial_rows = output_rows(p.mode, p.groups.count, p.m);
    if (how.tile == TILE_FEW) return launch_block_few(args, p.mode, how.few_b, how.fragments, sums_fp32(sums), p.stream);
    const hipError_t e = p.mode == BLOCK_DENSE ? launch_mode<BLOCK_DENSE>(p, args, sums, how.tile)
                         : p.mode == BLOCK_ROWS ? launch_mode<BLOCK_ROWS>(p, args, sums, how.tile) : launch_mode<BLOCK_SUM>(p, args, sums, how.tile);
    if (e != hipSuccess || how.slices == 1) return e;
    const int64_t quads = args.partial_rows * ceil_div(p.n, 4);
    block_add_slices_kernel<<<static_cast<uint32_t>(ceil_div(quads, 256)), 256, 0, p.stream>>>(args);
    return hipGetLastError();
}

}  // namespace mg
