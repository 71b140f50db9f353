// Products of 8-bit matrices whose rows start on 16 bytes: operand tiles and their scales go from global memory straight into LDS, `STAGES` K-tiles of
// one scale block (128 bytes of a row) each.
//
// A wavefront's tile is FM x FN fragments of 16 x 16 outputs.  All FM fragments of A stay in registers for a K-tile, those of B follow one another
// (phase j: fragment j of B times all of A's) and are read one phase ahead.  The one barrier of a K-tile stands in front of its last phase: behind
// it the next K-tile's stage is complete, so A's fragments are replaced one by one as the last phase uses them, and the stage that was read is free,
// so the loads of the K-tile `STAGES` further on start there and have a whole K-tile (2048 clocks of 256 x 256) to land.
//
// LDS rows of 128 bytes as in lds_layout.h for 16-row fragments: a lane's 32 bytes of a fragment are the chunks l / 16 and l / 16 + 4 of row
// l % 16, in either operand, so that both see the same order of the sum.
//
// Bound by the matrix pipes at the part's power limit, and by what a tile does before and behind its loop (4 us until the first K-tile of 256 x 256 is there, 8 for C).
// Calls in a row, activations times weights: 4096^3 into bfloat16 67 to 74 us (2.0 PFLOP/s; 72 to 75 with scales of any value and square blocks), 8192 x 4096 x 4096 121
// (2.3; 139, and 160 with row blocks on both sides), with FP32 sums 4096 x 4096 x 8192 240 to 248 (1.1 PFLOP/s).
// Under a profiler's kernel trace the same kernels take a fifth longer (148 and 296).
// A work-group that stays for its next tile and loads it while C leaves has no registers for it with 256 x 256, and gains nothing with 256 x 128.
//
// Ends: rows behind an operand's last one are its last one again (their products are not stored).  Pieces of 16 bytes behind the end of the sum are not
// fetched: their lanes name an offset outside the descriptor's range, for which zeros arrive in LDS.  Where the sum ends inside a piece, its last
// K-tile is staged through registers behind the loop (in the loop that code cost the 256 x 256 tiles their registers).
#pragma once

#include "block_gemm_kernel.h"
#include "mfma_dma_kernel.h"

namespace mg {

#if defined(__HIP_DEVICE_COMPILE__)
// An operand's tile: ROWS rows of 128 bytes in 1 KB blocks of eight rows; a wavefront of W owns COUNT consecutive blocks.
template <int ROWS, int W> struct BlockLoader {
    static constexpr int COUNT = ROWS / 8 / W;
    static constexpr uint32_t MISSING = 0x80000000u;
    static_assert(COUNT >= 1 && COUNT * 8 * W == ROWS, "whole blocks for every wavefront");

    uint32_t offset[COUNT];       // of the lane's piece from the descriptor's base
    int piece[2];                 // first byte of the lane's piece in its row, even and odd blocks
    __amdgpu_buffer_rsrc_t rsrc;

    static __device__ inline int piece_of(int block, int lane) { return ((lane % 8) ^ ldsmap::swizzle16(block * 8 + lane / 8)) * 16; }
    // row_bytes(r): offset of the tile's row r from the base
    template <typename F> __device__ inline void prepare(const uint8_t *base, int wave, int lane, F &&row_bytes)
    {
        rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(base), 0, 0x7fffffff, 0x00020000);
        piece[0] = piece_of(wave * COUNT, lane);
        piece[1] = piece_of(wave * COUNT + 1, lane);
#pragma unroll
        for (int q = 0; q < COUNT; ++q) offset[q] = row_bytes((wave * COUNT + q) * 8 + lane / 8) + static_cast<uint32_t>(piece[q % 2]);
    }
    // left: bytes of the sum from this K-tile on; along: its distance from the base (wave-uniform)
    __device__ inline void issue(lds_char *mine, int left, uint32_t along) const
    {
#pragma unroll
        for (int q = 0; q < COUNT; ++q)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, reinterpret_cast<lds_void *>(mine + q * 1024), 16, piece[q % 2] < left ? offset[q] : MISSING, along, 0, 0);
    }
};

template <int OFFSET> __device__ inline float lds_read_b32_untracked(uint32_t at)
{
    static_assert(OFFSET >= 0 && OFFSET < 65536, "LDS instruction offsets have 16 bits");
    float r;
    asm volatile("ds_read_b32 %0, %1 offset:%2" : "=&v"(r) : "v"(at), "n"(OFFSET) : "memory");
    return r;
}
// A register that an LDS read has written by now (behind the wait): what uses it stays behind this
template <typename T> __device__ inline void landed(T &x) { asm volatile("" : "+v"(x)); }
#endif

constexpr int dma_waitcnt(int loads) { return 0x0F70 | (loads & 15) | ((loads >> 4) << 14); }      // vmcnt alone

template <int BM, int BN, int W> constexpr int block_scale_slots() { return (BM + BN + 64 * W - 1) / (64 * W) * 64 * W; }
template <int BM, int BN, int W, int STAGES> constexpr int block_dma_lds() { return STAGES * ((BM + BN) * 128 + block_scale_slots<BM, BN, W>() * 4); }

template <int MODE, int SUMS, int BM, int BN, int WM, int WN, int STAGES>
__global__ __launch_bounds__(WM *WN * 64) void block_dma_kernel(const BlockArgs args)
{
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int W = WM * WN, WTM = BM / WM, WTN = BN / WN, FM = WTM / 16, FN = WTN / 16;
    constexpr int LOG_BM = BM == 256 ? 8 : BM == 128 ? 7 : 6;
    static_assert(1 << LOG_BM == BM && BN % 64 == 0 && WTM % 16 == 0 && FN % 2 == 0, "tile shape");
    static_assert(WTN <= 128, "one block of 128 rows of B for a wavefront");
    using LoadA = BlockLoader<BM, W>;
    using LoadB = BlockLoader<BN, W>;
    constexpr int A_BYTES = BM * 128, B_BYTES = BN * 128, SLOTS = block_scale_slots<BM, BN, W>(), SCALE_LOADS = SLOTS / (64 * W);
    constexpr int B_AT = STAGES * A_BYTES, S_AT = B_AT + STAGES * B_BYTES;
    constexpr int PIECES = LoadA::COUNT + LoadB::COUNT + SCALE_LOADS;
    static_assert(STAGES >= 2 && (STAGES - 2) * PIECES < 64, "the wait count has six bits");

    extern __shared__ __attribute__((aligned(1024))) char lds[];
    lds_char *const lds3 = (lds_char *)lds;

    BlockTile tile;
    if (!block_tile<MODE, LOG_BM, BN>(args, &tile)) return;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), wm = wave / WN, wn = wave % WN;
    // a last K-tile that ends inside a piece of 16 bytes is not in the loop
    const bool ragged = tile.b_end > tile.b0 && static_cast<int64_t>(tile.b_end) * SCALE_BLOCK > tile.k && tile.k % 16 != 0;
    const int ktiles = tile.b_end - tile.b0 - (ragged ? 1 : 0);
    const bool indexed = MODE == BLOCK_ROWS && args.groups.source != nullptr;
    const int rows_a = static_cast<int>(tile.m_end - tile.m0 < BM ? tile.m_end - tile.m0 : BM);
    const int rows_b = static_cast<int>(args.n - tile.n0 < BN ? args.n - tile.n0 : BN);
    const uint8_t *const B = args.B + (MODE == BLOCK_ROWS ? tile.group * args.stride_b : 0);
    const float *const SB = args.SB + (MODE == BLOCK_ROWS ? tile.group * args.stride_sb : 0);
    // row r of the tile, seen from the operand's first row where rows are indexed, otherwise from the tile's
    auto row_a = [&](int r) -> int64_t {
        const int64_t row = r < rows_a ? r : rows_a - 1;
        return indexed ? source_row(args.groups, tile.m0 + row) : row;
    };

    floatx4 acc[FN][FM];
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int i = 0; i < FM; ++i) acc[j][i] = floatx4{0.f, 0.f, 0.f, 0.f};

    if (ktiles > 0) {
        const int64_t column = tile.column + static_cast<int64_t>(tile.b0) * SCALE_BLOCK;
        LoadA la;
        LoadB lb;
        la.prepare(args.A + (indexed ? 0 : tile.m0 * args.lda) + column, wave, lane, [&](int r) { return static_cast<uint32_t>(row_a(r) * args.lda); });
        lb.prepare(B + tile.n0 * args.ldb + column, wave, lane, [&](int r) { return static_cast<uint32_t>((r < rows_b ? r : rows_b - 1) * args.ldb); });
        // scales: 64 slots for a load of a wavefront, A's BM first, B's BN behind them; what is left over loads B's first one
        uint32_t scale_offset[SCALE_LOADS];
        __amdgpu_buffer_rsrc_t scale_rsrc[SCALE_LOADS];
#pragma unroll
        for (int q = 0; q < SCALE_LOADS; ++q) {
            const int first = (wave * SCALE_LOADS + q) * 64;
            const bool of_a = first < BM;
            const int64_t base_row = of_a ? (indexed ? 0 : tile.m0) : tile.n0;
            const float *base = of_a ? args.SA + (base_row >> args.a_shift) * args.ldsa : SB + (base_row >> args.b_shift) * args.ldsb;
            const int r = first + lane - (of_a ? 0 : BM);
            const int64_t row = of_a ? row_a(r) : r < rows_b ? r : r < BN ? rows_b - 1 : 0;
            // (rows counted from base_row, which square blocks need not divide)
            const int64_t from = of_a ? ((base_row + row) >> args.a_shift) - (base_row >> args.a_shift) : ((base_row + row) >> args.b_shift) - (base_row >> args.b_shift);
            scale_offset[q] = static_cast<uint32_t>(from * (of_a ? args.ldsa : args.ldsb) * 4);
            scale_rsrc[q] = __builtin_amdgcn_make_buffer_rsrc(const_cast<float *>(base + column / SCALE_BLOCK), 0, 0x7fffffff, 0x00020000);
        }
        auto left_from = [&](int t) { return tile.k - (tile.b0 + t) * SCALE_BLOCK; };
        auto mine_a = [&](int stage) { return lds3 + stage * A_BYTES + wave * (LoadA::COUNT * 1024); };
        auto mine_b = [&](int stage) { return lds3 + B_AT + stage * B_BYTES + wave * (LoadB::COUNT * 1024); };
        auto load_tile = [&](int t, int stage) {
            const int left = left_from(t);
            la.issue(mine_a(stage), left, static_cast<uint32_t>(t) * 128);
            lb.issue(mine_b(stage), left, static_cast<uint32_t>(t) * 128);
#pragma unroll
            for (int q = 0; q < SCALE_LOADS; ++q)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(scale_rsrc[q], reinterpret_cast<lds_void *>(lds3 + S_AT + stage * (SLOTS * 4) + (wave * SCALE_LOADS + q) * 256), 4,
                                                         scale_offset[q], static_cast<uint32_t>(t) * 4, 0, 0);
        };
        auto fence = [] { __builtin_amdgcn_sched_barrier(0); };
        auto wait_reads = [&] { __builtin_amdgcn_s_waitcnt(0xC07F); fence(); };
        // K-tile t complete in LDS for every wavefront; this one's loads of the K-tiles behind it may still be on their way
        auto complete = [&](int t) {
            if (t + STAGES - 2 < ktiles) __builtin_amdgcn_s_waitcnt(dma_waitcnt((STAGES - 2) * PIECES));
            else __builtin_amdgcn_s_waitcnt(dma_waitcnt(0));
            fence();
            __builtin_amdgcn_s_barrier();
            fence();
        };

        const uint32_t lds_at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(lds3));
        const uint32_t at_a = lds_at + ldsmap::kcontig_base<16>(lane, wm * WTM), at_b = lds_at + B_AT + ldsmap::kcontig_base<16>(lane, wn * WTN);
        const uint32_t at_sa = lds_at + S_AT + (wm * WTM + lane % 16) * 4;
        const uint32_t at_sb = lds_at + S_AT + (BM + wn * WTN + (SUMS == SUMS_POW2 || SUMS == SUMS_FP32_POW2 ? lane % 16 : SUMS == SUMS_SQUARE ? 0 : lane / 16 * 4)) * 4;

        u32x4 ra[FM][2], rb[2][2];                // fragments as they come from LDS
        float sa[FM], sb1[2];
        u32x4 sb4[2];
        auto read_a = [&](auto I, int stage) {
            constexpr int i = decltype(I)::value;
            ra[i][0] = lds_read_b128_untracked<i * 2048>(at_a + stage * A_BYTES);
            ra[i][1] = lds_read_b128_untracked<i * 2048>((at_a + stage * A_BYTES) ^ 64);
            sa[i] = lds_read_b32_untracked<i * 64>(at_sa + stage * (SLOTS * 4));
        };
        auto read_b = [&](auto J, int stage) {
            constexpr int j = decltype(J)::value;
            rb[j % 2][0] = lds_read_b128_untracked<j * 2048>(at_b + stage * B_BYTES);
            rb[j % 2][1] = lds_read_b128_untracked<j * 2048>((at_b + stage * B_BYTES) ^ 64);
            if constexpr (SUMS == SUMS_POW2 || SUMS == SUMS_FP32_POW2) sb1[j % 2] = lds_read_b32_untracked<j * 64>(at_sb + stage * (SLOTS * 4));
            else if constexpr (SUMS == SUMS_SQUARE) sb1[j % 2] = lds_read_b32_untracked<0>(at_sb + stage * (SLOTS * 4));
            else sb4[j % 2] = lds_read_b128_untracked<j * 64>(at_sb + stage * (SLOTS * 4));
        };
        auto landed_b = [&](auto J) {
            constexpr int j = decltype(J)::value;
            landed(rb[j % 2][0]);
            landed(rb[j % 2][1]);
            if constexpr (SUMS == SUMS_ANY || SUMS == SUMS_FP32) landed(sb4[j % 2]);
            else landed(sb1[j % 2]);
        };
        auto landed_a = [&] {
            static_for<FM>([&](auto I) {
                landed(ra[decltype(I)::value][0]);
                landed(ra[decltype(I)::value][1]);
                landed(sa[decltype(I)::value]);
            });
        };

        static_for<STAGES>([&](auto S) {
            if (decltype(S)::value < ktiles) load_tile(decltype(S)::value, decltype(S)::value);
        });
        // (of the K-tiles loaded here all but the first may be on their way, unless there are fewer)
        if (STAGES - 1 < ktiles) __builtin_amdgcn_s_waitcnt(dma_waitcnt((STAGES - 1) * PIECES < 63 ? (STAGES - 1) * PIECES : 63));
        else __builtin_amdgcn_s_waitcnt(dma_waitcnt(0));
        fence();
        __builtin_amdgcn_s_barrier();
        fence();
        // behind the last read of a stage: the next K-tile is there, and the loads of the one `STAGES` on start
        auto turn = [&](int t, int stage) {
            if (t + 1 < ktiles) {
                complete(t + 1);
                if (t + STAGES < ktiles) load_tile(t + STAGES, stage);
            }
        };
        // Nothing to multiply: this wavefront only loads.  (A SIMD's two wavefronts lie along m, so that in an expert's last tile every SIMD has one
        // less: 16 experts of 61 to 2879 rows, 4096 x 2048: 208 -> 203 us.)
        const bool idle = wm * WTM >= rows_a || wn * WTN >= rows_b;
        if (idle) {
            int stage = 0;
            for (int t = 0; t < ktiles; ++t) {
                turn(t, stage);
                stage = stage + 1 < STAGES ? stage + 1 : 0;
            }
        } else {
            read_b(std::integral_constant<int, 0>{}, 0);
            static_for<FM>([&](auto I) { read_a(I, 0); });

            // (here and now: otherwise the compiler moves the additions behind the branch of the last phase and keeps every block's sum until then)
            auto add_scaled = [&](floatx4 &sum, const floatx4 &d, float s, const u32x4 &sb) {
                scale_add(sum, d, s, std::integral_constant<bool, SUMS == SUMS_SQUARE>{}, sb);
                landed(sum);
            };
            int stage = 0;
            if constexpr (SUMS == SUMS_FP32_POW2) {
                // Operands are widened beside the matrix instructions: A's fragments in phase 0, each in front of its first use, B's in the
                // second half of the phase before theirs.  (Widened all at once, both wavefronts of a SIMD did so at the same time: 1.65 us
                // for a K-tile of 256 x 128 instead of 1.57.)
                Bf16Fragment fa[FM], fb[2];
                wait_reads();
                landed_b(std::integral_constant<int, 0>{});
                landed_a();
                fb[0].set(rb[0], sb1[0]);
                auto multiply = [&](auto J, auto I, auto Q) {
                    constexpr int j = decltype(J)::value, i = decltype(I)::value, q = decltype(Q)::value;
                    acc[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[j % 2].v[q], fa[i].v[q], acc[j][i], 0, 0, 0);
                };
                for (int t = 0; t < ktiles; ++t) {
                    const int next = stage + 1 < STAGES ? stage + 1 : 0;
                    static_for<FN>([&](auto J) {
                        constexpr int j = decltype(J)::value, following = (j + 1) % FN;
                        using Following = std::integral_constant<int, following>;
                        if constexpr (j == FN - 1) turn(t, stage);
                        read_b(Following{}, j == FN - 1 ? next : stage);
                        fence();
                        if constexpr (j == 0) {
                            fa[0].set(ra[0], sa[0]);
                            static_for<4 * FM>([&](auto S) {
                                constexpr int i = decltype(S)::value / 4, q = decltype(S)::value % 4;
                                if constexpr (i + 1 < FM) fa[i + 1].template quarter<q>(ra[i + 1], sa[i + 1]);
                                if constexpr (i + 1 == FM && q == 0) {
                                    wait_reads();
                                    landed_b(Following{});
                                }
                                if constexpr (i + 1 == FM) fb[1].template quarter<q>(rb[1], sb1[1]);
                                multiply(J, std::integral_constant<int, i>{}, std::integral_constant<int, q>{});
                                fence();
                            });
                        } else {
                            // (a quarter of the block for all fragments of A, so that no instruction waits for the one in front of it)
                            static_for<4 * FM>([&](auto S) {
                                constexpr int s = decltype(S)::value, q = s / FM, i = s % FM;
                                if constexpr (s == 2 * FM) {
                                    wait_reads();
                                    landed_b(Following{});
                                    if constexpr (j == FN - 1) landed_a();
                                }
                                if constexpr (s >= 2 * FM && (s - 2 * FM) % (FM / 2) == 0) fb[following % 2].template quarter<(s - 2 * FM) / (FM / 2)>(rb[following % 2], sb1[following % 2]);
                                multiply(J, std::integral_constant<int, i>{}, std::integral_constant<int, q>{});
                                if constexpr (j == FN - 1 && s < FM) read_a(std::integral_constant<int, s>{}, next);
                                fence();
                            });
                        }
                    });
                    stage = next;
                }
            } else
            for (int t = 0; t < ktiles; ++t) {
                const int next = stage + 1 < STAGES ? stage + 1 : 0;
                typename FragmentOf<SUMS>::type fa[FM];
                int ea[FM];
                float s[FM];
                static_for<FN>([&](auto J) {
                    constexpr int j = decltype(J)::value;
                    wait_reads();
                    landed_b(J);
                    if constexpr (j == 0) {
                        landed_a();
                        static_for<FM>([&](auto I) {
                            constexpr int i = decltype(I)::value;
                            fa[i].set(join(ra[i][0], ra[i][1]));
                            if constexpr (SUMS == SUMS_POW2) ea[i] = scale_bits(sa[i]);
                            else if constexpr (SUMS == SUMS_SQUARE) s[i] = sa[i] * sb1[0];
                            else s[i] = sa[i];
                        });
                    }
                    typename FragmentOf<SUMS>::type fb;
                    fb.set(join(rb[j % 2][0], rb[j % 2][1]));
                    if constexpr (j + 1 < FN) {
                        read_b(std::integral_constant<int, j + 1>{}, stage);
                    } else {
                        turn(t, stage);
                        read_b(std::integral_constant<int, 0>{}, next);       // (behind the last K-tile: nobody uses them)
                    }
                    fence();
                    constexpr int LATER = FM < 3 ? FM - 1 : 2;      // a block's sum is scaled that many fragments later, when it is there
                    floatx4 d[LATER + 1];
                    static_for<FM>([&](auto I) {
                        constexpr int i = decltype(I)::value;
                        if constexpr (SUMS == SUMS_POW2) {
                            add_block_pow2(acc[j][i], fb, fa[i], scale_bits(sb1[j % 2]), ea[i]);
                        } else {
                            d[i % (LATER + 1)] = block_sum(fb, fa[i]);
                            if constexpr (i >= LATER) add_scaled(acc[j][i - LATER], d[(i - LATER) % (LATER + 1)], s[i - LATER], sb4[j % 2]);
                            if constexpr (i == FM - 1)
                                static_for<LATER>([&](auto L) {
                                    constexpr int l = FM - LATER + decltype(L)::value;
                                    add_scaled(acc[j][l], d[l % (LATER + 1)], s[l], sb4[j % 2]);
                                });
                        }
                        if constexpr (j == FN - 1) read_a(I, next);
                        fence();
                    });
                });
                stage = next;
            }
            wait_reads();                     // the reads behind the last K-tile still write registers
            landed_b(std::integral_constant<int, 0>{});
            landed_a();
        }
    }
    if (ragged) {
        const int64_t at = static_cast<int64_t>(tile.b_end - 1) * SCALE_BLOCK;
        const int left = static_cast<int>(tile.k - at);
        const int64_t first_a = indexed ? 0 : tile.m0;
        __syncthreads();
        for (int p = threadIdx.x; p < (BM + BN) * 8; p += W * 64) {
            const bool of_a = p < BM * 8;
            const int r = p / 8 - (of_a ? 0 : BM), piece = p % 8;
            const uint8_t *from = of_a ? args.A + (first_a + row_a(r)) * args.lda : B + (tile.n0 + (r < rows_b ? r : rows_b - 1)) * args.ldb;
            *reinterpret_cast<u32x4 *>(lds + (of_a ? 0 : B_AT) + ldsmap::kcontig_slot<16>(r, piece)) = load_aligned16(from + tile.column + at + 16 * piece, left - 16 * piece);
        }
        float *const scales = reinterpret_cast<float *>(lds + S_AT);
        for (int r = threadIdx.x; r < BM + BN; r += W * 64) {
            const bool of_a = r < BM;
            const int64_t row = of_a ? first_a + row_a(r) : tile.n0 + (r - BM < rows_b ? r - BM : rows_b - 1);
            scales[r] = (of_a ? args.SA + (row >> args.a_shift) * args.ldsa : SB + (row >> args.b_shift) * args.ldsb)[(tile.column + at) / SCALE_BLOCK];
        }
        __syncthreads();
        auto fragment = [&](int base, int row, float s) {
            typename FragmentOf<SUMS>::type f;
            const u32x4 x[2] = {*reinterpret_cast<const u32x4 *>(lds + base + ldsmap::kcontig_slot<16>(row, lane / 16)),
                                *reinterpret_cast<const u32x4 *>(lds + base + ldsmap::kcontig_slot<16>(row, lane / 16 + 4))};
            if constexpr (SUMS == SUMS_FP32_POW2) f.set(x, s);
            else f.set(join(x[0], x[1]));
            return f;
        };
        static_for<FM>([&](auto I) {
            constexpr int i = decltype(I)::value;
            const int row = wm * WTM + 16 * i + lane % 16;
            const float s = scales[row];
            const auto fa = fragment(0, row, s);
            static_for<FN>([&](auto J) {
                constexpr int j = decltype(J)::value;
                const int of_b = wn * WTN + 16 * j;
                const float sb = scales[BM + of_b + lane % 16];
                const auto fb = fragment(B_AT, of_b + lane % 16, sb);
                if constexpr (SUMS == SUMS_FP32_POW2)
                    static_for<4>([&](auto Q) { acc[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb.v[decltype(Q)::value], fa.v[decltype(Q)::value], acc[j][i], 0, 0, 0); });
                else if constexpr (SUMS == SUMS_POW2) add_block_pow2(acc[j][i], fb, fa, scale_bits(sb), scale_bits(s));
                else add_block(acc[j][i], fb, fa, *reinterpret_cast<const floatx4 *>(scales + BM + of_b + 4 * (lane / 16)), s);
                __builtin_amdgcn_sched_barrier(0);           // (one after the other: the registers are taken)
            });
        });
    }
    __syncthreads();                      // nobody reads operands from LDS any more
    static_assert(STORE_REGION * W <= block_dma_lds<BM, BN, W, STAGES>(), "a region for every wavefront");
    store_tile(args, tile, acc, lds + wave * STORE_REGION, tile.m0 + wm * WTM, tile.n0 + wn * WTN, lane);
#else
    (void)args;
#endif
}

template <int MODE, int SUMS, int BM, int BN, int WM, int WN, int STAGES> hipError_t launch_block_dma_as(const BlockArgs &args, hipStream_t stream)
{
    constexpr int LDS = block_dma_lds<BM, BN, WM * WN, STAGES>();
    static bool raised = false;                   // raising the limit twice is harmless
    auto kernel = block_dma_kernel<MODE, SUMS, BM, BN, WM, WN, STAGES>;
    if (!raised) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
        if (e != hipSuccess) return e;
        raised = true;
    }
    const dim3 grid(static_cast<uint32_t>(args.tiles_m) * args.tiles_n, args.slices, MODE == BLOCK_SUM ? args.groups.count : 1);
    kernel<<<grid, WM * WN * 64, LDS, stream>>>(args);
    return hipGetLastError();
}

template <int MODE> hipError_t launch_block_dma(const BlockArgs &args, int sums, int tile, hipStream_t stream)
{
    if (tile == DMA_256) {
        if (sums == SUMS_POW2) return launch_block_dma_as<MODE, SUMS_POW2, 256, 256, 2, 4, 2>(args, stream);
        if constexpr (MODE != BLOCK_SUM) {                 // (sums over experts' rows have row blocks on both sides)
            if (sums == SUMS_SQUARE) return launch_block_dma_as<MODE, SUMS_SQUARE, 256, 256, 2, 4, 2>(args, stream);
        }
        if (sums == SUMS_ANY) return launch_block_dma_as<MODE, SUMS_ANY, 256, 256, 4, 2, 2>(args, stream);
        if (sums == SUMS_FP32_POW2) return launch_block_dma_as<MODE, SUMS_FP32_POW2, 256, 128, 4, 2, 2>(args, stream);
        return launch_block_dma_as<MODE, SUMS_FP32, 256, 128, 4, 2, 2>(args, stream);
    }
    if (tile == DMA_64) {
        if (sums == SUMS_POW2) return launch_block_dma_as<MODE, SUMS_POW2, 64, 64, 2, 2, 4>(args, stream);
        if (sums == SUMS_FP32_POW2) return launch_block_dma_as<MODE, SUMS_FP32_POW2, 64, 64, 2, 2, 4>(args, stream);
        if (sums == SUMS_FP32) return launch_block_dma_as<MODE, SUMS_FP32, 64, 64, 2, 2, 4>(args, stream);
        return launch_block_dma_as<MODE, SUMS_ANY, 64, 64, 2, 2, 4>(args, stream);
    }
    if (sums == SUMS_POW2) return launch_block_dma_as<MODE, SUMS_POW2, 128, 128, 2, 2, 2>(args, stream);
    if (sums == SUMS_FP32_POW2) return launch_block_dma_as<MODE, SUMS_FP32_POW2, 128, 128, 2, 2, 2>(args, stream);
    if (sums == SUMS_FP32) return launch_block_dma_as<MODE, SUMS_FP32, 128, 128, 2, 2, 2>(args, stream);
    return launch_block_dma_as<MODE, SUMS_ANY, 128, 128, 2, 2, 2>(args, stream);
}

}  // namespace mg
