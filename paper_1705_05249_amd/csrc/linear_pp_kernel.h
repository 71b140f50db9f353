// Products of 16-bit matrices on 256 x 256 tiles in which the two wavefronts that share a SIMD take turns: while one issues the matrix instructions of a K-tile
// from registers, the other fetches its operands of the next one from LDS and starts global -> LDS loads; a work-group barrier ends every turn.  The schedule is
// that of hgemm_pp_kernel (mfma_pp_kernel.h, where its turns and shares of the loads are drawn up), with Q as its A and P as its B; what is different is what
// linear_dma_kernel.h says: bfloat16, Q of two matrices, sizes that end inside a tile, what becomes of the sums; and P may lie across the sum, as two halves of 128 rows
// in LDS, since each half of the work-group reads one and its blocks are loaded apart from the other's.
// Measured, in us, against the kernel of linear_dma_kernel.h on the same tile: 4096 x 4096 x 8192 both along 226 -> 186 (1.48 PFLOP/s), 8192 x 2048 x 16384
// with Q across 484 -> 409; 8192^3 both across 947 -> 808 (1.36).
#pragma once

#include "linear_dma_kernel.h"

namespace mg {

// One operand tile (256 rows x 64 values of the sum): global -> LDS by the four wavefronts of one half of the work-group.  1 KB block b of the tile's LDS image
// belongs to wavefront b % 4 of the half, a wavefront's blocks Q = 0 .. 7 are blocks 4 Q + w.  Along the sum these are rows 32 Q + 8 w ..; across it
// lines 8 Q + 2 w .., whose swizzle repeats every second block.  GATED: w 0 and 1 have the gate matrix's features 16 Q + 8 w .., w 2 and 3 the up matrix's.
template <bool ALONG, bool GATED = false> struct LinearLoaderHalf {
    static constexpr uint32_t MISSING = 0x80000000u;
    uint32_t goff[2], other[2], now[2];
    int kpos;
    uint32_t step;                  // bytes between blocks Q and Q + 1 (across the sum: Q + 2)
    bool up;
    __amdgpu_buffer_rsrc_t rsrc;

    // as LinearLoader's
    __device__ inline void prepare(int64_t ld, int64_t ld1, int w, int lane, int left)
    {
        up = GATED && w >= 2;
        const int64_t mine = up ? ld1 : ld;
        if constexpr (ALONG) {
            const int r = 8 * w + lane / 8, chunk = lane % 8 ^ ldsmap::swizzle<16>(r), row = GATED ? r % 16 : r;
            kpos = chunk * 8;
            goff[0] = row < left ? static_cast<uint32_t>(row * mine * 2) + (chunk << 4) : MISSING;
            step = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>((GATED ? 16 : 32) * mine * 2));
        } else {
            static_for<2>([&](auto G) {
                constexpr int g = decltype(G)::value;
                const int kl = 8 * g + 2 * w + lane / 32, chunk = lane % 32 ^ ldsmap::line_swizzle(256, kl);
                goff[g] = chunk * 8 < left ? static_cast<uint32_t>(kl * ld * 2) + (chunk << 4) : MISSING;
                other[g] = chunk * 8 < left ? static_cast<uint32_t>(kl * ld1 * 2) + (chunk << 4) : MISSING;
            });
            step = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(16 * ld * 2));
        }
    }
    __device__ inline void aim(const _Float16 *X, int64_t ld, int64_t r0, int64_t l0, int left, int rows, bool second = false)
    {
        if constexpr (ALONG) {
            rsrc = linear_descriptor(X + r0 * ld + l0, rows < (GATED ? 128 : 256) ? rows : (GATED ? 128 : 256), ld, left);
            now[0] = kpos < left ? goff[0] : MISSING;
        } else {
            rsrc = linear_descriptor(X + r0 + l0 * ld, left < 64 ? left : 64, ld, rows);
            now[0] = second ? other[0] : goff[0];
            now[1] = second ? other[1] : goff[1];
            step = static_cast<uint32_t>(16 * ld * 2);
        }
    }
    // mine: this wavefront's block 0 in the destination stage (wave-uniform); flat: every block goes to `mine` itself (loads whose data nobody wants)
    template <int Q> __device__ inline void issue(lds_char *mine, bool flat = false) const
    {
        const uint32_t at = ALONG ? now[0] + Q * step : now[Q % 2] + (Q / 2) * step;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, reinterpret_cast<lds_void *>(mine + (flat ? 0 : Q * 4096)), 16, at, 0, 0, 0);
    }
};

// P across the sum, 256 columns in memory and two tiles of 128 in LDS (lines of 256 bytes, four to a block): blocks Q = 0 .. 3 of a wavefront are lines 16 Q + 4 w ..
// of the first, 4 .. 7 of the second.
struct LinearLoaderHalves {
    static constexpr uint32_t MISSING = 0x80000000u;
    uint32_t goff[2], step;
    __amdgpu_buffer_rsrc_t rsrc;

    __device__ inline void prepare(int64_t ld, int64_t, int w, int lane, int left)
    {
        const int kl = 4 * w + lane / 16, chunk = lane % 16 ^ ldsmap::line_swizzle(128, kl);
        static_for<2>([&](auto H) {
            constexpr int h = decltype(H)::value;
            goff[h] = 128 * h + chunk * 8 < left ? static_cast<uint32_t>(kl * ld * 2) + 256 * h + (chunk << 4) : MISSING;
        });
        step = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(16 * ld * 2));
    }
    __device__ inline void aim(const _Float16 *X, int64_t ld, int64_t r0, int64_t l0, int left, int rows)
    {
        rsrc = linear_descriptor(X + r0 + l0 * ld, left < 64 ? left : 64, ld, rows);
    }
    template <int Q> __device__ inline void issue(lds_char *mine, bool flat = false) const
    {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, reinterpret_cast<lds_void *>(mine + (flat ? 0 : Q * 4096)), 16, goff[Q / 4] + (Q % 4) * step, 0, 0, 0);
    }
};

// (as mma_in_place of mfma_pp_kernel.h, and for its reasons)
template <typename T> __device__ inline void multiply_in_place(floatx4 &acc, const u32x4 &frag_p, const u32x4 &frag_q)
{
    if constexpr (std::is_same_v<T, _Float16>) asm("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+v"(acc) : "v"(frag_q), "v"(frag_p));
    else asm("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+v"(acc) : "v"(frag_q), "v"(frag_p));
}

constexpr int LINEAR_PP_LDS = 4 * 32768 + 1024;

// PAST: what a block keeps (END_GATED, END_GATED_GRAD) or dz (END_SCORES_GRAD) passes the caches by
template <typename T, int FORM, int END, bool PAST> __global__ __launch_bounds__(512) void linear_pp_kernel(const LinearArgs args)
{
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr bool P_ALONG = FORM != FORM_NN, Q_ALONG = FORM == FORM_KK, GATED = END == END_GATED;
    constexpr int BC = 256, BR = 256, WC = 2, WR = 4, BK = 64, RB = 16, KSTEPS = 2;
    constexpr int WTC = BC / WC, WTR = BR / WR, FM = WTC / RB, FN = WTR / RB;
    using LoadQ = LinearLoaderHalf<Q_ALONG, GATED>;
    using LoadP = std::conditional_t<P_ALONG, LinearLoaderHalf<true>, LinearLoaderHalves>;
    constexpr int Q_BYTES = 32768, P_BYTES = 32768;              // LDS: [Q stage 0][Q stage 1][P stage 0][P stage 1][dump]
    constexpr int SLOTS = FM * FN, NMMA = KSTEPS * SLOTS, NM = 2, MEM_LOADS = 8 - NM;       // NM: loads a wavefront issues inside its run of MFMAs
    constexpr int REGION = end_region<WTC>(), DUMP = 2 * (Q_BYTES + P_BYTES);
    static_assert(WC * WR * REGION + WC * BR * 8 <= DUMP, "the end's memory lies in front of the dump area");

    extern __shared__ __attribute__((aligned(1024))) char lds[];
    lds_char *const lds3 = (lds_char *)lds;

    int tile_c, tile_r;
    tile_coords(blockIdx.x, args.tiles_c, args.tiles_r, 8, tile_c, tile_r);
    const int col0 = tile_c * BC, row0 = tile_r * BR;
    const int kb = blockIdx.z * args.k_per_slice, ke = kb + args.k_per_slice < args.k ? kb + args.k_per_slice : args.k;
    const int ktiles = (ke - kb + BK - 1) / BK;

    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int wc = wave % WC, wr = wave / WC;
    const int wave_u = __builtin_amdgcn_readfirstlane(wave), w4 = wave_u % 4;
    auto first_fragment = [&](bool along, int wrow, int base, int rows) {
        const int p = base + (along ? ldsmap::kcontig_base<RB>(lane, wrow) : ldsmap::transposed_base<RB>(lane, wrow, rows));
        return static_cast<uint32_t>(reinterpret_cast<uintptr_t>(lds3)) + static_cast<uint32_t>(p);
    };
    const uint32_t frag_q = first_fragment(Q_ALONG, wc * WTC, 0, BC);
    const uint32_t frag_p = P_ALONG ? first_fragment(true, wr * WTR, 2 * Q_BYTES, BR) : first_fragment(false, wr % 2 * WTR, 2 * Q_BYTES + wr / 2 * (P_BYTES / 2), BR / 2);

    floatx4 acc[FN][FM];
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int i = 0; i < FM; ++i) acc[j][i] = floatx4{0.f, 0.f, 0.f, 0.f};

    lds_char *const dump = lds3 + DUMP;
    auto fence = [] { __builtin_amdgcn_sched_barrier(0); };
    // until at most LEFT of this wavefront's loads are outstanding (they return in order)
    auto wait_loads = [&](auto LEFT) { __builtin_amdgcn_s_waitcnt(0x0F70 + decltype(LEFT)::value); fence(); };
    auto wait_reads = [&] { __builtin_amdgcn_s_waitcnt(0xC07F); fence(); };         // lgkmcnt(0)
    auto barrier = [&] { fence(); __builtin_amdgcn_s_barrier(); fence(); };

    u32x4 fq[KSTEPS][FM], fp[KSTEPS][FN];
    auto read_tile = [&](auto PAR) __attribute__((always_inline)) {                  // mem(t): every operand of the K-tile in stage PAR
        constexpr int par = decltype(PAR)::value;
        static_for<KSTEPS>([&](auto S) {
            constexpr int s = decltype(S)::value;
            static_for<FN>([&](auto F) { fp[s][decltype(F)::value] = read_linear<P_ALONG, P_ALONG ? BR : BR / 2, decltype(F)::value, s, par * P_BYTES>(frag_p); });
            static_for<FM>([&](auto F) { fq[s][decltype(F)::value] = read_linear<Q_ALONG, BC, decltype(F)::value, s, par * Q_BYTES>(frag_q); });
        });
    };
    // the MFMAs of one K-tile; between(i) may issue a load after MFMA i
    auto mma_tile = [&](auto &&between) __attribute__((always_inline)) {
        fence();
        __builtin_amdgcn_s_setprio(2);
        static_for<KSTEPS>([&](auto S) __attribute__((always_inline)) {
            constexpr int s = decltype(S)::value;
            static_for<SLOTS>([&](auto N) __attribute__((always_inline)) {
                constexpr int q = decltype(N)::value;
                multiply_in_place<T>(acc[q / FM][q % FM], fp[s][q / FM], fq[s][q % FM]);
                between(std::integral_constant<int, s * SLOTS + q>{});
                fence();
            });
        });
        __builtin_amdgcn_s_setprio(0);
        fence();
    };
    using Stage0 = std::integral_constant<int, 0>;
    using Stage1 = std::integral_constant<int, 1>;
    // all K-tiles, two per round of the loop (compile-time LDS stages)
    auto run_tiles = [&](auto &&turn_pair) __attribute__((always_inline)) {
        int t = 0;
        for (; t + 1 < ktiles; t += 2) {
            turn_pair(Stage0{}, t);
            turn_pair(Stage1{}, t + 1);
        }
        if (t < ktiles) turn_pair(Stage0{}, t);
    };

    if (ktiles > 0) {
        const _Float16 *const P = static_cast<const _Float16 *>(args.P), *const Q0 = static_cast<const _Float16 *>(args.Q0), *const Q1 = static_cast<const _Float16 *>(args.Q1);
        LoadQ lq;
        LoadP lp;
        lq.prepare(args.ldq0, args.ldq1, w4, lane, GATED ? args.hidden - col0 / 2 : args.cols - col0);
        lp.prepare(args.ldp, args.ldp, w4, lane, args.rows - row0);
        lds_char *const mine_q = lds3 + w4 * 1024;
        lds_char *const mine_p = lds3 + 2 * Q_BYTES + w4 * 1024;
        // l: the K-tile's first value; left: how many there are from it on (behind the end none: zeros, without memory being touched)
        auto place = [&](int t, int &l, int &left, bool &second) {
            l = kb + t * BK;
            left = ke - l;
            if (left <= 0) l = kb;
            second = false;
            if constexpr (FORM == FORM_KN && END == END_STORE) {
                second = args.segment > 0 && l >= args.segment;
                const int line = second ? l - args.segment : l;
                if (args.segment > 0 && args.lines - line < left) left = args.lines - line;
            }
        };
        auto aim_q = [&](int t) {
            int l, left;
            bool second;
            place(t, l, left, second);
            if constexpr (GATED) lq.aim(lq.up ? Q1 : Q0, lq.up ? args.ldq1 : args.ldq0, col0 / 2, l, left, args.hidden - col0 / 2);
            else lq.aim(second ? Q1 : Q0, second ? args.ldq1 : args.ldq0, col0, second ? l - args.segment : l, left, args.cols - col0, second);
        };
        auto aim_p = [&](int t) {
            int l, left;
            bool second;
            place(t, l, left, second);
            lp.aim(P, args.ldp, row0, l, left, args.rows - row0);
        };
        // piece J (0..7) of a turn's P loads: J < 4 -> block 4 + J of P(t+1) (rows 128-255), else block J - 4 of P(t+2)
        auto issue_p = [&](auto J, lds_char *to1, lds_char *to2) {
            constexpr int j = decltype(J)::value;
            if constexpr (j < 4) lp.template issue<4 + j>(to1, to1 == dump);
            else lp.template issue<j - 4>(to2, to2 == dump);
        };
        constexpr int GAP = NMMA / NM;
        if (wave_u < 4) {
            aim_q(0);
            static_for<8>([&](auto N) { lq.template issue<decltype(N)::value>(mine_q); });
            wait_loads(std::integral_constant<int, 0>{});
            barrier();
            auto turn_pair = [&](auto CUR, int t) __attribute__((always_inline)) {          // turns 2t and 2t+1
                using Cur = decltype(CUR);
                constexpr int cur = Cur::value, nxt = 1 - cur;
                lds_char *const q1 = t + 1 < ktiles ? mine_q + nxt * Q_BYTES : dump;      // wave-uniform selects
                lds_char *const p1 = t + 1 < ktiles ? mine_p + nxt * P_BYTES : dump;
                lds_char *const p2 = t + 2 < ktiles ? mine_p + cur * P_BYTES : dump;
                read_tile(Cur{});
                aim_q(t + 1);
                static_for<MEM_LOADS>([&](auto N) { lq.template issue<decltype(N)::value>(q1, q1 == dump); });
                wait_reads();
                wait_loads(std::integral_constant<int, MEM_LOADS>{});                      // the P pieces of the run before
                barrier();
                aim_p(t + 2);
                mma_tile([&](auto I) __attribute__((always_inline)) {
                    constexpr int i = decltype(I)::value;
                    if constexpr (i % GAP == GAP / 2) issue_p(std::integral_constant<int, MEM_LOADS + i / GAP>{}, p1, p2);
                });
                wait_loads(std::integral_constant<int, NM>{});                             // the Q pieces of this tile's mem turn
                barrier();
            };
            run_tiles(turn_pair);
        } else {
            aim_p(0);
            static_for<8>([&](auto N) { lp.template issue<decltype(N)::value>(mine_p); });
            aim_p(1);
            {
                lds_char *const p1 = 1 < ktiles ? mine_p + P_BYTES : dump;
                static_for<4>([&](auto N) { lp.template issue<decltype(N)::value>(p1, p1 == dump); });
            }
            wait_loads(std::integral_constant<int, 0>{});
            barrier();
            {                                                   // turn 0: this half's share of Q(1)
                lds_char *const q1 = 1 < ktiles ? mine_q + Q_BYTES : dump;
                aim_q(1);
                static_for<NM>([&](auto N) { lq.template issue<MEM_LOADS + decltype(N)::value>(q1, q1 == dump); });
            }
            barrier();
            auto turn_pair = [&](auto CUR, int t) __attribute__((always_inline)) {          // turns 2t+1 and 2t+2
                using Cur = decltype(CUR);
                constexpr int cur = Cur::value, nxt = 1 - cur;
                lds_char *const p1 = t + 1 < ktiles ? mine_p + nxt * P_BYTES : dump;
                lds_char *const p2 = t + 2 < ktiles ? mine_p + cur * P_BYTES : dump;
                lds_char *const q2 = t + 2 < ktiles ? mine_q + cur * Q_BYTES : dump;
                read_tile(Cur{});
                aim_p(t + 1);
                static_for<MEM_LOADS>([&](auto J) {
                    if constexpr (decltype(J)::value == 4) aim_p(t + 2);
                    issue_p(J, p1, p2);
                });
                wait_reads();
                wait_loads(std::integral_constant<int, MEM_LOADS>{});                      // the Q pieces of the run before
                barrier();
                aim_q(t + 2);
                mma_tile([&](auto I) __attribute__((always_inline)) {
                    constexpr int i = decltype(I)::value;
                    if constexpr (i % GAP == GAP / 2) lq.template issue<MEM_LOADS + i / GAP>(q2, q2 == dump);
                });
                wait_loads(std::integral_constant<int, NM>{});                             // the P pieces of this tile's mem turn
                if (t + 1 < ktiles) barrier();                 // the last run of MFMAs ends the K loop
            };
            run_tiles(turn_pair);
        }
    }
    // Every operand read of the work-group is complete (the first half has passed the barrier that ends the last mem turn of the second half), and loads in flight
    // go to the dump area: each wavefront may use its own region of the LDS.  The last MFMAs (16 passes at most) must have written their results before
    // anything reads them.
    asm volatile("s_nop 15\n\ts_nop 15");
    fence();
    linear_end<T, END, FM, FN, WR, WC, PAST>(args, acc, lds + wave * REGION, reinterpret_cast<float2 *>(lds + WC * WR * REGION), row0, col0, wr, wc, lane, blockIdx.z);
    __builtin_amdgcn_s_waitcnt(0x0F70);
#else
    (void)args;
#endif
}

template <typename T, int FORM, int END, bool PAST> hipError_t launch_linear_pp_as(LinearArgs args, int slices, hipStream_t stream)
{
    static RaisedLds raised;
    auto kernel = linear_pp_kernel<T, FORM, END, PAST>;
    if (const hipError_t e = raised(reinterpret_cast<const void *>(kernel), LINEAR_PP_LDS)) return e;
    args.tiles_c = (args.cols + 255) / 256;
    args.tiles_r = (args.rows + 255) / 256;
    kernel<<<dim3(static_cast<uint32_t>(args.tiles_c) * args.tiles_r, 1, slices), 512, LINEAR_PP_LDS, stream>>>(args);
    return hipGetLastError();
}

// What does not stay in the last-level cache (256 MB) until the backward pass comes for it leaves it to what does.  302 MB (8192 x 8192 elements in bfloat16): the forward product of
// width 2048 453 -> 438 us, the backward one 294 -> 279; 52 MB: backward 39.7 through the caches and 42.3 past them.  dz of 256 MB and more: the step of the loss of
// 8192 x 2048 x 65536, 537 MB a piece, 6633 -> 6545 us.
template <typename T, int FORM, int END> hipError_t launch_linear_pp(const LinearArgs &args, int slices, hipStream_t stream)
{
    if constexpr (END == END_GATED || END == END_GATED_GRAD)
        if (args.kept != nullptr && kept_blocks(args.hidden) * ((args.rows + 15) / 16) * kept_block_bytes(std::is_same_v<T, bfloat> ? MG_BF16 : MG_F16) >= int64_t(128) << 20)
            return launch_linear_pp_as<T, FORM, END, true>(args, slices, stream);
    if constexpr (END == END_SCORES_GRAD)
        if (static_cast<int64_t>(args.rows) * args.cols >= int64_t(1) << 27) return launch_linear_pp_as<T, FORM, END, true>(args, slices, stream);
    return launch_linear_pp_as<T, FORM, END, false>(args, slices, stream);
}

}  // namespace mg
