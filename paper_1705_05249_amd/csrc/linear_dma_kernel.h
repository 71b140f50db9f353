// Products of 16-bit matrices whose rows start on 16 bytes: operand tiles go from global memory straight into LDS.
//
// Loads, LDS layouts, fragment reads and the order of the K loop are those of hgemm_dma_tile (mfma_dma_kernel.h), with Q as its A and P as its B: the
// instruction's output registers run along C's columns, its lanes along C's rows.  What is different: bfloat16 beside FP16, Q of two matrices (gate and up
// weights, 16 rows of each in turn; the two halves of a sum), and what becomes of the sums (linear_end.h).  Every size may end inside a tile: lanes whose
// 16 bytes do not exist name an offset outside the descriptor, for which zeros arrive without memory being touched.
#pragma once

#include "linear_end.h"
#include "mfma_dma_kernel.h"

namespace mg {

typedef __bf16 bfloatx8 __attribute__((ext_vector_type(8)));
__device__ inline void mma(floatx4 &acc, const u32x4 &frag_n, const u32x4 &frag_m, bfloat)
{
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bfloatx8, frag_m), __builtin_bit_cast(bfloatx8, frag_n), acc, 0, 0, 0);
}

// `rows` rows of `ld` elements in reach of a descriptor, the last one `last` long (in whole pieces: what a range cuts is lost in words)
__device__ inline __amdgpu_buffer_rsrc_t linear_descriptor(const _Float16 *base, int64_t rows, int64_t ld, int last)
{
    const int64_t range = ((rows - 1) * ld + (last + 7) / 8 * 8) * 2;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<_Float16 *>(base), 0, rows <= 0 || last <= 0 ? 0 : static_cast<int>(range < 0x7fffffff ? range : 0x7fffffff), 0x00020000);
}

// One operand tile, ROWS rows x 64 values of the sum: global -> LDS, in blocks of 1 KB that a wavefront's instruction fills; a wavefront has COUNT
// consecutive ones.  The swizzles of lds_layout.h repeat: two lane offsets (`group`) and a multiple of a scalar step name the place of every block.
//   along the sum:    eight rows a block, 16 rows a step; what lies behind the sum's end in a row is left out by the lane's place in the K-tile, rows
//                     behind the last one by the descriptor's range;
//   across it:        1024 / (2 ROWS) lines a block, four lines a step; columns behind the last one by a lane offset outside the range, lines by the range.
// ONCE: the operand is read once in a call and not kept in the caches (the 134 MB of a served token's gate and up weights: 28.8 -> 25.5 us).
// GATED (along the sum): rows 32 f .. 32 f + 15 of the tile are features 16 f .. of the gate matrix, the next 16 the same features of the up matrix.
template <int ROWS, int NT, bool ALONG, bool GATED = false, bool ONCE = false> struct LinearLoader {
    static constexpr int AUX = ONCE ? 2 : 0;            // nontemporal
    static constexpr int LDS_BYTES = ROWS * 128;
    static constexpr int COUNT = LDS_BYTES / (NT * 16);
    static constexpr uint32_t MISSING = 0x80000000u;                // no range is that long; no step carries it past 2^32
    static_assert((COUNT == 2 || COUNT == 4 || (COUNT == 8 && ALONG && !GATED)) && COUNT * NT * 16 == LDS_BYTES && (ALONG || !GATED), "tile / work-group size");
    static constexpr int group(int q) { return ALONG ? q % 2 : ROWS == 128 ? q / 2 : q; }
    static constexpr int steps(int q) { return ALONG ? q / 2 : ROWS == 128 ? q % 2 : 0; }

    uint32_t goff[2], now[2];           // lane's byte offset of a group's first block; what the K-tile aimed at makes of it
    uint32_t other[2];                  // the same in a second matrix
    int kpos[2];                        // ALONG: the lane's first value of the sum inside the K-tile
    uint32_t step;                      // bytes
    bool up;                            // GATED, COUNT 2: this wavefront's rows are of the up matrix
    __amdgpu_buffer_rsrc_t rsrc, rsrc_up;

    // left: rows of the operand (GATED: features) from the tile's first one on; ld1: of the second matrix (GATED: up)
    __device__ inline void prepare(int64_t ld, int64_t ld1, int wave, int lane, int left)
    {
        up = GATED && COUNT == 2 && __builtin_amdgcn_readfirstlane(wave) % 2 != 0;
        static_for<2>([&](auto G) {
            constexpr int g = decltype(G)::value;
            const int q = ALONG || ROWS != 128 ? g : 2 * g;                         // the group's first block
            const int o = (wave * COUNT + q) * 1024 + lane * 16;
            if constexpr (ALONG) {
                const int r = o / 128, chunk = (o / 16) % 8 ^ ldsmap::swizzle<16>(r);
                const int row = GATED ? r / 32 * 16 + r % 16 : r;
                kpos[g] = chunk * 8;
                goff[g] = static_cast<uint32_t>(row * (up ? ld1 : ld) * 2) + (chunk << 4);
                other[g] = static_cast<uint32_t>(row * ld1 * 2) + (chunk << 4);
                if (row >= left) goff[g] = other[g] = MISSING;                      // (of an operand of fewer rows than a group's)
            } else {
                const int kl = o / (2 * ROWS), chunk = (o / 16) % (ROWS / 8) ^ ldsmap::line_swizzle(ROWS, kl);
                goff[g] = chunk * 8 < left ? static_cast<uint32_t>(kl * ld * 2) + (chunk << 4) : MISSING;
                other[g] = chunk * 8 < left ? static_cast<uint32_t>(kl * ld1 * 2) + (chunk << 4) : MISSING;
            }
        });
        step = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>((ALONG ? 16 : 4) * ld * 2));
    }
    // The K-tile that starts at value l0 of the sum, of which `left` are there (none: zeros).  rows: of the operand from r0 on (GATED: features).
    __device__ inline void aim(const _Float16 *X, int64_t ld, int64_t r0, int64_t l0, int left, int rows, bool second = false)
    {
        if constexpr (ALONG) {
            rsrc = linear_descriptor(X + r0 * ld + l0, rows < ROWS ? rows : ROWS, ld, left);
            now[0] = kpos[0] < left ? goff[0] : MISSING;
            now[1] = kpos[1] < left ? goff[1] : MISSING;
        } else {
            rsrc = linear_descriptor(X + r0 + l0 * ld, left < 64 ? left : 64, ld, rows);
            now[0] = second ? other[0] : goff[0];
            now[1] = second ? other[1] : goff[1];
            step = static_cast<uint32_t>(4 * ld * 2);                               // (the matrices' rows need not be equally far apart)
        }
    }
    __device__ inline void aim_gated(const _Float16 *gate, int64_t ldg, const _Float16 *upper, int64_t ldu, int64_t feature, int64_t l0, int left, int features)
    {
        const int rows = features < ROWS / 2 ? features : ROWS / 2;
        rsrc = linear_descriptor(gate + feature * ldg + l0, rows, ldg, left);
        rsrc_up = linear_descriptor(upper + feature * ldu + l0, rows, ldu, left);
        if (COUNT == 2 && up) rsrc = rsrc_up;
    }
    // mine: this wavefront's first block in the destination stage (wave-uniform); left: values of the sum from the K-tile's first one on (GATED)
    template <int Q> __device__ inline void issue(lds_char *mine, int left) const
    {
        constexpr int g = group(Q);
        if constexpr (GATED) {
            constexpr bool UP = COUNT == 4 && Q >= 2;
            const uint32_t at = kpos[g] < left ? (UP ? other[g] : goff[g]) : MISSING;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(UP ? rsrc_up : rsrc, reinterpret_cast<lds_void *>(mine + Q * 1024), 16, at, 0, 0, AUX);
        } else {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, reinterpret_cast<lds_void *>(mine + Q * 1024), 16, now[g] + steps(Q) * step, 0, 0, AUX);
        }
    }
};

// MFMA operand of fragment F, K-step S, from the operand stage at byte offset STAGE; `at`: the lane's LDS address of fragment 0, step 0
template <bool ALONG, int ROWS, int F, int S, int STAGE> __device__ inline u32x4 read_linear(uint32_t at)
{
    if constexpr (ALONG) {
        constexpr int OFFSET = F * 16 * 128 + STAGE, FAR = OFFSET >= 65536 ? OFFSET / 32768 * 32768 : 0;
        return lds_read_b128_untracked<OFFSET - FAR>((at ^ static_cast<uint32_t>(ldsmap::kcontig_xor<16>(F, S))) + FAR);
    } else {
        constexpr int LINE = 2 * ROWS, OFFSET = S * (32 * LINE) + STAGE, FAR = OFFSET + 4 * LINE >= 65536 ? OFFSET / 32768 * 32768 : 0;
        // (the fragment's address is made beside its reads: the compiler would otherwise hold all of them in registers through the K loop, and spill)
        static_assert(FAR == 0 || (FAR & 0xff) == 0, "the XOR stays below what is added");
        shortx4 lo, hi;
        uint32_t ax;
        asm volatile("v_xor_b32 %2, %6, %3\n\tds_read_b64_tr_b16 %0, %2 offset:%4\n\tds_read_b64_tr_b16 %1, %2 offset:%5"
                     : "=&v"(lo), "=&v"(hi), "=&v"(ax)
                     : "v"(FAR != 0 ? at + FAR : at), "n"(OFFSET - FAR), "n"(OFFSET - FAR + 4 * LINE), "n"(ldsmap::transposed_xor<16>(F))
                     : "memory");
        return __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
}

// BC x BR: columns and rows of a work-group's tile; WC x WR wavefronts.  FORM, END: LinearForm, LinearEnd.  group: among the tiles of a slice.
// HALVES 2: twice the wavefronts, two sets that take K-tiles in turn, each with LDS of its own, and share the end.  For launches that leave a compute unit one tile of 64: alone, a K-tile there waits
// for itself from load to matrix instruction (0.3 us), and two at a time take hardly longer.
template <typename T, int FORM, int END, int BC, int BR, int WC, int WR, int STAGES, int HALVES> __device__ __forceinline__ void linear_dma_tile(const LinearArgs &args, int group, int slice)
{
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr bool P_ALONG = FORM != FORM_NN, Q_ALONG = FORM == FORM_KK;
    constexpr bool GATED = END == END_GATED;
    constexpr int RB = 16, BK = 64, NT = WC * WR * 64;
    constexpr int WTC = BC / WC, WTR = BR / WR;
    constexpr int FM = WTC / RB, FN = WTR / RB, KSTEPS = 2;
    using LoadQ = LinearLoader<BC, NT, Q_ALONG, GATED>;
    using LoadP = LinearLoader<BR, NT, P_ALONG>;
    constexpr int Q_BYTES = LoadQ::LDS_BYTES, P_BYTES = LoadP::LDS_BYTES;        // LDS: [Q stage 0][Q stage 1] ... [P stage 0] ...
    constexpr int SLOTS = FM * FN, FRAGS = FM + FN, PIECES = LoadQ::COUNT + LoadP::COUNT;

    constexpr int HALF_BYTES = STAGES * (Q_BYTES + P_BYTES);
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int half = HALVES == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / NT);
    lds_char *const lds3 = (lds_char *)lds + half * HALF_BYTES;

    int tile_c, tile_r;
    tile_coords(group, args.tiles_c, args.tiles_r, 8, tile_c, tile_r);
    const int col0 = tile_c * BC, row0 = tile_r * BR;
    const int kb = slice * args.k_per_slice, ke = kb + args.k_per_slice < args.k ? kb + args.k_per_slice : args.k;
    const int ktiles = (ke - kb + BK * HALVES - 1) / (BK * HALVES);

    const int lane = threadIdx.x % 64, wave = threadIdx.x % NT / 64;
    const int wc = wave % WC, wr = wave / WC;
    const int wave_u = __builtin_amdgcn_readfirstlane(wave);

    auto first_fragment = [&](bool along, int wrow, int base, int rows) {
        const int p = base + (along ? ldsmap::kcontig_base<RB>(lane, wrow) : ldsmap::transposed_base<RB>(lane, wrow, rows));
        return static_cast<uint32_t>(reinterpret_cast<uintptr_t>(lds3)) + static_cast<uint32_t>(p);
    };
    const uint32_t frag_q = first_fragment(Q_ALONG, wc * WTC, 0, BC), frag_p = first_fragment(P_ALONG, wr * WTR, STAGES * Q_BYTES, BR);

    floatx4 acc[FN][FM];
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int i = 0; i < FM; ++i) acc[j][i] = floatx4{0.f, 0.f, 0.f, 0.f};

    const _Float16 *const P = static_cast<const _Float16 *>(args.P), *const Q0 = static_cast<const _Float16 *>(args.Q0), *const Q1 = static_cast<const _Float16 *>(args.Q1);
    LoadQ lq;
    LoadP lp;
    lq.prepare(args.ldq0, args.ldq1, wave, lane, GATED ? args.hidden - col0 / 2 : args.cols - col0);
    lp.prepare(args.ldp, args.ldp, wave, lane, args.rows - row0);
    int left = 0;                               // values of the sum from the K-tile aimed at on
    auto aim_tile = [&](int t) {
        int l0 = kb + (t * HALVES + half) * BK;
        left = ke - l0;                         // (behind the end nothing is fetched)
        if (left <= 0) l0 = kb;
        if constexpr (GATED) {
            lq.aim_gated(Q0, args.ldq0, Q1, args.ldq1, col0 / 2, l0, left, args.hidden - col0 / 2);
        } else if constexpr (FORM == FORM_KN && END == END_STORE) {
            const bool second = args.segment > 0 && l0 >= args.segment;
            const int line = second ? l0 - args.segment : l0;
            if (args.segment > 0 && args.lines - line < left) left = args.lines - line;
            lq.aim(second ? Q1 : Q0, second ? args.ldq1 : args.ldq0, col0, line, left, args.cols - col0, second);
        } else {
            lq.aim(Q0, args.ldq0, col0, l0, left, args.cols - col0);
        }
        lp.aim(P, args.ldp, row0, l0, left, args.rows - row0);
    };
    lds_char *const mine_q = lds3 + wave_u * (LoadQ::COUNT * 1024);
    lds_char *const mine_p = lds3 + STAGES * Q_BYTES + wave_u * (LoadP::COUNT * 1024);
    auto issue_piece = [&](auto N, auto PAR) {          // piece N of the tile aimed at, into stage PAR
        constexpr int n = decltype(N)::value, par = decltype(PAR)::value;
        if constexpr (n < LoadQ::COUNT) lq.template issue<n>(mine_q + par * Q_BYTES, left);
        else lp.template issue<n - LoadQ::COUNT>(mine_p + par * P_BYTES, left);
    };
    constexpr int AHEAD = (STAGES - 2) * PIECES;
    static_assert(STAGES >= 2 && AHEAD < 64, "six bits of the wait count");
    auto wait_loads = [] { __builtin_amdgcn_s_waitcnt(0x0F70 | (AHEAD & 15) | (AHEAD / 16) << 14); };

    u32x4 fq[2][FM], fp[2][FN];
    auto read_frag = [&](auto F, auto PAR, auto S, int buf) {
        constexpr int f = decltype(F)::value, par = decltype(PAR)::value, s = decltype(S)::value;
        if constexpr (f < FM) fq[buf][f] = read_linear<Q_ALONG, BC, f, s, par * Q_BYTES>(frag_q);
        else fp[buf][f - FM] = read_linear<P_ALONG, BR, f - FM, s, par * P_BYTES>(frag_p);
    };
    auto wait_fragments = [] {                   // (the compiler does not know that the reads are in flight)
        __builtin_amdgcn_s_waitcnt(0xC07F);      // lgkmcnt(0)
        __builtin_amdgcn_sched_barrier(0);
    };
    using Step0 = std::integral_constant<int, 0>;
    using Stage0 = std::integral_constant<int, 0>;
    // (a barrier with the memory model's fences would wait for every load in flight)
    auto barrier = [] {
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
    };

    if (ktiles > 0) {
        static_for<STAGES - 1>([&](auto PAR) {
            aim_tile(decltype(PAR)::value);
            static_for<PIECES>([&](auto N) { issue_piece(N, PAR); });
        });
        wait_loads();
        barrier();
        static_for<FRAGS>([&](auto F) { read_frag(F, Stage0{}, Step0{}, 0); });
    }
    constexpr int TAIL = (SLOTS * MG_TAIL_SIXTEENTHS / 16) > 0 ? (SLOTS * MG_TAIL_SIXTEENTHS / 16) : 1;
    constexpr int BARRIER_SLOT = KSTEPS * SLOTS - TAIL;
    constexpr int READ_SLOTS = SLOTS >= 4 ? SLOTS * 3 / 4 : SLOTS;
    constexpr int TAIL_READ_SLOTS = TAIL >= 4 ? TAIL * 3 / 4 : TAIL;
    constexpr int PER_SLOT = (PIECES + BARRIER_SLOT - 1) / BARRIER_SLOT;     // loads issued in a slot of the first ones
    auto tile_body = [&](auto CUR, int t) __attribute__((always_inline)) {        // (too large for the inliner to do so by itself)
        using Cur = decltype(CUR);
        using Nxt = std::integral_constant<int, (Cur::value + 1) % STAGES>;
        using Far = std::integral_constant<int, (Cur::value + STAGES - 1) % STAGES>;      // read last one tile ago
        aim_tile(t + STAGES - 1);
        static_for<KSTEPS>([&](auto S) {
            constexpr int s = decltype(S)::value;
            static_for<SLOTS>([&](auto N) {
                constexpr int q = decltype(N)::value, g = s * SLOTS + q;
                if constexpr (g == BARRIER_SLOT) {
                    wait_loads();
                    barrier();                           // tile t+1 is complete in its stage
                }
                if constexpr (q == 0) wait_fragments();  // this step's operands, read during the previous step
                mma(acc[q / FM][q % FM], fp[s & 1][q / FM], fq[s & 1][q % FM], T{});
                if constexpr (s + 1 < KSTEPS) {
                    if constexpr (q < READ_SLOTS)
                        static_for<share_begin(q + 1, FRAGS, READ_SLOTS) - share_begin(q, FRAGS, READ_SLOTS)>([&](auto R) {
                            constexpr int o = share_begin(q, FRAGS, READ_SLOTS) + decltype(R)::value;
                            constexpr int f = o < FM ? o : FM + (FRAGS - 1 - o);
                            read_frag(std::integral_constant<int, f>{}, Cur{}, std::integral_constant<int, s + 1>{}, (s + 1) & 1);
                        });
                } else if constexpr (g >= BARRIER_SLOT && g - BARRIER_SLOT < TAIL_READ_SLOTS) {
                    constexpr int h = g - BARRIER_SLOT;
                    static_for<share_begin(h + 1, FRAGS, TAIL_READ_SLOTS) - share_begin(h, FRAGS, TAIL_READ_SLOTS)>([&](auto R) {
                        constexpr int o = share_begin(h, FRAGS, TAIL_READ_SLOTS) + decltype(R)::value;
                        constexpr int f = o < FM ? o : FM + (FRAGS - 1 - o);
                        read_frag(std::integral_constant<int, f>{}, Nxt{}, Step0{}, 0);
                    });
                }
                static_for<PER_SLOT>([&](auto R) {
                    constexpr int n = g * PER_SLOT + decltype(R)::value;
                    if constexpr (n < PIECES) issue_piece(std::integral_constant<int, n>{}, Far{});
                });
                __builtin_amdgcn_sched_barrier(0);
            });
        });
    };
    int t = 0;
    for (; t + STAGES - 1 < ktiles; t += STAGES) static_for<STAGES>([&](auto CUR) __attribute__((always_inline)) { tile_body(CUR, t + decltype(CUR)::value); });
    static_for<STAGES - 1>([&](auto CUR) __attribute__((always_inline)) {
        if (t + decltype(CUR)::value < ktiles) tile_body(CUR, t + decltype(CUR)::value);
    });

    __builtin_amdgcn_s_waitcnt(0x0F70);          // the loads behind the end of the sum
    wait_fragments();                            // the reads issued behind the last barrier still write registers: let them land
    hold_registers(fq[0]);
    hold_registers(fp[0]);
    __syncthreads();        // all loads have landed and all fragment reads are done
    constexpr int REGION = end_region<WTC>();
    if constexpr (HALVES == 1) {
        linear_end<T, END, FM, FN, WR, WC>(args, acc, lds + wave * REGION, reinterpret_cast<float2 *>(lds + WC * WR * REGION), row0, col0, wr, wc, lane, slice);
    } else {
        // each set leaves the other one its sums of a half of the rows
        static_assert(HALVES == 2 && FN == 2, "a row of blocks for each");
        end_floatx4 *const sums = reinterpret_cast<end_floatx4 *>(lds);
        end_floatx4 mine[1][FM];
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            sums[((half * WC * WR + wave) * FM + i) * 64 + lane] = half == 0 ? acc[1][i] : acc[0][i];
            mine[0][i] = half == 0 ? acc[0][i] : acc[1][i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < FM; ++i) mine[0][i] += sums[(((1 - half) * WC * WR + wave) * FM + i) * 64 + lane];
        constexpr int SUMS = HALVES * WC * WR * FM * 1024;
        linear_end<T, END, FM, 1, WR * 2, WC>(args, mine, lds + SUMS + (half * WC * WR + wave) * REGION, reinterpret_cast<float2 *>(lds + SUMS + 2 * WC * WR * REGION), row0, col0,
                                              wr * 2 + half, wc, lane, slice);
    }
#else
    (void)args, (void)group, (void)slice;
#endif
}

template <typename T, int FORM, int END, int BC, int BR, int WC, int WR, int STAGES, int HALVES> __global__ __launch_bounds__(WC *WR *HALVES * 64) void linear_dma_kernel(const LinearArgs args)
{
    linear_dma_tile<T, FORM, END, BC, BR, WC, WR, STAGES, HALVES>(args, blockIdx.x, blockIdx.z);
}

template <int BC, int BR, int WC, int WR, int STAGES> constexpr int linear_dma_lds()
{
    const int stages = STAGES * (BC + BR) * 128, end = WC * WR * end_region<BC / WC>() + WC * BR * 8;
    return stages > end ? stages : end;
}

template <typename T, int FORM, int END, int BC, int BR, int WC, int WR, int STAGES, int HALVES> hipError_t launch_linear_dma_as(LinearArgs args, int slices, hipStream_t stream)
{
    constexpr int LDS = HALVES * linear_dma_lds<BC, BR, WC, WR, STAGES>();
    static_assert(LDS <= 160 * 1024, "LDS of a compute unit");
    static RaisedLds raised;
    auto kernel = linear_dma_kernel<T, FORM, END, BC, BR, WC, WR, STAGES, HALVES>;
    if (const hipError_t e = raised(reinterpret_cast<const void *>(kernel), LDS)) return e;
    args.tiles_c = (args.cols + BC - 1) / BC;
    args.tiles_r = (args.rows + BR - 1) / BR;
    kernel<<<dim3(static_cast<uint32_t>(args.tiles_c) * args.tiles_r, 1, slices), WC * WR * HALVES * 64, LDS, stream>>>(args);
    return hipGetLastError();
}

template <typename T, int FORM, int END> hipError_t launch_linear_pp(const LinearArgs &args, int slices, hipStream_t stream);      // linear_pp_kernel.h

// the kernels of one form and end, all tiles
template <int FORM, int END> hipError_t launch_linear_dma(int dtype, int tile, const LinearArgs &args, int slices, hipStream_t stream)
{
    auto with = [&](auto type) {
        using T = decltype(type);
        if (tile == LINEAR_256) return launch_linear_pp<T, FORM, END>(args, slices, stream);
        if (tile == LINEAR_128) return launch_linear_dma_as<T, FORM, END, 128, 128, 2, 2, 2, 1>(args, slices, stream);
        if (tile == LINEAR_128_DEEP) return launch_linear_dma_as<T, FORM, END, 128, 128, 2, 2, 4, 1>(args, slices, stream);
        if (tile == LINEAR_64_TWICE) return launch_linear_dma_as<T, FORM, END, 64, 64, 2, 2, 4, 2>(args, slices, stream);
        return launch_linear_dma_as<T, FORM, END, 64, 64, 2, 2, 4, 1>(args, slices, stream);
    };
    return dtype == MG_F16 ? with(_Float16{}) : with(bfloat{});
}

}  // namespace mg
