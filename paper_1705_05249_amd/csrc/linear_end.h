// What becomes of the sums of a product (LinearEnd): from the registers of a wavefront's tile to memory.
//
// acc[j][i] is the 16 x 16 block of rows row0 + 16 j and columns col0 + 16 i: lane l holds row l % 16, columns 4 (l / 16) .. + 3.  Stored from there, a
// wavefront's store would write 16 pieces of 8 bytes in each of 16 rows; the rows of a block go through LDS instead, so that a store instruction
// writes 16 bytes a lane and rows of the wavefront's tile whole (4096 x 4096 in bfloat16 behind one K-tile of an 8-bit product: 29 us from registers, 11.6 so).
#pragma once

#include "layers.h"

namespace mg {

#if defined(__HIPCC__)

typedef float end_floatx4 __attribute__((ext_vector_type(4)));
typedef uint32_t end_u32x4 __attribute__((ext_vector_type(4), aligned(2)));

// LDS bytes of a wavefront's region: 16 rows of its columns in FP32 or two matrices of 16 bits, 16 bytes apart from each other's banks
template <int WTM> constexpr int end_region() { return 16 * (WTM * 4 + 16); }

// waits for nothing in hardware (a wavefront's LDS operations run in order); keeps the compiler from moving reads across other lanes' writes
__device__ inline void end_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

template <typename T> struct __attribute__((packed, aligned(8))) Four {
    T v[4];
};

// COLS columns of 16 rows, U elements, in the wavefront's region -> base(row) + col; rows below `rows`, columns below `cols`
template <typename U, int COLS, bool PAST = false, typename Row> __device__ inline void end_drain(const char *region, int row_bytes, int row, int col, int rows, int cols, int lane, Row &&at)
{
    constexpr int PER = 16 / static_cast<int>(sizeof(U)), CH = COLS / PER;
    static_assert(COLS % PER == 0, "whole pieces");
#pragma unroll
    for (int pass = 0; pass < (16 * CH + 63) / 64; ++pass) {
        const int id = lane + 64 * pass, c = id % CH, r = id / CH;
        if (16 * CH % 64 != 0 && r >= 16) continue;
        const int left = cols - (col + c * PER);
        if (row + r >= rows || left <= 0) continue;
        const Piece<U, PER> x = __builtin_bit_cast(Piece<U, PER>, *reinterpret_cast<const end_floatx4 *>(region + r * row_bytes + c * 16));
        U *to = at(row + r) + col + c * PER;
        if (left >= PER) {
            if constexpr (PAST) __builtin_nontemporal_store(__builtin_bit_cast(end_u32x4, x), reinterpret_cast<end_u32x4 *>(to));
            else *reinterpret_cast<Piece<U, PER> *>(to) = x;
        } else {
#pragma unroll
            for (int e = 0; e < PER; ++e)
                if (e < left) to[e] = x.v[e];
        }
    }
}

template <typename T> __device__ inline void end_stage(char *at, float a, float b, float c, float d)
{
    if constexpr (sizeof(T) == 4) *reinterpret_cast<end_floatx4 *>(at) = end_floatx4{a, b, c, d};
    else *reinterpret_cast<Four<T> *>(at) = Four<T>{{static_cast<T>(a), static_cast<T>(b), static_cast<T>(c), static_cast<T>(d)}};
}

// A block of a and b of what is kept (kept_block), this lane's four of each.  bfloat16: 16 bytes a lane, then the lanes' exponents.
// PAST: by the caches
template <bool PAST, typename V> __device__ inline void put_kept(V v, void *at)
{
    if constexpr (PAST) __builtin_nontemporal_store(v, static_cast<V *>(at));
    else *static_cast<V *>(at) = v;
}
template <bool PAST, typename V> __device__ inline V get_kept(const void *at)
{
    if constexpr (PAST) return __builtin_nontemporal_load(static_cast<const V *>(at));
    else return *static_cast<const V *>(at);
}
template <typename T, bool PAST> __device__ inline void keep(void *kept, int64_t block, int lane, const float (&a)[4], const float (&b)[4])
{
    if constexpr (std::is_same_v<T, bfloat>) {
        char *const at = static_cast<char *>(kept) + block * kept_block_bytes(MG_BF16);
        // the largest finite one of four goes to 2^14 .. 2^15 (infinities stay what they are)
        auto shift = [](const float (&v)[4]) {
            float largest = fmaxf(fmaxf(fabsf(v[0]), fabsf(v[1])), fmaxf(fabsf(v[2]), fabsf(v[3])));
            if (__builtin_expect(__any(largest == __builtin_inff()), 0)) {
                largest = 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) largest = fmaxf(largest, fabsf(v[i]) < __builtin_inff() ? fabsf(v[i]) : 0.f);
            }
            const int e = __builtin_amdgcn_frexp_expf(largest);
            return 15 - e < 126 ? 15 - e : 126;
        };
        const int ka = shift(a), kb = shift(b);
        Four<_Float16> x, y;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x.v[e] = static_cast<_Float16>(ldexpf(a[e], ka));
            y.v[e] = static_cast<_Float16>(ldexpf(b[e], kb));
        }
        const uint64_t both[2] = {__builtin_bit_cast(uint64_t, x), __builtin_bit_cast(uint64_t, y)};
        put_kept<PAST>(__builtin_bit_cast(end_floatx4, both), at + 16 * lane);
        put_kept<PAST>(static_cast<uint16_t>((ka & 0xff) | (kb & 0xff) << 8), at + 1024 + 2 * lane);
    } else {
        float *const at = reinterpret_cast<float *>(static_cast<char *>(kept) + block * kept_block_bytes(MG_F16)) + 4 * lane;
        put_kept<PAST>(end_floatx4{a[0], a[1], a[2], a[3]}, at);
        put_kept<PAST>(end_floatx4{b[0], b[1], b[2], b[3]}, at + 256);
    }
}
// The way back: a block's load, which may be early, and what it holds
template <typename T> struct Kept {
    end_floatx4 x, y;
    template <bool PAST> __device__ inline void load(const void *kept, int64_t block, int lane)
    {
        const float *const at = reinterpret_cast<const float *>(static_cast<const char *>(kept) + block * kept_block_bytes(MG_F16)) + 4 * lane;
        x = get_kept<PAST, end_floatx4>(at);
        y = get_kept<PAST, end_floatx4>(at + 256);
    }
    __device__ inline void recall(float (&a)[4], float (&b)[4]) const
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            a[e] = x[e];
            b[e] = y[e];
        }
    }
};
template <> struct Kept<bfloat> {
    end_floatx4 x;
    uint16_t k;
    template <bool PAST> __device__ inline void load(const void *kept, int64_t block, int lane)
    {
        const char *const at = static_cast<const char *>(kept) + block * kept_block_bytes(MG_BF16);
        x = get_kept<PAST, end_floatx4>(at + 16 * lane);
        k = get_kept<PAST, uint16_t>(at + 1024 + 2 * lane);
    }
    __device__ inline void recall(float (&a)[4], float (&b)[4]) const
    {
        struct Both {
            Four<_Float16> x, y;
        };
        const Both v = __builtin_bit_cast(Both, x);
        const int ka = static_cast<int8_t>(k & 0xff), kb = static_cast<int8_t>(k >> 8);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            a[e] = ldexpf(static_cast<float>(v.x.v[e]), -ka);
            b[e] = ldexpf(static_cast<float>(v.y.v[e]), -kb);
        }
    }
};

// Columns of H, dG and dU that are written: zeros from `hidden` on
__device__ inline int held_columns(int hidden) { return (hidden + 15) / 16 * 16; }

template <int ACT, typename T, bool PAST, int FM, int FN> __device__ __forceinline__ void end_gated(const LinearArgs &args, const end_floatx4 (&acc)[FN][FM], char *region, int row0, int col0, int lane)
{
    constexpr int HALF = FM / 2, ROWB = HALF * 32 + 16;
    const int out0 = col0 / 2, held = held_columns(args.hidden);
    T *const C = static_cast<T *>(args.C0);
#pragma unroll
    for (int j = 0; j < FN; ++j) {
        const int row = row0 + 16 * j;
        end_fence();
#pragma unroll
        for (int i = 0; i < HALF; ++i) {
            const end_floatx4 g = acc[j][2 * i], u = acc[j][2 * i + 1];
            float a[4], b[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float slope;
                activation_of<ACT>(g[e], a[e], slope);
                b[e] = u[e] * slope;
            }
            if (args.kept != nullptr && row < args.rows && out0 + 16 * i < held) keep<T, PAST>(args.kept, kept_block(row, out0 + 16 * i, args.hidden), lane, a, b);
            end_stage<T>(region + (lane % 16) * ROWB + i * 32 + (lane / 16) * 8, a[0] * u[0], a[1] * u[1], a[2] * u[2], a[3] * u[3]);
        }
        end_fence();
        end_drain<T, HALF * 16>(region, ROWB, row, out0, args.rows, held, lane, [&](int r) { return C + r * args.ldc0; });
    }
}

template <typename T, bool PAST, int FM, int FN> __device__ __forceinline__ void end_gated_grad(const LinearArgs &args, const end_floatx4 (&acc)[FN][FM], char *region, int row0, int col0, int lane)
{
    constexpr int ROWB = FM * 32 + 16;
    const int held = held_columns(args.hidden);
    T *const C = static_cast<T *>(args.C0);
    const int64_t beside = args.ldc0 / 2;                   // dU's columns behind dG's
    // what a row of blocks needs is asked for while the row before it is stored, as far as there are registers
    constexpr int EARLY = std::is_same_v<T, bfloat> ? FM : FM / 4;
    Kept<T> kept[2][FM];
    auto ask = [&](int j, int from, int to) __attribute__((always_inline)) {
        // (blocks outside are not there: a block that is, is read for them, and not used)
        const int row = row0 + 16 * j < args.rows ? row0 + 16 * j : args.rows - 1;
#pragma unroll
        for (int i = from; i < to; ++i) {
            const int col = col0 + 16 * i < held ? col0 + 16 * i : held - 1;
            kept[j % 2][i].template load<PAST>(args.kept, kept_block(row, col, args.hidden), lane);
        }
    };
    ask(0, 0, EARLY);
#pragma unroll
    for (int j = 0; j < FN; ++j) {
        const int row = row0 + 16 * j;
        Four<T> du[FM];
        ask(j, EARLY, FM);
        if (j + 1 < FN) ask(j + 1, 0, EARLY);
        end_fence();
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            const int col = col0 + 16 * i;
            float a[4], b[4];
            kept[j % 2][i].recall(a, b);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                // (columns behind the last one are sums of whatever lies behind the rows of WD)
                const bool there = col + 4 * (lane / 16) + e < args.hidden;
                a[e] = there ? acc[j][i][e] * a[e] : 0.f;
                b[e] = there ? acc[j][i][e] * b[e] : 0.f;
            }
            end_stage<T>(region + (lane % 16) * ROWB + i * 32 + (lane / 16) * 8, b[0], b[1], b[2], b[3]);
            du[i] = Four<T>{{static_cast<T>(a[0]), static_cast<T>(a[1]), static_cast<T>(a[2]), static_cast<T>(a[3])}};
        }
        end_fence();
        end_drain<T, FM * 16>(region, ROWB, row, col0, args.rows, held, lane, [&](int r) { return C + r * args.ldc0; });
        end_fence();
#pragma unroll
        for (int i = 0; i < FM; ++i) *reinterpret_cast<Four<T> *>(region + (lane % 16) * ROWB + i * 32 + (lane / 16) * 8) = du[i];
        end_fence();
        end_drain<T, FM * 16>(region, ROWB, row, col0, args.rows, held, lane, [&](int r) { return C + beside + r * args.ldc0; });
    }
}

// A row's target among this lane's 4 FM columns (element e of block i is 4 i + e), -1: not there.  wanted: behind the wavefront's first column; left: columns from that on.
// A vocabulary has many tiles and a row one target: what is done for it stands behind a branch that few wavefronts take.
template <int FM> __device__ inline int wanted_column(int64_t wanted, int left, int lane)
{
    if (wanted < 0 || wanted >= 16 * FM || wanted >= left) return -1;
    const int at = static_cast<int>(wanted);
    return at % 16 / 4 == lane / 16 ? at / 16 * 4 + at % 4 : -1;
}
template <int FM> __device__ inline float wanted_of(const end_floatx4 (&row)[FM], int at)
{
    float z = 0.f;
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) z = at == 4 * i + e ? row[i][e] : z;
    return z;
}

// (largest, sum of exp(z - largest)) of two sets of logits
__device__ inline float2 join_scores(float2 a, float2 b)
{
    const float m = fmaxf(a.x, b.x), from = m == -__builtin_inff() ? 0.f : m;
    return make_float2(m, a.y * exp_fast(a.x - from) + b.y * exp_fast(b.x - from));
}

// All WR x WC wavefronts that share a tile come here, and nobody uses the LDS any more.  The wavefront's tile starts at (row0, col0) and is wavefront
// (wr, wc) of WR x WC; region: its own; shared: WR * FN * 16 * WC float2 that no region overlaps (END_SCORES).
template <typename T, int END, int FM, int FN, int WR, int WC, bool PAST = false>
__device__ __forceinline__ void linear_end(const LinearArgs &args, end_floatx4 (&acc)[FN][FM], char *region, float2 *shared, int tile_row, int tile_col, int wr, int wc, int lane, int slice = 0)
{
    const int row0 = tile_row + wr * FN * 16, col0 = tile_col + wc * FM * 16;
    if constexpr (END == END_STORE) {
        if (args.partial != nullptr) {
            constexpr int ROWB = FM * 64 + 16;
            float *const to = args.partial + slice * args.partial_stride;
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                end_fence();
#pragma unroll
                for (int i = 0; i < FM; ++i) *reinterpret_cast<end_floatx4 *>(region + (lane % 16) * ROWB + i * 64 + (lane / 16) * 16) = acc[j][i];
                end_fence();
                end_drain<float, FM * 16>(region, ROWB, row0 + 16 * j, col0, args.rows, args.cols, lane, [&](int r) { return to + r * args.partial_ld; });
            }
        } else {
            constexpr int ROWB = FM * 32 + 16;
            const float scale = args.scale == nullptr ? 1.f : *args.scale;
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                end_fence();
#pragma unroll
                for (int i = 0; i < FM; ++i)
                    end_stage<T>(region + (lane % 16) * ROWB + i * 32 + (lane / 16) * 8, acc[j][i][0] * scale, acc[j][i][1] * scale, acc[j][i][2] * scale, acc[j][i][3] * scale);
                end_fence();
                // (16 rows are of one matrix: `second` is a multiple of 64)
                const int row = row0 + 16 * j;
                const bool other = args.second > 0 && row >= args.second;
                T *const C = static_cast<T *>(other ? args.C1 : args.C0) - (other ? args.second * args.ldc1 : 0);
                const int64_t ldc = other ? args.ldc1 : args.ldc0;
                const int rows = args.second == 0 ? args.rows : other ? args.second + args.rows0 : args.rows0;
                if ((other ? args.C1 : args.C0) != nullptr) end_drain<T, FM * 16>(region, ROWB, row, col0, rows, args.cols, lane, [&](int r) { return C + r * ldc; });
            }
        }
    } else if constexpr (END == END_GATED) {
        if (args.activation == MG_ACT_SILU) end_gated<MG_ACT_SILU, T, PAST>(args, acc, region, row0, col0, lane);
        else if (args.activation == MG_ACT_GELU) end_gated<MG_ACT_GELU, T, PAST>(args, acc, region, row0, col0, lane);
        else if (args.activation == MG_ACT_GELU_TANH) end_gated<MG_ACT_GELU_TANH, T, PAST>(args, acc, region, row0, col0, lane);
        else end_gated<MG_ACT_RELU2, T, PAST>(args, acc, region, row0, col0, lane);
    } else if constexpr (END == END_GATED_GRAD) {
        end_gated_grad<T, PAST>(args, acc, region, row0, col0, lane);
    } else if constexpr (END == END_SCORES) {
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const int row = row0 + 16 * j + lane % 16;
            const int at = wanted_column<FM>(row < args.rows ? args.targets[row] - args.first - col0 : -1, args.cols - col0, lane);
            if (col0 + 16 * FM > args.cols) {
#pragma unroll
                for (int i = 0; i < FM; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (col0 + 16 * i + 4 * (lane / 16) + e >= args.cols) acc[j][i][e] = -__builtin_inff();
            }
            if (__any(at >= 0)) {
                const float z = wanted_of<FM>(acc[j], at);
                if (at >= 0) args.target_score[row] = z;
            }
            float m = -__builtin_inff(), s = 0.f;
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) m = fmaxf(m, acc[j][i][e]);
            m = fmaxf(m, __shfl_xor(m, 16));
            m = fmaxf(m, __shfl_xor(m, 32));
            // exp(z - m) as 2 to the power of z log2(e) - (m log2(e)), the product in front rounded: off by half a step of m for all of a row's terms, as m itself is
            const float from = m == -__builtin_inff() ? 0.f : -LOG2_E * m;
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) s += __builtin_amdgcn_exp2f(fmaf(acc[j][i][e], LOG2_E, from));
            s += __shfl_xor(s, 16);
            s += __shfl_xor(s, 32);
            if (lane < 16) shared[wc * (WR * FN * 16) + wr * FN * 16 + 16 * j + lane] = make_float2(m, s);
        }
        if constexpr (WR * WC == 1) end_fence();
        else __syncthreads();
        for (int r = (wr * WC + wc) * 64 + lane; r < WR * FN * 16; r += WR * WC * 64) {
            if (tile_row + r >= args.rows) continue;
            float2 all = shared[r];
#pragma unroll
            for (int w = 1; w < WC; ++w) all = join_scores(all, shared[w * (WR * FN * 16) + r]);
            args.scores[static_cast<int64_t>(tile_col / (WC * FM * 16)) * args.rows + tile_row + r] = all;
        }
    } else {
        constexpr int ROWB = FM * 32 + 16;
        T *const C = static_cast<T *>(args.C0);
        const int held = (args.cols + 15) / 16 * 16;
        const float weight_scale = args.weight_scale == nullptr ? 1.f : *args.weight_scale;
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const int row = row0 + 16 * j + lane % 16;
            int64_t wanted = -1;
            float w = 0.f, from = 0.f;
            if (row < args.rows) {
                wanted = args.targets[row];
                if (wanted >= 0 && wanted < args.vocab) {
                    w = (args.weights == nullptr ? 1.f : args.weights[row]) * weight_scale;
                    from = -LOG2_E * args.lse[row];
                }
                wanted -= args.first + col0;
            }
            const int at = wanted_column<FM>(wanted, args.cols - col0, lane);
            const bool ends = col0 + 16 * FM > args.cols;
            end_fence();
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                const int col = col0 + 16 * i + 4 * (lane / 16);
                float d[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float p = __builtin_amdgcn_exp2f(fmaf(acc[j][i][e], LOG2_E, from));
                    d[e] = w != 0.f ? w * p : 0.f;                                  // (a token that adds nothing adds nothing, whatever its logits are)
                }
                if (ends) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (col + e >= args.cols) d[e] = 0.f;
                }
                end_stage<T>(region + (lane % 16) * ROWB + i * 32 + (lane / 16) * 8, d[0], d[1], d[2], d[3]);
            }
            if (__any(at >= 0)) {
                // the target's own: w (p - 1), in the place of w p
                const float p = __builtin_amdgcn_exp2f(fmaf(wanted_of<FM>(acc[j], at), LOG2_E, from)) - 1.f;
                if (at >= 0) *reinterpret_cast<T *>(region + (lane % 16) * ROWB + (at / 4 * 16 + lane / 16 * 4 + at % 4) * 2) = static_cast<T>(w != 0.f ? w * p : 0.f);
            }
            end_fence();
            end_drain<T, FM * 16, PAST>(region, ROWB, row0 + 16 * j, col0, args.rows, held, lane, [&](int r) { return C + r * args.ldc0; });
        }
    }
}
#endif

}  // namespace mg
