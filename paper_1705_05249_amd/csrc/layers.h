// What the kernels of mg_layers.h share: the products of 16-bit matrices and what becomes of their results.
//
// Every product of the block and of the loss is C(r, c) = sum over l of P(r, l) Q(c, l), C row-major.  P and Q each lie along the sum
// (element (r, l) at P[r*ld + l]) or across it (at P[l*ld + r]); the results stay in registers until they have become what the operator stores.
#pragma once

#include <atomic>

#include "experts.h"
#include "../../include/mg_layers.h"

namespace mg {

constexpr int64_t LAYER_PIECE = 64;               // columns of the matrices that the library lays out itself are padded to this, with zeros

__host__ __device__ inline int64_t padded(int64_t v) { return (v + LAYER_PIECE - 1) / LAYER_PIECE * LAYER_PIECE; }

// What becomes of the sums
enum LinearEnd {
    END_STORE = 0,          // C in the operands' type, its rows in one matrix or two, or slices of FP32 sums
    END_GATED = 1,          // Q is gate and up weights, 16 rows of each in turn: H = act(G) * U, and what the backward pass needs of G and U
    END_GATED_GRAD = 2,     // the sums are dH: dG and dU beside each other
    END_SCORES = 3,         // the sums are logits: largest one and sum of exponentials of a tile's columns, the target's logit
    END_SCORES_GRAD = 4     // the sums are logits: dz
};

// Operands.  Matrix 1 is the second half of Q: END_GATED (up weights), or with `segment` the lines from l = segment on.
struct LinearArgs {
    const void *P, *Q0, *Q1;
    int64_t ldp, ldq0, ldq1;
    int rows, cols;             // of C; END_GATED: cols is 32 * ceil(hidden / 16), the interleaved columns
    int k;                      // length of the sum
    int segment;                // 0, or where in the sum Q1 takes over (a multiple of 64; P has zeros between `lines` and it)
    int lines;                  // with `segment`: lines that Q0 and Q1 have
    int hidden;                 // END_GATED, END_GATED_GRAD
    bool p_padded, q_padded;    // the operand has zeros up to a whole piece behind the sum's end
    int tiles_r, tiles_c;
    int k_per_slice;            // a multiple of 64; slice z of the sum starts at z * k_per_slice
    // results
    void *C0, *C1;              // END_STORE: rows from `second` on are rows 0.. of C1 (`second` rows: of C0, `rows0` of which exist, as many of C1)
    int64_t ldc0, ldc1;
    int second, rows0;
    float *partial;             // END_STORE: instead of C, FP32 sums: slice z at partial + z * partial_stride, rows x partial_ld
    int64_t partial_ld, partial_stride;
    const float *scale;         // END_STORE: device scalar that every result is multiplied with; null: 1
    int activation;
    void *kept;                 // END_GATED (null: nothing is kept), END_GATED_GRAD: see kept_block
    // END_SCORES, END_SCORES_GRAD: columns are the vocabulary's from `first` on
    int64_t first, vocab;
    const int64_t *targets;
    float2 *scores;             // [tile of columns][row]: (largest, sum of exp(z - largest))
    float *target_score;        // [row]
    const float *lse;
    const float *weights;       // null: 1
    const float *weight_scale;  // device scalar beside the weights; null: 1
};

// What a block keeps of 16-bit types for its backward pass: a = act(G) and b = U act'(G), of which dU = dH a and dG = dH b, in blocks of 16 x 16 in the order in which a
// matrix instruction leaves them (lane l: row l % 16, columns 4 (l / 16) .. + 3): a wavefront moves a block on end.  FP16: FP32 numbers.  bfloat16: FP16
// numbers with a power of two for every four of a row, which puts the largest into 2^14 .. 2^15: 11 bits, three more than dG and dU are rounded to afterwards, whatever the range
// (bfloat16 would add as much error as that rounding), down to 2^-28 of the largest of the four, fewer below, in 1152 bytes instead of 2048.
__host__ __device__ inline int64_t kept_blocks(int64_t hidden) { return (hidden + 15) / 16; }
__host__ __device__ inline int64_t kept_block(int64_t row, int64_t col, int64_t hidden) { return (row / 16) * kept_blocks(hidden) + col / 16; }
constexpr int kept_block_bytes(int dtype) { return dtype == MG_BF16 ? 1024 + 128 : 2048; }

// Products of END_STORE in one launch (linear_together.hip): the first of FORM_KN, the others of FORM_NN; none where rows is 0.  begin: first work-group
struct LinearTogether {
    LinearArgs of[3];
    uint32_t begin[4];
};

// Which of P and Q lie along the sum
enum LinearForm { FORM_KK = 0, FORM_KN = 1, FORM_NN = 2 };       // both; P along, Q across; both across

// Tiles of C, square; ANY: the kernel for operands at any address.  128_DEEP: four K-tiles in LDS instead of two, for launches that leave a compute unit one
// work-group (2048^3: 30.2 -> 21.7 us; with two work-groups to a compute unit the other one is ahead, 4096 x 4096 x 2048: 72 against 82).  64_TWICE: two sets of
// wavefronts for such launches (512 x 1024 x 2048: 10.6 -> 9.0 us, 1024 x 1024 x 1024 7.3 -> 6.9).
enum LinearTile { LINEAR_256 = 0, LINEAR_128 = 1, LINEAR_64 = 2, LINEAR_128_DEEP = 3, LINEAR_FEW = 4, LINEAR_64_TWICE = 5, LINEAR_ANY = -1, LINEAR_ANY_FEW = -2 };
constexpr int linear_tile_size(int tile) { return tile == LINEAR_256 ? 256 : tile == LINEAR_128 || tile == LINEAR_128_DEEP ? 128 : 64; }
// slices: of the sum, each from z * k_per_slice on
hipError_t launch_linear_any(int dtype, int form, int end, LinearArgs args, int slices, hipStream_t stream);
// FORM_KK, few rows of P, operands at any address or on 16 bytes; columns that a work-group has there
hipError_t launch_linear_few_any(int dtype, int end, const LinearArgs &args, hipStream_t stream);
hipError_t launch_linear_few_dma(int dtype, int end, const LinearArgs &args, hipStream_t stream);
constexpr int linear_few_columns(int end) { return end == END_SCORES ? 64 : end == END_GATED ? 32 : 16; }
constexpr int LINEAR_FEW_ROWS = 32;
// dtype MG_F16 or MG_BF16, operands that linear_aligned() is true for
hipError_t launch_linear_dma_kk_store(int dtype, int tile, const LinearArgs &args, int slices, hipStream_t stream);
hipError_t launch_linear_dma_kk_gated(int dtype, int tile, const LinearArgs &args, int slices, hipStream_t stream);
hipError_t launch_linear_dma_kk_scores(int dtype, int tile, const LinearArgs &args, int slices, hipStream_t stream);
hipError_t launch_linear_dma_kk_scores_grad(int dtype, int tile, const LinearArgs &args, int slices, hipStream_t stream);
hipError_t launch_linear_dma_kn_store(int dtype, int tile, const LinearArgs &args, int slices, hipStream_t stream);
hipError_t launch_linear_dma_kn_gated_grad(int dtype, int tile, const LinearArgs &args, int slices, hipStream_t stream);
hipError_t launch_linear_dma_nn_store(int dtype, int tile, const LinearArgs &args, int slices, hipStream_t stream);

// All of them, in one launch or one by one (linear_plan.h); room: for slices of the first one's sum
hipError_t launch_linear_together(int dtype, LinearTogether all, void *room, size_t room_bytes, hipStream_t stream);
// tile: LINEAR_128 or LINEAR_64; slices: of the first product, whose k_per_slice and `partial` say so
hipError_t launch_linear_together_on(int dtype, int tile, LinearTogether all, int slices, hipStream_t stream);

// adds the slices of END_STORE and writes C in dtype (MG_F32: C may be the first slice)
hipError_t launch_linear_sum(int dtype, const LinearArgs &args, int slices, hipStream_t stream);

// The product on the kernel that its plan (linear_plan.h) takes, `room` for slices of its sum; scores_columns, of END_SCORES: columns that one entry of args.scores stands for
hipError_t launch_linear(int dtype, int form, int end, LinearArgs args, void *room, size_t room_bytes, hipStream_t stream, int *scores_columns = nullptr);
// bytes of room with which a product of aligned operands takes its preferred number of slices
size_t linear_room(int form, int end, int64_t rows, int64_t cols, int64_t k);

// Copies of matrices of 16-bit units whose rows do not start on 16 bytes, or end inside a piece along a sum: rows x padded(cols), zeros behind the columns
struct LinearCopies {
    const void *from[6];
    void *to[6];
    int64_t ld[6];
    int cols[6];
    int64_t rows[6];
    uint32_t begin[7];               // first work-group
    int count;
    // the gradient of the loss (targets null: other callers): rows of matrix 0 are tokens, and zeros where the token's target is no row of the vocabulary or its weight
    // is zero; scale (or null): what dz is scaled with, see weight_scale
    const int64_t *targets;
    int64_t vocab;
    const float *weights;
    float most, *scale;
};
hipError_t launch_linear_copies(LinearCopies copies, hipStream_t stream);
// Rows of `cols` units whose pieces of eight a launch counts in 32 bits.  Matrices of 16 bits (2^34 elements, fewer than 2^24 rows) have no more pieces than that; X of FP32, two
// units an element, may have: 16 760 000 x 1025 has 4.4e9.  It is alone in its list and goes in parts.
inline int64_t copy_rows(int64_t cols) { return cols == 0 ? INT64_MAX : (int64_t(1) << 32) / (padded(cols) / 8); }
// the first rows of a list's only matrix leave the list
inline LinearCopies take_copy_rows(LinearCopies &c, int64_t rows)
{
    LinearCopies first = c;
    first.rows[0] = rows;
    c.rows[0] -= rows;
    c.from[0] = static_cast<const uint16_t *>(c.from[0]) + rows * c.ld[0];
    c.to[0] = static_cast<uint16_t *>(c.to[0]) + rows * padded(c.cols[0]);
    if (c.targets != nullptr) c.targets += rows;
    if (c.weights != nullptr) c.weights += rows;
    return first;
}

// Memory of a workspace, handed out on 256 bytes; without a base it only counts
struct Arena {
    char *base;
    size_t bytes, used;
    void *take(size_t wanted)
    {
        void *const at = base == nullptr ? nullptr : base + used;
        used += (wanted + 255) / 256 * 256;
        return at;
    }
    size_t left() const { return used < bytes ? bytes - used : 0; }
};

struct GatedProblem {
    int dtype, activation;
    int64_t tokens, width, hidden;
    const void *X, *WG, *WU, *WD, *dY;
    int64_t ldx, ldwg, ldwu, ldwd, lddy;
    void *Y, *dX, *dWG, *dWU, *dWD;
    int64_t ldy, lddx, lddwg, lddwu, lddwd;
    void *kept;
    Arena workspace;
    hipStream_t stream;
};
size_t gated_kept(int dtype, int64_t tokens, int64_t hidden);
size_t gated_workspace(int dtype, int64_t tokens, int64_t width, int64_t hidden, bool backward);
mg_status gated_forward(const GatedProblem &p);          // sizes above zero
mg_status gated_backward(const GatedProblem &p);

struct LossProblem {
    int dtype;
    int64_t tokens, width, vocab;
    const void *X, *W;
    int64_t ldx, ldw;
    const int64_t *targets;
    float *loss;
    float *lse;                       // read by the gradient
    const float *weights;
    void *dX, *dW;
    int64_t lddx, lddw;
    Arena workspace;
    hipStream_t stream;
};
size_t loss_workspace(int dtype, int64_t tokens, int64_t width, int64_t vocab, bool gradient);
mg_status vocab_loss(const LossProblem &p);              // vocab may be zero, tokens not
mg_status vocab_loss_grad(const LossProblem &p);         // sizes above zero

struct ClipProblem {
    int64_t count;
    const int32_t *types;
    const void *const *sources;
    void *const *results;             // null: in place
    const int64_t *sizes;
    bool scales;
    float max_norm;
    float *norm;
    void *workspace;
    hipStream_t stream;
};
size_t clip_workspace(int64_t count);
hipError_t launch_clip(const ClipProblem &p);

// Devices on which a kernel may take more than 64 KB of LDS: the limit belongs to a kernel on a device
struct RaisedLds {
    std::atomic<uint64_t> devices{0};
    hipError_t operator()(const void *kernel, int bytes)
    {
        int device = 0;
        if (const hipError_t e = hipGetDevice(&device)) return e;
        const uint64_t bit = device < 64 ? uint64_t(1) << device : 0;
        if ((devices.load(std::memory_order_relaxed) & bit) != 0) return hipSuccess;
        const hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);      // (raising it twice is harmless)
        if (e == hipSuccess) devices.fetch_or(bit, std::memory_order_relaxed);
        return e;
    }
};

// zeros in a matrix (rows x cols elements of `size` bytes)
hipError_t launch_zero_rows(void *X, int64_t rows, int64_t cols, int64_t ld, int size, hipStream_t stream);

#if defined(__HIPCC__)

// e^x by the hardware's exponential of base two: relative error below 2^-23 (1 + |x|)
constexpr float LOG2_E = 1.44269504088896340736f;
__device__ inline float exp_fast(float x) { return __builtin_amdgcn_exp2f(x * LOG2_E); }
template <bool PRECISE> __device__ inline float exp_of(float x)
{
    if constexpr (PRECISE) return expf(x);
    else return exp_fast(x);
}
// 1 / x, PRECISE: rounded, otherwise off by a step (one instruction in the place of ten)
template <bool PRECISE> __device__ inline float one_over(float x)
{
    if constexpr (PRECISE) return 1.f / x;
    else return __builtin_amdgcn_rcpf(x);
}

// act(g) and its derivative (PRECISE: for results in FP32).  GELU_TANH: (1 + tanh(b)) / 2 = 1 / (1 + exp(-2 b)), which loses nothing for small results; GELU: the normal
// distribution function as erfc(-g / sqrt 2) / 2, for the same reason.  That is exp(-g^2 / 2) times a function without poles, of which the 16-bit types take a
// polynomial in t = 1 / (1 + 0.27 |g|), of degree 9 and without constant term, fitted to the least relative error (2^-25; evaluated in FP32 2^-21.3); the exponential is in the slope
// too.  Gate and up product of 8192 tokens, width 2048, hidden 8192, with what is kept: 528 us with erfcf, 484 so; SILU with the reciprocal for a division 466 -> 453.
template <int ACT, bool PRECISE = false> __device__ inline void activation_of(float g, float &a, float &slope)
{
    if constexpr (ACT == MG_ACT_SILU) {
        const float p = one_over<PRECISE>(1.f + exp_of<PRECISE>(-g));
        a = g * p;
        slope = fmaf(a, 1.f - p, p);
    } else if constexpr (ACT == MG_ACT_RELU2) {
        const float v = g > 0.f ? g : g != g ? g : 0.f;
        a = v * v;
        slope = 2.f * v;
    } else if constexpr (ACT == MG_ACT_GELU) {
        constexpr float DENSITY = 0.39894228040143267794f;               // 1 / sqrt(2 pi)
        const float e = exp_of<PRECISE>(-0.5f * g * g);
        float below;
        if constexpr (PRECISE) {
            below = 0.5f * erfcf(-0.70710678118654752440f * g);
        } else {
            const float t = one_over<false>(fmaf(fabsf(g), 0.27f, 1.f));
            float s = 0.028915580362081528f;
            s = fmaf(s, t, -0.1262567639350891f);
            s = fmaf(s, t, 0.16929452121257782f);
            s = fmaf(s, t, -0.06862454861402512f);
            s = fmaf(s, t, 0.10740189999341965f);
            s = fmaf(s, t, 0.07223924249410629f);
            s = fmaf(s, t, 0.10175943374633789f);
            s = fmaf(s, t, 0.1075504720211029f);
            s = fmaf(s, t, 0.10772018134593964f);
            const float tail = s * t * e;
            below = g < 0.f ? tail : 1.f - tail;
        }
        a = g * below;
        slope = fmaf(g * e, DENSITY, below);
    } else {
        constexpr float A = 1.59576912160573071176f, B = 0.044715f;       // 2 sqrt(2 / pi)
        const float g2 = fminf(g * g, 1e30f), p = one_over<PRECISE>(1.f + exp_of<PRECISE>(-g * fmaf(g2, A * B, A)));
        a = g * p;
        slope = fmaf(a * (1.f - p), fmaf(g2, 3.f * A * B, A), p);
    }
}
#endif

}  // namespace mg
