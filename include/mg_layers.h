/*
 * mg_layers.h  --  C ABI of the dense layers of a language model's training step: gated feed-forward blocks, the softmax cross
 * entropy over a vocabulary with the last projection in it, and clipping by the global norm of all gradients.
 *
 * Same library and conventions as mg_gemm.h and mg_experts.h: device pointers owned by the caller, nothing allocated, copied to the
 * host or synchronised, every call only enqueues kernels on `stream`, arguments are checked on the host before any GPU work, errors are
 * negative status codes, the errors of smaller magnitude come first.  Matrices are row-major: element (r, c) at X[r*ld + c]; any address
 * that is a multiple of an element's size and any leading dimension that holds a row will do.  dtype is MG_F32, MG_F16 or MG_BF16, for
 * all matrices of a call.  Results do not depend on timing: the same call gives the same bits.  A result may not
 * overlap what the call reads, nor another result.
 *
 * Sums are in FP32 (MG_F32: as mg_sgemm's).  With 16-bit types a number is rounded to dtype where it becomes an operand of the next product
 * (H, dG and dU of a block, dz of the loss) and where it is a result; activations and exponentials are in FP32, and so is what a block keeps for its
 * backward pass, but for MG_BF16, where that has 11 bits and an exponent for four neighbouring features (numbers below 2^-28 of the largest of the four may
 * have fewer, below 2^-40 none).  MG_F16: an element of H, dG or dU beyond 65504 is an infinity, as it is in any program that stores it in that type; dG and dU are
 * not scaled as dz is, so that gradients in that range are the caller's (a loss scale).
 *
 * Workspaces: 256-byte aligned, at least the bytes that the query of the call answers (MG_ERR_WORKSPACE otherwise), which is 0 for sizes that
 * the call refuses.  With 16-bit types, operands whose rows start on 16 bytes (pointer and leading dimension) and are whole 16-byte pieces
 * along a sum take the fastest kernels as they are.  Others are copied into the workspace first where it has room: the queries count that
 * room where `width` or `hidden` is no multiple of eight; without it the products run on a slower kernel (large calls take 2.7 to 4.5 times as long), with the
 * same result up to the order of sums.  So do matrices of whole widths whose rows lie off 16 bytes in a workspace of the query's size: room for a copy of
 * each, rows x (columns up to a multiple of 64) x 2 bytes, beyond it is used.  Two calls that may run at the same time need a workspace each.
 *
 * A kernel may read an aligned 16-byte piece of memory whole when at least one of its bytes belongs to an operand.
 *
 * MG_ERR_DIM also covers what 32-bit counts and a launch cannot hold: extents of 2^24 and more, matrices of more than 2^40 stored elements
 * and products with more than 2^34 results (logits are such results; of a block, rows of 2 hidden).
 */
#ifndef MG_LAYERS_H
#define MG_LAYERS_H

#include "mg_experts.h"

#ifdef __cplusplus
extern "C" {
#endif

enum {
    MG_ERR_ACTIVATION = -30,  /* activation is none of MG_ACT_...                                           */
    MG_ERR_KEPT = -31,        /* what a forward pass keeps: missing, misaligned or too small                */
    MG_ERR_LIMIT = -32        /* max_norm is negative or not a number                                      */
};

/* ---- gated feed-forward block ------------------------------------------------------------------------------------------
 *     G = X WG^T,  U = X WU^T,  H = act(G) * U,  Y = H WD^T
 * X tokens x width, WG and WU hidden x width, WD width x hidden, Y tokens x width.
 *   MG_ACT_SILU g / (1 + exp(-g));  MG_ACT_GELU g times the normal distribution function;  MG_ACT_GELU_TANH its form with tanh:
 *   g / 2 (1 + tanh(sqrt(2/pi) (g + 0.044715 g^3)));  MG_ACT_RELU2 max(g, 0)^2. */
typedef enum { MG_ACT_SILU = 171, MG_ACT_GELU = 172, MG_ACT_GELU_TANH = 173, MG_ACT_RELU2 = 174 } mg_activation;

/* kept: what mg_gated_backward reads of this forward pass (act(G), U act'(G) and H, in an order of their own), 256-byte aligned, at least
 * mg_gated_kept_bytes() bytes; NULL where no backward pass will come (tokens that are served).  Calls of few tokens without it read the
 * weights once, at the memory's rate.
 * Errors: MG_ERR_DIM, MG_ERR_LDA (ldx), MG_ERR_LDB (a weight matrix's), MG_ERR_LDC (ldy), MG_ERR_NULL, MG_ERR_WORKSPACE, MG_ERR_TYPE,
 * MG_ERR_ACTIVATION, MG_ERR_KEPT.  No tokens or no width: nothing happens.  hidden == 0: Y becomes zero. */
mg_status mg_gated_forward(int dtype, int activation, int64_t tokens, int64_t width, int64_t hidden, const void *X, int64_t ldx,
                           const void *WG, int64_t ldwg, const void *WU, int64_t ldwu, const void *WD, int64_t ldwd, void *Y, int64_t ldy,
                           void *kept, size_t kept_bytes, void *workspace, size_t workspace_bytes, void *stream);
size_t mg_gated_forward_workspace_bytes(int dtype, int64_t tokens, int64_t width, int64_t hidden);
size_t mg_gated_kept_bytes(int dtype, int64_t tokens, int64_t width, int64_t hidden);

/* Gradients for dY (tokens x width), from the same X and weights and what the forward pass of the same dtype, activation and sizes kept:
 *     dH = dY WD,  dU = dH * act(G),  dG = dH * U * act'(G)
 *     dX = dG WG + dU WU,  dWG = dG^T X,  dWU = dU^T X,  dWD = dY^T H
 * The activation's slope is in what was kept; `activation` is checked, nothing else.  Each of the four results may be NULL.  `kept` is not changed: the call can be made again.  No tokens: the weights' gradients become zero.
 * Errors: as above, MG_ERR_LDA also for lddy, MG_ERR_LDC for a result's. */
mg_status mg_gated_backward(int dtype, int activation, int64_t tokens, int64_t width, int64_t hidden, const void *X, int64_t ldx,
                            const void *WG, int64_t ldwg, const void *WU, int64_t ldwu, const void *WD, int64_t ldwd, const void *dY, int64_t lddy,
                            const void *kept, size_t kept_bytes, void *dX, int64_t lddx, void *dWG, int64_t lddwg, void *dWU, int64_t lddwu,
                            void *dWD, int64_t lddwd, void *workspace, size_t workspace_bytes, void *stream);
size_t mg_gated_backward_workspace_bytes(int dtype, int64_t tokens, int64_t width, int64_t hidden);

/* ---- softmax cross entropy over a vocabulary ---------------------------------------------------------------------------
 *     z = X W^T,  lse[t] = log(sum over v of exp(z(t, v))),  loss[t] = lse[t] - z(t, targets[t])
 * X tokens x width, W vocab x width; targets: device array of tokens; loss, lse: FP32 device arrays.  A target outside 0 .. vocab-1 is
 * ignored: its loss is 0 (lse is written all the same; vocab == 0: minus infinity).  The logits z exist a piece at a time, in registers
 * (MG_F32: in the workspace), and are not kept.
 * Errors: MG_ERR_DIM, MG_ERR_LDA (ldx), MG_ERR_LDB (ldw), MG_ERR_NULL, MG_ERR_WORKSPACE, MG_ERR_TYPE. */
mg_status mg_vocab_loss(int dtype, int64_t tokens, int64_t width, int64_t vocab, const void *X, int64_t ldx, const void *W, int64_t ldw,
                        const int64_t *targets, float *loss, float *lse, void *workspace, size_t workspace_bytes, void *stream);
size_t mg_vocab_loss_workspace_bytes(int dtype, int64_t tokens, int64_t width, int64_t vocab);

/* Gradients of sum over t of weights[t] * loss[t], from the lse that mg_vocab_loss wrote:
 *     dz(t, v) = weights[t] * (exp(z(t, v) - lse[t]) - (v == targets[t])),  0 for ignored targets
 *     dX = dz W,  dW = dz^T X
 * weights: FP32 device array of tokens (a mean over `count` tokens has 1/count in it, and a loss scale), NULL: 1.  A token that is ignored or has weight zero adds
 * nothing, whatever its row of X holds, infinities and NaN among it; its row of dX is zero (a product of zeros with W: no number where W is not finite).
 * dz exists for a piece of the vocabulary at a time, in the workspace.  dX or dW may be NULL.  No tokens: dW becomes zero; vocab == 0: dX.
 * 16 bits: dz is rounded in units of the largest weight of a token that counts (MG_F16: of 2^-13 of it), so that equal weights cost no bits and small probabilities keep theirs.
 * Errors: as above, MG_ERR_LDC (lddx, lddw). */
mg_status mg_vocab_loss_grad(int dtype, int64_t tokens, int64_t width, int64_t vocab, const void *X, int64_t ldx, const void *W, int64_t ldw,
                             const int64_t *targets, const float *lse, const float *weights, void *dX, int64_t lddx, void *dW, int64_t lddw,
                             void *workspace, size_t workspace_bytes, void *stream);
size_t mg_vocab_loss_grad_workspace_bytes(int dtype, int64_t tokens, int64_t width, int64_t vocab);

/* ---- the norm of all gradients, and clipping ---------------------------------------------------------------------------
 * Host arrays of `count` entries: types[i], device address sources[i] and number of elements sizes[i] of tensor i, dense.  They are read
 * during the call and not after it: a captured graph holds their values.
 *     norm[0] = sqrt(sum over all elements of g^2)      (device; summed in 64 bits, rounded once to FP32)
 * mg_gradient_clip also writes every tensor, multiplied by max_norm / norm where max_norm < norm (formed in 64 bits and rounded to FP32, as each
 * product is to the tensor's type) and as it is otherwise, to results[i]
 * (the same type and size; the same address is fine, any other overlap of results with sources is not; results NULL: all in place).  Where
 * norm[0] is infinite (also of finite elements whose norm FP32 does not hold) or no number, tensors stay as they are.  max_norm infinite: nothing is ever clipped.
 * Errors: MG_ERR_DIM (count outside 0 .. 2^16, a negative size, more than 2^40 elements in all), MG_ERR_NULL (an array, or an address of a tensor with elements),
 * MG_ERR_WORKSPACE, MG_ERR_TYPE, MG_ERR_LIMIT.  count == 0: norm[0] = 0. */
mg_status mg_gradient_norm(int64_t count, const int32_t *types, const void *const *sources, const int64_t *sizes, float *norm,
                           void *workspace, size_t workspace_bytes, void *stream);
mg_status mg_gradient_clip(int64_t count, const int32_t *types, const void *const *sources, void *const *results, const int64_t *sizes,
                           float max_norm, float *norm, void *workspace, size_t workspace_bytes, void *stream);
size_t mg_gradient_workspace_bytes(int64_t count);

#ifdef __cplusplus
}
#endif
#endif
