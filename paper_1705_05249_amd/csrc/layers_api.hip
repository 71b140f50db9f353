// Boundary of mg_layers.h: argument checks in status-code order, calls without work.  As in api.hip nothing is allocated, copied or synchronised, and
// validation touches no HIP API.
#include "internal.h"
#include "layers.h"

namespace mg {
namespace {

constexpr int64_t MOST_EXTENT = int64_t(1) << 24;                 // every extent below it
constexpr __int128 MOST_STORED = __int128(1) << 40;
constexpr __int128 MOST_RESULTS = __int128(1) << 34;
constexpr int64_t MOST_TENSORS = int64_t(1) << 16;

bool extent(int64_t v) { return v >= 0 && v < MOST_EXTENT; }
bool stored(int64_t rows, int64_t ld) { return __int128(rows) * ld <= MOST_STORED; }
bool results_fit(int64_t rows, int64_t cols) { return __int128(rows) * cols <= MOST_RESULTS; }
bool type_known(int dtype) { return dtype == MG_F32 || dtype == MG_F16 || dtype == MG_BF16; }
bool at_least(int64_t ld, int64_t width) { return ld >= (width > 1 ? width : 1); }
bool aligned(const void *p) { return p != nullptr && reinterpret_cast<uintptr_t>(p) % 256 == 0; }
mg_status launched(hipError_t e) { return e == hipSuccess ? MG_OK : MG_ERR_LAUNCH; }
int size_of(int dtype) { return dtype == MG_F32 ? 4 : 2; }

// every product of a block has two of these extents as its results
bool block_fits(int64_t tokens, int64_t width, int64_t hidden)
{
    return extent(tokens) && extent(width) && extent(hidden) && results_fit(tokens, 2 * padded(hidden)) && results_fit(tokens, width) && results_fit(2 * padded(hidden), width);
}
bool activation_known(int act) { return act >= MG_ACT_SILU && act <= MG_ACT_RELU2; }

bool loss_fits(int64_t tokens, int64_t width, int64_t vocab)
{
    return extent(tokens) && extent(width) && extent(vocab) && results_fit(tokens, width) && results_fit(vocab, width) && results_fit(tokens, vocab);
}

Arena arena(void *workspace, size_t bytes) { return Arena{static_cast<char *>(workspace), bytes, 0}; }

mg_status check_clip(const ClipProblem &p, size_t workspace_bytes)
{
    if (p.count < 0 || p.count > MOST_TENSORS) return MG_ERR_DIM;
    if (p.count > 0 && (p.sizes == nullptr || p.types == nullptr || p.sources == nullptr)) return MG_ERR_NULL;
    int64_t total = 0;
    for (int64_t i = 0; i < p.count; ++i) {
        if (p.sizes[i] < 0 || p.sizes[i] > (int64_t(1) << 40)) return MG_ERR_DIM;
        total += p.sizes[i];
        if (total > (int64_t(1) << 40)) return MG_ERR_DIM;
    }
    if (p.norm == nullptr) return MG_ERR_NULL;
    for (int64_t i = 0; i < p.count; ++i)
        if (p.sizes[i] > 0 && (p.sources[i] == nullptr || (p.results != nullptr && p.results[i] == nullptr))) return MG_ERR_NULL;
    const size_t need = clip_workspace(p.count);
    if (need > 0 && (!aligned(p.workspace) || workspace_bytes < need)) return MG_ERR_WORKSPACE;
    for (int64_t i = 0; i < p.count; ++i)
        if (!type_known(p.types[i])) return MG_ERR_TYPE;
    return MG_OK;
}

}  // namespace
}  // namespace mg

using namespace mg;

extern "C" {

mg_status mg_gated_forward(int dtype, int activation, int64_t tokens, int64_t width, int64_t hidden, const void *X, int64_t ldx, const void *WG, int64_t ldwg, const void *WU,
                           int64_t ldwu, const void *WD, int64_t ldwd, void *Y, int64_t ldy, void *kept, size_t kept_bytes, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!block_fits(tokens, width, hidden)) return MG_ERR_DIM;
    if (!at_least(ldx, width)) return MG_ERR_LDA;
    if (!at_least(ldwg, width) || !at_least(ldwu, width) || !at_least(ldwd, hidden)) return MG_ERR_LDB;
    if (!at_least(ldy, width)) return MG_ERR_LDC;
    if (!stored(tokens, ldx) || !stored(hidden, ldwg) || !stored(hidden, ldwu) || !stored(width, ldwd) || !stored(tokens, ldy)) return MG_ERR_DIM;
    const bool empty = tokens == 0 || width == 0, sums = !empty && hidden > 0;
    if (!empty && (Y == nullptr || (sums && (X == nullptr || WG == nullptr || WU == nullptr || WD == nullptr)))) return MG_ERR_NULL;
    if (sums && type_known(dtype)) {
        if (!aligned(workspace) || workspace_bytes < gated_workspace(dtype, tokens, width, hidden, false)) return MG_ERR_WORKSPACE;
    }
    if (!type_known(dtype)) return MG_ERR_TYPE;
    if (!activation_known(activation)) return MG_ERR_ACTIVATION;
    if (kept != nullptr && sums && (!aligned(kept) || kept_bytes < gated_kept(dtype, tokens, hidden))) return MG_ERR_KEPT;
    if (empty) return MG_OK;
    if (!sums) return launched(launch_zero_rows(Y, tokens, width, ldy, size_of(dtype), static_cast<hipStream_t>(stream)));
    GatedProblem p{};
    p.dtype = dtype; p.activation = activation;
    p.tokens = tokens; p.width = width; p.hidden = hidden;
    p.X = X; p.ldx = ldx; p.WG = WG; p.ldwg = ldwg; p.WU = WU; p.ldwu = ldwu; p.WD = WD; p.ldwd = ldwd;
    p.Y = Y; p.ldy = ldy; p.kept = kept;
    p.workspace = arena(workspace, workspace_bytes);
    p.stream = static_cast<hipStream_t>(stream);
    return gated_forward(p);
}

size_t mg_gated_forward_workspace_bytes(int dtype, int64_t tokens, int64_t width, int64_t hidden)
{
    if (!type_known(dtype) || !block_fits(tokens, width, hidden) || tokens == 0 || width == 0 || hidden == 0) return 0;
    return gated_workspace(dtype, tokens, width, hidden, false);
}

size_t mg_gated_kept_bytes(int dtype, int64_t tokens, int64_t width, int64_t hidden)
{
    if (!type_known(dtype) || !block_fits(tokens, width, hidden) || tokens == 0 || width == 0 || hidden == 0) return 0;
    return gated_kept(dtype, tokens, hidden);
}

mg_status mg_gated_backward(int dtype, int activation, int64_t tokens, int64_t width, int64_t hidden, const void *X, int64_t ldx, const void *WG, int64_t ldwg, const void *WU,
                            int64_t ldwu, const void *WD, int64_t ldwd, const void *dY, int64_t lddy, const void *kept, size_t kept_bytes, void *dX, int64_t lddx, void *dWG,
                            int64_t lddwg, void *dWU, int64_t lddwu, void *dWD, int64_t lddwd, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!block_fits(tokens, width, hidden)) return MG_ERR_DIM;
    if (!at_least(ldx, width) || !at_least(lddy, width)) return MG_ERR_LDA;
    if (!at_least(ldwg, width) || !at_least(ldwu, width) || !at_least(ldwd, hidden)) return MG_ERR_LDB;
    if ((dX != nullptr && !at_least(lddx, width)) || (dWG != nullptr && !at_least(lddwg, width)) || (dWU != nullptr && !at_least(lddwu, width)) ||
        (dWD != nullptr && !at_least(lddwd, hidden)))
        return MG_ERR_LDC;
    if (!stored(tokens, ldx) || !stored(tokens, lddy) || !stored(hidden, ldwg) || !stored(hidden, ldwu) || !stored(width, ldwd)) return MG_ERR_DIM;
    if ((dX != nullptr && !stored(tokens, lddx)) || (dWG != nullptr && !stored(hidden, lddwg)) || (dWU != nullptr && !stored(hidden, lddwu)) ||
        (dWD != nullptr && !stored(width, lddwd)))
        return MG_ERR_DIM;
    const bool wanted = dX != nullptr || dWG != nullptr || dWU != nullptr || dWD != nullptr;
    const bool sums = wanted && tokens > 0 && width > 0 && hidden > 0;
    if (sums && (X == nullptr || WG == nullptr || WU == nullptr || WD == nullptr || dY == nullptr)) return MG_ERR_NULL;
    if (sums && type_known(dtype)) {
        if (!aligned(workspace) || workspace_bytes < gated_workspace(dtype, tokens, width, hidden, true)) return MG_ERR_WORKSPACE;
    }
    if (!type_known(dtype)) return MG_ERR_TYPE;
    if (!activation_known(activation)) return MG_ERR_ACTIVATION;
    if (sums && (!aligned(kept) || kept_bytes < gated_kept(dtype, tokens, hidden))) return MG_ERR_KEPT;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (!sums) {
        const int size = size_of(dtype);
        if (const hipError_t e = launch_zero_rows(dX, tokens, width, lddx, size, s)) return launched(e);
        if (const hipError_t e = launch_zero_rows(dWG, hidden, width, lddwg, size, s)) return launched(e);
        if (const hipError_t e = launch_zero_rows(dWU, hidden, width, lddwu, size, s)) return launched(e);
        return launched(launch_zero_rows(dWD, width, hidden, lddwd, size, s));
    }
    GatedProblem p{};
    p.dtype = dtype; p.activation = activation;
    p.tokens = tokens; p.width = width; p.hidden = hidden;
    p.X = X; p.ldx = ldx; p.WG = WG; p.ldwg = ldwg; p.WU = WU; p.ldwu = ldwu; p.WD = WD; p.ldwd = ldwd; p.dY = dY; p.lddy = lddy;
    p.dX = dX; p.lddx = lddx; p.dWG = dWG; p.lddwg = lddwg; p.dWU = dWU; p.lddwu = lddwu; p.dWD = dWD; p.lddwd = lddwd;
    p.kept = const_cast<void *>(kept);
    p.workspace = arena(workspace, workspace_bytes);
    p.stream = s;
    return gated_backward(p);
}

size_t mg_gated_backward_workspace_bytes(int dtype, int64_t tokens, int64_t width, int64_t hidden)
{
    if (!type_known(dtype) || !block_fits(tokens, width, hidden) || tokens == 0 || width == 0 || hidden == 0) return 0;
    return gated_workspace(dtype, tokens, width, hidden, true);
}

mg_status mg_vocab_loss(int dtype, int64_t tokens, int64_t width, int64_t vocab, const void *X, int64_t ldx, const void *W, int64_t ldw, const int64_t *targets, float *loss, float *lse,
                        void *workspace, size_t workspace_bytes, void *stream)
{
    if (!loss_fits(tokens, width, vocab)) return MG_ERR_DIM;
    if (!at_least(ldx, width)) return MG_ERR_LDA;
    if (!at_least(ldw, width)) return MG_ERR_LDB;
    if (!stored(tokens, ldx) || !stored(vocab, ldw)) return MG_ERR_DIM;
    const bool empty = tokens == 0, sums = width > 0 && vocab > 0;
    if (!empty && (targets == nullptr || loss == nullptr || lse == nullptr || (sums && (X == nullptr || W == nullptr)))) return MG_ERR_NULL;
    if (!empty && type_known(dtype) && (!aligned(workspace) || workspace_bytes < loss_workspace(dtype, tokens, width, vocab, false))) return MG_ERR_WORKSPACE;
    if (!type_known(dtype)) return MG_ERR_TYPE;
    if (empty) return MG_OK;
    LossProblem p{};
    p.dtype = dtype;
    p.tokens = tokens; p.width = width; p.vocab = vocab;
    p.X = X; p.ldx = ldx; p.W = W; p.ldw = ldw;
    p.targets = targets; p.loss = loss; p.lse = lse;
    p.workspace = arena(workspace, workspace_bytes);
    p.stream = static_cast<hipStream_t>(stream);
    return vocab_loss(p);
}

size_t mg_vocab_loss_workspace_bytes(int dtype, int64_t tokens, int64_t width, int64_t vocab)
{
    if (!type_known(dtype) || !loss_fits(tokens, width, vocab) || tokens == 0) return 0;
    return loss_workspace(dtype, tokens, width, vocab, false);
}

mg_status mg_vocab_loss_grad(int dtype, int64_t tokens, int64_t width, int64_t vocab, const void *X, int64_t ldx, const void *W, int64_t ldw, const int64_t *targets, const float *lse,
                             const float *weights, void *dX, int64_t lddx, void *dW, int64_t lddw, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!loss_fits(tokens, width, vocab)) return MG_ERR_DIM;
    if (!at_least(ldx, width)) return MG_ERR_LDA;
    if (!at_least(ldw, width)) return MG_ERR_LDB;
    if ((dX != nullptr && !at_least(lddx, width)) || (dW != nullptr && !at_least(lddw, width))) return MG_ERR_LDC;
    if (!stored(tokens, ldx) || !stored(vocab, ldw) || (dX != nullptr && !stored(tokens, lddx)) || (dW != nullptr && !stored(vocab, lddw))) return MG_ERR_DIM;
    const bool sums = tokens > 0 && vocab > 0 && width > 0 && (dX != nullptr || dW != nullptr);
    if (sums && (targets == nullptr || lse == nullptr || X == nullptr || W == nullptr)) return MG_ERR_NULL;
    if (sums && type_known(dtype) && (!aligned(workspace) || workspace_bytes < loss_workspace(dtype, tokens, width, vocab, true))) return MG_ERR_WORKSPACE;
    if (!type_known(dtype)) return MG_ERR_TYPE;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (!sums) {
        if (const hipError_t e = launch_zero_rows(dX, tokens, width, lddx, size_of(dtype), s)) return launched(e);
        return launched(launch_zero_rows(dW, vocab, width, lddw, size_of(dtype), s));
    }
    LossProblem p{};
    p.dtype = dtype;
    p.tokens = tokens; p.width = width; p.vocab = vocab;
    p.X = X; p.ldx = ldx; p.W = W; p.ldw = ldw;
    p.targets = targets; p.lse = const_cast<float *>(lse); p.weights = weights;
    p.dX = dX; p.lddx = lddx; p.dW = dW; p.lddw = lddw;
    p.workspace = arena(workspace, workspace_bytes);
    p.stream = s;
    return vocab_loss_grad(p);
}

size_t mg_vocab_loss_grad_workspace_bytes(int dtype, int64_t tokens, int64_t width, int64_t vocab)
{
    if (!type_known(dtype) || !loss_fits(tokens, width, vocab) || tokens == 0 || vocab == 0 || width == 0) return 0;
    return loss_workspace(dtype, tokens, width, vocab, true);
}

mg_status mg_gradient_norm(int64_t count, const int32_t *types, const void *const *sources, const int64_t *sizes, float *norm, void *workspace, size_t workspace_bytes, void *stream)
{
    const ClipProblem p{count, types, sources, nullptr, sizes, false, 0.f, norm, workspace, static_cast<hipStream_t>(stream)};
    if (const mg_status st = check_clip(p, workspace_bytes)) return st;
    return launched(launch_clip(p));
}

mg_status mg_gradient_clip(int64_t count, const int32_t *types, const void *const *sources, void *const *results, const int64_t *sizes, float max_norm, float *norm, void *workspace,
                           size_t workspace_bytes, void *stream)
{
    const ClipProblem p{count, types, sources, results, sizes, true, max_norm, norm, workspace, static_cast<hipStream_t>(stream)};
    if (const mg_status st = check_clip(p, workspace_bytes)) return st;
    if (!(max_norm >= 0.f)) return MG_ERR_LIMIT;
    return launched(launch_clip(p));
}

size_t mg_gradient_workspace_bytes(int64_t count) { return count > 0 && count <= MOST_TENSORS ? clip_workspace(count) : 0; }

}  // extern "C"
