// Gated feed-forward blocks: which products a call is made of, and the elementwise kernels between the products of FP32.
//
// Forward, 16 bits: one product with gate and up weights as one matrix, 16 rows of each in turn, so that a lane holds g and u of the same element and
// H leaves the kernel (6 tokens width hidden operations in two launches); then Y.  Backward: dH never exists in memory, dG and dU leave its product, made of what
// the forward pass kept without another look at the activation;
// dX is one sum over 2 hidden, dG's half and dU's; the gradients of gate and up weights are one product with twice the rows; these and the down weights' go in one
// launch where that pays (linear_together.hip).
// FP32: products as mg_sgemm makes them, with G and U in memory.
#include "linear_end.h"
#include "internal.h"

namespace mg {
namespace {

constexpr int64_t F = sizeof(float);

// H = act(G) * U; KEEP: act(G) and U act'(G) take the places of G and U
template <int ACT, bool KEEP> __global__ __launch_bounds__(256) void gated_act_kernel(float *G, float *U, float *H, int64_t count)
{
    const int64_t at = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 4;
    if (at >= count) return;
    const int valid = static_cast<int>(count - at < 4 ? count - at : 4);
    float g[4], u[4], h[4];
    load_piece<float, 4>(G + at, valid, g);
    load_piece<float, 4>(U + at, valid, u);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float a, slope;
        activation_of<ACT, true>(g[e], a, slope);
        h[e] = a * u[e];
        g[e] = a;
        u[e] *= slope;
    }
    store_piece<float, 4>(H + at, valid, h);
    if (KEEP) {
        store_piece<float, 4>(G + at, valid, g);
        store_piece<float, 4>(U + at, valid, u);
    }
}

// dG = dH b (where dH is) and dU = dH a, from what the forward pass kept
__global__ __launch_bounds__(256) void gated_grad_kernel(const float *A, const float *B, float *dH, float *dU, int64_t count)
{
    const int64_t at = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 4;
    if (at >= count) return;
    const int valid = static_cast<int>(count - at < 4 ? count - at : 4);
    float a[4], b[4], d[4];
    load_piece<float, 4>(A + at, valid, a);
    load_piece<float, 4>(B + at, valid, b);
    load_piece<float, 4>(dH + at, valid, d);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        a[e] *= d[e];
        b[e] *= d[e];
    }
    store_piece<float, 4>(dH + at, valid, b);
    store_piece<float, 4>(dU + at, valid, a);
}

uint32_t pieces(int64_t count) { return static_cast<uint32_t>(ceil_div(count, 1024)); }

// calls fn with the activation as a type
template <typename Fn> hipError_t with_activation(int act, Fn &&fn)
{
    if (act == MG_ACT_SILU) fn(std::integral_constant<int, MG_ACT_SILU>{});
    else if (act == MG_ACT_GELU) fn(std::integral_constant<int, MG_ACT_GELU>{});
    else if (act == MG_ACT_GELU_TANH) fn(std::integral_constant<int, MG_ACT_GELU_TANH>{});
    else fn(std::integral_constant<int, MG_ACT_RELU2>{});
    return hipGetLastError();
}

// what a forward pass of FP32 keeps, tokens x hidden each: act(G) and U act'(G), where G and U were, and H
struct KeptF32 {
    float *G, *U, *H;
    KeptF32(void *at, int64_t tokens, int64_t hidden) : G(static_cast<float *>(at)), U(G + tokens * hidden), H(U + tokens * hidden) {}
};

size_t sgemm_workspace(int ta, int tb, int64_t m, int64_t n, int64_t k, int64_t lda, int64_t ldb, int64_t ldc)
{
    return mg_gemm_workspace_bytes(MG_F32, MG_ROW_MAJOR, ta, tb, m, n, k, lda, ldb, ldc);
}

// room for the products of dense matrices; with other leading dimensions a product may want more, and runs in what there is
size_t sgemm_room(int64_t tokens, int64_t width, int64_t hidden, bool backward)
{
    size_t most = 0;
    auto add = [&](size_t v) { most = v > most ? v : most; };
    add(sgemm_workspace(MG_NO_TRANS, MG_TRANS, tokens, hidden, width, width, width, hidden));
    add(sgemm_workspace(MG_NO_TRANS, MG_TRANS, tokens, width, hidden, hidden, hidden, width));
    if (backward) {
        add(sgemm_workspace(MG_NO_TRANS, MG_NO_TRANS, tokens, hidden, width, width, hidden, hidden));
        add(sgemm_workspace(MG_NO_TRANS, MG_NO_TRANS, tokens, width, hidden, hidden, width, width));
        add(sgemm_workspace(MG_TRANS, MG_NO_TRANS, hidden, width, tokens, hidden, width, width));
        add(sgemm_workspace(MG_TRANS, MG_NO_TRANS, width, hidden, tokens, width, hidden, hidden));
    }
    return most;
}

mg_status forward_f32(const GatedProblem &p)
{
    Arena ws = p.workspace;
    const KeptF32 kept(p.kept != nullptr ? p.kept : ws.take(3 * p.tokens * p.hidden * F), p.tokens, p.hidden);
    const size_t room = ws.left();
    void *const scratch = ws.take(0);
    const float *X = static_cast<const float *>(p.X);
    auto product = [&](const float *A, int64_t lda, const void *B, int64_t ldb, int64_t n, int64_t k, float *C, int64_t ldc) {
        return mg_sgemm(MG_ROW_MAJOR, MG_NO_TRANS, MG_TRANS, p.tokens, n, k, 1.f, A, lda, static_cast<const float *>(B), ldb, 0.f, C, ldc, scratch, room, p.stream);
    };
    if (const mg_status st = product(X, p.ldx, p.WG, p.ldwg, p.hidden, p.width, kept.G, p.hidden)) return st;
    if (const mg_status st = product(X, p.ldx, p.WU, p.ldwu, p.hidden, p.width, kept.U, p.hidden)) return st;
    const int64_t count = p.tokens * p.hidden;
    const hipError_t e = with_activation(p.activation, [&](auto act) {
        constexpr int ACT = decltype(act)::value;
        if (p.kept != nullptr) gated_act_kernel<ACT, true><<<pieces(count), 256, 0, p.stream>>>(kept.G, kept.U, kept.H, count);
        else gated_act_kernel<ACT, false><<<pieces(count), 256, 0, p.stream>>>(kept.G, kept.U, kept.H, count);
    });
    if (e != hipSuccess) return MG_ERR_LAUNCH;
    return product(kept.H, p.hidden, p.WD, p.ldwd, p.width, p.hidden, static_cast<float *>(p.Y), p.ldy);
}

mg_status backward_f32(const GatedProblem &p)
{
    Arena ws = p.workspace;
    const int64_t count = p.tokens * p.hidden;
    const KeptF32 kept(p.kept, p.tokens, p.hidden);
    float *const dG = static_cast<float *>(ws.take(2 * count * F)), *const dU = dG + count;
    const size_t room = ws.left();
    void *const scratch = ws.take(0);
    auto product = [&](int ta, int64_t m, int64_t n, int64_t k, const void *A, int64_t lda, const void *B, int64_t ldb, float beta, void *C, int64_t ldc) {
        return mg_sgemm(MG_ROW_MAJOR, ta, MG_NO_TRANS, m, n, k, 1.f, static_cast<const float *>(A), lda, static_cast<const float *>(B), ldb, beta, static_cast<float *>(C),
                        ldc, scratch, room, p.stream);
    };
    mg_status st = MG_OK;
    if (p.dX != nullptr || p.dWG != nullptr || p.dWU != nullptr) {
        st = product(MG_NO_TRANS, p.tokens, p.hidden, p.width, p.dY, p.lddy, p.WD, p.ldwd, 0.f, dG, p.hidden);
        if (st != MG_OK) return st;
        gated_grad_kernel<<<pieces(count), 256, 0, p.stream>>>(kept.G, kept.U, dG, dU, count);
        if (hipGetLastError() != hipSuccess) return MG_ERR_LAUNCH;
    }
    if (p.dX != nullptr) {
        st = product(MG_NO_TRANS, p.tokens, p.width, p.hidden, dG, p.hidden, p.WG, p.ldwg, 0.f, p.dX, p.lddx);
        if (st == MG_OK) st = product(MG_NO_TRANS, p.tokens, p.width, p.hidden, dU, p.hidden, p.WU, p.ldwu, 1.f, p.dX, p.lddx);
    }
    if (st == MG_OK && p.dWG != nullptr) st = product(MG_TRANS, p.hidden, p.width, p.tokens, dG, p.hidden, p.X, p.ldx, 0.f, p.dWG, p.lddwg);
    if (st == MG_OK && p.dWU != nullptr) st = product(MG_TRANS, p.hidden, p.width, p.tokens, dU, p.hidden, p.X, p.ldx, 0.f, p.dWU, p.lddwu);
    if (st == MG_OK && p.dWD != nullptr) st = product(MG_TRANS, p.width, p.hidden, p.tokens, p.dY, p.lddy, kept.H, p.hidden, 0.f, p.dWD, p.lddwd);
    return st;
}

// 16 bits: a and b in front of H
size_t kept_front(int dtype, int64_t tokens, int64_t hidden) { return static_cast<size_t>(kept_block((tokens + 15) / 16 * 16, 0, hidden) * kept_block_bytes(dtype) + 255) / 256 * 256; }
size_t held_rows(int64_t tokens, int64_t cols) { return static_cast<size_t>(tokens * padded(cols)) * 2; }

mg_status launched(hipError_t e) { return e == hipSuccess ? MG_OK : MG_ERR_LAUNCH; }

// An operand of the caller, or its copy
struct Operand {
    const void *at;
    int64_t ld;
    bool padded;
};

// Operands that the direct-to-LDS kernels do not take as they are get a copy while the workspace has room.  `along`: the operand lies along a sum.
class Copies {
  public:
    Copies(Arena &ws, bool wanted) : ws_(ws), wanted_(wanted) {}
    Operand operator()(const void *X, int64_t ld, int64_t rows, int64_t cols, bool along)
    {
        const bool fine = reinterpret_cast<uintptr_t>(X) % 16 == 0 && ld % 8 == 0 && (!along || cols % 8 == 0);
        const size_t bytes = static_cast<size_t>(rows * padded(cols)) * 2;
        if (fine || !wanted_ || ws_.left() < bytes) return {X, ld, false};
        const int n = list_.count++;
        list_.from[n] = X; list_.to[n] = ws_.take(bytes); list_.ld[n] = ld; list_.rows[n] = rows; list_.cols[n] = static_cast<int>(cols);
        return {list_.to[n], padded(cols), true};
    }
    hipError_t launch(hipStream_t stream) const { return launch_linear_copies(list_, stream); }

  private:
    Arena &ws_;
    bool wanted_;
    LinearCopies list_{};
};

// A forward pass of few tokens reads its weights once, wherever their rows start; all else is faster with copies (width 1000, hidden 2000, rows at odd elements, without and
// with copies: 33 tokens forward 38 and 25 us, backward 75 and 45; 1024 tokens 73 and 38, 232 and 77).
bool copies_pay(int64_t tokens, bool backward) { return backward || tokens > LINEAR_FEW_ROWS; }
size_t copy_bytes(int64_t rows, int64_t cols) { return (static_cast<size_t>(rows * padded(cols)) * 2 + 255) / 256 * 256; }

// what dense operands need
size_t copies_room(int64_t tokens, int64_t width, int64_t hidden, bool backward)
{
    if (!copies_pay(tokens, backward)) return 0;
    size_t room = 0;
    if (width % 8 != 0) room += copy_bytes(tokens, width) * (backward ? 2 : 1) + 2 * copy_bytes(hidden, width);
    if (hidden % 8 != 0) room += copy_bytes(width, hidden);
    return room;
}

size_t forward_room(int64_t tokens, int64_t width, int64_t hidden) { return linear_room(FORM_KK, END_STORE, tokens, width, hidden); }
size_t backward_room(int64_t tokens, int64_t width, int64_t hidden)
{
    size_t most = linear_room(FORM_KN, END_STORE, tokens, width, 2 * padded(hidden));
    for (const size_t v : {linear_room(FORM_NN, END_STORE, 2 * padded(hidden), width, tokens), linear_room(FORM_NN, END_STORE, width, hidden, tokens)}) most = v > most ? v : most;
    return most;
}

void gate(LinearArgs &a, const Operand &q) { a.Q0 = q.at; a.ldq0 = q.ld; a.q_padded = q.padded; }
void left(LinearArgs &a, const Operand &p) { a.P = p.at; a.ldp = p.ld; a.p_padded = p.padded; }

mg_status forward_16(const GatedProblem &p)
{
    Arena ws = p.workspace;
    void *const H = p.kept != nullptr ? static_cast<char *>(p.kept) + kept_front(p.dtype, p.tokens, p.hidden) : ws.take(held_rows(p.tokens, p.hidden));
    const size_t wanted = forward_room(p.tokens, p.width, p.hidden), room_bytes = wanted < ws.left() ? wanted : ws.left();
    void *const room = ws.take(room_bytes);
    Copies copied(ws, copies_pay(p.tokens, false));
    const Operand x = copied(p.X, p.ldx, p.tokens, p.width, true), wg = copied(p.WG, p.ldwg, p.hidden, p.width, true), wu = copied(p.WU, p.ldwu, p.hidden, p.width, true),
                  wd = copied(p.WD, p.ldwd, p.width, p.hidden, true);
    if (const hipError_t e = copied.launch(p.stream)) return launched(e);
    LinearArgs a{};
    left(a, x);
    gate(a, wg);
    a.Q1 = wu.at; a.ldq1 = wu.ld; a.q_padded = wg.padded && wu.padded;
    a.rows = static_cast<int>(p.tokens); a.cols = static_cast<int>(kept_blocks(p.hidden) * 32); a.k = static_cast<int>(p.width);
    a.hidden = static_cast<int>(p.hidden); a.activation = p.activation; a.kept = p.kept;
    a.C0 = H; a.ldc0 = padded(p.hidden);
    if (const hipError_t e = launch_linear(p.dtype, FORM_KK, END_GATED, a, nullptr, 0, p.stream)) return launched(e);
    LinearArgs b{};
    left(b, {H, padded(p.hidden), true});
    gate(b, wd);
    b.rows = a.rows; b.cols = static_cast<int>(p.width); b.k = static_cast<int>(p.hidden);
    b.C0 = p.Y; b.ldc0 = p.ldy;
    return launched(launch_linear(p.dtype, FORM_KK, END_STORE, b, room, room_bytes, p.stream));
}

mg_status backward_16(const GatedProblem &p)
{
    Arena ws = p.workspace;
    const int64_t half = padded(p.hidden);
    void *const d = ws.take(held_rows(p.tokens, p.hidden) * 2);         // dG and dU, side by side
    const size_t wanted = backward_room(p.tokens, p.width, p.hidden), room_bytes = wanted < ws.left() ? wanted : ws.left();
    void *const room = ws.take(room_bytes);
    const bool inner = p.dX != nullptr || p.dWG != nullptr || p.dWU != nullptr, gates = p.dWG != nullptr || p.dWU != nullptr;
    Copies copied(ws, copies_pay(p.tokens, true));
    const Operand none{nullptr, 0, false};
    const Operand dy = copied(p.dY, p.lddy, p.tokens, p.width, inner), x = gates ? copied(p.X, p.ldx, p.tokens, p.width, false) : none,
                  wd = inner ? copied(p.WD, p.ldwd, p.width, p.hidden, false) : none, wg = p.dX != nullptr ? copied(p.WG, p.ldwg, p.hidden, p.width, false) : none,
                  wu = p.dX != nullptr ? copied(p.WU, p.ldwu, p.hidden, p.width, false) : none;
    if (const hipError_t e = copied.launch(p.stream)) return launched(e);
    const int tokens = static_cast<int>(p.tokens), width = static_cast<int>(p.width), hidden = static_cast<int>(p.hidden);
    const Operand both{d, 2 * half, true};
    if (inner) {
        LinearArgs a{};
        left(a, dy);
        gate(a, wd);
        a.rows = tokens; a.cols = hidden; a.k = width;
        a.hidden = hidden; a.kept = p.kept;
        a.C0 = d; a.ldc0 = 2 * half;
        if (const hipError_t e = launch_linear(p.dtype, FORM_KN, END_GATED_GRAD, a, nullptr, 0, p.stream)) return launched(e);
    }
    LinearTogether last{};
    if (p.dX != nullptr) {
        LinearArgs &a = last.of[0];
        left(a, both);
        gate(a, wg);
        a.Q1 = wu.at; a.ldq1 = wu.ld;
        a.segment = static_cast<int>(half); a.lines = hidden;
        a.rows = tokens; a.cols = width; a.k = static_cast<int>(2 * half);
        a.C0 = p.dX; a.ldc0 = p.lddx;
    }
    if (gates) {
        LinearArgs &a = last.of[1];
        left(a, both);
        gate(a, x);
        a.rows = static_cast<int>(2 * half); a.cols = width; a.k = tokens;
        a.second = static_cast<int>(half); a.rows0 = hidden;
        a.C0 = p.dWG; a.ldc0 = p.lddwg; a.C1 = p.dWU; a.ldc1 = p.lddwu;
    }
    if (p.dWD != nullptr) {
        LinearArgs &a = last.of[2];
        left(a, dy);
        gate(a, {static_cast<char *>(p.kept) + kept_front(p.dtype, p.tokens, p.hidden), half, true});
        a.rows = width; a.cols = hidden; a.k = tokens;
        a.C0 = p.dWD; a.ldc0 = p.lddwd;
    }
    return launched(launch_linear_together(p.dtype, last, room, room_bytes, p.stream));
}

}  // namespace

size_t gated_kept(int dtype, int64_t tokens, int64_t hidden)
{
    return dtype == MG_F32 ? static_cast<size_t>(3 * tokens * hidden) * F : kept_front(dtype, tokens, hidden) + held_rows(tokens, hidden);
}

size_t gated_workspace(int dtype, int64_t tokens, int64_t width, int64_t hidden, bool backward)
{
    Arena ws{nullptr, 0, 0};
    if (dtype == MG_F32) {
        ws.take(static_cast<size_t>((backward ? 2 : 3) * tokens * hidden) * F);
        ws.take(sgemm_room(tokens, width, hidden, backward));
    } else {
        ws.take(held_rows(tokens, hidden) * (backward ? 2 : 1));
        ws.take(backward ? backward_room(tokens, width, hidden) : forward_room(tokens, width, hidden));
        ws.take(copies_room(tokens, width, hidden, backward));
    }
    return ws.used;
}

mg_status gated_forward(const GatedProblem &p) { return p.dtype == MG_F32 ? forward_f32(p) : forward_16(p); }
mg_status gated_backward(const GatedProblem &p) { return p.dtype == MG_F32 ? backward_f32(p) : backward_16(p); }

}  // namespace mg
