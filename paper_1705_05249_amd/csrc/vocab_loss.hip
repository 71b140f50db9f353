// Softmax cross entropy over a vocabulary, with the projection in it.
//
// Logits of 16-bit matrices stay in the registers of the product's kernel: a tile leaves the largest one and the sum of exponentials of each of its
// rows, and a second kernel joins the tiles (the running maximum and sum of a softmax, over tiles).  The gradient makes the logits again, a piece of the
// vocabulary at a time, and leaves dz = w (exp(z - lse) - [target]) in the operands' type for the two products that read it: dX is a sum over all
// pieces, in FP32 slices that are added in the pieces' order, dW's rows belong to one piece each.  FP32: pieces of logits in memory, products as mg_sgemm makes them.
#include "linear_end.h"
#include "internal.h"

namespace mg {
namespace {

constexpr int64_t F = sizeof(float);
constexpr int64_t PIECE_ELEMENTS = int64_t(1) << 28;              // of dz in 16 bits; FP32: logits, a quarter as many

// FP32 slices of dX, one for each piece.  Where there are more pieces, the first slice takes the sum of all whenever they are full, in the order in which one launch would add
// them: the bits are the same.  A slice for every piece, whose columns are 2^28 / tokens, would take memory that grows with tokens^2 (131072 tokens of width 4096, 131072 words:
// 130 GiB, 9.6 so).  Gradient of 32768 x 2048 x 131072, 16 pieces: 4.63 -> 1.63 GiB, 40.7 -> 40.9 ms; of 65536 x 1024 x 65536: 4.69 -> 1.69 GiB, 23.7 -> 24.0.
constexpr int64_t MOST_SLICES = 4;

// columns of a piece: a multiple of 256, or the vocabulary
int64_t piece_columns(int dtype, int64_t tokens, int64_t vocab)
{
    const int64_t most = (dtype == MG_F32 ? PIECE_ELEMENTS / 4 : PIECE_ELEMENTS) / tokens / 256 * 256;
    const int64_t columns = most < 256 ? 256 : most;
    return columns < vocab ? columns : vocab;
}

mg_status launched(hipError_t e) { return e == hipSuccess ? MG_OK : MG_ERR_LAUNCH; }

constexpr int CHUNK = 4096;             // logits of a row that a work-group of the FP32 kernels has, 16 in a thread

// FP32: (largest, sum of exponentials) of a chunk of a row of logits, and the target's logit.  z is read once.
__global__ __launch_bounds__(256) void scores_kernel(const float *Z, int64_t ldz, int cols, int64_t first, int tokens, const int64_t *targets, float2 *scores, float *target_score)
{
    __shared__ float parts[4];
    const int row = blockIdx.x, lane = threadIdx.x % 64, wave = threadIdx.x / 64, start = blockIdx.y * CHUNK;
    const float *z = Z + row * ldz + start;
    const int here = cols - start < CHUNK ? cols - start : CHUNK;
    float v[4][4], m = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = (i * 256 + static_cast<int>(threadIdx.x)) * 4;
        load_piece<float, 4>(z + c, here - c > 0 ? here - c : 0, v[i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (c + e >= here) v[i][e] = -__builtin_inff();
            m = fmaxf(m, v[i][e]);
        }
    }
    for (int d = 32; d > 0; d /= 2) m = fmaxf(m, __shfl_xor(m, d));
    if (lane == 0) parts[wave] = m;
    __syncthreads();
    m = fmaxf(fmaxf(parts[0], parts[1]), fmaxf(parts[2], parts[3]));
    __syncthreads();
    const float from = m == -__builtin_inff() ? 0.f : m;
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) s += expf(v[i][e] - from);
    for (int d = 32; d > 0; d /= 2) s += __shfl_xor(s, d);
    if (lane == 0) parts[wave] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        scores[static_cast<int64_t>(blockIdx.y) * tokens + row] = make_float2(m, (parts[0] + parts[1]) + (parts[2] + parts[3]));
        const int64_t t = targets[row] - first - start;
        if (t >= 0 && t < here) target_score[row] = z[t];
    }
}

// FP32: dz in the place of z
__global__ __launch_bounds__(256) void scores_grad_kernel(float *Z, int64_t ldz, int cols, int64_t first, int64_t vocab, const int64_t *targets, const float *lse,
                                                          const float *weights)
{
    const int row = blockIdx.x, start = blockIdx.y * CHUNK, here = cols - start < CHUNK ? cols - start : CHUNK;
    const int64_t target = targets[row], at = target - first - start;
    const float w = target >= 0 && target < vocab ? weights == nullptr ? 1.f : weights[row] : 0.f, l = lse[row];
    float *z = Z + row * ldz + start;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = (i * 256 + static_cast<int>(threadIdx.x)) * 4, left = here - c > 0 ? here - c : 0;
        float v[4];
        load_piece<float, 4>(z + c, left, v);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = w != 0.f ? w * (expf(v[e] - l) - (c + e == at ? 1.f : 0.f)) : 0.f;
        store_piece<float, 4>(z + c, left, v);
    }
}

// Joins the tiles' scores in a fixed order: TOKENS tokens a work-group, 256 / TOKENS lanes a token.
template <int TOKENS> __global__ __launch_bounds__(256) void join_scores_kernel(const float2 *scores, int tiles, int tokens, int64_t vocab, const int64_t *targets, const float *target_score,
                                                                                float *loss, float *lse)
{
    constexpr int LANES = 256 / TOKENS;
    const int row = blockIdx.x * TOKENS + threadIdx.x % TOKENS, part = threadIdx.x / TOKENS;
    __shared__ float2 parts[256];
    float2 all = make_float2(-__builtin_inff(), 0.f);
    if (row < tokens)
        for (int t = part; t < tiles; t += LANES) all = join_scores(all, scores[static_cast<int64_t>(t) * tokens + row]);
    parts[threadIdx.x] = all;
    for (int d = LANES / 2; d > 0; d /= 2) {
        __syncthreads();
        if (part < d) parts[threadIdx.x] = all = join_scores(all, parts[threadIdx.x + d * TOKENS]);
    }
    if (part != 0 || row >= tokens) return;
    const float total = all.x + logf(all.y);
    const int64_t target = targets[row];
    lse[row] = total;
    loss[row] = target >= 0 && target < vocab ? total - target_score[row] : 0.f;
}

// FP32: how many scores a token has when the vocabulary goes in pieces
int64_t score_chunks(int64_t vocab, int64_t columns) { return vocab / columns * ceil_div(columns, CHUNK) + ceil_div(vocab % columns, CHUNK); }

struct LossMemory {
    float2 *scores;
    float *target_score, *pieces;          // pieces: FP32 logits
    size_t left;
    void *rest;
};

LossMemory loss_memory(Arena &ws, int dtype, int64_t tokens, int64_t vocab)
{
    LossMemory m{};
    const int64_t columns = vocab > 0 ? piece_columns(dtype, tokens, vocab) : 0;
    m.target_score = static_cast<float *>(ws.take(tokens * F));
    if (dtype == MG_F32) {
        m.scores = static_cast<float2 *>(ws.take(vocab > 0 ? score_chunks(vocab, columns) * tokens * 8 : 0));
        m.pieces = static_cast<float *>(ws.take(tokens * columns * F));
    } else {
        m.scores = static_cast<float2 *>(ws.take(ceil_div(vocab, 64) * tokens * 8));
    }
    m.left = ws.left();
    m.rest = ws.take(0);
    return m;
}

struct LossGradMemory {
    void *x;                               // X without the tokens that do not count, rows of x_lead elements
    int64_t x_lead;
    void *dz;                              // a piece
    float *scale;
    float *slices;
    int64_t slice;                         // elements of one
    void *room;                            // 16 bits: for slices of a product
    size_t room_bytes;
    size_t left;
    void *rest;
};

LossGradMemory loss_grad_memory(Arena &ws, int dtype, int64_t tokens, int64_t width, int64_t vocab)
{
    LossGradMemory m{};
    const int64_t columns = piece_columns(dtype, tokens, vocab), count = ceil_div(vocab, columns);
    m.scale = static_cast<float *>(ws.take(2 * F));
    const int64_t units = dtype == MG_F32 ? 2 : 1;               // of 16 bits
    m.x = ws.take(tokens * padded(width * units) * 2);
    m.x_lead = padded(width * units) / units;
    m.dz = ws.take(tokens * padded(columns) * (dtype == MG_F32 ? 4 : 2));
    m.slice = tokens * padded(width);
    if (dtype != MG_F32) {
        if (count > 1) m.slices = static_cast<float *>(ws.take((count < MOST_SLICES ? count : MOST_SLICES) * m.slice * F));
        else m.room_bytes = linear_room(FORM_KN, END_STORE, tokens, width, columns);
        const size_t other = linear_room(FORM_NN, END_STORE, columns, width, tokens);
        m.room_bytes = other > m.room_bytes ? other : m.room_bytes;
        m.room = ws.take(m.room_bytes);
    }
    m.left = ws.left();
    m.rest = ws.take(0);
    return m;
}

size_t sgemm_room(int64_t tokens, int64_t width, int64_t vocab, bool gradient)
{
    const int64_t columns = piece_columns(MG_F32, tokens, vocab);
    size_t most = 0;
    auto add = [&](int ta, int tb, int64_t m, int64_t n, int64_t k, int64_t lda, int64_t ldb, int64_t ldc) {
        const size_t v = mg_gemm_workspace_bytes(MG_F32, MG_ROW_MAJOR, ta, tb, m, n, k, lda, ldb, ldc);
        most = v > most ? v : most;
    };
    for (int64_t some : {columns, vocab % columns})
        if (some > 0) {
            add(MG_NO_TRANS, MG_TRANS, tokens, some, width, width, width, columns);
            if (gradient) {
                add(MG_NO_TRANS, MG_NO_TRANS, tokens, width, some, columns, width, width);
                add(MG_TRANS, MG_NO_TRANS, some, width, tokens, columns, width, width);
            }
        }
    return most;
}

const float *row_of(const void *X, int64_t row, int64_t ld) { return static_cast<const float *>(X) + row * ld; }

// The loss alone reads W once; where it has rows at odd elements, copying it pays from about 192 tokens on (vocabulary of 32768, width 2048, without and with copies: 128 tokens
// 75 and 74 us, 256 tokens 151 and 88).  The gradient reads it twice more: 33 tokens 210 and 154 us.
bool copies_pay(int64_t tokens, bool gradient) { return gradient || tokens >= 192; }
size_t copies_room(int64_t tokens, int64_t width, int64_t vocab, bool gradient)
{
    return width % 8 != 0 && copies_pay(tokens, gradient) ? static_cast<size_t>(((gradient ? 0 : tokens) + vocab) * padded(width)) * 2 + 512 : 0;
}

// The caller's matrices or copies of them
struct LossOperands {
    const void *X, *W;
    int64_t ldx, ldw;
    bool x_padded, w_padded;
};

// adds a copy to the list, where the direct-to-LDS kernels do not take a matrix along the sum as it is and there is room
bool copy_of(LinearCopies &list, Arena &ws, const void *&at, int64_t &ld, int64_t rows, int64_t width)
{
    const size_t bytes = static_cast<size_t>(rows * padded(width)) * 2;
    if (bytes == 0 || (width % 8 == 0 && reinterpret_cast<uintptr_t>(at) % 16 == 0 && ld % 8 == 0) || ws.left() < bytes) return false;
    const int m = list.count++;
    list.from[m] = at; list.to[m] = ws.take(bytes); list.ld[m] = ld; list.rows[m] = rows; list.cols[m] = static_cast<int>(width);
    at = list.to[m];
    ld = padded(width);
    return true;
}

// the copy of X without the tokens that do not count, first in a list; the scale
void masked_copy(LinearCopies &list, const LossProblem &p, const LossGradMemory &m, float most, float *scale)
{
    const int units = p.dtype == MG_F32 ? 2 : 1;
    list.count = 1;
    list.from[0] = p.X; list.to[0] = m.x; list.ld[0] = p.ldx * units; list.rows[0] = p.tokens; list.cols[0] = static_cast<int>(p.width) * units;
    list.targets = p.targets; list.vocab = p.vocab; list.weights = p.weights;
    list.most = most; list.scale = scale;
}

mg_status loss_f32(const LossProblem &p, const LossMemory &m)
{
    const int64_t columns = piece_columns(MG_F32, p.tokens, p.vocab);
    int64_t done = 0;
    for (int64_t first = 0; first < p.vocab; first += columns) {
        const int64_t some = p.vocab - first < columns ? p.vocab - first : columns, chunks = ceil_div(some, CHUNK);
        const mg_status st = mg_sgemm(MG_ROW_MAJOR, MG_NO_TRANS, MG_TRANS, p.tokens, some, p.width, 1.f, static_cast<const float *>(p.X), p.ldx, row_of(p.W, first, p.ldw), p.ldw, 0.f,
                                      m.pieces, columns, m.rest, m.left, p.stream);
        if (st != MG_OK) return st;
        scores_kernel<<<dim3(static_cast<uint32_t>(p.tokens), static_cast<uint32_t>(chunks)), 256, 0, p.stream>>>(m.pieces, columns, static_cast<int>(some), first, static_cast<int>(p.tokens),
                                                                                                                 p.targets, m.scores + done * p.tokens, m.target_score);
        if (hipGetLastError() != hipSuccess) return MG_ERR_LAUNCH;
        done += chunks;
    }
    return MG_OK;
}

mg_status grad_f32(const LossProblem &p, const LossGradMemory &m)
{
    const int64_t columns = piece_columns(MG_F32, p.tokens, p.vocab);
    float *const Z = static_cast<float *>(m.dz);
    const float *const X = static_cast<const float *>(m.x);
    LinearCopies list{};
    masked_copy(list, p, m, 1.f, nullptr);
    if (const hipError_t e = launch_linear_copies(list, p.stream)) return launched(e);
    for (int64_t first = 0; first < p.vocab; first += columns) {
        const int64_t some = p.vocab - first < columns ? p.vocab - first : columns;
        const float *W = row_of(p.W, first, p.ldw);
        mg_status st = mg_sgemm(MG_ROW_MAJOR, MG_NO_TRANS, MG_TRANS, p.tokens, some, p.width, 1.f, X, m.x_lead, W, p.ldw, 0.f, Z, columns, m.rest, m.left, p.stream);
        if (st != MG_OK) return st;
        scores_grad_kernel<<<dim3(static_cast<uint32_t>(p.tokens), static_cast<uint32_t>(ceil_div(some, CHUNK))), 256, 0, p.stream>>>(Z, columns, static_cast<int>(some), first, p.vocab, p.targets, p.lse, p.weights);
        if (hipGetLastError() != hipSuccess) return MG_ERR_LAUNCH;
        if (p.dX != nullptr)
            st = mg_sgemm(MG_ROW_MAJOR, MG_NO_TRANS, MG_NO_TRANS, p.tokens, p.width, some, 1.f, Z, columns, W, p.ldw, first > 0 ? 1.f : 0.f, static_cast<float *>(p.dX), p.lddx, m.rest,
                          m.left, p.stream);
        if (st == MG_OK && p.dW != nullptr)
            st = mg_sgemm(MG_ROW_MAJOR, MG_TRANS, MG_NO_TRANS, some, p.width, p.tokens, 1.f, Z, columns, X, m.x_lead, 0.f, static_cast<float *>(p.dW) + first * p.lddw, p.lddw, m.rest, m.left,
                          p.stream);
        if (st != MG_OK) return st;
    }
    return MG_OK;
}

LinearArgs logits(const LossProblem &p, const LossOperands &o, int64_t first, int64_t columns)
{
    LinearArgs a{};
    a.P = o.X; a.ldp = o.ldx; a.p_padded = o.x_padded; a.q_padded = o.w_padded;
    a.Q0 = static_cast<const uint16_t *>(o.W) + first * o.ldw; a.ldq0 = o.ldw;
    a.rows = static_cast<int>(p.tokens); a.cols = static_cast<int>(columns); a.k = static_cast<int>(p.width);
    a.first = first; a.vocab = p.vocab; a.targets = p.targets;
    return a;
}

mg_status grad_16(const LossProblem &p, const LossGradMemory &m, Arena &ws)
{
    LossOperands o{m.x, p.W, m.x_lead, p.ldw, true, false};
    LinearCopies list{};
    float *const scale = p.weights != nullptr || p.dtype == MG_F16 ? m.scale : nullptr;
    masked_copy(list, p, m, p.dtype == MG_F16 ? 8192.f : 1.f, scale);
    if (copies_pay(p.tokens, true)) o.w_padded = copy_of(list, ws, o.W, o.ldw, p.vocab, p.width);
    if (const hipError_t e = launch_linear_copies(list, p.stream)) return launched(e);
    const int64_t columns = piece_columns(p.dtype, p.tokens, p.vocab), lead = padded(columns);
    const int64_t count = ceil_div(p.vocab, columns);
    int held = 0;                                          // slices of dX that are full
    LinearTogether both{};
    LinearArgs x{};                                        // dX
    x.P = m.dz; x.ldp = lead; x.p_padded = true; x.ldq0 = o.ldw;
    x.rows = static_cast<int>(p.tokens); x.cols = static_cast<int>(p.width);
    x.C0 = p.dX; x.ldc0 = p.lddx;
    x.scale = scale == nullptr ? nullptr : scale + 1;
    x.partial_ld = padded(p.width);
    x.partial_stride = m.slice;
    for (int64_t first = 0; first < p.vocab; first += columns) {
        const int64_t some = p.vocab - first < columns ? p.vocab - first : columns;
        LinearArgs z = logits(p, o, first, some);
        z.lse = p.lse; z.weights = p.weights; z.weight_scale = scale;
        z.C0 = m.dz; z.ldc0 = lead;
        if (const hipError_t e = launch_linear(p.dtype, FORM_KK, END_SCORES_GRAD, z, nullptr, 0, p.stream)) return launched(e);
        if (p.dX != nullptr) {
            x.Q0 = z.Q0;
            x.k = static_cast<int>(some);
            if (held == MOST_SLICES) {
                LinearArgs sum = x;
                sum.partial = m.slices;
                sum.C0 = m.slices; sum.ldc0 = x.partial_ld; sum.scale = nullptr;
                if (const hipError_t e = launch_linear_sum(MG_F32, sum, held, p.stream)) return launched(e);
                held = 1;
            }
            x.partial = count > 1 ? m.slices + held++ * m.slice : nullptr;
            both.of[0] = x;
        }
        if (p.dW != nullptr) {
            LinearArgs &w = both.of[1];
            w.P = m.dz; w.ldp = lead; w.Q0 = o.X; w.ldq0 = o.ldx;
            w.rows = static_cast<int>(some); w.cols = static_cast<int>(p.width); w.k = static_cast<int>(p.tokens);
            w.C0 = static_cast<uint16_t *>(p.dW) + first * p.lddw; w.ldc0 = p.lddw;
            w.scale = x.scale;
        }
        if (const hipError_t e = launch_linear_together(p.dtype, both, m.room, m.room_bytes, p.stream)) return launched(e);
    }
    if (p.dX != nullptr && count > 1) {
        x.partial = m.slices;
        return launched(launch_linear_sum(p.dtype, x, held, p.stream));
    }
    return MG_OK;
}

}  // namespace

size_t loss_workspace(int dtype, int64_t tokens, int64_t width, int64_t vocab, bool gradient)
{
    Arena ws{nullptr, 0, 0};
    if (gradient) loss_grad_memory(ws, dtype, tokens, width, vocab);
    else loss_memory(ws, dtype, tokens, vocab);
    if (vocab > 0) ws.take(dtype == MG_F32 ? sgemm_room(tokens, width, vocab, gradient) : copies_room(tokens, width, vocab, gradient));
    return ws.used;
}

mg_status vocab_loss(const LossProblem &p)
{
    Arena ws = p.workspace;
    const LossMemory m = loss_memory(ws, p.dtype, p.tokens, p.vocab);
    int tiles = 0;
    if (p.vocab > 0 && p.dtype == MG_F32) {
        if (const mg_status st = loss_f32(p, m)) return st;
        tiles = static_cast<int>(score_chunks(p.vocab, piece_columns(MG_F32, p.tokens, p.vocab)));
    } else if (p.vocab > 0) {
        LossOperands o{p.X, p.W, p.ldx, p.ldw, false, false};
        LinearCopies list{};
        if (copies_pay(p.tokens, false)) {
            o.x_padded = copy_of(list, ws, o.X, o.ldx, p.tokens, p.width);
            o.w_padded = copy_of(list, ws, o.W, o.ldw, p.vocab, p.width);
        }
        if (const hipError_t e = launch_linear_copies(list, p.stream)) return launched(e);
        LinearArgs a = logits(p, o, 0, p.vocab);
        a.scores = m.scores;
        a.target_score = m.target_score;
        int columns = 0;
        if (const hipError_t e = launch_linear(p.dtype, FORM_KK, END_SCORES, a, nullptr, 0, p.stream, &columns)) return launched(e);
        tiles = static_cast<int>(ceil_div(p.vocab, columns));
    }
    auto join = [&](auto each) {
        constexpr int TOKENS = decltype(each)::value;
        join_scores_kernel<TOKENS><<<static_cast<uint32_t>(ceil_div(p.tokens, TOKENS)), 256, 0, p.stream>>>(m.scores, tiles, static_cast<int>(p.tokens), p.vocab, p.targets, m.target_score, p.loss,
                                                                                                          p.lse);
    };
    // (few tokens: a work-group each, 16 tokens of 512 tiles 11.9 us otherwise)
    if (p.tokens <= 512) join(std::integral_constant<int, 1>{});
    else join(std::integral_constant<int, 16>{});
    return launched(hipGetLastError());
}

mg_status vocab_loss_grad(const LossProblem &p)
{
    Arena ws = p.workspace;
    const LossGradMemory m = loss_grad_memory(ws, p.dtype, p.tokens, p.width, p.vocab);
    return p.dtype == MG_F32 ? grad_f32(p, m) : grad_16(p, m, ws);
}

}  // namespace mg
