// Boundary of mg_experts.h: argument checks in status-code order, canonical problems, launches.  As in api.hip nothing is allocated, copied or
// synchronised, and validation touches no HIP API.
#include "internal.h"
#include "experts.h"

namespace mg {
namespace {

constexpr int64_t MOST_EXTENT = (int64_t(1) << 31) - 1024;        // every extent below it (kernels round them up in 32 bits)
constexpr __int128 MOST_ELEMENTS = __int128(1) << 40;             // of a stored matrix
constexpr __int128 MOST_PIECES = __int128(1) << 24;               // work-groups of 256 threads that a launch does not reach

bool extent(int64_t v) { return v >= 0 && v < MOST_EXTENT; }
bool stored(int64_t rows, int64_t ld) { return __int128(rows) * ld <= MOST_ELEMENTS; }
bool type_known(int dtype) { return dtype == MG_F32 || dtype == MG_F16 || dtype == MG_BF16; }
bool block_known(int block) { return block == MG_BLOCK_ROW || block == MG_BLOCK_SQUARE; }
bool groups_known(int groups) { return groups >= 1 && groups <= MG_MOST_GROUPS; }
bool fan_known(int fan) { return fan >= 1 && fan <= MG_MOST_FAN; }
bool at_least(int64_t ld, int64_t width) { return ld >= (width > 1 ? width : 1); }
int64_t blocks(int64_t size) { return ceil_div(size, SCALE_BLOCK); }
mg_status launched(hipError_t e) { return e == hipSuccess ? MG_OK : MG_ERR_LAUNCH; }
// a missing, misaligned or small workspace is none
size_t usable(const void *workspace, size_t bytes) { return workspace != nullptr && reinterpret_cast<uintptr_t>(workspace) % 256 == 0 ? bytes : 0; }

// turned_cols: width of the transposed result
mg_status quantize(QuantizeProblem &p, int block, int64_t turned_cols)
{
    if (!extent(p.rows) || !extent(p.cols)) return MG_ERR_DIM;
    if (__int128(blocks(p.rows) + p.groups.count) * blocks(p.cols) * 8 >= MOST_PIECES) return MG_ERR_DIM;
    const bool q = p.Q != nullptr || p.S != nullptr, t = p.T != nullptr || p.ST != nullptr;
    if (!at_least(p.ldx, p.cols)) return MG_ERR_LDA;
    if (q && !at_least(p.ldq, p.cols)) return MG_ERR_LDB;
    if (t && !at_least(p.ldt, turned_cols)) return MG_ERR_LDC;
    if (!stored(p.rows, p.ldx) || (q && !stored(p.rows, p.ldq)) || (t && !stored(p.cols, p.ldt))) return MG_ERR_DIM;
    const bool empty = p.rows == 0 || p.cols == 0 || p.batch == 0;
    if (!empty && (p.X == nullptr || (p.groups.count > 0 && p.groups.offsets == nullptr) || (!q && !t) || (q && (p.Q == nullptr || p.S == nullptr)) || (t && (p.T == nullptr || p.ST == nullptr)))) return MG_ERR_NULL;
    if (p.batch < 0 || p.batch > 65535) return MG_ERR_BATCH;
    if (p.stride_x < 0 || p.stride_q < 0 || p.stride_s < 0 || p.stride_t < 0 || p.stride_st < 0) return MG_ERR_STRIDE;
    if (!type_known(p.dtype)) return MG_ERR_TYPE;
    if (!block_known(block)) return MG_ERR_BLOCK;
    p.square = block == MG_BLOCK_SQUARE;
    if ((q && !at_least(p.lds, blocks(p.cols))) || (t && !at_least(p.ldst, blocks(turned_cols)))) return MG_ERR_SCALES;
    return empty ? MG_OK : launched(launch_quantize(p));
}

// `scales` without the flag that asks for FP32 sums
int kind_of(int scales) { return scales & ~MG_SUMS_FP32; }
bool scales_known(int scales) { return kind_of(scales) == MG_SCALES_ANY || kind_of(scales) == MG_SCALES_POW2; }
bool sums_fp32(int scales, int c_type) { return c_type == MG_F32 || (scales & MG_SUMS_FP32) != 0; }

// The tiles of a product fit a launch
bool tiles_fit(int64_t m, int64_t n, int groups) { return __int128(blocks(m) + groups) * 2 * blocks(n) * 8 <= MOST_PIECES; }

}  // namespace
}  // namespace mg

using namespace mg;

extern "C" {

mg_status mg_block_quantize(int dtype, int block, int64_t rows, int64_t cols, const void *X, int64_t ldx, uint8_t *Q, int64_t ldq, float *S,
                            int64_t lds, uint8_t *T, int64_t ldt, float *ST, int64_t ldst, void *stream)
{
    return mg_block_quantize_batched(dtype, block, 1, rows, cols, X, ldx, 0, Q, ldq, 0, S, lds, 0, T, ldt, 0, ST, ldst, 0, stream);
}

mg_status mg_block_quantize_batched(int dtype, int block, int64_t batch, int64_t rows, int64_t cols, const void *X, int64_t ldx, int64_t stride_x,
                                    uint8_t *Q, int64_t ldq, int64_t stride_q, float *S, int64_t lds, int64_t stride_s,
                                    uint8_t *T, int64_t ldt, int64_t stride_t, float *ST, int64_t ldst, int64_t stride_st, void *stream)
{
    QuantizeProblem p{dtype, false, rows, cols, batch, X, ldx, stride_x, Q, ldq, stride_q, S, lds, stride_s, T, ldt, stride_t, ST, ldst, stride_st,
                      Groups{nullptr, 0, rows, nullptr, 1}, static_cast<hipStream_t>(stream)};
    return quantize(p, block, rows);
}

mg_status mg_block_quantize_grouped(int dtype, int groups, const int32_t *offsets, int64_t rows, int64_t cols, const void *X, int64_t ldx,
                                    const int32_t *source, int fan, uint8_t *Q, int64_t ldq, float *S, int64_t lds, uint8_t *T, int64_t ldt,
                                    float *ST, int64_t ldst, void *stream)
{
    QuantizeProblem p{dtype, false, rows, cols, 1, X, ldx, 0, Q, ldq, 0, S, lds, 0, T, ldt, 0, ST, ldst, 0,
                      Groups{offsets, groups, rows, source, fan}, static_cast<hipStream_t>(stream)};
    if (!extent(rows) || !extent(cols)) return MG_ERR_DIM;
    if (!groups_known(groups) || !fan_known(fan)) {
        p.groups.count = 1;
        p.rows = 0;                                   // (the errors of arguments with smaller codes come first)
        p.lds = p.ldst = MOST_EXTENT;
        const mg_status st = quantize(p, MG_BLOCK_ROW, rows);
        return st != MG_OK ? st : MG_ERR_GROUPS;
    }
    return quantize(p, MG_BLOCK_ROW, mg_grouped_columns(rows, groups));
}

int64_t mg_grouped_columns(int64_t rows, int groups)
{
    return extent(rows) && groups_known(groups) ? (blocks(rows) + groups) * SCALE_BLOCK : -1;
}

mg_status mg_block_gemm(int layout, int64_t m, int64_t n, int64_t k, float alpha, int scales, int a_block, const uint8_t *A, int64_t lda,
                        const float *SA, int64_t ldsa, int b_block, const uint8_t *B, int64_t ldb, const float *SB, int64_t ldsb, float beta,
                        int c_type, void *C, int64_t ldc, void *workspace, size_t workspace_bytes, void *stream)
{
    if (layout != MG_ROW_MAJOR && layout != MG_COL_MAJOR) return MG_ERR_LAYOUT;
    const bool row = layout == MG_ROW_MAJOR;
    if (!extent(m) || !extent(n) || !extent(k) || !tiles_fit(m, n, 0) || !tiles_fit(n, m, 0)) return MG_ERR_DIM;
    if (!at_least(lda, k)) return MG_ERR_LDA;
    if (!at_least(ldb, k)) return MG_ERR_LDB;
    if (!at_least(ldc, row ? n : m)) return MG_ERR_LDC;
    if (!stored(m, lda) || !stored(n, ldb) || !stored(row ? m : n, ldc)) return MG_ERR_DIM;
    const bool empty = m == 0 || n == 0, reads = alpha != 0.f && k > 0;
    if (!empty && (C == nullptr || (reads && (A == nullptr || B == nullptr || SA == nullptr || SB == nullptr)))) return MG_ERR_NULL;
    if (!type_known(c_type)) return MG_ERR_TYPE;
    if (!block_known(a_block) || !block_known(b_block) || !scales_known(scales)) return MG_ERR_BLOCK;
    if (!at_least(ldsa, blocks(k)) || !at_least(ldsb, blocks(k))) return MG_ERR_SCALES;
    if (empty) return MG_OK;
    BlockProblem p{};
    p.mode = BLOCK_DENSE;
    p.k = k;
    p.alpha = alpha;
    p.beta = beta;
    p.pow2 = kind_of(scales) == MG_SCALES_POW2;
    p.fp32_sums = sums_fp32(scales, c_type);
    p.A = A; p.lda = lda; p.SA = SA; p.ldsa = ldsa; p.a_square = a_block == MG_BLOCK_SQUARE; p.m = m;
    p.B = B; p.ldb = ldb; p.SB = SB; p.ldsb = ldsb; p.b_square = b_block == MG_BLOCK_SQUARE; p.n = n;
    if (!row) {                                       // column-major C = A B^T is row-major C^T = B A^T on the same bytes
        p.A = B; p.lda = ldb; p.SA = SB; p.ldsa = ldsb; p.a_square = b_block == MG_BLOCK_SQUARE; p.m = n;
        p.B = A; p.ldb = lda; p.SB = SA; p.ldsb = ldsa; p.b_square = a_block == MG_BLOCK_SQUARE; p.n = m;
    }
    p.c_type = c_type; p.C = C; p.ldc = ldc;
    p.groups = Groups{nullptr, 0, m, nullptr, 1};
    p.workspace_bytes = usable(workspace, workspace_bytes);
    p.workspace = workspace;
    p.stream = static_cast<hipStream_t>(stream);
    return launched(launch_block_gemm(p));
}

size_t mg_block_gemm_workspace_bytes(int64_t m, int64_t n, int64_t k)
{
    if (!extent(m) || !extent(n) || !extent(k) || m == 0 || n == 0) return 0;
    const size_t a = block_gemm_workspace(BLOCK_DENSE, 0, m, n, k), b = block_gemm_workspace(BLOCK_DENSE, 0, n, m, k);      // (either layout)
    return a > b ? a : b;
}

mg_status mg_block_gemm_grouped(int groups, const int32_t *offsets, int64_t rows, int64_t n, int64_t k, float alpha, int scales, const uint8_t *A,
                                int64_t lda, const float *SA, int64_t ldsa, const int32_t *source, int fan, int b_block, const uint8_t *B,
                                int64_t ldb, int64_t stride_b, const float *SB, int64_t ldsb, int64_t stride_sb, float beta, int c_type, void *C,
                                int64_t ldc, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!extent(rows) || !extent(n) || !extent(k) || !tiles_fit(rows, n, groups_known(groups) ? groups : 1)) return MG_ERR_DIM;
    if (!at_least(lda, k)) return MG_ERR_LDA;
    if (!at_least(ldb, k)) return MG_ERR_LDB;
    if (!at_least(ldc, n)) return MG_ERR_LDC;
    if (!stored(rows, lda) || !stored(n, ldb) || !stored(rows, ldc)) return MG_ERR_DIM;
    const bool empty = rows == 0 || n == 0, reads = alpha != 0.f && k > 0;
    if (!empty && (C == nullptr || offsets == nullptr || (reads && (A == nullptr || B == nullptr || SA == nullptr || SB == nullptr)))) return MG_ERR_NULL;
    if (stride_b < 0 || stride_sb < 0) return MG_ERR_STRIDE;
    if (!type_known(c_type)) return MG_ERR_TYPE;
    if (!block_known(b_block) || !scales_known(scales)) return MG_ERR_BLOCK;
    if (!groups_known(groups) || !fan_known(fan)) return MG_ERR_GROUPS;
    if (!at_least(ldsa, blocks(k)) || !at_least(ldsb, blocks(k))) return MG_ERR_SCALES;
    if (empty) return MG_OK;
    BlockProblem p{};
    p.mode = BLOCK_ROWS;
    p.m = rows; p.n = n; p.k = k;
    p.alpha = alpha; p.beta = beta;
    p.pow2 = kind_of(scales) == MG_SCALES_POW2;
    p.fp32_sums = sums_fp32(scales, c_type);
    p.A = A; p.lda = lda; p.SA = SA; p.ldsa = ldsa; p.a_square = false;
    p.B = B; p.ldb = ldb; p.stride_b = stride_b; p.SB = SB; p.ldsb = ldsb; p.stride_sb = stride_sb; p.b_square = b_block == MG_BLOCK_SQUARE;
    p.c_type = c_type; p.C = C; p.ldc = ldc;
    p.groups = Groups{offsets, groups, rows, source, fan};
    p.workspace_bytes = usable(workspace, workspace_bytes);
    p.workspace = workspace;
    p.stream = static_cast<hipStream_t>(stream);
    return launched(launch_block_gemm(p));
}

size_t mg_block_gemm_grouped_workspace_bytes(int groups, int64_t rows, int64_t n, int64_t k)
{
    if (!groups_known(groups) || !extent(rows) || !extent(n) || !extent(k) || rows == 0 || n == 0) return 0;
    return block_gemm_workspace(BLOCK_ROWS, groups, rows, n, k);
}

mg_status mg_block_gemm_grouped_sum(int groups, const int32_t *offsets, int64_t rows, int64_t m, int64_t n, float alpha, int scales, const uint8_t *A,
                                    int64_t lda, const float *SA, int64_t ldsa, const uint8_t *B, int64_t ldb, const float *SB, int64_t ldsb,
                                    float beta, int c_type, void *C, int64_t ldc, int64_t stride_c, void *workspace, size_t workspace_bytes,
                                    void *stream)
{
    if (!extent(rows) || !extent(m) || !extent(n) || !tiles_fit(m, n, 0)) return MG_ERR_DIM;
    const int64_t columns = groups_known(groups) ? mg_grouped_columns(rows, groups) : 0;
    if (!at_least(lda, columns)) return MG_ERR_LDA;
    if (!at_least(ldb, columns)) return MG_ERR_LDB;
    if (!at_least(ldc, n)) return MG_ERR_LDC;
    if (!stored(m, lda) || !stored(n, ldb) || !stored(m, ldc)) return MG_ERR_DIM;
    const bool empty = m == 0 || n == 0, reads = alpha != 0.f && rows > 0;
    if (!empty && (C == nullptr || offsets == nullptr || (reads && (A == nullptr || B == nullptr || SA == nullptr || SB == nullptr)))) return MG_ERR_NULL;
    if (stride_c < 0) return MG_ERR_STRIDE;
    if (!type_known(c_type)) return MG_ERR_TYPE;
    if (!scales_known(scales)) return MG_ERR_BLOCK;
    if (!groups_known(groups)) return MG_ERR_GROUPS;
    if (!at_least(ldsa, blocks(columns)) || !at_least(ldsb, blocks(columns))) return MG_ERR_SCALES;
    if (empty) return MG_OK;
    BlockProblem p{};
    p.mode = BLOCK_SUM;
    p.m = m; p.n = n; p.k = rows;
    p.alpha = alpha; p.beta = beta;
    p.pow2 = kind_of(scales) == MG_SCALES_POW2;
    p.fp32_sums = sums_fp32(scales, c_type);
    p.A = A; p.lda = lda; p.SA = SA; p.ldsa = ldsa;
    p.B = B; p.ldb = ldb; p.SB = SB; p.ldsb = ldsb;
    p.c_type = c_type; p.C = C; p.ldc = ldc; p.stride_c = stride_c;
    p.groups = Groups{offsets, groups, rows, nullptr, 1};
    p.workspace_bytes = usable(workspace, workspace_bytes);
    p.workspace = workspace;
    p.stream = static_cast<hipStream_t>(stream);
    return launched(launch_block_gemm(p));
}

size_t mg_block_gemm_grouped_sum_workspace_bytes(int groups, int64_t rows, int64_t m, int64_t n)
{
    if (!groups_known(groups) || !extent(rows) || !extent(m) || !extent(n) || m == 0 || n == 0) return 0;
    return block_gemm_workspace(BLOCK_SUM, groups, m, n, rows);
}

mg_status mg_expert_sort(int64_t tokens, int fan, int experts, const int32_t *ids, int32_t *offsets, int32_t *position, int32_t *source,
                         void *workspace, size_t workspace_bytes, void *stream)
{
    if (!extent(tokens) || __int128(tokens) * fan > (__int128(1) << 30)) return MG_ERR_DIM;
    if (offsets == nullptr || (tokens > 0 && (ids == nullptr || position == nullptr || source == nullptr))) return MG_ERR_NULL;
    if (fan_known(fan) && groups_known(experts) && usable(workspace, workspace_bytes) < expert_sort_workspace(tokens, fan, experts)) return MG_ERR_WORKSPACE;
    if (!fan_known(fan) || !groups_known(experts)) return MG_ERR_GROUPS;
    return launched(launch_expert_sort(tokens, fan, experts, ids, offsets, position, source, workspace, static_cast<hipStream_t>(stream)));
}

size_t mg_expert_sort_workspace_bytes(int64_t tokens, int fan, int experts)
{
    if (!extent(tokens) || !fan_known(fan) || !groups_known(experts) || tokens * fan > (int64_t(1) << 30)) return 0;
    return expert_sort_workspace(tokens, fan, experts);
}

// What the three routines on rows check alike.  A launch has a thread for each piece of 16 bytes of tokens x fan rows, whose number is rounded up in every
// row, to less than twice as many, or a work-group for each token.
static mg_status check_rows(int64_t tokens, int fan, int64_t cols)
{
    if (!extent(tokens) || !extent(cols) || __int128(tokens) * fan > (__int128(1) << 30)) return MG_ERR_DIM;
    if (fan > 0 && __int128(tokens) * fan * ceil_div(cols, 4) > MOST_PIECES * 128) return MG_ERR_DIM;
    if (tokens >= MOST_PIECES) return MG_ERR_DIM;
    return MG_OK;
}

mg_status mg_expert_gather(int dtype, int64_t tokens, int fan, int64_t cols, const void *X, int64_t ldx, const int32_t *source, const float *weights,
                           void *Y, int64_t ldy, void *stream)
{
    if (const mg_status st = check_rows(tokens, fan, cols)) return st;
    if (!at_least(ldx, cols)) return MG_ERR_LDA;
    if (!at_least(ldy, cols)) return MG_ERR_LDB;
    if (!stored(tokens, ldx) || !stored(tokens * (fan > 0 ? fan : 0), ldy)) return MG_ERR_DIM;
    const bool empty = tokens == 0 || cols == 0;
    if (!empty && (X == nullptr || source == nullptr || Y == nullptr)) return MG_ERR_NULL;
    if (!type_known(dtype)) return MG_ERR_TYPE;
    if (!fan_known(fan)) return MG_ERR_GROUPS;
    return empty ? MG_OK : launched(launch_expert_gather(dtype, tokens, fan, cols, X, ldx, source, weights, Y, ldy, static_cast<hipStream_t>(stream)));
}

mg_status mg_expert_combine(int dtype, int64_t tokens, int fan, int64_t cols, const void *Y, int64_t ldy, const int32_t *position,
                            const float *weights, void *O, int64_t ldo, void *stream)
{
    if (const mg_status st = check_rows(tokens, fan, cols)) return st;
    if (!at_least(ldy, cols)) return MG_ERR_LDA;
    if (!at_least(ldo, cols)) return MG_ERR_LDB;
    if (!stored(tokens, ldo) || !stored(tokens * (fan > 0 ? fan : 0), ldy)) return MG_ERR_DIM;
    const bool empty = tokens == 0 || cols == 0;
    if (!empty && (Y == nullptr || position == nullptr || O == nullptr)) return MG_ERR_NULL;
    if (!type_known(dtype)) return MG_ERR_TYPE;
    if (!fan_known(fan)) return MG_ERR_GROUPS;
    return empty ? MG_OK : launched(launch_expert_combine(dtype, tokens, fan, cols, Y, ldy, position, weights, O, ldo, static_cast<hipStream_t>(stream)));
}

mg_status mg_expert_combine_grad(int dtype, int64_t tokens, int fan, int64_t cols, const void *dO, int64_t lddo, const void *Y, int64_t ldy,
                                 const int32_t *position, const float *weights, void *dY, int64_t lddy, float *dweights, void *stream)
{
    if (const mg_status st = check_rows(tokens, fan, cols)) return st;
    const int64_t slots = tokens * (fan > 0 ? fan : 0);
    if (!at_least(lddo, cols)) return MG_ERR_LDA;
    if (dweights != nullptr && !at_least(ldy, cols)) return MG_ERR_LDB;
    if (dY != nullptr && !at_least(lddy, cols)) return MG_ERR_LDC;
    if (!stored(tokens, lddo) || (dweights != nullptr && !stored(slots, ldy)) || (dY != nullptr && !stored(slots, lddy))) return MG_ERR_DIM;
    const bool empty = tokens == 0;
    if (!empty && (dY != nullptr || dweights != nullptr) && ((cols > 0 && dO == nullptr) || position == nullptr || (cols > 0 && dweights != nullptr && Y == nullptr)))
        return MG_ERR_NULL;
    if (!type_known(dtype)) return MG_ERR_TYPE;
    if (!fan_known(fan)) return MG_ERR_GROUPS;
    if (empty || (dY == nullptr && dweights == nullptr) || (cols == 0 && dweights == nullptr)) return MG_OK;
    return launched(launch_expert_combine_grad(dtype, tokens, fan, cols, dO, lddo, Y, ldy, position, weights, dY, lddy, dweights,
                                               static_cast<hipStream_t>(stream)));
}

}  // extern "C"
