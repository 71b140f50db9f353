// Routing: slots sorted by expert, rows copied into that order and summed back with weights, and the gradient of that.
//
// Sorting is a stable counting sort, the same result whatever the timing: a wavefront walks its slots 64 at a time; which lanes before a lane
// have the same expert follows from a ballot for every bit of the expert's number, and only one wavefront counts in a row of the table.
// Everything else is bound by memory (rows) or by the launch (few tokens): 131072 slots of 64 experts sorted in 13 us, their rows of 2048 bfloat16 gathered in 150
// (604 MB, 4.0 TB/s), with weights in 170; 8192 tokens of four choices and 4096 columns combined in 73 (336 MB, 4.6 TB/s), the gradient 139 (604 MB, 4.3 TB/s); 16 tokens 3.
#include "internal.h"
#include "experts.h"

namespace mg {
namespace {

// ---- sort --------------------------------------------------------------------------------------------------------------
constexpr int SORT_KEYS = 4;                     // slots of a lane, 64 apart
constexpr int SORT_WAVES = 16;
constexpr int SORT_CHUNK = SORT_WAVES * 64 * SORT_KEYS;          // slots of a work-group
constexpr int SORT_ROW = MG_MOST_GROUPS + 1;     // experts and, behind them, the dropped slots
// Chunks up to which every one of them adds up what is in front of it by itself; with more a launch in between does.  64 experts, 64 chunks: 13.1 us alone, 15.5 with
// the launch; 128: 16.2 and 15.7; 2048 (8 M slots): 411 and 105; 1024 experts: 19.3 and 19.6, 25.2 and 21.1, 1477 and 155.
constexpr int SORT_UNSCANNED = 64;

// Lanes with the same key, as a mask (keys below 2^bits; all 64 lanes take part)
__device__ inline uint64_t same_key(int key, int bits)
{
    uint64_t same = ~uint64_t(0);
    for (int b = 0; b < bits; ++b) {
        const uint64_t one = __ballot((key >> b) & 1);
        same &= ((key >> b) & 1) ? one : ~one;
    }
    return same;
}

// Sum over a work-group's threads in front of this one; `total`: over all of them
__device__ inline int sum_before(int v, int *scratch, int *total)
{
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, waves = blockDim.x / 64;
    int sum = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(sum, d);
        if (lane >= d) sum += o;
    }
    if (lane == 63) scratch[wave] = sum;
    __syncthreads();
    int before = 0, all = 0;
    for (int w = 0; w < waves; ++w) {
        if (w < wave) before += scratch[w];
        all += scratch[w];
    }
    __syncthreads();
    *total = all;
    return before + sum - v;
}

// key of slot i of the call: its expert, or `experts` for a dropped one; behind the last slot a key that nobody counts
__device__ inline int slot_key(const int32_t *ids, int64_t i, int64_t end, int experts)
{
    if (i >= end) return experts + 1;
    const int e = ids[i];
    return e >= 0 && e < experts ? e : experts;
}

// counts[chunk][key] of a chunk of slots
__global__ __launch_bounds__(SORT_WAVES * 64) void sort_count_kernel(int64_t slots, int experts, const int32_t *ids, int32_t *counts)
{
    __shared__ int count[SORT_ROW + 1];
    const int64_t first = static_cast<int64_t>(blockIdx.x) * SORT_CHUNK + threadIdx.x;
    int key[SORT_KEYS];
#pragma unroll
    for (int q = 0; q < SORT_KEYS; ++q) key[q] = slot_key(ids, first + q * (SORT_WAVES * 64), slots, experts);
    for (int e = threadIdx.x; e <= experts; e += SORT_WAVES * 64) count[e] = 0;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < SORT_KEYS; ++q) atomicAdd(&count[key[q]], 1);               // (whole numbers: any order)
    __syncthreads();
    for (int e = threadIdx.x; e <= experts; e += SORT_WAVES * 64) counts[static_cast<int64_t>(blockIdx.x) * (experts + 1) + e] = count[e];
}

// counts[chunk][key] -> sums over the chunks in front of each, and over all of them in a row behind the last.  A lane has a key, a wavefront a
// run of chunks.
__global__ __launch_bounds__(SORT_WAVES * 64) void sort_scan_kernel(int keys, int chunks, int32_t *counts)
{
    __shared__ int sums[SORT_WAVES][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, key = blockIdx.x * 64 + lane;
    const int each = (chunks + SORT_WAVES - 1) / SORT_WAVES, first = wave * each < chunks ? wave * each : chunks;
    const int end = key < keys ? first + each < chunks ? first + each : chunks : first;
    int sum = 0;
#pragma unroll 8
    for (int c = first; c < end; ++c) sum += counts[static_cast<int64_t>(c) * keys + key];
    sums[wave][lane] = sum;
    __syncthreads();
    int before = 0;
    for (int w = 0; w < wave; ++w) before += sums[w][lane];
#pragma unroll 8
    for (int c = first; c < end; ++c) {
        int32_t *const at = counts + static_cast<int64_t>(c) * keys + key;
        const int v = *at;
        *at = before;
        before += v;
    }
    if (wave == SORT_WAVES - 1 && key < keys) counts[static_cast<int64_t>(chunks) * keys + key] = before;
}

// Rows of a chunk's slots; a wavefront has 64 SORT_KEYS of them in a row.  counts null: the call's only chunk, counted here.  scanned: counts as
// sort_scan_kernel leaves them.
__global__ __launch_bounds__(SORT_WAVES * 64) void sort_place_kernel(int64_t slots, int experts, const int32_t *ids, const int32_t *counts, int chunks, bool scanned,
                                                                     int32_t *offsets, int32_t *position, int32_t *source)
{
    extern __shared__ int next[];                 // [wave][key]: how many slots of that key the wavefront has, then the row of its first one
    __shared__ int scratch[SORT_WAVES];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, waves = blockDim.x / 64, keys = experts + 1;
    const int bits = 32 - __builtin_clz(experts + 1);
    const int64_t mine = static_cast<int64_t>(blockIdx.x) * SORT_CHUNK + wave * (64 * SORT_KEYS) + lane;
    const uint64_t below = (uint64_t(1) << lane) - 1;

    int key[SORT_KEYS], rank[SORT_KEYS];
#pragma unroll
    for (int q = 0; q < SORT_KEYS; ++q) key[q] = slot_key(ids, mine + 64 * q, slots, experts);
    for (int i = threadIdx.x; i < waves * keys; i += blockDim.x) next[i] = 0;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < SORT_KEYS; ++q) {
        const uint64_t same = same_key(key[q], bits);
        const int earlier = key[q] < keys ? next[wave * keys + key[q]] : 0;
        __builtin_amdgcn_wave_barrier();
        rank[q] = earlier + __popcll(same & below);
        if (key[q] < keys && (same & below) == 0) next[wave * keys + key[q]] = earlier + __popcll(same);       // (one lane for each key)
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    // thread e: rows in front of key e's, and of this chunk's share of them
    int carried = 0;
    for (int base = 0; base < keys; base += blockDim.x) {
        const int e = base + threadIdx.x;
        int all = 0, earlier = 0;
        if (e < keys) {
            if (scanned) {
                all = counts[static_cast<int64_t>(chunks) * keys + e];
                earlier = counts[static_cast<int64_t>(blockIdx.x) * keys + e];
            } else if (counts != nullptr) {
#pragma unroll 8
                for (int c = 0; c < chunks; ++c) {
                    const int v = counts[static_cast<int64_t>(c) * keys + e];
                    all += v;
                    earlier += c < static_cast<int>(blockIdx.x) ? v : 0;
                }
            } else {
                for (int w = 0; w < waves; ++w) all += next[w * keys + e];
            }
        }
        int total;
        const int before = carried + sum_before(all, scratch, &total);
        carried += total;
        if (e < keys) {
            int at = before + earlier;
            for (int w = 0; w < waves; ++w) {
                const int v = next[w * keys + e];
                next[w * keys + e] = at;
                at += v;
            }
            if (blockIdx.x == 0) offsets[e] = before;         // (the dropped slots' start is offsets[experts])
        }
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < SORT_KEYS; ++q) {
        if (key[q] >= keys) continue;
        const int row = next[wave * keys + key[q]] + rank[q];
        const bool kept = key[q] < experts;
        position[mine + 64 * q] = kept ? row : -1;
        source[row] = kept ? static_cast<int32_t>(mine + 64 * q) : -1;
    }
}

// ---- rows --------------------------------------------------------------------------------------------------------------
template <typename T> struct RowPiece { static constexpr int N = 16 / sizeof(T); };            // elements of 16 bytes

// Threads of a work-group on rows of `pieces` 16-byte pieces: 2^log of them beside each other on a row, the rest on the rows behind it, and as many
// work-groups beside each other as the row takes
struct RowShape {
    int log;
    uint32_t beside;
};
inline RowShape row_shape(int64_t pieces)
{
    int log = 0;
    while (log < 8 && (1 << log) < pieces) ++log;
    return {log, static_cast<uint32_t>(ceil_div(pieces, int64_t(1) << log))};
}

// 16 bytes past the caches.  What that does depends on the size and on who reads them next; rows of 2048 bfloat16, past the caches / as usual, alone and with a pass
// behind it that quantises them: 8192 rows 8.9 / 10.4 us and 21.8 / 20.3; 32768 rows 38 / 39 and 71 / 70; 131072 rows (more than the last-level cache holds) 151 / 150 and
// 290 / 318; 2048 rows and fewer the same.
template <typename T, int N> __device__ inline void store_streaming(T *p, const Piece<T, N> &x)
{
    typedef uint32_t words __attribute__((ext_vector_type(4), aligned(2)));
    words w;
    __builtin_memcpy(&w, &x, 16);
    __builtin_nontemporal_store(w, reinterpret_cast<words *>(p));
}

// GATHER_ROWS pieces a thread, so that as many loads are in flight; without weights the bytes are moved as they are
constexpr int GATHER_ROWS = 4;
template <typename T, bool WEIGHTED>
__global__ __launch_bounds__(256) void gather_kernel(int rows, int fan, int64_t cols, const T *X, int64_t ldx, const int32_t *source, const float *weights,
                                                     T *Y, int64_t ldy, int log, uint32_t beside)
{
    constexpr int N = RowPiece<T>::N, U = GATHER_ROWS;
    const int64_t col = (static_cast<int64_t>(blockIdx.x % beside << log) + (threadIdx.x & ((1 << log) - 1))) * N;
    if (col >= cols) return;
    const int valid = static_cast<int>(cols - col < N ? cols - col : N);
    const int per_pass = 256 >> log, first = static_cast<int>(blockIdx.x / beside) * per_pass * U + static_cast<int>(threadIdx.x >> log);
    int slot[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int row = first + u * per_pass;
        slot[u] = row < rows ? source[row] : -1;
        if (slot[u] >= rows) slot[u] = -1;
    }
    if (valid == N && !WEIGHTED) {
        Piece<T, N> x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            x[u] = Piece<T, N>{};
            if (slot[u] >= 0) x[u] = *reinterpret_cast<const Piece<T, N> *>(X + slot[u] / fan * ldx + col);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t row = first + u * per_pass;
            if (row < rows) store_streaming(Y + row * ldy + col, x[u]);
        }
        return;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t row = first + u * per_pass;
        if (row >= rows) continue;
        float v[N];
        load_piece<T, N>(X + (slot[u] >= 0 ? slot[u] / fan * ldx + col : 0), slot[u] >= 0 ? valid : 0, v);
        if (WEIGHTED && slot[u] >= 0) {
            const float w = weights[slot[u]];
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] *= w;
        }
        store_piece<T, N>(Y + row * ldy + col, valid, v);
    }
}

// One piece of a token's row a thread; the rows of COMBINE_SLOTS choices are on their way at a time
constexpr int COMBINE_SLOTS = 4;
template <typename T>
__global__ __launch_bounds__(256) void combine_kernel(int64_t tokens, int fan, int64_t cols, const T *Y, int64_t ldy, const int32_t *position,
                                                      const float *weights, T *O, int64_t ldo, int log, uint32_t beside)
{
    constexpr int N = RowPiece<T>::N, U = COMBINE_SLOTS;
    const int64_t col = (static_cast<int64_t>(blockIdx.x % beside << log) + (threadIdx.x & ((1 << log) - 1))) * N;
    const int64_t token = static_cast<int64_t>(blockIdx.x / beside) * (256 >> log) + (threadIdx.x >> log);
    if (col >= cols || token >= tokens) return;
    const int valid = static_cast<int>(cols - col < N ? cols - col : N);
    const int rows = static_cast<int>(tokens) * fan;
    const int32_t *at = position + token * fan;
    const float *of = weights == nullptr ? nullptr : weights + token * fan;
    float sum[N];
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] = 0.f;
    for (int j0 = 0; j0 < fan; j0 += U) {
        float v[U][N], w[U];
        int row[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            row[u] = j0 + u < fan ? at[j0 + u] : -1;
            if (row[u] >= rows) row[u] = -1;
            w[u] = j0 + u < fan && of != nullptr ? of[j0 + u] : 1.f;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) load_piece<T, N>(Y + (row[u] >= 0 ? row[u] * ldy + col : 0), row[u] >= 0 ? valid : 0, v[u]);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (row[u] >= 0) {
#pragma unroll
                for (int i = 0; i < N; ++i) sum[i] = __builtin_fmaf(w[u], v[u][i], sum[i]);
            }
    }
    store_piece<T, N>(O + token * ldo + col, valid, sum);
}

// WAVES wavefronts take a token (one for short rows, so that a work-group takes four) and U of its choices: they walk the row, with dO's piece read once for
// all of them, and add up the weights' gradients in registers.
template <typename T, int WAVES, int U>
__global__ __launch_bounds__(256) void combine_grad_kernel(int64_t tokens, int fan, int64_t cols, const T *dO, int64_t lddo, const T *Y, int64_t ldy,
                                                           const int32_t *position, const float *weights, T *dY, int64_t lddy, float *dweights)
{
    constexpr int N = RowPiece<T>::N, THREADS = WAVES * 64;
    __shared__ float part[4][U];
    const int wave = threadIdx.x / 64, me = threadIdx.x % THREADS;
    const int64_t token = static_cast<int64_t>(blockIdx.x) * (4 / WAVES) + wave / WAVES;
    if (WAVES == 1 && token >= tokens) return;
    const int rows = static_cast<int>(tokens) * fan;
    const int j0 = blockIdx.y * U;
    int row[U];
    float w[U], dot[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        row[u] = j0 + u < fan ? position[token * fan + j0 + u] : -1;
        if (row[u] >= rows) row[u] = -1;
        w[u] = j0 + u < fan && weights != nullptr ? weights[token * fan + j0 + u] : 1.f;
        dot[u] = 0.f;
    }
    for (int64_t col = me * N; col < cols; col += THREADS * N) {
        const int valid = static_cast<int>(cols - col < N ? cols - col : N);
        float g[N], y[U][N];
        load_piece<T, N>(dO + token * lddo + col, valid, g);
        if (dweights != nullptr) {
#pragma unroll
            for (int u = 0; u < U; ++u) load_piece<T, N>(Y + (row[u] >= 0 ? row[u] * ldy + col : 0), row[u] >= 0 ? valid : 0, y[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (row[u] < 0) continue;
            if (dweights != nullptr) {
#pragma unroll
                for (int i = 0; i < N; ++i) dot[u] = __builtin_fmaf(g[i], y[u][i], dot[u]);
            }
            if (dY != nullptr) {
                float d[N];
#pragma unroll
                for (int i = 0; i < N; ++i) d[i] = w[u] * g[i];
                store_piece<T, N>(dY + row[u] * lddy + col, valid, d);
            }
        }
    }
    if (dweights == nullptr) return;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) dot[u] += __shfl_xor(dot[u], d);
    if constexpr (WAVES > 1) {
        if (threadIdx.x % 64 == 0) {
#pragma unroll
            for (int u = 0; u < U; ++u) part[wave][u] = dot[u];
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < U; ++u) dot[u] = (part[0][u] + part[1][u]) + (part[2][u] + part[3][u]);
    }
    if (me == 0) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (j0 + u < fan) dweights[token * fan + j0 + u] = dot[u];
    }
}

// f(T{}) for the type that dtype names
template <typename F> hipError_t with_type(int dtype, F &&f)
{
    if (dtype == MG_F32) f(float{});
    else if (dtype == MG_F16) f(_Float16{});
    else f(bfloat{});
    return hipGetLastError();
}

template <typename T> int64_t row_pieces(int64_t cols) { return ceil_div(cols, RowPiece<T>::N); }

}  // namespace

size_t expert_sort_workspace(int64_t tokens, int fan, int experts)
{
    const int64_t chunks = ceil_div(tokens * fan, SORT_CHUNK);
    return chunks > 1 ? static_cast<size_t>(chunks + (chunks > SORT_UNSCANNED ? 1 : 0)) * (experts + 1) * sizeof(int32_t) : 0;
}

hipError_t launch_expert_sort(int64_t tokens, int fan, int experts, const int32_t *ids, int32_t *offsets, int32_t *position, int32_t *source,
                              void *workspace, hipStream_t stream)
{
    const int64_t slots = tokens * fan;
    const int chunks = static_cast<int>(ceil_div(slots, SORT_CHUNK));
    int32_t *counts = chunks > 1 ? static_cast<int32_t *>(workspace) : nullptr;
    if (counts != nullptr) {
        sort_count_kernel<<<chunks, SORT_WAVES * 64, 0, stream>>>(slots, experts, ids, counts);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const bool scanned = chunks > SORT_UNSCANNED;
    if (scanned) {
        sort_scan_kernel<<<static_cast<uint32_t>(ceil_div(experts + 1, 64)), SORT_WAVES * 64, 0, stream>>>(experts + 1, chunks, counts);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    // a short call in as few wavefronts as its slots and its experts keep busy
    const int64_t wanted = ceil_div(slots, 64 * SORT_KEYS) > ceil_div(experts + 1, 256) ? ceil_div(slots, 64 * SORT_KEYS) : ceil_div(experts + 1, 256);
    const int waves = static_cast<int>(wanted < SORT_WAVES ? wanted : SORT_WAVES);
    const size_t lds = static_cast<size_t>(waves) * (experts + 1) * sizeof(int);
    static bool raised = false;                   // raising the limit twice is harmless
    if (lds > 48 * 1024 && !raised) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(sort_place_kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                                                 SORT_WAVES * SORT_ROW * sizeof(int));
        if (e != hipSuccess) return e;
        raised = true;
    }
    sort_place_kernel<<<chunks > 0 ? chunks : 1, waves * 64, lds, stream>>>(slots, experts, ids, counts, chunks, scanned, offsets, position, source);
    return hipGetLastError();
}

hipError_t launch_expert_gather(int dtype, int64_t tokens, int fan, int64_t cols, const void *X, int64_t ldx, const int32_t *source,
                                const float *weights, void *Y, int64_t ldy, hipStream_t stream)
{
    return with_type(dtype, [&](auto zero) {
        using T = decltype(zero);
        const RowShape s = row_shape(row_pieces<T>(cols));
        const int rows = static_cast<int>(tokens * fan);
        const uint32_t grid = static_cast<uint32_t>(ceil_div(rows, (256 >> s.log) * GATHER_ROWS)) * s.beside;
        if (weights != nullptr)
            gather_kernel<T, true><<<grid, 256, 0, stream>>>(rows, fan, cols, static_cast<const T *>(X), ldx, source, weights, static_cast<T *>(Y), ldy, s.log, s.beside);
        else
            gather_kernel<T, false><<<grid, 256, 0, stream>>>(rows, fan, cols, static_cast<const T *>(X), ldx, source, weights, static_cast<T *>(Y), ldy, s.log, s.beside);
    });
}

hipError_t launch_expert_combine(int dtype, int64_t tokens, int fan, int64_t cols, const void *Y, int64_t ldy, const int32_t *position,
                                 const float *weights, void *O, int64_t ldo, hipStream_t stream)
{
    return with_type(dtype, [&](auto zero) {
        using T = decltype(zero);
        const RowShape s = row_shape(row_pieces<T>(cols));
        combine_kernel<T><<<static_cast<uint32_t>(ceil_div(tokens, 256 >> s.log)) * s.beside, 256, 0, stream>>>(tokens, fan, cols, static_cast<const T *>(Y), ldy, position, weights,
                                                                                                              static_cast<T *>(O), ldo, s.log, s.beside);
    });
}

hipError_t launch_expert_combine_grad(int dtype, int64_t tokens, int fan, int64_t cols, const void *dO, int64_t lddo, const void *Y, int64_t ldy,
                                      const int32_t *position, const float *weights, void *dY, int64_t lddy, float *dweights, hipStream_t stream)
{
    return with_type(dtype, [&](auto zero) {
        using T = decltype(zero);
        auto launch = [&](auto waves, auto choices) {
            constexpr int W = decltype(waves)::value, U = decltype(choices)::value;
            combine_grad_kernel<T, W, U><<<dim3(static_cast<uint32_t>(ceil_div(tokens, 4 / W)), static_cast<uint32_t>(ceil_div(fan, U))), 256, 0, stream>>>(
                tokens, fan, cols, static_cast<const T *>(dO), lddo, static_cast<const T *>(Y), ldy, position, weights, static_cast<T *>(dY), lddy, dweights);
        };
        // One wavefront for a token where it holds the row in two pieces a lane.  Few tokens: a work-group for every choice (1 token, 6 choices, 4873 columns:
        // 14 -> 4.6 us); many: four choices share their token's row of dO.
        using One = std::integral_constant<int, 1>;
        using Four = std::integral_constant<int, 4>;
        const bool narrow = row_pieces<T>(cols) <= 128, few = tokens * ceil_div(fan, 4) < 512;
        if (narrow && few) launch(One{}, One{});
        else if (narrow) launch(One{}, Four{});
        else if (few) launch(Four{}, One{});
        else launch(Four{}, Four{});
    });
}

}  // namespace mg
