// Routing: slots sorted by expert, rows copied into that order and summed back with weights, and the gradient of that.
//
// Sorting is a stable counting sort, the same result whatever the timing: a wavefront walks its slots 64 at a time; which lanes before a lane
// have the same expert follows from a ballot for every bit of the expert's number, and only one wavefront counts in a row of the table.
// Everything else is bound by memory (rows) or by the launch (few tokens).
#include "internal.h"
#include "experts.h"

namespace mg {
namespace {

// ---- sort --------------------------------------------------------------------------------------------------------------
constexpr int SORT_THREADS = 1024, SORT_WAVES = 16;
constexpr int SORT_CHUNK = 8192;                 // slots of a work-group: 512 for each wavefront
constexpr int SORT_ROW = MG_MOST_GROUPS + 1;     // experts and, behind them, the dropped slots

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
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    int sum = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(sum, d);
        if (lane >= d) sum += o;
    }
    if (lane == 63) scratch[wave] = sum;
    __syncthreads();
    int before = 0, all = 0;
    for (int w = 0; w < SORT_WAVES; ++w) {
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
__global__ __launch_bounds__(SORT_THREADS) void sort_count_kernel(int64_t slots, int experts, const int32_t *ids, int32_t *counts)
{
    __shared__ int count[SORT_ROW];
    for (int e = threadIdx.x; e <= experts; e += SORT_THREADS) count[e] = 0;
    __syncthreads();
    const int64_t first = static_cast<int64_t>(blockIdx.x) * SORT_CHUNK, end = first + SORT_CHUNK < slots ? first + SORT_CHUNK : slots;
    for (int64_t i = first + threadIdx.x; i < end; i += SORT_THREADS) atomicAdd(&count[slot_key(ids, i, end, experts)], 1);     // (whole numbers: any order)
    __syncthreads();
    for (int e = threadIdx.x; e <= experts; e += SORT_THREADS) counts[static_cast<int64_t>(blockIdx.x) * (experts + 1) + e] = count[e];
}

// Rows of a chunk's slots.  counts null: the call's only chunk, counted here.
__global__ __launch_bounds__(SORT_THREADS) void sort_place_kernel(int64_t slots, int experts, const int32_t *ids, const int32_t *counts, int chunks,
                                                                  int32_t *offsets, int32_t *position, int32_t *source)
{
    extern __shared__ int next[];                 // [wave][key]: the row of the wavefront's next slot of that key
    __shared__ int scratch[SORT_WAVES];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, keys = experts + 1;
    const int bits = 32 - __builtin_clz(experts + 1);
    const int64_t first = static_cast<int64_t>(blockIdx.x) * SORT_CHUNK;
    const int64_t end = first + SORT_CHUNK < slots ? first + SORT_CHUNK : slots;
    const int64_t each = ((end - first + SORT_WAVES - 1) / SORT_WAVES + 63) / 64 * 64;
    const int64_t mine = first + wave * each, mine_end = mine + each < end ? mine + each : end;
    const uint64_t below = (uint64_t(1) << lane) - 1;

    for (int i = threadIdx.x; i < SORT_WAVES * keys; i += SORT_THREADS) next[i] = 0;
    __syncthreads();
    for (int64_t i = mine; i < mine_end; i += 64) {
        const int key = slot_key(ids, i + lane, mine_end, experts);
        const uint64_t same = same_key(key, bits);
        if (key < keys && (same & below) == 0) next[wave * keys + key] += __popcll(same);        // (one lane for each key)
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    // thread e: rows in front of key e's, and of this chunk's share of them; MG_MOST_GROUPS + 1 keys take two rounds
    int carried = 0;
    for (int base = 0; base < keys; base += SORT_THREADS) {
        const int e = base + threadIdx.x;
        int all = 0, earlier = 0;
        if (e < keys) {
            if (counts != nullptr) {
                for (int c = 0; c < chunks; ++c) {
                    const int v = counts[static_cast<int64_t>(c) * keys + e];
                    all += v;
                    if (c < static_cast<int>(blockIdx.x)) earlier += v;
                }
            } else {
                for (int w = 0; w < SORT_WAVES; ++w) all += next[w * keys + e];
            }
        }
        int total;
        const int before = carried + sum_before(all, scratch, &total);
        carried += total;
        if (e < keys) {
            int at = before + earlier;
            for (int w = 0; w < SORT_WAVES; ++w) {
                const int v = next[w * keys + e];
                next[w * keys + e] = at;
                at += v;
            }
            if (blockIdx.x == 0) offsets[e] = before;         // (the dropped slots' start is offsets[experts])
        }
    }
    __syncthreads();
    for (int64_t i = mine; i < mine_end; i += 64) {
        const int key = slot_key(ids, i + lane, mine_end, experts);
        const uint64_t same = same_key(key, bits);
        const int row = key < keys ? next[wave * keys + key] + __popcll(same & below) : 0;
        __builtin_amdgcn_wave_barrier();
        if (key < keys && (same & below) == 0) next[wave * keys + key] = row + __popcll(same);
        __builtin_amdgcn_wave_barrier();
        if (key < keys) {
            position[i + lane] = key < experts ? row : -1;
            source[row] = key < experts ? static_cast<int32_t>(i + lane) : -1;
        }
    }
}

// ---- rows --------------------------------------------------------------------------------------------------------------
template <typename T> struct RowPiece { static constexpr int N = 16 / sizeof(T); };            // elements of 16 bytes

// one thread for 16 bytes of a row
template <typename T>
__global__ __launch_bounds__(256) void gather_kernel(int64_t rows, int fan, int64_t cols, const T *X, int64_t ldx, const int32_t *source,
                                                     const float *weights, T *Y, int64_t ldy, uint32_t pieces)
{
    constexpr int N = RowPiece<T>::N;
    const int64_t id = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const int64_t row = id / pieces, col = id % pieces * N;
    if (row >= rows) return;
    const int valid = static_cast<int>(cols - col < N ? cols - col : N);
    const int slot = source[row];
    float v[N];
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = 0.f;
    if (slot >= 0 && slot < rows) {
        load_piece<T, N>(X + slot / fan * ldx + col, valid, v);
        if (weights != nullptr) {
            const float w = weights[slot];
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] *= w;
        }
    }
    store_piece<T, N>(Y + row * ldy + col, valid, v);
}

template <typename T>
__global__ __launch_bounds__(256) void combine_kernel(int64_t tokens, int fan, int64_t cols, const T *Y, int64_t ldy, const int32_t *position,
                                                      const float *weights, T *O, int64_t ldo, uint32_t pieces)
{
    constexpr int N = RowPiece<T>::N;
    const int64_t id = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const int64_t token = id / pieces, col = id % pieces * N;
    if (token >= tokens) return;
    const int valid = static_cast<int>(cols - col < N ? cols - col : N);
    float sum[N];
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] = 0.f;
    for (int j = 0; j < fan; ++j) {
        const int64_t slot = token * fan + j;
        const int row = position[slot];
        if (row < 0 || row >= tokens * fan) continue;
        const float w = weights != nullptr ? weights[slot] : 1.f;
        float v[N];
        load_piece<T, N>(Y + row * ldy + col, valid, v);
#pragma unroll
        for (int i = 0; i < N; ++i) sum[i] = __builtin_fmaf(w, v[i], sum[i]);
    }
    store_piece<T, N>(O + token * ldo + col, valid, sum);
}

// A work-group takes a token: its row of dO is read once for all of its slots.
template <typename T>
__global__ __launch_bounds__(256) void combine_grad_kernel(int64_t tokens, int fan, int64_t cols, const T *dO, int64_t lddo, const T *Y, int64_t ldy,
                                                           const int32_t *position, const float *weights, T *dY, int64_t lddy, float *dweights)
{
    constexpr int N = RowPiece<T>::N;
    __shared__ float part[4];
    const int64_t token = blockIdx.x;
    for (int j = 0; j < fan; ++j) {
        const int64_t slot = token * fan + j;
        const int row = position[slot];
        const bool kept = row >= 0 && row < tokens * fan;                 // (the same in all threads)
        float dot = 0.f;
        if (kept) {
            const float w = weights != nullptr ? weights[slot] : 1.f;
            for (int64_t col = threadIdx.x * N; col < cols; col += 256 * N) {
                const int valid = static_cast<int>(cols - col < N ? cols - col : N);
                float g[N], y[N];
                load_piece<T, N>(dO + token * lddo + col, valid, g);
                if (dweights != nullptr) {
                    load_piece<T, N>(Y + row * ldy + col, valid, y);
#pragma unroll
                    for (int i = 0; i < N; ++i) dot = __builtin_fmaf(g[i], y[i], dot);
                }
                if (dY != nullptr) {
#pragma unroll
                    for (int i = 0; i < N; ++i) g[i] *= w;
                    store_piece<T, N>(dY + row * lddy + col, valid, g);
                }
            }
        }
        if (dweights == nullptr) continue;
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) dot += __shfl_xor(dot, d);
        if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = dot;
        __syncthreads();
        if (threadIdx.x == 0) dweights[slot] = (part[0] + part[1]) + (part[2] + part[3]);
        __syncthreads();
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

template <typename T> uint32_t row_pieces(int64_t cols) { return static_cast<uint32_t>(ceil_div(cols, RowPiece<T>::N)); }
uint32_t groups_of_256(int64_t threads) { return static_cast<uint32_t>(ceil_div(threads, 256)); }

}  // namespace

size_t expert_sort_workspace(int64_t tokens, int fan, int experts)
{
    const int64_t chunks = ceil_div(tokens * fan, SORT_CHUNK);
    return chunks > 1 ? static_cast<size_t>(chunks) * (experts + 1) * sizeof(int32_t) : 0;
}

hipError_t launch_expert_sort(int64_t tokens, int fan, int experts, const int32_t *ids, int32_t *offsets, int32_t *position, int32_t *source,
                              void *workspace, hipStream_t stream)
{
    const int64_t slots = tokens * fan;
    const int chunks = static_cast<int>(ceil_div(slots, SORT_CHUNK));
    int32_t *counts = chunks > 1 ? static_cast<int32_t *>(workspace) : nullptr;
    if (counts != nullptr) {
        sort_count_kernel<<<chunks, SORT_THREADS, 0, stream>>>(slots, experts, ids, counts);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const size_t lds = static_cast<size_t>(SORT_WAVES) * (experts + 1) * sizeof(int);
    static bool raised = false;                   // raising the limit twice is harmless
    if (lds > 48 * 1024 && !raised) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(sort_place_kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                                                 SORT_WAVES * SORT_ROW * sizeof(int));
        if (e != hipSuccess) return e;
        raised = true;
    }
    sort_place_kernel<<<chunks > 0 ? chunks : 1, SORT_THREADS, lds, stream>>>(slots, experts, ids, counts, chunks, offsets, position, source);
    return hipGetLastError();
}

hipError_t launch_expert_gather(int dtype, int64_t tokens, int fan, int64_t cols, const void *X, int64_t ldx, const int32_t *source,
                                const float *weights, void *Y, int64_t ldy, hipStream_t stream)
{
    return with_type(dtype, [&](auto zero) {
        using T = decltype(zero);
        const uint32_t pieces = row_pieces<T>(cols);
        gather_kernel<T><<<groups_of_256(tokens * fan * pieces), 256, 0, stream>>>(tokens * fan, fan, cols, static_cast<const T *>(X), ldx, source, weights,
                                                                                   static_cast<T *>(Y), ldy, pieces);
    });
}

hipError_t launch_expert_combine(int dtype, int64_t tokens, int fan, int64_t cols, const void *Y, int64_t ldy, const int32_t *position,
                                 const float *weights, void *O, int64_t ldo, hipStream_t stream)
{
    return with_type(dtype, [&](auto zero) {
        using T = decltype(zero);
        const uint32_t pieces = row_pieces<T>(cols);
        combine_kernel<T><<<groups_of_256(tokens * pieces), 256, 0, stream>>>(tokens, fan, cols, static_cast<const T *>(Y), ldy, position, weights,
                                                                              static_cast<T *>(O), ldo, pieces);
    });
}

hipError_t launch_expert_combine_grad(int dtype, int64_t tokens, int fan, int64_t cols, const void *dO, int64_t lddo, const void *Y, int64_t ldy,
                                      const int32_t *position, const float *weights, void *dY, int64_t lddy, float *dweights, hipStream_t stream)
{
    return with_type(dtype, [&](auto zero) {
        using T = decltype(zero);
        combine_grad_kernel<T><<<static_cast<uint32_t>(tokens), 256, 0, stream>>>(tokens, fan, cols, static_cast<const T *>(dO), lddo,
                                                                                  static_cast<const T *>(Y), ldy, position, weights, static_cast<T *>(dY),
                                                                                  lddy, dweights);
    });
}

}  // namespace mg
