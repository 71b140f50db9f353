// The norm of all gradients and clipping by it.
//
// Tensors are cut into chunks of 16 KB; a work-group has a range of consecutive chunks, whatever tensors they are of, so that many small tensors cost what one
// large one does.  A launch takes a table of tensors among its arguments.  First pass: every work-group's sum of squares, in 64 bits (a square of a
// bfloat16 does not fit FP32, and sums of 10^9 squares lose nothing that way); second pass: every work-group adds all work-groups' sums in the same order,
// so that no launch stands between the passes, and scales.  Bound by memory: read once, read again and written.  The second pass goes from the last chunks to
// the first, which it finds in the last-level cache while they are, and large results pass that by: 800 MB of 300 tensors 633 -> 507 us (the first
// pass at 5.3 TB/s, the second at 4.7).
#include "layers.h"
#include "internal.h"

namespace mg {
namespace {

constexpr int TENSORS = 120;                 // of a launch: 3.4 KB of arguments
constexpr int MOST_GROUPS = 1280;            // work-groups of a launch: five for every compute unit (four 2.5 % slower, three and six 8)
constexpr int MOST_SUMS = 8192;              // of all launches, unless there are more launches than that
constexpr int CHUNK_BYTES = 16384;
constexpr int64_t PAST_CACHES = int64_t(128) << 20;      // results of so many bytes do not stay in the last-level cache (256 MB) for their reader

// 16 bytes at the alignment of an element of SIZE bytes
template <int SIZE> struct ClipPiece;
template <> struct ClipPiece<4> {
    typedef uint32_t type __attribute__((ext_vector_type(4), aligned(4)));
};
template <> struct ClipPiece<2> {
    typedef uint32_t type __attribute__((ext_vector_type(4), aligned(2)));
};

struct ClipTable {
    const void *source[TENSORS];
    void *result[TENSORS];
    int64_t size_type[TENSORS];              // 4 * elements + type
    uint32_t begin[TENSORS + 1];             // the tensor's first chunk
    int count;
    uint32_t per_group;                      // chunks
};

__host__ __device__ inline int64_t chunk_elements(int type) { return CHUNK_BYTES / (type == MG_F32 ? 4 : 2); }

// calls fn(tensor, first element, elements) for the work-group's chunks, BACK from the last one on
template <bool BACK, typename Fn> __device__ inline void for_chunks(const ClipTable &t, Fn &&fn)
{
    const uint32_t total = t.begin[t.count], start = blockIdx.x * t.per_group, end = start + t.per_group < total ? start + t.per_group : total;
    if (start >= end) return;
    uint32_t chunk = BACK ? end - 1 : start;
    int at = 0, high = t.count - 1;          // the tensor with begin <= chunk < the next one's
    while (at < high) {
        const int mid = (at + high + 1) / 2;
        if (t.begin[mid] <= chunk) at = mid;
        else high = mid - 1;
    }
    for (uint32_t n = end - start; n > 0; --n) {
        if (BACK) while (chunk < t.begin[at]) --at;
        else while (chunk >= t.begin[at + 1]) ++at;
        const int type = static_cast<int>(t.size_type[at] & 3);
        const int64_t size = t.size_type[at] >> 2, each = chunk_elements(type), first = (chunk - t.begin[at]) * each;
        fn(at, type, first, size - first < each ? static_cast<int>(size - first) : static_cast<int>(each));
        chunk += BACK ? -1 : 1;
    }
}

template <typename T> __device__ inline double squares(const T *at, int count)
{
    constexpr int PER = 16 / static_cast<int>(sizeof(T));
    float v[4][PER];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int e = (i * 256 + static_cast<int>(threadIdx.x)) * PER;
        load_piece<T, PER>(at + e, count - e > 0 ? count - e : 0, v[i]);
    }
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < PER; ++e) sum = fma(static_cast<double>(v[i][e]), static_cast<double>(v[i][e]), sum);
    return sum;
}

// the sum over 256 threads, in thread 0, in a fixed order
__device__ inline double group_sum(double v, double *parts)
{
    for (int d = 32; d > 0; d /= 2) v += __shfl_xor(v, d);
    if (threadIdx.x % 64 == 0) parts[threadIdx.x / 64] = v;
    __syncthreads();
    return (parts[0] + parts[1]) + (parts[2] + parts[3]);
}

__global__ __launch_bounds__(256) void squares_kernel(const ClipTable t, double *sums)
{
    __shared__ double parts[4];
    double sum = 0.0;
    for_chunks<false>(t, [&](int tensor, int type, int64_t first, int count) {
        if (type == MG_F32) sum += squares(static_cast<const float *>(t.source[tensor]) + first, count);
        else if (type == MG_F16) sum += squares(static_cast<const _Float16 *>(t.source[tensor]) + first, count);
        else sum += squares(static_cast<const bfloat *>(t.source[tensor]) + first, count);
    });
    sum = group_sum(sum, parts);
    if (threadIdx.x == 0) sums[blockIdx.x] = sum;
}

__device__ inline double norm_of(const double *sums, int count, double *parts)
{
    double sum = 0.0;
    for (int i = threadIdx.x; i < count; i += 256) sum += sums[i];
    return sqrt(group_sum(sum, parts));
}

__global__ __launch_bounds__(256) void norm_kernel(const double *sums, int count, float *norm)
{
    __shared__ double parts[4];
    const double n = norm_of(sums, count, parts);
    if (threadIdx.x == 0) norm[0] = static_cast<float>(n);
}

// PASS: the results pass the caches by
template <typename T, bool PASS> __device__ inline void scale_chunk(const T *from, T *to, int count, float factor)
{
    constexpr int PER = 16 / static_cast<int>(sizeof(T));
    float v[4][PER];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int e = (i * 256 + static_cast<int>(threadIdx.x)) * PER;
        load_piece<T, PER>(from + e, count - e > 0 ? count - e : 0, v[i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int e = (i * 256 + static_cast<int>(threadIdx.x)) * PER;
#pragma unroll
        for (int k = 0; k < PER; ++k) v[i][k] *= factor;
        if constexpr (PASS) {
            if (count - e >= PER) {
                Piece<T, PER> x;
#pragma unroll
                for (int k = 0; k < PER; ++k) x.v[k] = static_cast<T>(v[i][k]);
                __builtin_nontemporal_store(__builtin_bit_cast(typename ClipPiece<sizeof(T)>::type, x), reinterpret_cast<typename ClipPiece<sizeof(T)>::type *>(to + e));
                continue;
            }
        }
        store_piece<T, PER>(to + e, count - e > 0 ? count - e : 0, v[i]);
    }
}

// factor 1 does not touch what is scaled in place and copies what is not, infinities and NaN among it.  Whether the norm is finite goes by what the caller is told, in FP32.
template <bool PASS> __global__ __launch_bounds__(256) void clip_kernel(const ClipTable t, const double *sums, int count, double max_norm, float *norm)
{
    __shared__ double parts[4];
    const double n = norm_of(sums, count, parts);
    if (norm != nullptr && blockIdx.x == 0 && threadIdx.x == 0) norm[0] = static_cast<float>(n);
    const float factor = n > max_norm && static_cast<float>(n) < __builtin_inff() ? static_cast<float>(max_norm / n) : 1.f;
    for_chunks<true>(t, [&](int tensor, int type, int64_t first, int some) {
        if (factor == 1.f && t.source[tensor] == t.result[tensor]) return;
        if (type == MG_F32) scale_chunk<float, PASS>(static_cast<const float *>(t.source[tensor]) + first, static_cast<float *>(t.result[tensor]) + first, some, factor);
        else if (type == MG_F16) scale_chunk<_Float16, PASS>(static_cast<const _Float16 *>(t.source[tensor]) + first, static_cast<_Float16 *>(t.result[tensor]) + first, some, factor);
        else scale_chunk<bfloat, PASS>(static_cast<const bfloat *>(t.source[tensor]) + first, static_cast<bfloat *>(t.result[tensor]) + first, some, factor);
    });
}

int64_t launches(int64_t count) { return ceil_div(count, TENSORS); }
// work-groups of a launch, at most
int groups_of(int64_t count)
{
    const int64_t each = MOST_SUMS / (launches(count) > 0 ? launches(count) : 1);
    return static_cast<int>(each > MOST_GROUPS ? MOST_GROUPS : each < 16 ? 16 : each);
}

// tensors first .. of a table; its work-groups
uint32_t fill(ClipTable &t, const ClipProblem &p, int64_t first)
{
    t.count = 0;
    t.begin[0] = 0;
    for (int64_t i = first; i < p.count && i < first + TENSORS; ++i) {
        const int n = t.count++;
        t.source[n] = p.sources[i];
        t.result[n] = p.results == nullptr ? const_cast<void *>(p.sources[i]) : p.results[i];
        t.size_type[n] = p.sizes[i] * 4 + p.types[i];
        t.begin[n + 1] = t.begin[n] + static_cast<uint32_t>(ceil_div(p.sizes[i], chunk_elements(p.types[i])));
    }
    const uint32_t total = t.begin[t.count], most = static_cast<uint32_t>(groups_of(p.count));
    t.per_group = static_cast<uint32_t>(ceil_div(total > 0 ? total : 1, most));
    return static_cast<uint32_t>(ceil_div(total, t.per_group));
}

}  // namespace

size_t clip_workspace(int64_t count) { return static_cast<size_t>(launches(count)) * groups_of(count) * sizeof(double); }

hipError_t launch_clip(const ClipProblem &p)
{
    double *const sums = static_cast<double *>(p.workspace);
    int64_t bytes = 0;
    for (int64_t i = 0; i < p.count; ++i) bytes += p.sizes[i] * (p.types[i] == MG_F32 ? 4 : 2);
    const bool past = bytes >= PAST_CACHES;
    ClipTable t;
    int written = 0;
    for (int64_t first = 0; first < p.count; first += TENSORS) {
        const uint32_t groups = fill(t, p, first);
        if (groups == 0) continue;
        squares_kernel<<<groups, 256, 0, p.stream>>>(t, sums + written);
        written += static_cast<int>(groups);
        if (const hipError_t e = hipGetLastError()) return e;
    }
    bool told = false;
    if (p.scales)
        for (int64_t first = (p.count - 1) / TENSORS * TENSORS; first >= 0; first -= TENSORS) {
            const uint32_t groups = fill(t, p, first);
            if (groups == 0) continue;
            auto kernel = past ? clip_kernel<true> : clip_kernel<false>;
            kernel<<<groups, 256, 0, p.stream>>>(t, sums, written, static_cast<double>(p.max_norm), told ? nullptr : p.norm);
            told = true;
            if (const hipError_t e = hipGetLastError()) return e;
        }
    if (!told) norm_kernel<<<1, 256, 0, p.stream>>>(sums, written, p.norm);
    return hipGetLastError();
}

}  // namespace mg
