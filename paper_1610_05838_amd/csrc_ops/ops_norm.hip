// ops_norm.hip -- the global norm of many gradients, and what is done with it:
//   norm = sqrt(sum over all tensors of g^2),
//   c    = norm <= max_norm or max_norm infinite ? 1 : max_norm / norm,
//   clip g <- c g,  or  step p <- p - lr (c g + lambda p).
//
// Bound by memory: a norm reads g once; clipping reads it again and writes it; a
// step reads g again and p and writes p.  ONCE: gradients that are together
// larger than the Infinity Cache are loaded past the caches, which have lost
// their beginning by the time it is read again (276 MB binary32: norm 45.7 us,
// 6.0 TB/s, against 50.1; 1.6 GB: 230 against 258; 64 MB, which stay in the
// caches: 15.2 against 14.5).  A step's update of 69 M binary32 parameters, 828 MB:
// 128 us, 6.5 TB/s.
//
// Squares are summed in binary64 from the first: the square of a binary32 or
// bfloat16 value leaves binary32's range at either end, a binary64 sum of such
// squares never does.  A workgroup adds a fixed set of chunks, the sums of all
// workgroups are added in one fixed order, so the norm is the same bits every
// time.
//
// The tensors' addresses travel in the kernel's arguments, kGroup of them a
// launch: nothing is copied to the device, kept there or waited for.
#include <algorithm>

#include "ops_common.hpp"

namespace mfsgd {
namespace ops {

namespace {

constexpr int kThreads = 256;
constexpr int kGroup = 112;     // tensors of one launch: 4 KB of arguments
constexpr int kChunk = 8192;    // elements a workgroup takes at a time
constexpr int kMostWgs = 2048;  // 8 workgroups on each of 256 CUs
constexpr int kFold = 2048;     // up to so many sums every workgroup of the update adds up by itself

struct Group {
    const void* g[kGroup];
    void* p[kGroup];
    int64_t n[kGroup];
    uint32_t first[kGroup + 1]; // first chunk of every tensor, then the chunks in all
    uint8_t dtype[kGroup];
    int count;
};
static_assert(sizeof(Group) <= 3500, "the arguments of a launch");

// Workgroup b's tensor of chunk `chunk`, from the last one on (chunks ascend).
__device__ __forceinline__ int tensor_of(const Group& a, uint32_t chunk, int from)
{
    int lo = from, hi = a.count; // a.first[lo] <= chunk < a.first[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.first[mid] <= chunk)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

__device__ __forceinline__ double block_sum(double x, double* sums)
{
    x = lanes_sum(x);
    if ((threadIdx.x & 63) == 0)
        sums[threadIdx.x >> 6] = x;
    __syncthreads();
    x = (sums[0] + sums[1]) + (sums[2] + sums[3]);
    __syncthreads();
    return x;
}

template <typename T, int V, bool ONCE>
__device__ __forceinline__ Vec<T, V> load_some(const T* p)
{
    return ONCE ? load_once<T, V>(p) : load_vec<T, V>(p);
}

template <typename T, bool ONCE>
__device__ __forceinline__ double squares(const T* __restrict__ g, int n, double sum)
{
    constexpr int V = 16 / (int)sizeof(T), ahead = 4;
    const int whole = n / V;
    double part[V];
#pragma unroll
    for (int e = 0; e < V; ++e)
        part[e] = 0.0;
    for (int i0 = threadIdx.x; i0 < whole; i0 += kThreads * ahead) {
        Vec<T, V> x[ahead];
#pragma unroll
        for (int u = 0; u < ahead; ++u)
            x[u] = load_some<T, V, ONCE>(g + (int64_t)(i0 + u * kThreads < whole ? i0 + u * kThreads : i0) * V);
#pragma unroll
        for (int u = 0; u < ahead; ++u)
            if (i0 + u * kThreads < whole) {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const double d = (double)(float)x[u].v[e];
                    part[e] += d * d;
                }
            }
    }
    const int rest = whole * V + (int)threadIdx.x;
    if (rest < n) {
        const double d = (double)(float)g[rest];
        sum += d * d;
    }
#pragma unroll
    for (int e = 0; e < V; ++e)
        sum += part[e];
    return sum;
}

template <bool ONCE>
__global__ __launch_bounds__(kThreads) void k_norm_part(Group a, double* __restrict__ part)
{
    __shared__ double sums[4];
    double sum = 0.0;
    int t = 0;
    for (uint32_t chunk = blockIdx.x; chunk < a.first[a.count]; chunk += gridDim.x) {
        t = tensor_of(a, chunk, t);
        const int64_t at = (int64_t)(chunk - a.first[t]) * kChunk;
        const int n = (int)(a.n[t] - at < kChunk ? a.n[t] - at : kChunk);
        if (a.dtype[t] == kF32)
            sum = squares<float, ONCE>((const float*)a.g[t] + at, n, sum);
        else if (a.dtype[t] == kF16)
            sum = squares<_Float16, ONCE>((const _Float16*)a.g[t] + at, n, sum);
        else
            sum = squares<__bf16, ONCE>((const __bf16*)a.g[t] + at, n, sum);
    }
    sum = block_sum(sum, sums);
    if (threadIdx.x == 0)
        part[blockIdx.x] = sum;
}

// The sum of `parts` partial sums, by every thread of a workgroup.
__device__ __forceinline__ double fold(const double* __restrict__ part, int64_t parts, double* sums)
{
    double x = 0.0;
    for (int64_t i0 = threadIdx.x; i0 < parts; i0 += kThreads * 8) {
        double y[8];
#pragma unroll
        for (int u = 0; u < 8; ++u)
            y[u] = i0 + u * kThreads < parts ? part[i0 + u * kThreads] : 0.0;
#pragma unroll
        for (int u = 0; u < 8; ++u)
            x += y[u];
    }
    return block_sum(x, sums);
}

// The norm alone, or (total) the sum of squares for many partial sums.
__global__ __launch_bounds__(kThreads) void k_norm_fold(const double* __restrict__ part, int64_t parts,
                                                        double* __restrict__ norm, double* __restrict__ total)
{
    __shared__ double sums[4];
    const double x = fold(part, parts, sums);
    if (threadIdx.x == 0) {
        *norm = sqrt(x);
        if (total)
            *total = x;
    }
}

template <typename T, bool STEP, bool ONCE>
__device__ __forceinline__ void apply_to(T* p, const T* g, int n, float c, float lr, float lam)
{ // clipping: p is g
    constexpr int V = 16 / (int)sizeof(T), ahead = 4;
    const int whole = n / V;
    for (int i0 = threadIdx.x; i0 < whole; i0 += kThreads * ahead) {
        Vec<T, V> x[ahead], y[ahead];
#pragma unroll
        for (int u = 0; u < ahead; ++u) {
            const int i = i0 + u * kThreads < whole ? i0 + u * kThreads : i0;
            x[u] = load_some<T, V, ONCE>(g + (int64_t)i * V);
            if (STEP)
                y[u] = load_some<T, V, ONCE>(p + (int64_t)i * V);
        }
#pragma unroll
        for (int u = 0; u < ahead; ++u) {
            const int i = i0 + u * kThreads;
            if (i < whole) {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float d = c * (float)x[u].v[e];
                    x[u].v[e] = STEP ? T((float)y[u].v[e] - lr * (d + lam * (float)y[u].v[e])) : T(d);
                }
                store_vec<T, V>(p + (int64_t)i * V, x[u]);
            }
        }
    }
    const int i = whole * V + (int)threadIdx.x;
    if (i < n) {
        const float d = c * (float)g[i];
        p[i] = STEP ? T((float)p[i] - lr * (d + lam * (float)p[i])) : T(d);
    }
}

// The clipping factor is rounded once, from binary64 to the binary32 that the
// elements are computed in.
template <bool STEP, bool ONCE>
__global__ __launch_bounds__(kThreads) void k_norm_apply(Group a, const double* __restrict__ part, int64_t parts,
                                                         double max_norm, float lr, float lam,
                                                         double* __restrict__ norm_out)
{
    __shared__ double sums[4];
    const double norm = sqrt(fold(part, parts, sums));
    if (norm_out && blockIdx.x == 0 && threadIdx.x == 0)
        *norm_out = norm;
    const bool within = norm <= max_norm || isinf(max_norm); // a NaN is within no finite bound
    const float c = within ? 1.0f : (float)(max_norm / norm);
    if (!STEP && within)
        return; // c g = g
    int t = 0;
    for (uint32_t chunk = blockIdx.x; chunk < a.first[a.count]; chunk += gridDim.x) {
        t = tensor_of(a, chunk, t);
        const int64_t at = (int64_t)(chunk - a.first[t]) * kChunk;
        const int n = (int)(a.n[t] - at < kChunk ? a.n[t] - at : kChunk);
        if (a.dtype[t] == kF32)
            apply_to<float, STEP, ONCE>((float*)a.p[t] + at, (const float*)a.g[t] + at, n, c, lr, lam);
        else if (a.dtype[t] == kF16)
            apply_to<_Float16, STEP, ONCE>((_Float16*)a.p[t] + at, (const _Float16*)a.g[t] + at, n, c, lr, lam);
        else
            apply_to<__bf16, STEP, ONCE>((__bf16*)a.p[t] + at, (const __bf16*)a.g[t] + at, n, c, lr, lam);
    }
}

int64_t chunks_of(int64_t n) { return (n + kChunk - 1) / kChunk; }

// The next launch's tensors from list[i] on, empty ones left out; returns where
// the one after it begins.  (The caller has checked that all chunks together
// are below 2^31.)
int64_t next_group(const NormTensor* list, int64_t count, int64_t i, Group& a)
{
    int64_t chunks = 0;
    a.count = 0;
    for (; i < count && a.count < kGroup; ++i) {
        const NormTensor& t = list[i];
        if (t.n == 0)
            continue;
        a.g[a.count] = t.g;
        a.p[a.count] = t.p;
        a.n[a.count] = t.n;
        a.dtype[a.count] = (uint8_t)t.dtype;
        a.first[a.count] = (uint32_t)chunks;
        chunks += chunks_of(t.n);
        ++a.count;
    }
    a.first[a.count] = (uint32_t)chunks;
    return i;
}

} // namespace

// A partial sum for every workgroup of every launch, and the sum of all.
size_t norm_bytes(int64_t count)
{
    const int64_t launches = (count + kGroup - 1) / kGroup + 1;
    return round256(sizeof(double) * (size_t)(launches * kMostWgs + 1));
}

hipError_t norm_apply(const NormTensor* list, int64_t count, int apply, double max_norm, float lr, float lam,
                      double* norm_out, void* work, hipStream_t st)
{
    double* part = (double*)work + 1;
    double* total = (double*)work;
    Group a;
    int64_t bytes = 0;
    for (int64_t i = 0; i < count; ++i)
        bytes += list[i].n * (list[i].dtype == kF32 ? 4 : 2);
    const bool once = bytes > kInfinityCache;
    int64_t parts = 0;
    for (int64_t i = 0; i < count;) {
        i = next_group(list, count, i, a);
        if (!a.count)
            break;
        const int64_t wgs = std::min<int64_t>(a.first[a.count], kMostWgs);
        hipLaunchKernelGGL((once ? k_norm_part<true> : k_norm_part<false>), dim3((unsigned)wgs), dim3(kThreads), 0, st,
                           a, part + parts);
        parts += wgs;
    }
    const bool folded = !apply || parts > kFold || parts == 0;
    if (folded)
        hipLaunchKernelGGL(k_norm_fold, dim3(1), dim3(kThreads), 0, st, part, parts, norm_out,
                           apply ? total : nullptr);
    if (!apply || parts == 0)
        return hipGetLastError();
    if (parts > kFold) {
        part = total;
        parts = 1;
    }
    double* norm = folded ? nullptr : norm_out;
    for (int64_t i = 0; i < count;) {
        i = next_group(list, count, i, a);
        if (!a.count)
            break;
        const int64_t wgs = std::min<int64_t>(a.first[a.count], kMostWgs);
        if (apply == 2)
            hipLaunchKernelGGL((once ? k_norm_apply<true, true> : k_norm_apply<true, false>), dim3((unsigned)wgs),
                               dim3(kThreads), 0, st, a, part, parts, max_norm, lr, lam, norm);
        else
            hipLaunchKernelGGL((once ? k_norm_apply<false, true> : k_norm_apply<false, false>), dim3((unsigned)wgs),
                               dim3(kThreads), 0, st, a, part, parts, max_norm, lr, lam, norm);
        norm = nullptr; // written by the first
    }
    return hipGetLastError();
}

} // namespace ops
} // namespace mfsgd
