// ops_common.hpp -- element types and vector accesses shared by the operator
// kernels (row lookups, products, gradient norms).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ops_launch.hpp"

namespace mfsgd {
namespace ops {

// Vectors of E elements at any element alignment: global accesses of 4 to 16
// bytes need not be aligned on this target, so a row of odd width or pitch is
// read and written in the same wide accesses as an aligned one.
template <typename T, int E>
struct Vec {
    T v[E];
};

template <int BYTES>
struct Raw;
template <>
struct Raw<2> {
    typedef uint16_t type;
};
template <>
struct Raw<4> {
    typedef uint32_t type;
};
template <>
struct Raw<8> {
    typedef uint32_t type __attribute__((ext_vector_type(2)));
};
template <>
struct Raw<16> {
    typedef uint32_t type __attribute__((ext_vector_type(4)));
};

template <typename T, int E>
__device__ __forceinline__ Vec<T, E> load_vec(const T* p)
{
    Vec<T, E> x;
    __builtin_memcpy(&x, p, sizeof(x));
    return x;
}

template <typename T, int E>
__device__ __forceinline__ void store_vec(T* p, const Vec<T, E>& x)
{
    __builtin_memcpy(p, &x, sizeof(x));
}

constexpr int64_t kInfinityCache = 256 << 20; // bytes

// Streams that are read or written once and are larger than the caches.
template <typename T, int E>
__device__ __forceinline__ Vec<T, E> load_once(const T* p)
{
    typedef typename Raw<int(sizeof(T)) * E>::type R;
    typedef R U __attribute__((aligned(sizeof(T))));
    U r = __builtin_nontemporal_load(reinterpret_cast<const U*>(p));
    Vec<T, E> x;
    __builtin_memcpy(&x, &r, sizeof(x));
    return x;
}

template <typename T, int E>
__device__ __forceinline__ void store_once(T* p, const Vec<T, E>& x)
{
    typedef typename Raw<int(sizeof(T)) * E>::type R;
    typedef R U __attribute__((aligned(sizeof(T))));
    U r;
    __builtin_memcpy(&r, &x, sizeof(x));
    __builtin_nontemporal_store(r, reinterpret_cast<U*>(p));
}

// Sum over the 64 lanes (a fixed tree), the same in every lane.
template <typename A>
__device__ __forceinline__ A lanes_sum(A x)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1)
        x += __shfl_xor(x, d, 64);
    return x;
}

// n / d for n < 2^31 and 1 <= d < 2^31 by one multiply: m = floor(2^(31 + s) / d) + 1
// with s = ceil(log2 d); n * m >> (31 + s) is exact for n < 2^31.
struct FastDiv {
    uint64_t mul;
    uint32_t d, shift;
};

inline FastDiv fast_div(uint32_t d)
{
    uint32_t s = 0;
    while ((uint64_t(1) << s) < d)
        ++s;
    FastDiv f;
    f.d = d;
    f.shift = 31 + s;
    f.mul = ((uint64_t(1) << (31 + s)) / d) + 1; // below 2^33 for s <= 31
    return f;
}

__device__ __forceinline__ uint32_t div_by(uint32_t n, const FastDiv& f)
{
    // n < 2^31 and mul <= 2^32 + ..., so the product stays below 2^64
    return (uint32_t)((uint64_t)n * f.mul >> f.shift);
}

} // namespace ops
} // namespace mfsgd
