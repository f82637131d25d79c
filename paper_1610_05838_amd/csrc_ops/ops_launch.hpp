// ops_launch.hpp -- host-side launch interface between the operators' C-ABI
// layer (ops_api.hip) and their kernels.  Every function only enqueues kernels
// on `st` (no allocation, no copy, no wait), so a caller may capture it.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace mfsgd {
namespace ops {

constexpr int kF32 = 0, kF16 = 1, kBF16 = 2; // MFSGD_FP32, MFSGD_FP16, MFSGD_BF16

inline size_t elem_bytes(int dtype) { return dtype == kF32 ? 4 : 2; }

// Workspaces are cut into parts that start at multiples of 256 bytes.
inline size_t round256(size_t b) { return (b + 255) / 256 * 256; }

// Sizes that no memory holds: sums and products of sizes stop at the largest
// value, and a call whose workspace is above kMostBytes is refused.
constexpr size_t kMostBytes = size_t(1) << 62;
inline size_t times(size_t a, size_t b)
{
    size_t r;
    return __builtin_mul_overflow(a, b, &r) ? SIZE_MAX : r;
}
inline size_t plus(size_t a, size_t b)
{
    size_t r;
    return __builtin_add_overflow(a, b, &r) ? SIZE_MAX : r;
}

// ---- rows of a table (ops_rows.hip) ----
struct RowsLaunch {
    const void* table;
    int64_t rows, ld;
    int k, dtype;
    const int32_t* ids;
    int64_t ids_stride, count;
    float scale;
    void* out;
    int64_t ld_out;
};
hipError_t rows_get(const RowsLaunch& a, hipStream_t st);

struct RowsGradLaunch {
    const void* dout;
    int64_t ld_dout;
    const int32_t* ids;
    int64_t ids_stride, count;
    int k, dtype;
    float scale;
    void* dtable;
    int64_t rows, ld;
    int accumulate;
    void* work;
};
size_t rows_grad_bytes(int64_t count, int k, int64_t rows); // most for rows = 1
hipError_t rows_grad(const RowsGradLaunch& a, hipStream_t st);

// ---- products (ops_linear.hip) ----
struct LinearLaunch {
    const void *x, *w, *bias, *residual;
    int64_t ldx, ldw, ldr, M, N, K;
    int dtype, act;
    void *y, *z;
    int64_t ldy, ldz;
    void* work;
};
size_t linear_bytes(int64_t M, int64_t N, int64_t K, int dtype);
hipError_t linear(const LinearLaunch& a, hipStream_t st);

struct LinearGradLaunch {
    const void *dy, *z, *x, *w;
    int64_t lddy, ldz, ldx, ldw, M, N, K;
    int dtype, act;
    void *dx, *dw, *dbias;
    int64_t lddx, lddw;
    void* work;
};
size_t linear_grad_bytes(int64_t M, int64_t N, int64_t K, int dtype);
hipError_t linear_grad(const LinearGradLaunch& a, hipStream_t st);

// ---- norms over many tensors (ops_norm.hip) ----
struct NormTensor {
    void* p; // updated tensor (clip: the gradient itself); nullptr for a norm alone
    const void* g;
    int64_t n;
    int dtype;
};
size_t norm_bytes(int64_t count);
// *norm_out = sqrt(sum of squares); then, for apply != 0, with c = norm <=
// max_norm ? 1 : max_norm / norm:  1: g <- c g,  2: p <- p - lr (c g + lam p)
hipError_t norm_apply(const NormTensor* list, int64_t count, int apply, double max_norm, float lr, float lam,
                      double* norm_out, void* work, hipStream_t st);

} // namespace ops
} // namespace mfsgd
