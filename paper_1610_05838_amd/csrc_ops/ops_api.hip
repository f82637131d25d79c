// ops_api.hip -- the C ABI of the operators (include/mfsgd.h): argument checks
// and dispatch.  They keep no state; the model's factors and the error text
// come from mfsgd_api.hip.
#include <algorithm>
#include <cmath>
#include <cstdio>
#include <initializer_list>
#include <new>
#include <vector>

#include "mfsgd.h"
#include "mfsgd_launch.hpp"
#include "ops_launch.hpp"

namespace {

using namespace mfsgd;
using namespace mfsgd::ops;

static_assert(kF32 == MFSGD_FP32 && kF16 == MFSGD_FP16 && kBF16 == MFSGD_BF16, "element types");

int bad(const char* msg) { return set_error(MFSGD_EINVAL, msg); }

int launched(hipError_t e) { return e == hipSuccess ? MFSGD_OK : set_error(MFSGD_EHIP, hipGetErrorString(e)); }

// No exception crosses the ABI; a call that returns MFSGD_OK leaves no text.
template <typename F>
int guarded(F&& f) noexcept
{
    try {
        set_error(MFSGD_OK, "");
        return f();
    } catch (const std::bad_alloc&) {
        return set_error(MFSGD_ENOMEM, "host allocation failed");
    } catch (...) {
        return set_error(MFSGD_EHIP, "unexpected exception");
    }
}

#define REQUIRE(cond, msg)                                                                                         \
    do {                                                                                                           \
        if (!(cond))                                                                                               \
            return bad(msg);                                                                                       \
    } while (0)

bool aligned(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

// rows x width elements at p, rows ld elements apart: present, aligned, and its extent in bytes fits 62 bits
bool matrix_ok(const void* p, int64_t rows, int64_t width, int64_t ld, int dtype)
{
    if (ld < width || ld > (int64_t(1) << 40))
        return false;
    if (rows == 0 || width == 0)
        return true;
    return p && aligned(p, elem_bytes(dtype)) && (rows - 1 < (int64_t(1) << 60) / ((int64_t)elem_bytes(dtype) * ld));
}

bool dtype_ok(int32_t d) { return d == kF32 || d == kF16 || d == kBF16; }

constexpr int32_t kMostColumns = 1 << 22; // 64 to 512 columns a workgroup, on the grid's second axis

int check_bytes(size_t need)
{
    REQUIRE(need <= kMostBytes, "the sizes ask for a workspace of more than 2^62 bytes");
    return MFSGD_OK;
}

int check_work(const void* work, int64_t have, size_t need)
{
    if (int rc = check_bytes(need))
        return rc;
    REQUIRE(need == 0 || (work && have >= 0 && (uint64_t)have >= need), "the workspace is too small");
    REQUIRE(need == 0 || aligned(work, 256), "the workspace is not aligned to 256 bytes");
    return MFSGD_OK;
}

// What a call reads or writes: rows of `width` bytes, `pitch` bytes apart.
struct Area {
    uintptr_t at;
    int64_t rows, width, pitch;
    bool written;

    uintptr_t end() const { return at + (uintptr_t)((rows - 1) * pitch + width); }
};

Area matrix(const void* p, int64_t rows, int64_t width, int64_t ld, int dtype, bool written = false)
{
    const int64_t es = (int64_t)elem_bytes(dtype);
    if (!p || rows == 0 || width == 0)
        return Area{0, 0, 0, 0, false};
    if (rows == 1 || ld == width)
        return Area{(uintptr_t)p, 1, rows * width * es, rows * width * es, written};
    return Area{(uintptr_t)p, rows, width * es, ld * es, written};
}

Area row(const void* p, int64_t n, int dtype, bool written = false) { return matrix(p, 1, n, n, dtype, written); }

Area ids_area(const int32_t* ids, int64_t stride, int64_t count) { return matrix(ids, count, 1, stride, kF32); }

Area bytes_area(const void* p, size_t bytes) // a workspace
{
    return Area{(uintptr_t)p, p && bytes ? 1 : 0, (int64_t)bytes, (int64_t)bytes, true};
}

// Whether [from, to) holds a byte of a.
bool reaches(const Area& a, uintptr_t from, uintptr_t to)
{
    if (to <= a.at || from >= a.end())
        return false;
    // the first row that ends behind `from`
    const int64_t i = from < a.at + (uintptr_t)a.width ? 0 : (int64_t)(from - a.at - (uintptr_t)a.width) / a.pitch + 1;
    return i < a.rows && a.at + (uintptr_t)(i * a.pitch) < to;
}

// Whether the two share a byte.  Columns of one buffer lie inside each other's
// extent without doing so: with equal pitches the remainders of their starts
// tell; otherwise the rows of one are looked for in the other, which ends at the
// first that is there.
bool share(const Area& a, const Area& b)
{
    if (a.rows == 0 || b.rows == 0 || a.end() <= b.at || b.end() <= a.at)
        return false;
    if (a.rows == 1)
        return reaches(b, a.at, a.end());
    if (b.rows == 1)
        return reaches(a, b.at, b.end());
    if (a.pitch == b.pitch) {
        const uintptr_t pitch = (uintptr_t)a.pitch;
        const uintptr_t behind = b.at >= a.at ? (b.at - a.at) % pitch : (pitch - (a.at - b.at) % pitch) % pitch;
        if (behind >= (uintptr_t)a.width && behind + (uintptr_t)b.width <= pitch)
            return false;
    }
    const Area &few = a.rows < b.rows ? a : b, &other = a.rows < b.rows ? b : a;
    const int64_t skip = few.at < other.at ? (int64_t)(other.at - few.at) / few.pitch : 0;
    for (int64_t i = skip; i < few.rows; ++i) {
        const uintptr_t at = few.at + (uintptr_t)(i * few.pitch);
        if (at >= other.end())
            break;
        if (reaches(other, at, at + (uintptr_t)few.width))
            return true;
    }
    return false;
}

int check_apart(std::initializer_list<Area> all)
{
    for (const Area* a = all.begin(); a != all.end(); ++a)
        for (const Area* b = a + 1; b != all.end(); ++b)
            REQUIRE(!(a->written || b->written) || !share(*a, *b), "an array that is written overlaps another one");
    return MFSGD_OK;
}

int check_ids(const int32_t* ids, int64_t stride, int64_t count)
{
    REQUIRE(count >= 0 && count <= INT32_MAX, "count must be in [0, 2^31-1]");
    REQUIRE(stride >= 1 && stride <= (int64_t(1) << 28), "ids_stride must be in [1, 2^28]");
    REQUIRE(count == 0 || (ids && aligned(ids, 4)), "ids is NULL or not aligned to 4 bytes");
    return MFSGD_OK;
}

int embed_impl(const RowsLaunch& a, void* stream)
{
    REQUIRE(dtype_ok(a.dtype), "unknown dtype");
    REQUIRE(a.rows >= 1 && a.rows <= INT32_MAX, "rows must be in [1, 2^31-1]");
    REQUIRE(a.k >= 1 && a.k <= kMostColumns, "k must be in [1, 2^22]");
    if (int rc = check_ids(a.ids, a.ids_stride, a.count))
        return rc;
    REQUIRE(matrix_ok(a.table, a.rows, a.k, a.ld, a.dtype), "table is NULL or misaligned, or ld is below k");
    REQUIRE(matrix_ok(a.out, a.count, a.k, a.ld_out, a.dtype), "out is NULL or misaligned, or ld_out is below k");
    if (int rc = check_apart({matrix(a.table, a.rows, a.k, a.ld, a.dtype), ids_area(a.ids, a.ids_stride, a.count),
                              matrix(a.out, a.count, a.k, a.ld_out, a.dtype, true)}))
        return rc;
    return a.count ? launched(rows_get(a, (hipStream_t)stream)) : MFSGD_OK;
}

int embed_grad_impl(RowsGradLaunch a, void* work, int64_t bytes, void* stream)
{
    REQUIRE(dtype_ok(a.dtype), "unknown dtype");
    REQUIRE(a.rows >= 1 && a.rows <= INT32_MAX, "rows must be in [1, 2^31-1]");
    REQUIRE(a.k >= 1 && a.k <= kMostColumns, "k must be in [1, 2^22]");
    if (int rc = check_ids(a.ids, a.ids_stride, a.count))
        return rc;
    REQUIRE(matrix_ok(a.dout, a.count, a.k, a.ld_dout, a.dtype), "dout is NULL or misaligned, or ld_dout is below k");
    REQUIRE(matrix_ok(a.dtable, a.rows, a.k, a.ld, a.dtype), "dtable is NULL or misaligned, or ld is below k");
    const size_t need = rows_grad_bytes(a.count, a.k, a.rows);
    if (int rc = check_work(work, bytes, need))
        return rc;
    if (int rc = check_apart({matrix(a.dout, a.count, a.k, a.ld_dout, a.dtype),
                              ids_area(a.ids, a.ids_stride, a.count),
                              matrix(a.dtable, a.rows, a.k, a.ld, a.dtype, true), bytes_area(work, need)}))
        return rc;
    a.work = work;
    return launched(rows_grad(a, (hipStream_t)stream));
}

// The model's table of `side`, if the current device holds it.
int table_of(int32_t side, int32_t k, int32_t dtype, ModelView& v, void*& table, int64_t& rows)
{
    int dev = -1;
    if (!model_view(&v))
        return set_error(MFSGD_ESTATE, "mfsgd_init has not been called");
    if (hipGetDevice(&dev) != hipSuccess || dev != v.device)
        return set_error(MFSGD_ESTATE, "the current device is not the one mfsgd_init ran on");
    REQUIRE(side == MFSGD_P || side == MFSGD_Q, "side must be MFSGD_P or MFSGD_Q");
    REQUIRE(k == v.k && dtype == v.dtype, "k or dtype is not the model's");
    table = side == MFSGD_P ? v.P : v.Q;
    rows = side == MFSGD_P ? v.m : v.n;
    return MFSGD_OK;
}

// ---- products ----

int check_product(int64_t M, int64_t N, int64_t K, int32_t dtype)
{
    REQUIRE(M >= 0 && N >= 0 && K >= 0 && M <= INT32_MAX && N <= INT32_MAX && K <= INT32_MAX,
            "M, N and K must be in [0, 2^31-1]");
    REQUIRE(dtype_ok(dtype), "unknown dtype");
    return MFSGD_OK;
}

int linear_impl(LinearLaunch a, void* work, int64_t bytes, void* stream)
{
    if (int rc = check_product(a.M, a.N, a.K, a.dtype))
        return rc;
    REQUIRE(a.act >= MFSGD_ACT_NONE && a.act <= MFSGD_ACT_GELU, "unknown act");
    REQUIRE(matrix_ok(a.x, a.M, a.K, a.ldx, a.dtype), "x is NULL or misaligned, or ldx is below K");
    REQUIRE(matrix_ok(a.w, a.N, a.K, a.ldw, a.dtype), "w is NULL or misaligned, or ldw is below K");
    REQUIRE(aligned(a.bias, elem_bytes(a.dtype)), "bias is misaligned");
    REQUIRE(!a.residual || matrix_ok(a.residual, a.M, a.N, a.ldr, a.dtype),
            "residual is misaligned, or ldr is below N");
    REQUIRE(matrix_ok(a.y, a.M, a.N, a.ldy, a.dtype), "y is NULL or misaligned, or ldy is below N");
    REQUIRE(!a.z || matrix_ok(a.z, a.M, a.N, a.ldz, a.dtype), "z is misaligned, or ldz is below N");
    const size_t need = linear_bytes(a.M, a.N, a.K, a.dtype);
    if (int rc = check_work(work, bytes, need))
        return rc;
    const bool in_place = a.residual == a.y && (a.ldr == a.ldy || a.M == 1);
    if (int rc = check_apart({matrix(a.x, a.M, a.K, a.ldx, a.dtype), matrix(a.w, a.N, a.K, a.ldw, a.dtype),
                              row(a.bias, a.N, a.dtype),
                              matrix(in_place ? nullptr : a.residual, a.M, a.N, a.ldr, a.dtype),
                              matrix(a.y, a.M, a.N, a.ldy, a.dtype, true), matrix(a.z, a.M, a.N, a.ldz, a.dtype, true),
                              bytes_area(work, need)}))
        return rc;
    a.work = work;
    return launched(linear(a, (hipStream_t)stream));
}

int linear_grad_impl(LinearGradLaunch a, void* work, int64_t bytes, void* stream)
{
    if (int rc = check_product(a.M, a.N, a.K, a.dtype))
        return rc;
    REQUIRE(a.act >= MFSGD_ACT_NONE && a.act <= MFSGD_ACT_GELU, "unknown act");
    REQUIRE(matrix_ok(a.dy, a.M, a.N, a.lddy, a.dtype), "dy is NULL or misaligned, or lddy is below N");
    REQUIRE(a.act == MFSGD_ACT_NONE || matrix_ok(a.z, a.M, a.N, a.ldz, a.dtype),
            "z is NULL or misaligned, or ldz is below N");
    REQUIRE(!a.dw || matrix_ok(a.x, a.M, a.K, a.ldx, a.dtype), "x is NULL or misaligned, or ldx is below K");
    REQUIRE(!a.dx || matrix_ok(a.w, a.N, a.K, a.ldw, a.dtype), "w is NULL or misaligned, or ldw is below K");
    REQUIRE(!a.dx || matrix_ok(a.dx, a.M, a.K, a.lddx, a.dtype), "dx is misaligned, or lddx is below K");
    REQUIRE(!a.dw || matrix_ok(a.dw, a.N, a.K, a.lddw, a.dtype), "dw is misaligned, or lddw is below K");
    REQUIRE(aligned(a.dbias, elem_bytes(a.dtype)), "dbias is misaligned");
    const size_t need = linear_grad_bytes(a.M, a.N, a.K, a.dtype);
    if (int rc = check_work(work, bytes, need))
        return rc;
    if (int rc = check_apart({matrix(a.dy, a.M, a.N, a.lddy, a.dtype),
                              matrix(a.act == MFSGD_ACT_NONE ? nullptr : a.z, a.M, a.N, a.ldz, a.dtype),
                              matrix(a.dw ? a.x : nullptr, a.M, a.K, a.ldx, a.dtype),
                              matrix(a.dx ? a.w : nullptr, a.N, a.K, a.ldw, a.dtype),
                              matrix(a.dx, a.M, a.K, a.lddx, a.dtype, true),
                              matrix(a.dw, a.N, a.K, a.lddw, a.dtype, true), row(a.dbias, a.N, a.dtype, true),
                              bytes_area(work, need)}))
        return rc;
    a.work = work;
    return launched(linear_grad(a, (hipStream_t)stream));
}

// The model's scores: the users' rows into the workspace, whole (their padding is zero, as the items' is), then the
// product with Q as it lies.
size_t scores_rows_bytes(const ModelView& v, int64_t count)
{
    return round256((size_t)count * (size_t)v.KP * elem_bytes(v.dtype));
}

int scores_impl(const int32_t* users, int64_t stride, int64_t count, int64_t n, int32_t dtype, const void* bias,
                int32_t act, void* out, int64_t ld_out, void* work, int64_t bytes, void* stream)
{
    ModelView v;
    void* P = nullptr;
    int64_t m = 0;
    if (!model_view(&v))
        return set_error(MFSGD_ESTATE, "mfsgd_init has not been called");
    if (int rc = table_of(MFSGD_P, v.k, dtype, v, P, m))
        return rc;
    REQUIRE(n == v.n, "n is not the model's");
    if (int rc = check_ids(users, stride, count))
        return rc;
    REQUIRE(act >= MFSGD_ACT_NONE && act <= MFSGD_ACT_GELU, "unknown act");
    REQUIRE(aligned(bias, elem_bytes(dtype)), "bias is misaligned");
    REQUIRE(matrix_ok(out, count, n, ld_out, dtype), "out is NULL or misaligned, or ld_out is below n");
    const size_t rows = scores_rows_bytes(v, count), need = rows + linear_bytes(count, n, v.KP, dtype);
    if (int rc = check_work(work, bytes, need))
        return rc;
    if (count == 0)
        return MFSGD_OK;
    if (int rc = check_apart({ids_area(users, stride, count), row(bias, n, dtype), matrix(P, m, v.KP, v.KP, dtype),
                              matrix(v.Q, n, v.KP, v.KP, dtype), matrix(out, count, n, ld_out, dtype, true),
                              bytes_area(work, need)}))
        return rc;
    if (int rc = embed_impl(RowsLaunch{P, m, v.KP, v.KP, dtype, users, stride, count, 1.0f, work, v.KP}, stream))
        return rc;
    return linear_impl(LinearLaunch{work, v.Q, bias, nullptr, v.KP, v.KP, 0, count, n, v.KP, dtype, act, out, nullptr,
                                    ld_out, 0, nullptr},
                       (char*)work + rows, bytes - (int64_t)rows, stream);
}

// ---- norms ----

constexpr int64_t kMostTensors = 1 << 20;

int check_tensors(const mfsgd_tensor* list, int64_t count)
{
    REQUIRE(count >= 0 && count <= kMostTensors, "the number of tensors must be in [0, 2^20]");
    REQUIRE(count == 0 || list, "NULL list of tensors");
    int64_t all = 0;
    for (int64_t i = 0; i < count; ++i) {
        const mfsgd_tensor& t = list[i];
        REQUIRE(dtype_ok(t.dtype), "unknown dtype");
        REQUIRE(t.n >= 0 && t.n <= (int64_t(1) << 40), "a tensor's n must be in [0, 2^40]");
        REQUIRE(t.n == 0 || (t.data && aligned(t.data, elem_bytes(t.dtype))), "a tensor is NULL or misaligned");
        all += t.n;
        REQUIRE(all <= (int64_t(1) << 43), "the tensors hold more than 2^43 elements");
    }
    return MFSGD_OK;
}

struct Span {
    uintptr_t from, to;
    bool written;
};

void add_spans(std::vector<Span>& s, const mfsgd_tensor* list, int64_t count, bool written)
{
    for (int64_t i = 0; i < count; ++i)
        if (list[i].n)
            s.push_back(Span{(uintptr_t)list[i].data,
                             (uintptr_t)list[i].data + (size_t)list[i].n * elem_bytes(list[i].dtype), written});
}

// Whether a written span shares a byte with any other.
bool overlap(std::vector<Span>& s)
{
    std::sort(s.begin(), s.end(), [](const Span& a, const Span& b) { return a.from < b.from; });
    uintptr_t any = 0, written = 0; // furthest ends so far
    for (const Span& x : s) {
        if (x.from < written || (x.written && x.from < any))
            return true;
        any = std::max(any, x.to);
        if (x.written)
            written = std::max(written, x.to);
    }
    return false;
}

int norm_impl(const mfsgd_tensor* params, const mfsgd_tensor* grads, int64_t count, int apply, float lr, float lam,
              double max_norm, double* norm_dev, void* work, int64_t bytes, void* stream)
{
    if (int rc = check_tensors(grads, count))
        return rc;
    REQUIRE(norm_dev && aligned(norm_dev, 8), "norm_dev is NULL or not aligned to 8 bytes");
    if (apply)
        REQUIRE(max_norm >= 0.0, "max_norm is negative or NaN");
    if (apply == 2) {
        REQUIRE(std::isfinite(lr) && std::isfinite(lam), "lr or lambda is not finite");
        if (int rc = check_tensors(params, count))
            return rc;
        for (int64_t i = 0; i < count; ++i)
            REQUIRE(params[i].n == grads[i].n && params[i].dtype == grads[i].dtype,
                    "a parameter and its gradient differ in size or dtype");
    }
    const size_t need = norm_bytes(count);
    if (int rc = check_work(work, bytes, need))
        return rc;
    const Span norm{(uintptr_t)norm_dev, (uintptr_t)norm_dev + sizeof(double), true};
    const Span used{(uintptr_t)work, (uintptr_t)work + need, true};
    std::vector<Span> spans;
    spans.reserve((size_t)count * 2 + 2);
    add_spans(spans, grads, count, apply == 1);
    bool shared = norm.from < used.to && used.from < norm.to;
    if (apply) {
        if (apply == 2)
            add_spans(spans, params, count, true);
        spans.push_back(norm);
        spans.push_back(used);
        shared = overlap(spans);
    } else { // gradients that are only read may share what they like
        for (const Span& x : spans)
            shared |= (x.from < norm.to && norm.from < x.to) || (x.from < used.to && used.from < x.to);
    }
    REQUIRE(!shared, "an array that is written overlaps another one");
    std::vector<NormTensor> list((size_t)count);
    for (int64_t i = 0; i < count; ++i)
        list[i] = NormTensor{apply == 2 ? params[i].data : grads[i].data, grads[i].data, grads[i].n, grads[i].dtype};
    return launched(norm_apply(list.data(), count, apply, max_norm, lr, lam, norm_dev, work, (hipStream_t)stream));
}

} // namespace

extern "C" {

int mfsgd_embed(const void* table, int64_t rows, int64_t ld, int32_t k, int32_t dtype, const int32_t* ids,
                int64_t ids_stride, int64_t count, float scale, void* out, int64_t ld_out, void* stream)
{
    return guarded([&]() -> int {
        return embed_impl(RowsLaunch{table, rows, ld, k, dtype, ids, ids_stride, count, scale, out, ld_out}, stream);
    });
}

int mfsgd_embed_grad(const void* dout, int64_t ld_dout, const int32_t* ids, int64_t ids_stride, int64_t count,
                     int32_t k, int32_t dtype, float scale, void* dtable, int64_t rows, int64_t ld,
                     int32_t accumulate, void* workspace, int64_t workspace_bytes, void* stream)
{
    return guarded([&]() -> int {
        return embed_grad_impl(RowsGradLaunch{dout, ld_dout, ids, ids_stride, count, k, dtype, scale, dtable, rows, ld,
                                              accumulate != 0, nullptr},
                               workspace, workspace_bytes, stream);
    });
}

int mfsgd_embed_grad_workspace(int64_t count, int32_t k, int64_t* bytes)
{
    return mfsgd_embed_grad_workspace_rows(count, k, 1, bytes);
}

int mfsgd_embed_grad_workspace_rows(int64_t count, int32_t k, int64_t rows, int64_t* bytes)
{
    return guarded([&]() -> int {
        REQUIRE(bytes, "NULL bytes");
        REQUIRE(count >= 0 && count <= INT32_MAX, "count must be in [0, 2^31-1]");
        REQUIRE(k >= 1 && k <= kMostColumns, "k must be in [1, 2^22]");
        REQUIRE(rows >= 1 && rows <= INT32_MAX, "rows must be in [1, 2^31-1]");
        *bytes = (int64_t)rows_grad_bytes(count, k, rows);
        return MFSGD_OK;
    });
}

int mfsgd_rows(int32_t side, const int32_t* ids, int64_t ids_stride, int64_t count, int32_t k, int32_t dtype,
               float scale, void* out, int64_t ld_out, void* stream)
{
    return guarded([&]() -> int {
        ModelView v;
        void* table = nullptr;
        int64_t rows = 0;
        if (int rc = table_of(side, k, dtype, v, table, rows))
            return rc;
        return embed_impl(RowsLaunch{table, rows, v.KP, k, v.dtype, ids, ids_stride, count, scale, out, ld_out},
                          stream);
    });
}

int mfsgd_add_rows(int32_t side, const void* dout, int64_t ld_dout, const int32_t* ids, int64_t ids_stride,
                   int64_t count, int32_t k, int32_t dtype, float scale, void* workspace, int64_t workspace_bytes,
                   void* stream)
{
    return guarded([&]() -> int {
        ModelView v;
        void* table = nullptr;
        int64_t rows = 0;
        if (int rc = table_of(side, k, dtype, v, table, rows))
            return rc;
        return embed_grad_impl(RowsGradLaunch{dout, ld_dout, ids, ids_stride, count, k, v.dtype, scale, table, rows,
                                              v.KP, 1, nullptr},
                               workspace, workspace_bytes, stream);
    });
}

int mfsgd_linear(const void* x, int64_t ldx, const void* w, int64_t ldw, const void* bias, const void* residual,
                 int64_t ldr, int64_t M, int64_t N, int64_t K, int32_t dtype, int32_t act, void* y, int64_t ldy,
                 void* z, int64_t ldz, void* workspace, int64_t workspace_bytes, void* stream)
{
    return guarded([&]() -> int {
        return linear_impl(LinearLaunch{x, w, bias, residual, ldx, ldw, ldr, M, N, K, dtype, act, y, z, ldy, ldz,
                                        nullptr},
                           workspace, workspace_bytes, stream);
    });
}

int mfsgd_linear_workspace(int64_t M, int64_t N, int64_t K, int32_t dtype, int64_t* bytes)
{
    return guarded([&]() -> int {
        REQUIRE(bytes, "NULL bytes");
        if (int rc = check_product(M, N, K, dtype))
            return rc;
        *bytes = (int64_t)linear_bytes(M, N, K, dtype);
        return MFSGD_OK;
    });
}

int mfsgd_linear_grad(const void* dy, int64_t lddy, const void* z, int64_t ldz, const void* x, int64_t ldx,
                      const void* w, int64_t ldw, int64_t M, int64_t N, int64_t K, int32_t dtype, int32_t act,
                      void* dx, int64_t lddx, void* dw, int64_t lddw, void* dbias, void* workspace,
                      int64_t workspace_bytes, void* stream)
{
    return guarded([&]() -> int {
        return linear_grad_impl(LinearGradLaunch{dy, z, x, w, lddy, ldz, ldx, ldw, M, N, K, dtype, act, dx, dw, dbias,
                                                 lddx, lddw, nullptr},
                                workspace, workspace_bytes, stream);
    });
}

int mfsgd_linear_grad_workspace(int64_t M, int64_t N, int64_t K, int32_t dtype, int64_t* bytes)
{
    return guarded([&]() -> int {
        REQUIRE(bytes, "NULL bytes");
        if (int rc = check_product(M, N, K, dtype))
            return rc;
        const size_t need = linear_grad_bytes(M, N, K, dtype);
        if (int rc = check_bytes(need))
            return rc;
        *bytes = (int64_t)need;
        return MFSGD_OK;
    });
}

int mfsgd_scores(const int32_t* users, int64_t users_stride, int64_t count, int64_t n, int32_t dtype,
                 const void* bias, int32_t act, void* out, int64_t ld_out, void* workspace, int64_t workspace_bytes,
                 void* stream)
{
    return guarded([&]() -> int {
        return scores_impl(users, users_stride, count, n, dtype, bias, act, out, ld_out, workspace, workspace_bytes,
                           stream);
    });
}

int mfsgd_scores_workspace(int64_t count, int64_t* bytes)
{
    return guarded([&]() -> int {
        ModelView v;
        REQUIRE(bytes, "NULL bytes");
        REQUIRE(count >= 0 && count <= INT32_MAX, "count must be in [0, 2^31-1]");
        if (!model_view(&v))
            return set_error(MFSGD_ESTATE, "mfsgd_init has not been called");
        *bytes = (int64_t)(scores_rows_bytes(v, count) + linear_bytes(count, v.n, v.KP, v.dtype));
        return MFSGD_OK;
    });
}

int mfsgd_grad_norm(const mfsgd_tensor* grads, int64_t count, double* norm_dev, void* workspace,
                    int64_t workspace_bytes, void* stream)
{
    return guarded([&]() -> int {
        return norm_impl(nullptr, grads, count, 0, 0.0f, 0.0f, 0.0, norm_dev, workspace, workspace_bytes, stream);
    });
}

int mfsgd_clip_grads(const mfsgd_tensor* grads, int64_t count, double max_norm, double* norm_dev, void* workspace,
                     int64_t workspace_bytes, void* stream)
{
    return guarded([&]() -> int {
        return norm_impl(nullptr, grads, count, 1, 0.0f, 0.0f, max_norm, norm_dev, workspace, workspace_bytes, stream);
    });
}

int mfsgd_sgd_step(const mfsgd_tensor* params, const mfsgd_tensor* grads, int64_t count, float lr, float lambda,
                   double max_norm, double* norm_dev, void* workspace, int64_t workspace_bytes, void* stream)
{
    return guarded([&]() -> int {
        return norm_impl(params, grads, count, 2, lr, lambda, max_norm, norm_dev, workspace, workspace_bytes, stream);
    });
}

int mfsgd_norm_workspace(int64_t count, int64_t* bytes)
{
    return guarded([&]() -> int {
        REQUIRE(bytes, "NULL bytes");
        REQUIRE(count >= 0 && count <= kMostTensors, "the number of tensors must be in [0, 2^20]");
        *bytes = (int64_t)norm_bytes(count);
        return MFSGD_OK;
    });
}

} // extern "C"
