// ops_linear.hip -- products with bias, activation and residual, and their
// gradient:
//   Z = X W^T + b,  Y = act(Z) + R
//   dZ = dY o act'(Z),  dX = dZ W,  dW = dZ^T X,  db = column sums of dZ
//
// Every product is one form, C = A B^T with A (rows x depth) and B (cols x
// depth) both contiguous along the depth that is summed over.
#include <algorithm>
#include <cmath>

#include "ops_common.hpp"

namespace mfsgd {
namespace ops {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------ activations
//
// In binary32.  16-bit results take the hardware's exponential and reciprocal (1
// ulp) and for the normal distribution's tail the fit below; binary32 results the
// library functions.  No small result is the difference of two large numbers, so
// that the tails too are right relative to their own size: to the error of
// exp(-z^2 / 2) with a rounded argument, z^2 2^-22, and in 16 bits to 3e-5 (a 16th of
// half a step of binary16).
enum { kNone = 0, kRelu = 1, kSigmoid = 2, kSilu = 3, kGelu = 4 };

template <bool EXACT>
__device__ __forceinline__ float sigmoid(float z)
{
    if (EXACT)
        return 1.0f / (1.0f + expf(-z));
    return __builtin_amdgcn_rcpf(1.0f + __expf(-z));
}

template <bool EXACT>
__device__ __forceinline__ float normal_cdf(float z) // (1 + erf(z / sqrt 2)) / 2
{
    const float x = z * 0.70710678118654752f;
    if (EXACT)
        return 0.5f * erfcf(-x);
    // erfc(a) exp(a^2) for a >= 0 is t times a polynomial in t = 1 / (1 + 0.51 a), fitted so that the largest error is
    // least, counted in 1.2e-7 of 1 near a = 0 and in 3e-5 of erfc(a) in its tail
    const float a = fabsf(x), t = __builtin_amdgcn_rcpf(1.0f + 0.51f * a);
    float p = 0.085031174f;
    p = p * t - 0.32321757f;
    p = p * t + 0.30460083f;
    p = p * t + 0.09527203f;
    p = p * t + 0.2636423f;
    p = p * t + 0.28692773f;
    p = p * t + 0.2877436f;
    const float tail = 0.5f * p * t * __expf(-x * x); // (1 - erf a) / 2
    return z < 0.0f ? tail : 1.0f - tail;
}

// Beyond 128 on either side a result or slope equals its limit in every type; with
// z bounded there the formulas' products of an infinity and a zero become that
// limit.  (A NaN is lost in the bound and comes back with the other factor.)
__device__ __forceinline__ float above(float z) { return fmaxf(z, -128.0f); }
__device__ __forceinline__ float bounded(float z) { return __builtin_amdgcn_fmed3f(z, -128.0f, 128.0f); }

template <bool EXACT, int C>
__device__ __forceinline__ void activate(float (&v)[C], int act)
{
    switch (act) {
    case kRelu:
#pragma unroll
        for (int c = 0; c < C; ++c)
            v[c] = v[c] > 0.0f || v[c] != v[c] ? v[c] : 0.0f;
        break;
    case kSigmoid:
#pragma unroll
        for (int c = 0; c < C; ++c)
            v[c] = sigmoid<EXACT>(v[c]);
        break;
    case kSilu:
#pragma unroll
        for (int c = 0; c < C; ++c)
            v[c] = above(v[c]) * sigmoid<EXACT>(v[c]);
        break;
    case kGelu:
#pragma unroll
        for (int c = 0; c < C; ++c)
            v[c] = above(v[c]) * normal_cdf<EXACT>(v[c]);
        break;
    }
}

template <bool EXACT>
__device__ __forceinline__ float slope(float z, int act)
{
    switch (act) {
    case kRelu:
        return z > 0.0f ? 1.0f : z != z ? z : 0.0f; // a NaN stays one, as in the result
    case kSigmoid: { // s (1 - s) without the difference: the same on both sides of 0
        const float e = EXACT ? expf(-fabsf(z)) : __expf(-fabsf(z));
        const float r = EXACT ? 1.0f / (1.0f + e) : __builtin_amdgcn_rcpf(1.0f + e);
        return e * r * r;
    }
    case kSilu: {
        const float s = sigmoid<EXACT>(z);
        return s * (1.0f + bounded(z) * (1.0f - s));
    }
    case kGelu: {
        const float e = EXACT ? expf(-0.5f * z * z) : __expf(-0.5f * z * z);
        return normal_cdf<EXACT>(z) + bounded(z) * e * 0.39894228040143268f;
    }
    default:
        return 1.0f;
    }
}

// ---------------------------------------------------------------- epilogue
struct Epilogue {
    const void *bias, *residual;
    void *y, *z;
    int64_t ldr, ldy, ldz, M, N;
    int act;
    bool near; // 256 rows of each matrix are addressed by 31 bits
};

// C elements at p of which the first `n` exist (zeros for the rest).
template <typename T, int C>
__device__ __forceinline__ void read_some(const T* p, int n, float (&v)[C])
{
    constexpr int V = 16 / (int)sizeof(T) < C ? 16 / (int)sizeof(T) : C;
    if (n >= C) {
#pragma unroll
        for (int c = 0; c < C; c += V) {
            const Vec<T, V> x = load_vec<T, V>(p + c);
#pragma unroll
            for (int i = 0; i < V; ++i)
                v[c + i] = (float)x.v[i];
        }
    } else {
#pragma unroll
        for (int c = 0; c < C; ++c)
            v[c] = c < n ? (float)p[c] : 0.0f;
    }
}

template <typename T, int C>
__device__ __forceinline__ void write_some(T* p, int n, const float (&v)[C])
{
    constexpr int V = 16 / (int)sizeof(T) < C ? 16 / (int)sizeof(T) : C;
    if (n >= C) {
#pragma unroll
        for (int c = 0; c < C; c += V) {
            Vec<T, V> x;
#pragma unroll
            for (int i = 0; i < V; ++i)
                x.v[i] = T(v[c + i]);
            store_vec<T, V>(p + c, x);
        }
    } else {
#pragma unroll
        for (int c = 0; c < C; ++c)
            if (c < n)
                p[c] = T(v[c]);
    }
}

// Row m, columns n .. n + C: C sums of one lane.
template <typename T, int C>
__device__ __forceinline__ void finish(const Epilogue& e, int64_t m, int64_t n, float (&v)[C])
{
    if (m >= e.M || n >= e.N)
        return;
    const int some = e.N - n < C ? (int)(e.N - n) : C;
    if (e.bias) {
        float x[C];
        read_some<T, C>((const T*)e.bias + n, some, x);
#pragma unroll
        for (int c = 0; c < C; ++c)
            v[c] += x[c];
    }
    if (e.z)
        write_some<T, C>((T*)e.z + m * e.ldz + n, some, v);
    activate<sizeof(T) == 4, C>(v, e.act);
    if (e.residual) {
        float x[C];
        read_some<T, C>((const T*)e.residual + m * e.ldr + n, some, x);
#pragma unroll
        for (int c = 0; c < C; ++c)
            v[c] += x[c];
    }
    write_some<T, C>((T*)e.y + m * e.ldy + n, some, v);
}

// -------------------------------------------------------------- the product
//
// A workgroup computes BM rows x BN columns; its wavefronts WM x WN each, as
// 16 x 16 tiles of the matrix instructions.  A's and B's rows are staged in LDS
// kRow = 128 bytes of depth at a time; the copies of the next stages are on
// their way while one is computed on.
//
// The 16-byte pieces of a staged row are stored in the order piece ^ (row & 7),
// so that the 16 lanes that read one piece of 16 rows meet different banks; the
// copy writes LDS linearly, so the lanes' global addresses carry that order.
//
// B is the matrix instruction's row operand: a lane then holds 4 consecutive
// columns of C per tile (see column_of).
//
// Bound by the matrix instructions and what feeds them from LDS: 4096^3 bfloat16
// with bias, gelu, residual and Z kept 116-129 us, 1.1-1.2 PFLOP/s; by the epilogue
// where the depth is short: 2048 x 39,780 x 128 binary16 with bias and sigmoid 61
// us, 163 MB written at 2.7 TB/s (an exponential and a reciprocal per element are 17
// us of the vector units, the rest of the epilogue as much again).
constexpr int kRow = 128; // bytes of depth of a stage

__device__ __attribute__((aligned(16))) const uint32_t g_zeros[4] = {0, 0, 0, 0};

struct GemmArgs {
    const void *A, *B;
    int64_t lda, ldb, rows, cols, depth;
    uint32_t tiles_m, tiles_n, all, tile0; // of the whole product; with its slices; this launch's first
    int steps;                        // stages of one workgroup: a slice of the depth
    float* part;                      // the slices' sums [slice][rows][cols], or nullptr: one slice, finished here
};

// One launch's work: a product's tiles, slice by slice, the ids rounded up to
// whole turns of the XCDs; from id `second` on another product's;
// from id `sums` on the column sums of dZ (see k_turn).
struct Products {
    GemmArgs g[2];
    Epilogue e[2];
    uint32_t second, sums;
    const float* col_sums;
    int64_t row_tiles, cols;
    void* dbias;
};
constexpr uint32_t kNoWork = 0xffffffffu;

template <typename T>
__device__ __forceinline__ void mma(f32x4& c, const u32x4& b, const u32x4& a);

template <>
__device__ __forceinline__ void mma<_Float16>(f32x4& c, const u32x4& b, const u32x4& a)
{
    c = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, b), __builtin_bit_cast(f16x8, a), c, 0, 0, 0);
}

template <>
__device__ __forceinline__ void mma<__bf16>(f32x4& c, const u32x4& b, const u32x4& a)
{
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, b), __builtin_bit_cast(bf16x8, a), c, 0, 0,
                                                0);
}

// a lane's four values are depths 4 (lane / 16) + t: step t multiplies depths t, 4 + t, 8 + t, 12 + t
template <>
__device__ __forceinline__ void mma<float>(f32x4& c, const u32x4& b, const u32x4& a)
{
#pragma unroll
    for (int t = 0; t < 4; ++t)
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, (uint32_t)b[t]),
                                                 __builtin_bit_cast(float, (uint32_t)a[t]), c, 0, 0, 0);
}

// The 16-byte piece at p, of which the first n elements exist (zeros for the rest).
template <typename T>
__device__ __forceinline__ u32x4 piece_at(const T* p, int64_t n)
{
    constexpr int piece = 16 / (int)sizeof(T);
    Vec<T, piece> x;
    if (n >= piece) {
        x = load_vec<T, piece>(p);
    } else {
#pragma unroll
        for (int i = 0; i < piece; ++i)
            x.v[i] = i < n ? p[i] : T(0.0f);
    }
    u32x4 r;
    __builtin_memcpy(&r, &x, 16);
    return r;
}

// The column of C that row r of B's staged rows belongs to.  The matrix
// instruction leaves a lane columns 4 (lane / 16) + 0..3 of each 16; with 16-bit
// results two such tiles are made neighbours, so that a lane's 16-byte stores
// hold consecutive columns and four lanes write 64 bytes of a row in one
// instruction (binary32: they do as it is).
template <typename T>
__device__ __forceinline__ int column_of(int r)
{
    return sizeof(T) == 4 ? r : (r & ~31) + (r >> 2 & 3) * 8 + (r >> 4 & 1) * 4 + (r & 3);
}

// Workgroups are dealt to the 8 XCDs in turn: each XCD takes a run of
// consecutive tiles, slice by slice, and runs go down 8 tiles of rows before the
// next column, so that the tiles of an XCD share rows of A and B in its L2.
__device__ __forceinline__ void tile_place(const GemmArgs& g, uint32_t id, uint32_t& slice, uint32_t& tm, uint32_t& tn)
{
    const uint32_t tiles = g.tiles_m * g.tiles_n, x = id & 7;
    uint32_t t = x * (g.all >> 3) + (x < (g.all & 7) ? x : g.all & 7) + (id >> 3);
    slice = g.part ? t / tiles : 0;
    t -= slice * tiles;
    const uint32_t band = 8 * g.tiles_n, b = t / band, at = t - b * band;
    const uint32_t high = g.tiles_m - b * 8 < 8 ? g.tiles_m - b * 8 : 8;
    tn = at / high;
    tm = b * 8 + (at - tn * high);
}

// Wait until at most N of this wavefront's memory operations are outstanding.
template <int N>
__device__ __forceinline__ void wait_memory()
{
    static_assert(N >= 0 && N < 64, "a 6-bit count");
    __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | (N >> 4) << 14);
}

struct Yes {
    static constexpr bool value = true;
};
struct No {
    static constexpr bool value = false;
};
template <bool B, typename X, typename Y>
struct Pick {
    typedef X type;
};
template <typename X, typename Y>
struct Pick<false, X, Y> {
    typedef Y type;
};

template <typename T>
__device__ __forceinline__ void add_piece(float (&v)[16 / sizeof(T)], const u32x4& x)
{
    Vec<T, 16 / (int)sizeof(T)> p;
    __builtin_memcpy(&p, &x, 16);
#pragma unroll
    for (int c = 0; c < 16 / (int)sizeof(T); ++c)
        v[c] += (float)p.v[c];
}

// dbias from the column sums per 64 rows, 64 columns a workgroup of `parts`
// wavefronts: each adds a consecutive part of the tiles, the sums are joined in
// order.
template <typename T, int PARTS>
__device__ __forceinline__ void add_columns(const Products& p, int64_t block, float* lds)
{
    const int x = threadIdx.x & 63, y = threadIdx.x >> 6;
    const int64_t c = block * 64 + x, each = (p.row_tiles + PARTS - 1) / PARTS;
    const int64_t from = y * each, to = from + each < p.row_tiles ? from + each : p.row_tiles;
    float sum = 0.0f;
    if (c < p.cols)
        for (int64_t t0 = from; t0 < to; t0 += 8) {
            float v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u)
                v[u] = t0 + u < to ? p.col_sums[(t0 + u) * p.cols + c] : 0.0f;
#pragma unroll
            for (int u = 0; u < 8; ++u)
                sum += v[u];
        }
    lds[y * 64 + x] = sum;
    __syncthreads();
    if (y == 0 && c < p.cols) {
#pragma unroll
        for (int w = 1; w < PARTS; ++w)
            sum += lds[w * 64 + x];
        ((T*)p.dbias)[c] = T(sum);
    }
}

// DIRECT: rows of A and B start at 16-byte boundaries and the depth is whole
// pieces; the copies go from memory to LDS by themselves.  Otherwise (any
// alignment, any depth) they pass through registers.
template <typename T, int BM, int BN, int WM, int WN, bool DIRECT, int NB>
__global__ __launch_bounds__((BM / WM) * (BN / WN) * 64) void k_gemm(Products p)
{
    constexpr int pieces = kRow / 16, deep = kRow / 64; // of a staged row; steps of the matrix instructions in a stage
    constexpr int copied = 64 / pieces;                 // rows a wavefront copies at a time
    constexpr int waves = (BM / WM) * (BN / WN), groups = (BM + BN) / copied / waves;
    constexpr int TM = WM / 16, TN = WN / 16, piece = 16 / (int)sizeof(T), per_stage = kRow / (int)sizeof(T);
    constexpr int stage_bytes = (BM + BN) * kRow;
    static_assert(WN % 64 == 0 && (BM + BN) % (copied * waves) == 0 && BM % copied == 0, "tile shape");
    static_assert(DIRECT || NB == 2, "copies through registers have two stages in LDS");
    __shared__ __attribute__((aligned(128))) char lds[NB * stage_bytes];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / (BN / WN) * WM, wn = wave % (BN / WN) * WN;
    if (blockIdx.x >= p.sums) {
        add_columns<T, waves>(p, blockIdx.x - p.sums, (float*)lds);
        return;
    }
    const bool other = blockIdx.x >= p.second;
    const GemmArgs g = other ? p.g[1] : p.g[0];
    const Epilogue e = other ? p.e[1] : p.e[0];
    const uint32_t id = blockIdx.x + g.tile0 - (other ? p.second : 0);
    uint32_t slice, tm, tn;
    if (id >= g.all)
        return;
    tile_place(g, id, slice, tm, tn);
    const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
    const int64_t k0 = (int64_t)slice * g.steps * per_stage;
    const int64_t mine = (int64_t)g.steps * per_stage, depth = g.depth - k0 < mine ? g.depth - k0 : mine;
    const int steps = (int)((depth + per_stage - 1) / per_stage);

    // this lane's rows to copy: `copied` rows a group, a 16-byte piece of one each; rows past the end repeat the last
    // one (their sums are not written)
    auto turn = [](int row) { return row & (pieces - 1); };
    const int pc = (lane & (pieces - 1)) ^ turn(lane / pieces);
    const char* base[2] = {(const char*)((const T*)g.A + m0 * g.lda + k0), (const char*)((const T*)g.B + n0 * g.ldb + k0)};
    typedef typename Pick<DIRECT, uint32_t, uint64_t>::type Offset;
    Offset off[groups]; // from the tile's first row
    const int last_m = g.rows - m0 < BM ? (int)(g.rows - m0) - 1 : BM - 1;
    const int last_n = g.cols - n0 < BN ? (int)(g.cols - n0) - 1 : BN - 1;
#pragma unroll
    for (int u = 0; u < groups; ++u) {
        const int group = wave * groups + u, row = group * copied + lane / pieces;
        if (group < BM / copied) {
            off[u] = ((Offset)(row < last_m ? row : last_m) * (Offset)g.lda + pc * piece) * (Offset)sizeof(T);
        } else {
            const int n = column_of<T>(row - BM);
            off[u] = ((Offset)(n < last_n ? n : last_n) * (Offset)g.ldb + pc * piece) * (Offset)sizeof(T);
        }
    }
    // stages before `whole` lie inside the depth; in the last one pieces past it are zeros
    const int whole = (int)(depth / per_stage);
    const int64_t room = depth - (int64_t)whole * per_stage - pc * piece; // this lane's elements in that stage
    uint64_t zeros = (uint64_t)g_zeros;
    asm("" : "+v"(zeros)); // in registers: the copies' addresses are selected, not branched on
    u32x4 held[2][DIRECT ? 1 : groups]; // stages on their way through registers
    auto fetch = [&](int s, auto full, int half = 0) {
        constexpr bool FULL = decltype(full)::value;
        const char* from[2] = {base[0] + (int64_t)s * kRow, base[1] + (int64_t)s * kRow};
        if constexpr (DIRECT) {
            char* to = lds + s % NB * stage_bytes + wave * groups * copied * kRow;
            if (FULL || s < whole) {
#pragma unroll
                for (int u = 0; u < groups; ++u)
                    __builtin_amdgcn_global_load_lds(
                        (const __attribute__((address_space(1))) void*)(from[wave * groups + u >= BM / copied] + off[u]),
                        (__attribute__((address_space(3))) void*)(to + u * 1024), 16, 0, 0);
            } else {
#pragma unroll
                for (int u = 0; u < groups; ++u) {
                    const uint64_t at = room <= 0 ? zeros : (uint64_t)(from[wave * groups + u >= BM / copied] + off[u]);
                    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)at,
                                                     (__attribute__((address_space(3))) void*)(to + u * 1024), 16, 0, 0);
                }
            }
        } else {
            const int64_t some = FULL || s < whole ? piece : room;
#pragma unroll
            for (int u = 0; u < groups; ++u)
                held[half][u] = piece_at<T>((const T*)(from[wave * groups + u >= BM / copied] + off[u]), some);
        }
    };
    auto keep = [&](int s, int half) {
        char* to = lds + s % NB * stage_bytes + wave * groups * copied * kRow + lane * 16;
#pragma unroll
        for (int u = 0; u < groups; ++u)
            *(u32x4*)(to + u * 1024) = held[half][DIRECT ? 0 : u];
    };
    // all copies of this wavefront are in LDS that everyone's have to be in, and everyone is done reading before
    auto meet = [&] {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
    };

    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
            acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    const int quad = lane >> 4, r16 = lane & 15;
    u32x4 a[2][TM], b[2][TN]; // operands of this step and of the next
    auto read = [&](int to, int s, int kk) {
        const char* at = lds + s % NB * stage_bytes + ((kk * 4 + quad) ^ turn(r16)) * 16 + r16 * kRow;
#pragma unroll
        for (int j = 0; j < TN; ++j)
            b[to][j] = *(const u32x4*)(at + (BM + wn + j * 16) * kRow);
#pragma unroll
        for (int i = 0; i < TM; ++i)
            a[to][i] = *(const u32x4*)(at + (wm + i * 16) * kRow);
    };
    auto multiply = [&](int from) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
                mma<T>(acc[i][j], b[from][j], a[from][i]);
    };
    if constexpr (DIRECT) {
        // Of the ring of NB stages one is computed on and the others are on their way.  The operands of every step of
        // the matrix instructions are read from LDS during the step before, and everyone meets once a stage.
        auto stage = [&](int s, auto full) { // full: the stage to fetch exists and is whole
            constexpr bool FULL = decltype(full)::value;
#pragma unroll
            for (int kk = 0; kk < deep; ++kk) {
                if (kk + 1 < deep) {
                    read((kk + 1) & 1, s, kk + 1);
                } else if (FULL || s + 1 < steps) {
                    if (FULL || s + NB - 1 < steps)
                        wait_memory<(NB - 2) * groups>(); // stage s + 1 has landed
                    else
                        wait_memory<0>();
                    meet();
                    if (FULL || s + NB < steps)
                        fetch(s + NB, full);
                    read((kk + 1) & 1, s + 1, 0);
                }
                multiply(kk & 1);
                if constexpr (FULL) {
                    // spread the reads and copies among the products instead of before them (8192^3 bfloat16: 796 us
                    // against 828)
                    constexpr int products = TM * TN * (sizeof(T) == 4 ? 4 : 1), parts = products >= 64 ? 16 : 8;
#pragma unroll
                    for (int q = 0; q < parts; ++q) {
                        __builtin_amdgcn_sched_group_barrier(0x100, (TM + TN + parts - 1) / parts, 0); // LDS reads
                        if (kk + 1 == deep)
                            __builtin_amdgcn_sched_group_barrier(0x020, (groups + parts - 1) / parts, 0); // copies
                        __builtin_amdgcn_sched_group_barrier(0x008, products / parts, 0); // matrix instructions
                    }
                }
            }
        };
        static_assert(deep % 2 == 0, "a stage begins with the operands in half 0");
        int s = 0;
        if (steps > 0) {
#pragma unroll
            for (int i = 0; i < NB; ++i)
                if (i < steps)
                    fetch(i, No());
            if (steps >= NB)
                wait_memory<(NB - 1) * groups>();
            else
                wait_memory<0>();
            meet();
            read(0, 0, 0);
        }
        for (; s + NB < whole; ++s)
            stage(s, Yes());
        for (; s < steps; ++s)
            stage(s, No());
    } else {
        // One stage is computed on, the next one is in registers or on its way there, the one after it on its way.
        auto stage = [&](int s, int half, auto full) {
            constexpr bool FULL = decltype(full)::value;
            meet();
            if (FULL || s + 2 < steps)
                fetch(s + 2, full, half);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int kk = 0; kk < deep; ++kk) {
                read(0, s, kk);
                multiply(0);
            }
            if (FULL || s + 1 < steps)
                keep(s + 1, half ^ 1);
        };
        if (steps > 0) {
            fetch(0, No(), 0);
            if (steps > 1)
                fetch(1, No(), 1);
            keep(0, 0);
        }
        int s = 0;
        for (; s + 3 < whole; s += 2) {
            stage(s, 0, Yes());
            stage(s + 1, 1, Yes());
        }
        for (; s < steps; s += 2) {
            stage(s, 0, No());
            if (s + 1 < steps)
                stage(s + 1, 1, No());
        }
    }

    constexpr int together = sizeof(T) == 4 ? 1 : 2, chunks = TN / together; // tiles whose columns a lane holds together
    const int64_t mrow = m0 + wm + r16, ncol = n0 + wn + quad * piece;
    if (g.part) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < chunks; ++j) {
                const int64_t m = mrow + i * 16, n = ncol + j * 16 * together;
                float v[piece];
#pragma unroll
                for (int c = 0; c < piece; ++c)
                    v[c] = acc[i][j * together + c / 4][c % 4];
                if (m < g.rows && n < g.cols)
                    write_some<float, piece>(g.part + ((int64_t)slice * g.rows + m) * g.cols + n,
                                             g.cols - n < piece ? (int)(g.cols - n) : piece, v);
            }
        return;
    }
    // What the epilogue reads, several pieces at a time: one wait for memory instead of one a piece.  A tile that lies
    // inside C needs no checks, and its addresses are a scalar and a 32-bit offset of the lane: where the output is
    // most of the work the vector instructions of an epilogue with them took as long as its stores.
    auto epilogue = [&](auto inside) {
        constexpr bool INSIDE = decltype(inside)::value;
        constexpr int batch = TM * chunks <= 8 ? TM : 8 / chunks;
        const int lrow = wm + r16, lcol = wn + quad * piece;
        // piece (i, j) of a matrix of pitch ld
        auto at = [&](const void* p, int64_t ld, int i, int j) {
            const int far = i * 16, near = j * 16 * together;
            if (INSIDE) {
                const T* tile = (const T*)p + (m0 + far) * ld + n0 + near;
                return (T*)((char*)tile + (uint32_t)(lrow * (uint32_t)ld + lcol) * (uint32_t)sizeof(T));
            }
            return (T*)p + (mrow + far) * ld + ncol + near;
        };
        u32x4 bias[chunks];
        if (e.bias) {
#pragma unroll
            for (int j = 0; j < chunks; ++j)
                bias[j] = piece_at<T>(at(e.bias, 0, 0, j), INSIDE ? piece : e.N - ncol - j * 16 * together);
        }
#pragma unroll
        for (int i0 = 0; i0 < TM; i0 += batch) {
            u32x4 res[batch][chunks];
            if (e.residual) {
#pragma unroll
                for (int i = 0; i < batch; ++i)
#pragma unroll
                    for (int j = 0; j < chunks; ++j)
                        res[i][j] = piece_at<T>(at(e.residual, e.ldr, i0 + i, j),
                                                INSIDE                            ? piece
                                                : mrow + (i0 + i) * 16 < e.M ? e.N - ncol - j * 16 * together
                                                                                  : 0);
            }
#pragma unroll
            for (int i = 0; i < batch; ++i)
#pragma unroll
                for (int j = 0; j < chunks; ++j) {
                    const int64_t m = mrow + (i0 + i) * 16, n = ncol + j * 16 * together;
                    if (!INSIDE && (m >= e.M || n >= e.N))
                        continue;
                    const int some = INSIDE || e.N - n >= piece ? piece : (int)(e.N - n);
                    float v[piece];
#pragma unroll
                    for (int c = 0; c < piece; ++c)
                        v[c] = acc[i0 + i][j * together + c / 4][c % 4];
                    if (e.bias)
                        add_piece<T>(v, bias[j]);
                    if (e.z)
                        write_some<T, piece>(at(e.z, e.ldz, i0 + i, j), some, v);
                    activate<sizeof(T) == 4, piece>(v, e.act);
                    if (e.residual)
                        add_piece<T>(v, res[i][j]);
                    write_some<T, piece>(at(e.y, e.ldy, i0 + i, j), some, v);
                }
        }
    };
    if (e.near && m0 + BM <= e.M && n0 + BN <= e.N)
        epilogue(Yes());
    else
        epilogue(No());
}

// The slices' sums, added in order and finished: 4 columns a thread, BATCH of a
// column's sums on their way at a time (bound by that chain: few threads, many
// slices; 45 slices of 256 x 128: 7.5 us).  From
// workgroup `second` on another product's.
struct Join {
    const float* part[2];
    int slices[2];
    int64_t rows[2], cols[2];
    Epilogue e[2];
    uint32_t second;
};

template <typename T, int BATCH>
__global__ __launch_bounds__(256) void k_gemm_join(Join p)
{
    const bool other = blockIdx.x >= p.second;
    const float* part = other ? p.part[1] : p.part[0];
    const int slices = other ? p.slices[1] : p.slices[0];
    const int64_t rows = other ? p.rows[1] : p.rows[0], cols = other ? p.cols[1] : p.cols[0];
    const Epilogue e = other ? p.e[1] : p.e[0];
    const uint32_t block = other ? blockIdx.x - p.second : blockIdx.x;
    const uint32_t blocks = other || p.second > gridDim.x ? gridDim.x - (other ? p.second : 0) : p.second;
    const int64_t per_row = (cols + 3) / 4, all = rows * per_row, size = rows * cols;
    for (int64_t i = (int64_t)block * 256 + threadIdx.x; i < all; i += (int64_t)blocks * 256) {
        const int64_t m = all <= 0xffffffff ? (uint32_t)i / (uint32_t)per_row : i / per_row, n = (i - m * per_row) * 4;
        const int some = cols - n < 4 ? (int)(cols - n) : 4;
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int s0 = 0; s0 < slices; s0 += BATCH) {
            float x[BATCH][4];
#pragma unroll
            for (int u = 0; u < BATCH; ++u)
                read_some<float, 4>(part + (s0 + u < slices ? s0 + u : s0) * size + m * cols + n, some, x[u]);
#pragma unroll
            for (int u = 0; u < BATCH; ++u)
                if (s0 + u < slices) {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        sum[c] += x[u][c];
                }
        }
        finish<T, 4>(e, m, n, sum);
    }
}

// Up to 16 rows (a batch of queries, a single token; see few_rows): bound by reading B, which
// goes from memory to the matrix instructions' registers without a stop in LDS
// (one row against 4096 x 4096 bfloat16 in the caches: 8.2 us, 4.1 TB/s; with the
// tiles above 10.3), and by the latency of a launch and one trip to memory where B
// is small (17,770 x 128 binary16: 4.1 us, the tiles 5.1; 512 x 512 binary32, 16
// rows: 4.9 and 9.1).
// A wavefront takes 16 columns; KW of a workgroup's 4 wavefronts share one such
// tile, each a part of the depth, their sums joined in order.  Any alignment.
// Rows and columns past the end repeat one that exists; their sums are not
// written.
template <typename T, int KW>
__global__ __launch_bounds__(256) void k_gemm_few(GemmArgs g, Epilogue e)
{
    constexpr int piece = 16 / (int)sizeof(T), step = 4 * piece, ahead = 8;
    __shared__ f32x4 parts[4][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int quad = lane >> 4, r16 = lane & 15;
    const int64_t tiles = (g.cols + 15) / 16;
    const int64_t steps = (g.depth + step - 1) / step, each = (steps + KW - 1) / KW;
    const int64_t s0 = (wave % KW) * each, s1 = s0 + each < steps ? s0 + each : steps;
    const T* arow = (const T*)g.A + (r16 < g.rows ? r16 : 0) * g.lda + quad * piece;
    for (int64_t t0 = (int64_t)blockIdx.x * (4 / KW); t0 < tiles; t0 += (int64_t)gridDim.x * (4 / KW)) {
        const int64_t n = (t0 + wave / KW) * 16;
        const T* brow = (const T*)g.B + (n + r16 < g.cols ? n + r16 : g.cols - 1) * g.ldb + quad * piece;
        f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
        if (n < g.cols) {
            int64_t s = s0;
            for (; s + ahead <= s1 && (s + ahead) * step <= g.depth; s += ahead) {
                u32x4 a[ahead], b[ahead];
#pragma unroll
                for (int u = 0; u < ahead; ++u) {
                    b[u] = piece_at<T>(brow + (s + u) * step, piece);
                    a[u] = piece_at<T>(arow + (s + u) * step, piece);
                }
#pragma unroll
                for (int u = 0; u < ahead; ++u)
                    mma<T>(acc, b[u], a[u]);
            }
            for (; s < s1; s += 2) {
                u32x4 a[2], b[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int64_t k = (s + u) * step, here = s + u < s1 ? g.depth - k - quad * piece : 0;
                    b[u] = piece_at<T>(brow + k, here);
                    a[u] = piece_at<T>(arow + k, here);
                }
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    mma<T>(acc, b[u], a[u]);
            }
        }
        if (KW > 1) {
            parts[wave][lane] = acc;
            __syncthreads();
            if (wave % KW == 0)
#pragma unroll
                for (int w = 1; w < KW; ++w)
                    acc += parts[wave + w][lane];
            __syncthreads();
        }
        if (wave % KW == 0) {
            float v[4] = {acc[0], acc[1], acc[2], acc[3]};
            if (r16 < g.rows)
                finish<T, 4>(e, r16, n + quad * 4, v);
        }
    }
}

// The column sums alone.
template <typename T>
__global__ __launch_bounds__(512) void k_dbias(Products p, uint32_t from)
{
    __shared__ float lds[8 * 64];
    add_columns<T, 8>(p, (int64_t)from + blockIdx.x, lds);
}

// ------------------------------------------------- operands of the gradient
//
// dX sums over the columns of dZ, dW over its rows, so W, dZ and X are also
// needed with their rows and columns exchanged.  One launch does that, 64 x 64
// elements a workgroup through LDS: reads and writes are whole cache lines.  dZ
// is computed on the way and its unrounded column sums per 64 rows kept for
// dbias.  Rows of the results are whole 16-byte pieces, zeros behind their end.
//
// dZ is rounded to its type for the products, because the matrix instructions
// take no other: in 16 bits dX and dW then have the rounding of each dZ beside
// their own, about sqrt 2 of its size together (gelu, 4096 x 2048 x 2048 bfloat16:
// 0.0023 of the result's norm against 0.0017 from an unrounded dZ).  A second
// product with what the rounding left over would remove it for twice the products'
// time.  Without an activation, with relu and in binary32 nothing is lost.
//
// Bound by memory: 4096 x 2048 with gelu, X 4096 x 2048 and W 2048 x 2048 in
// bfloat16, 117 MB read and written: 22 us, 5.3 TB/s.  (Reading the matrix
// instructions' operands out of LDS the other way round would save the exchanged
// copies, about half of that.)
struct Turn {
    const void* src; // rows x cols
    int64_t ld, rows, cols;
    void* turned; // cols x rows, ld_turned apart; may be nullptr
    int64_t ld_turned;
    int64_t tiles; // of 64 x 64
};

struct Turns {
    Turn job[3]; // dZ first (src: dY), then W and X
    const void* z;
    int64_t ldz;
    int act;
    void* dz; // rows x cols, ld_dz apart; may be nullptr
    int64_t ld_dz;
    float* sums; // [tile of rows][cols]; may be nullptr
    int64_t tiles;
};

constexpr int kTurnThreads = 512;

template <typename T>
__global__ __launch_bounds__(kTurnThreads) void k_turn(Turns a)
{
    constexpr int V = 16 / (int)sizeof(T), across = 64 / V, down = kTurnThreads / across, turns = 64 / down;
    __shared__ T tile[64][64 + 4 / sizeof(T) * 1];
    __shared__ float sums[down][64];
    const int tx = threadIdx.x % across, ty = threadIdx.x / across;
    for (int64_t id0 = blockIdx.x; id0 < a.tiles; id0 += gridDim.x) {
        int which = 0;
        uint32_t id = (uint32_t)id0;
        while (which < 2 && id >= a.job[which].tiles)
            id -= (uint32_t)a.job[which++].tiles;
        const Turn& j = a.job[which];
        const uint32_t wide = (uint32_t)((j.cols + 63) / 64);
        const int64_t tr = id / wide, r0 = tr * 64, c0 = (int64_t)(id - (uint32_t)tr * wide) * 64;
        const int64_t c = c0 + tx * V;
        float sum[V];
#pragma unroll
        for (int i = 0; i < V; ++i)
            sum[i] = 0.0f;
        u32x4 raw[turns], rz[turns];
#pragma unroll
        for (int u = 0; u < turns; ++u) {
            const int64_t r = r0 + ty + u * down, some = r < j.rows ? j.cols - c : 0;
            raw[u] = piece_at<T>((const T*)j.src + r * j.ld + c, some);
            if (which == 0 && a.act != kNone)
                rz[u] = piece_at<T>((const T*)a.z + r * a.ldz + c, some);
        }
#pragma unroll
        for (int u = 0; u < turns; ++u) {
            const int64_t r = r0 + ty + u * down, some = r < j.rows ? j.cols - c : 0;
            Vec<T, V> x;
            __builtin_memcpy(&x, &raw[u], 16);
            if (which == 0) {
                if (a.act != kNone) {
                    Vec<T, V> z;
                    __builtin_memcpy(&z, &rz[u], 16);
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const float d = i < some ? (float)x.v[i] * slope<sizeof(T) == 4>((float)z.v[i], a.act) : 0.0f;
                        sum[i] += d;
                        x.v[i] = T(d);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < V; ++i)
                        sum[i] += (float)x.v[i];
                }
                // behind a row's end too, as far as its last piece
                if (a.dz && some > 0)
                    store_vec<T, V>((T*)a.dz + r * a.ld_dz + c, x);
            }
#pragma unroll
            for (int i = 0; i < V; ++i)
                tile[ty + u * down][tx * V + i] = x.v[i];
        }
        if (which == 0 && a.sums) {
#pragma unroll
            for (int i = 0; i < V; ++i)
                sums[ty][tx * V + i] = sum[i];
        }
        __syncthreads();
        if (which == 0 && a.sums && threadIdx.x < 64 && c0 + threadIdx.x < j.cols) {
            float s = 0.0f;
#pragma unroll
            for (int y = 0; y < down; ++y)
                s += sums[y][threadIdx.x];
            a.sums[tr * j.cols + c0 + threadIdx.x] = s;
        }
        if (j.turned) {
#pragma unroll
            for (int u = 0; u < turns; ++u) {
                const int64_t row = c0 + ty + u * down, at = r0 + tx * V; // of the result
                if (row < j.cols && at < j.rows) {
                    Vec<T, V> x;
#pragma unroll
                    for (int i = 0; i < V; ++i)
                        x.v[i] = tile[tx * V + i][ty + u * down];
                    store_vec<T, V>((T*)j.turned + row * j.ld_turned + at, x);
                }
            }
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------- host
constexpr uint32_t kMostWgs = 1 << 22; // of a launch: a grid's threads are counted in 32 bits
constexpr int64_t kCus = 256; // of an MI355X

int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to; }

// Which tile a product takes, and over how many slices of its depth.
//
// A tile of 256 x 256 moves half the bytes per product of one of 128 x 128 and
// runs at 1.25 times its rate where there are enough of them (4096^3 bfloat16:
// 116 us against 141), but only one fits a CU, so the last round of a product
// with few tiles leaves more of the chip idle: 4096 x 2048 x 2048 (128 large
// tiles for 256 CUs: 55 us against 40) takes the small one.
//
// Small tiles run two to a CU with two stages each, which hides one's barriers
// and epilogue behind the other's products; where there is at most one per CU it
// gets the LDS of both as four stages (2048 x 2048 x 4096: 37 us against 48).
struct Shape {
    int tile;       // 0: k_gemm_few; else rows of a tile
    int slices;     // > 1: sums to the workspace, joined afterwards
    int steps;      // stages of a slice
    int64_t groups; // workgroups
};

// The tile for `n` products of one launch.
int tile_for(const int64_t* rows, const int64_t* cols, const int64_t* stages, int n, int dtype)
{
    int64_t big = 0, mid = 0, low = 0, least = stages[0], most = 0, work = 0;
    for (int i = 0; i < n; ++i) {
        big += up(rows[i], 256) * up(cols[i], 256);
        work += up(rows[i], 256) * up(cols[i], 256) * stages[i];
        most = std::max(most, stages[i]);
        mid += up(rows[i], 128) * up(cols[i], 128);
        low += up(rows[i], 64) * up(cols[i], 128);
        least = std::min(least, stages[i]);
    }
    // Large tiles have no slices, so of two products the deeper one's tiles must not be what the launch waits for:
    // up to 1.25 times the evenly spread stages, which is the rate they gain.  (M, N, K = 24576, 512, 512 bfloat16,
    // where dW is 4 such tiles of 384 stages: 443 us, 65 with tiles of 128 and slices; 6144, 2048, 2048: 146, 117.)
    const bool even = n == 1 || (double)most * (double)kCus <= 1.25 * (double)work;
    if (least >= 8 && even && (double)up(big, kCus) <= 0.625 * 0.5 * (double)up(mid, kCus))
        return 256;
    // Tiles of 64 rows where they fill the last round better: one takes 0.55 of the other's time in binary32, 0.7 in
    // 16 bits (bound by what comes from L2), measured on 1000 x 5000 x 776 (88 us against 112; 21.6 against 20).
    return mid <= 128 || (dtype == kF32 ? 0.55 : 0.7) * (double)up(low, kCus) < (double)up(mid, kCus) ? 64 : 128;
}

int64_t tiles_of(int64_t rows, int64_t cols, int tile) { return up(rows, tile) * up(cols, tile == 256 ? 256 : 128); }

// How `n` products of one launch are cut: one tile for all, and slices of one
// length, the length by an estimate of the time.  A stage of a tile takes a CU 0.34
// us, or 0.58 with 128 rows (four times that in binary32): a product takes as many
// slices as the fullest CU has, two unequal ones as long as the work spread evenly
// and half a slice for the uneven end.  Slices cost the launch that joins them, 4
// us, and their sums' way to memory and back, which has to stay in the caches.
//
// 64 x 4096 x 1024 bfloat16: 8.8 us as one, 10.9 as two; 128 x 512 x 4096: 21.6 as
// one, 11.3 as eight; 333 x 500 x 1001 binary32: 43 and 16; the gradient for M, N, K
// = 16384, 512, 512 bfloat16, whose dW is 16 tiles of 256 stages beside 512 of 8: 172
// whole, 57 sliced; 20000, 256, 128 binary32: 114 and 63.
void shapes_of(const int64_t* rows, const int64_t* cols, const int64_t* depth, int n, int dtype, Shape* s)
{
    const int64_t least = dtype == kF32 ? 2 : 8; // stages
    int64_t stages[2], most = 1;
    double work = 0.0;
    for (int i = 0; i < n; ++i) {
        stages[i] = std::max<int64_t>(up(depth[i] * (int64_t)elem_bytes(dtype), kRow), 1);
        most = std::max(most, stages[i]);
    }
    const int tile = tile_for(rows, cols, stages, n, dtype);
    for (int i = 0; i < n; ++i)
        work += (double)tiles_of(rows[i], cols[i], tile) * (double)stages[i];
    int64_t steps = most;
    if (tile != 256) {
        const double stage_us = (tile == 64 ? 0.34 : 0.58) * (dtype == kF32 ? 4.0 : 1.0);
        double best = 0.0;
        // 1, 2, 3, 4, 6, 8, 12, ... slices of the deepest product
        for (int64_t slices = 1, more = 1; slices <= kCus; slices += more, more = slices & (slices - 1) ? more : slices / 2) {
            const int64_t len = up(most, slices);
            if (slices > 1 && len < least)
                break;
            double wgs = 0.0, sums = 0.0;
            for (int i = 0; i < n; ++i) {
                const double here = (double)up(stages[i], len);
                wgs += (double)tiles_of(rows[i], cols[i], tile) * here;
                sums += here > 1.0 ? here * (double)rows[i] * (double)cols[i] : 0.0;
            }
            if (slices > 1 && sums * 4.0 > (double)kInfinityCache)
                break;
            const double rounds = std::ceil(wgs / (double)kCus);
            const double span = n == 1 || rounds <= 1.0
                                    ? rounds * (double)len
                                    : std::max((double)len, work / (double)kCus + 0.5 * (double)len);
            const double us = span * stage_us + (sums > 0.0 ? 4.0 + sums * 8.0 / 4e6 : 0.0);
            if (slices == 1 || us < best) {
                best = us;
                steps = len;
            }
        }
    }
    int64_t groups = 0;
    for (int i = 0; i < n; ++i) {
        s[i].tile = tile;
        s[i].slices = (int)up(stages[i], steps);
        s[i].steps = (int)std::min(steps, stages[i]);
        groups += tiles_of(rows[i], cols[i], tile) * s[i].slices;
    }
    for (int i = 0; i < n; ++i)
        s[i].groups = groups;
}

// Up to 16 rows have a kernel of their own (k_gemm_few), which reads B once but
// splits no depth over workgroups: 16 columns each, so that up to 2048 columns
// leave half the chip idle while a wavefront goes down a quarter of the depth.  Of
// such a product at least 8192 deep the tiles take slices.  16 rows, columns x
// depth, bfloat16: 512 x 4096 4.6 us there, 8.7 in tiles (8192 deep: 16.6 and 9.5;
// 32,768: 58 and 15); 2048 x 8192: 17.2 and 11.4; 4096 x 8192: 17.9 and 17.4.  One
// row, binary32: 1024 x 4096 11.4 and 12.5; 2048 x 8192 28.9 and 25.2; 3000 x 8192
// 29.8 and 36.5.  dW of one output over a batch of 10^6 is of this form.
bool few_rows(int64_t rows, int64_t cols, int64_t depth) { return rows <= 16 && (depth < 8192 || cols > 2048); }

Shape shape_of(int64_t rows, int64_t cols, int64_t depth, int dtype)
{
    Shape s{0, 1, 1, 0};
    if (rows > 0 && cols > 0 && !few_rows(rows, cols, depth))
        shapes_of(&rows, &cols, &depth, 1, dtype, &s);
    return s;
}

size_t sums_bytes(const Shape& s, int64_t rows, int64_t cols)
{
    return s.slices > 1 ? round256(sizeof(float) * (size_t)s.slices * (size_t)rows * (size_t)cols) : 0;
}

size_t part_bytes(int64_t rows, int64_t cols, int64_t depth, int dtype)
{
    return sums_bytes(shape_of(rows, cols, depth, dtype), rows, cols);
}

// 256 rows are addressed by 31 bits from the first.
bool near(int64_t ld, int dtype) { return ld * (int64_t)elem_bytes(dtype) * 257 < (int64_t(1) << 31); }

bool rows_aligned(const void* p, int64_t ld, int dtype)
{
    return ((uintptr_t)p & 15) == 0 && ld * (int64_t)elem_bytes(dtype) % 16 == 0;
}

// Launches the products of p (the second one if its rows are set), and `sums`
// workgroups for the column sums.
template <typename T, int BM, int BN, int WM, int WN, bool DIRECT, int NB>
hipError_t gemm_launch(Products p, const Shape* s, int n, uint32_t sums, hipStream_t st)
{
    uint32_t ids[2] = {0, 0};
    for (int i = 0; i < n; ++i) {
        p.g[i].tiles_m = (uint32_t)up(p.g[i].rows, BM);
        p.g[i].tiles_n = (uint32_t)up(p.g[i].cols, BN);
        p.g[i].all = p.g[i].tiles_m * p.g[i].tiles_n * (uint32_t)s[i].slices;
        ids[i] = (uint32_t)up(p.g[i].all, 8) * 8;
    }
    p.second = n > 1 ? ids[0] : kNoWork;
    p.sums = sums ? ids[0] + ids[1] : kNoWork;
    const uint32_t all = ids[0] + ids[1] + sums;
    // (a part of a long launch begins with a whole turn of the XCDs; two products together are never that long)
    for (p.g[0].tile0 = 0; p.g[0].tile0 < all; p.g[0].tile0 += kMostWgs)
        hipLaunchKernelGGL((k_gemm<T, BM, BN, WM, WN, DIRECT, NB>), dim3(std::min(kMostWgs, all - p.g[0].tile0)),
                           dim3((BM / WM) * (BN / WN) * 64), 0, st, p);
    return hipGetLastError();
}

template <typename T>
hipError_t gemm_tiled(const Products& p, const Shape* s, int n, bool direct, uint32_t sums, hipStream_t st)
{
    if (s->tile == 256 && direct)
        return gemm_launch<T, 256, 256, 128, 64, true, 2>(p, s, n, sums, st);
    if (s->tile >= 128 && direct && s->groups <= kCus)
        return gemm_launch<T, 128, 128, 32, 64, true, 4>(p, s, n, sums, st);
    if (s->tile >= 128 && direct)
        return gemm_launch<T, 128, 128, 32, 64, true, 2>(p, s, n, sums, st);
    if (s->tile >= 128)
        return gemm_launch<T, 128, 128, 32, 64, false, 2>(p, s, n, sums, st);
    if (direct)
        return gemm_launch<T, 64, 128, 16, 64, true, 3>(p, s, n, sums, st);
    return gemm_launch<T, 64, 128, 16, 64, false, 2>(p, s, n, sums, st);
}

// The slices of those products that have several, joined.
template <typename T>
hipError_t join(const Products& p, const Shape* s, int n, hipStream_t st)
{
    Join j{};
    uint32_t wgs[2] = {0, 0};
    int m = 0;
    for (int i = 0; i < n; ++i)
        if (s[i].slices > 1) {
            j.part[m] = p.g[i].part;
            j.slices[m] = s[i].slices;
            j.rows[m] = p.g[i].rows;
            j.cols[m] = p.g[i].cols;
            j.e[m] = p.e[i];
            wgs[m] = (uint32_t)std::min<int64_t>(up(p.g[i].rows * up(p.g[i].cols, 4), 256), kMostWgs / 2);
            ++m;
        }
    if (!m)
        return hipSuccess;
    j.second = m > 1 ? wgs[0] : kNoWork;
    const bool many = std::max(j.slices[0], j.slices[1]) > 4; // slices in flight at a time
    hipLaunchKernelGGL((many ? k_gemm_join<T, 16> : k_gemm_join<T, 4>), dim3(wgs[0] + wgs[1]), dim3(256), 0, st, j);
    return hipGetLastError();
}

bool can_direct(const GemmArgs& g, int dtype)
{
    return rows_aligned(g.A, g.lda, dtype) && rows_aligned(g.B, g.ldb, dtype) &&
           g.depth * (int64_t)elem_bytes(dtype) % 16 == 0 && near(std::max(g.lda, g.ldb), dtype);
}

// C = A B^T with its epilogue; `part` holds part_bytes.
template <typename T>
hipError_t gemm(GemmArgs g, const Epilogue& e, int dtype, void* part, hipStream_t st)
{
    if (g.rows == 0 || g.cols == 0)
        return hipSuccess;
    const Shape s = shape_of(g.rows, g.cols, g.depth, dtype);
    g.steps = s.steps;
    g.part = s.slices > 1 ? (float*)part : nullptr;
    if (s.tile == 0) {
        // long rows: all four wavefronts on one tile (17,770 columns of 128 binary16: 4.1 us apart, 4.6 together; of
        // 256: 5.1 and 4.6; 4096 of 4096: 21.5 and 8.2)
        const bool shared = g.depth * (int64_t)sizeof(T) >= 512;
        const int64_t wgs = std::min<int64_t>(up(g.cols, shared ? 16 : 64), kMostWgs);
        if (shared)
            hipLaunchKernelGGL((k_gemm_few<T, 4>), dim3((unsigned)wgs), dim3(256), 0, st, g, e);
        else
            hipLaunchKernelGGL((k_gemm_few<T, 1>), dim3((unsigned)wgs), dim3(256), 0, st, g, e);
        return hipGetLastError();
    }
    Products p{};
    p.g[0] = g;
    p.e[0] = e;
    const hipError_t err = gemm_tiled<T>(p, &s, 1, can_direct(g, dtype), 0, st);
    return err == hipSuccess ? join<T>(p, &s, 1, st) : err;
}

template <typename T>
hipError_t linear_typed(const LinearLaunch& a, hipStream_t st)
{
    GemmArgs g{a.x, a.w, a.ldx, a.ldw, a.M, a.N, a.K, 0, 0, 0, 0, 0, nullptr};
    // the pitch of a matrix that is left out was not checked and counts for nothing
    const Epilogue e{a.bias, a.residual, a.y, a.z, a.ldr, a.ldy, a.ldz, a.M, a.N, a.act,
                     near(a.ldy, a.dtype) && (!a.residual || near(a.ldr, a.dtype)) && (!a.z || near(a.ldz, a.dtype))};
    return gemm<T>(g, e, a.dtype, a.work, st);
}

struct GradWork {
    void *dz, *dz_t, *x_t, *w_t, *sums, *part;
    int64_t Mp, Np; // rows of whole pieces
    size_t bytes;
};

// Whether dX and dW can share a launch (those of few rows mostly have a kernel of their own).
bool together(int64_t M, int64_t N, int64_t K) { return M > 16 && N > 16 && K > 0; }

void grad_shapes(int64_t M, int64_t N, int64_t K, int dtype, Shape* s)
{
    const int64_t rows[2] = {M, N}, cols[2] = {K, K}, depth[2] = {N, M};
    shapes_of(rows, cols, depth, 2, dtype, s);
}

GradWork grad_work(int64_t M, int64_t N, int64_t K, int dtype, void* base)
{
    GradWork w;
    size_t at = 0;
    const size_t es = elem_bytes(dtype);
    auto take = [&](size_t bytes) { // (an address is of use only where the sum is: the caller refuses others)
        char* p = (char*)base + at;
        at = bytes > kMostBytes ? SIZE_MAX : plus(at, round256(bytes));
        return (void*)p;
    };
    const int64_t piece = 16 / (int64_t)es;
    w.Mp = up(M, piece) * piece;
    w.Np = up(N, piece) * piece;
    w.dz = take(times(es * (size_t)M, (size_t)w.Np));
    w.dz_t = take(times(es * (size_t)N, (size_t)w.Mp));
    w.x_t = take(times(es * (size_t)K, (size_t)w.Mp));
    w.w_t = take(times(es * (size_t)K, (size_t)w.Np));
    w.sums = take(times(sizeof(float) * (size_t)up(M, 64), (size_t)N));
    size_t part = std::max(part_bytes(M, K, N, dtype), part_bytes(N, K, M, dtype));
    if (together(M, N, K)) {
        Shape s[2];
        grad_shapes(M, N, K, dtype, s);
        part = std::max(part, sums_bytes(s[0], M, K) + sums_bytes(s[1], N, K));
    }
    w.part = take(part);
    w.bytes = at;
    return w;
}

template <typename T>
hipError_t grad_typed(const LinearGradLaunch& a, hipStream_t st)
{
    const GradWork w = grad_work(a.M, a.N, a.K, a.dtype, a.work);
    const int64_t piece = 16 / (int64_t)sizeof(T);
    // dY itself serves as dZ where nothing is to be computed and its rows are whole pieces
    const bool as_is = a.act == kNone && rows_aligned(a.dy, a.lddy, a.dtype) && a.N % piece == 0;
    Turns t{};
    t.job[0] = Turn{a.dy, a.lddy, a.M, a.N, a.dw ? w.dz_t : nullptr, w.Mp, up(a.M, 64) * up(a.N, 64)};
    t.job[1] = Turn{a.w, a.ldw, a.N, a.K, w.w_t, w.Np, a.dx ? up(a.N, 64) * up(a.K, 64) : 0};
    t.job[2] = Turn{a.x, a.ldx, a.M, a.K, w.x_t, w.Mp, a.dw ? up(a.M, 64) * up(a.K, 64) : 0};
    t.z = a.z;
    t.ldz = a.ldz;
    t.act = a.act;
    t.dz = a.dx && !as_is ? w.dz : nullptr;
    t.ld_dz = w.Np;
    t.sums = a.dbias ? (float*)w.sums : nullptr;
    if (!t.job[0].turned && !t.dz && !t.sums)
        t.job[0].tiles = 0;
    t.tiles = t.job[0].tiles + t.job[1].tiles + t.job[2].tiles; // (64 x 64 elements each: below 2^32 in any memory)
    if (t.tiles)
        hipLaunchKernelGGL((k_turn<T>), dim3((unsigned)std::min<int64_t>(t.tiles, kMostWgs)),
                           dim3(kTurnThreads), 0, st, t);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess)
        return err;
    // (where dZ lies in the workspace the zeros behind a row are part of it: whole pieces)
    Products p{};
    p.g[0] = GemmArgs{as_is ? a.dy : w.dz, w.w_t, as_is ? a.lddy : w.Np, w.Np, a.M, a.K, as_is ? a.N : w.Np, 0, 0, 0, 0, 0,
                      nullptr};
    p.e[0] = Epilogue{nullptr, nullptr, a.dx, nullptr, 0, a.lddx, 0, a.M, a.K, kNone, near(a.lddx, a.dtype)};
    p.g[1] = GemmArgs{w.dz_t, w.x_t, w.Mp, w.Mp, a.N, a.K, w.Mp, 0, 0, 0, 0, 0, nullptr};
    p.e[1] = Epilogue{nullptr, nullptr, a.dw, nullptr, 0, a.lddw, 0, a.N, a.K, kNone, near(a.lddw, a.dtype)};
    p.col_sums = (const float*)w.sums;
    p.row_tiles = up(a.M, 64);
    p.cols = a.N;
    p.dbias = a.dbias;
    const uint32_t sums = a.dbias ? (uint32_t)up(a.N, 64) : 0;
    Shape s[2];
    const bool both = a.dx && a.dw && together(a.M, a.N, a.K) && can_direct(p.g[0], a.dtype) && can_direct(p.g[1], a.dtype);
    if (both)
        grad_shapes(a.M, a.N, a.K, a.dtype, s);
    if (both && s->groups + sums < kMostWgs / 2) {
        // both products and the column sums in one launch: the one fills what the other leaves idle, the deeper one
        // first (its tiles take longer; the shorter ones then even out the end)
        if (s[0].slices == 1 && s[1].slices == 1 && a.M > a.N) {
            std::swap(p.g[0], p.g[1]);
            std::swap(p.e[0], p.e[1]);
            std::swap(s[0], s[1]);
        }
        size_t at = 0;
        for (int i = 0; i < 2; ++i) {
            p.g[i].steps = s[i].steps;
            p.g[i].part = s[i].slices > 1 ? (float*)((char*)w.part + at) : nullptr;
            at += sums_bytes(s[i], p.g[i].rows, p.g[i].cols);
        }
        err = gemm_tiled<T>(p, s, 2, true, sums, st);
        return err == hipSuccess ? join<T>(p, s, 2, st) : err;
    }
    if (a.dx)
        err = gemm<T>(p.g[0], p.e[0], a.dtype, w.part, st);
    if (a.dw && err == hipSuccess)
        err = gemm<T>(p.g[1], p.e[1], a.dtype, w.part, st);
    for (uint32_t from = 0; from < sums && err == hipSuccess; from += kMostWgs) {
        hipLaunchKernelGGL((k_dbias<T>), dim3(std::min(kMostWgs, sums - from)), dim3(512), 0, st, p, from);
        err = hipGetLastError();
    }
    return err;
}

} // namespace

size_t linear_bytes(int64_t M, int64_t N, int64_t K, int dtype) { return part_bytes(M, N, K, dtype); }

hipError_t linear(const LinearLaunch& a, hipStream_t st)
{
    if (a.dtype == kF16)
        return linear_typed<_Float16>(a, st);
    if (a.dtype == kBF16)
        return linear_typed<__bf16>(a, st);
    return linear_typed<float>(a, st);
}

size_t linear_grad_bytes(int64_t M, int64_t N, int64_t K, int dtype)
{
    return grad_work(M, N, K, dtype, nullptr).bytes;
}

hipError_t linear_grad(const LinearGradLaunch& a, hipStream_t st)
{
    if (a.dtype == kF16)
        return grad_typed<_Float16>(a, st);
    if (a.dtype == kBF16)
        return grad_typed<__bf16>(a, st);
    return grad_typed<float>(a, st);
}

} // namespace ops
} // namespace mfsgd
