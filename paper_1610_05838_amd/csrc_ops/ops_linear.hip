// ops_linear.hip -- products with bias, activation and residual, and their
// gradient:
//   Z = X W^T + b,  Y = act(Z) + R
//   dZ = dY o act'(Z),  dX = dZ W,  dW = dZ^T X,  db = column sums of dZ
//
// Every product is one form, C = A B^T with A (rows x depth) and B (cols x
// depth) both contiguous along the depth that is summed over.
#include <algorithm>

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
// In binary32.  16-bit results take the hardware's exponential and reciprocal
// (1 ulp) and for erf the rational approximation 7.1.26 of Abramowitz and
// Stegun (1.5e-7), well below their own rounding; binary32 results the library
// functions.
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
        return 0.5f * (1.0f + erff(x));
    const float a = fabsf(x), t = __builtin_amdgcn_rcpf(1.0f + 0.3275911f * a);
    float p = 1.061405429f;
    p = p * t - 1.453152027f;
    p = p * t + 1.421413741f;
    p = p * t - 0.284496736f;
    p = p * t + 0.254829592f;
    const float tail = 0.5f * p * t * __expf(-x * x); // (1 - erf |x|) / 2
    return z < 0.0f ? tail : 1.0f - tail;
}

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
            v[c] = v[c] * sigmoid<EXACT>(v[c]);
        break;
    case kGelu:
#pragma unroll
        for (int c = 0; c < C; ++c)
            v[c] = v[c] * normal_cdf<EXACT>(v[c]);
        break;
    }
}

template <bool EXACT>
__device__ __forceinline__ float slope(float z, int act)
{
    switch (act) {
    case kRelu:
        return z > 0.0f ? 1.0f : 0.0f;
    case kSigmoid: {
        const float s = sigmoid<EXACT>(z);
        return s * (1.0f - s);
    }
    case kSilu: {
        const float s = sigmoid<EXACT>(z);
        return s * (1.0f + z * (1.0f - s));
    }
    case kGelu: {
        const float e = EXACT ? expf(-0.5f * z * z) : __expf(-0.5f * z * z);
        return normal_cdf<EXACT>(z) + z * e * 0.39894228040143268f;
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
// kRow = 128 bytes of depth at a time, two stages, copied by the memory
// pipeline itself while the other stage is computed on: one barrier a stage.
//
// The 16-byte pieces of a staged row are stored in the order piece ^ (row & 7),
// so that the 16 lanes that read one piece of 16 rows meet different banks; the
// copy writes LDS linearly, so the lanes' global addresses carry that order.
//
// B is the matrix instruction's row operand: a lane then holds 4 consecutive
// columns of C per tile.  B's rows are staged so that the four tiles of 64
// columns give a lane 16 consecutive ones, and a row of C is written in whole
// cache lines.
constexpr int kRow = 128; // bytes of depth of a stage

__device__ __attribute__((aligned(16))) const uint32_t g_zeros[4] = {0, 0, 0, 0};

struct GemmArgs {
    const void *A, *B;
    int64_t lda, ldb, rows, cols, depth;
    uint32_t tiles_m, tiles_n, tile0; // of the whole product; this launch's first
    int steps;                        // stages of one workgroup: a slice of the depth, blockIdx.y
    float* part;                      // the slices' sums [slice][rows][cols], or nullptr: one slice, finished here
};

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

// Workgroups are dealt to the 8 XCDs in turn: each XCD takes a run of
// consecutive tiles, and runs go down 8 tiles of rows before the next column, so
// that the tiles of an XCD share rows of A and B in its L2.
__device__ __forceinline__ void tile_place(const GemmArgs& g, uint32_t& tm, uint32_t& tn)
{
    const uint32_t all = g.tiles_m * g.tiles_n, id = blockIdx.x + g.tile0, x = id & 7;
    const uint32_t t = x * (all >> 3) + (x < (all & 7) ? x : all & 7) + (id >> 3);
    const uint32_t band = 8 * g.tiles_n, b = t / band, at = t - b * band;
    const uint32_t high = g.tiles_m - b * 8 < 8 ? g.tiles_m - b * 8 : 8;
    tn = at / high;
    tm = b * 8 + (at - tn * high);
}

// DIRECT: rows of A and B start at 16-byte boundaries and the depth is whole
// pieces; the copies go from memory to LDS by themselves.  Otherwise (any
// alignment, any depth) they pass through registers.
template <typename T, int BM, int BN, int WM, int WN, bool DIRECT>
__global__ __launch_bounds__((BM / WM) * (BN / WN) * 64) void k_gemm(GemmArgs g, Epilogue e)
{
    constexpr int waves = (BM / WM) * (BN / WN), groups = (BM + BN) / 8 / waves;
    constexpr int TM = WM / 16, TN = WN / 16, piece = 16 / (int)sizeof(T), per_stage = kRow / (int)sizeof(T);
    constexpr int stage_bytes = (BM + BN) * kRow;
    static_assert(WN % 64 == 0 && (BM + BN) % (8 * waves) == 0, "tile shape");
    __shared__ __attribute__((aligned(128))) char lds[2 * stage_bytes];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / (BN / WN) * WM, wn = wave % (BN / WN) * WN;
    uint32_t tm, tn;
    tile_place(g, tm, tn);
    const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
    const int64_t k0 = (int64_t)blockIdx.y * g.steps * per_stage, depth = g.depth - k0;
    const int64_t left = (depth + per_stage - 1) / per_stage;
    const int steps = (int)(left < g.steps ? left : g.steps);

    // this lane's rows to copy: 8 rows a group, a 16-byte piece of one each; rows past the end repeat the last one
    // (their sums are not written)
    const int pc = (lane & 7) ^ (lane >> 3);
    uint64_t src[groups];
#pragma unroll
    for (int u = 0; u < groups; ++u) {
        const int group = wave * groups + u, row = group * 8 + (lane >> 3);
        if (group < BM / 8) {
            const int64_t m = m0 + row < g.rows ? m0 + row : g.rows - 1;
            src[u] = (uint64_t)((const T*)g.A + m * g.lda + k0 + pc * piece);
        } else {
            const int r = row - BM, n = (r & ~63) + (r >> 2 & 3) * 16 + (r >> 4 & 3) * 4 + (r & 3);
            const int64_t col = n0 + n < g.cols ? n0 + n : g.cols - 1;
            src[u] = (uint64_t)((const T*)g.B + col * g.ldb + k0 + pc * piece);
        }
    }
    // stages before `whole` lie inside the depth; in the last one pieces past it are zeros
    const int whole = (int)(depth / per_stage);
    const int64_t room = depth - (int64_t)whole * per_stage - pc * piece; // this lane's elements in that stage
    uint64_t zeros = (uint64_t)g_zeros;
    asm("" : "+v"(zeros)); // in registers: the copies' addresses are selected, not branched on
    u32x4 held[DIRECT ? 1 : groups];
    auto fetch = [&](int s) {
        if constexpr (DIRECT) {
            char* to = lds + (s & 1) * stage_bytes + wave * groups * 8 * kRow;
            const bool none = s >= whole && room <= 0;
#pragma unroll
            for (int u = 0; u < groups; ++u) {
                const uint64_t from = none ? zeros : src[u];
                src[u] += kRow;
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                                 (__attribute__((address_space(3))) void*)(to + u * 8 * kRow), 16, 0,
                                                 0);
            }
        } else if (s < whole) {
#pragma unroll
            for (int u = 0; u < groups; ++u) {
                held[u] = piece_at<T>((const T*)src[u], piece);
                src[u] += kRow;
            }
        } else {
#pragma unroll
            for (int u = 0; u < groups; ++u)
                held[u] = piece_at<T>((const T*)src[u], room);
        }
    };
    auto keep = [&](int s) {
        char* to = lds + (s & 1) * stage_bytes + wave * groups * 8 * kRow + lane * 16;
#pragma unroll
        for (int u = 0; u < groups; ++u)
            *(u32x4*)(to + u * 8 * kRow) = held[DIRECT ? 0 : u];
    };

    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
            acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    const int quad = lane >> 4, r16 = lane & 15;
    if (steps > 0) {
        fetch(0);
        if constexpr (!DIRECT)
            keep(0);
    }
    for (int s = 0; s < steps; ++s) {
        // everyone's copies of stage s are in LDS, and everyone is done reading stage s - 1
        if constexpr (DIRECT) {
            __builtin_amdgcn_s_waitcnt(0x0f70); // vmcnt(0)
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
        } else {
            __syncthreads();
        }
        if (s + 1 < steps)
            fetch(s + 1);
        const char* at = lds + (s & 1) * stage_bytes;
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            const int sw = ((kk * 4 + quad) ^ (r16 & 7)) * 16;
            u32x4 a[TM], b[TN];
#pragma unroll
            for (int j = 0; j < TN; ++j)
                b[j] = *(const u32x4*)(at + (BM + wn + j * 16 + r16) * kRow + sw);
#pragma unroll
            for (int i = 0; i < TM; ++i)
                a[i] = *(const u32x4*)(at + (wm + i * 16 + r16) * kRow + sw);
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
                    mma<T>(acc[i][j], b[j], a[i]);
        }
        if constexpr (!DIRECT)
            if (s + 1 < steps)
                keep(s + 1);
    }

#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int64_t m = m0 + wm + i * 16 + r16;
#pragma unroll
        for (int q = 0; q < TN / 4; ++q) {
            const int64_t n = n0 + wn + q * 64 + quad * 16;
            float v[16];
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    v[j * 4 + c] = acc[i][q * 4 + j][c];
            if (!g.part)
                finish<T, 16>(e, m, n, v);
            else if (m < g.rows && n < g.cols)
                write_some<float, 16>(g.part + ((int64_t)blockIdx.y * g.rows + m) * g.cols + n,
                                      g.cols - n < 16 ? (int)(g.cols - n) : 16, v);
        }
    }
}

// The slices' sums, added in order and finished: 4 columns a thread.
template <typename T>
__global__ __launch_bounds__(256) void k_gemm_join(const float* __restrict__ part, int slices, int64_t rows,
                                                   int64_t cols, Epilogue e)
{
    const int64_t per_row = (cols + 3) / 4, all = rows * per_row, size = rows * cols;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const int64_t m = i / per_row, n = (i - m * per_row) * 4;
        const int some = cols - n < 4 ? (int)(cols - n) : 4;
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int s0 = 0; s0 < slices; s0 += 4) {
            float x[4][4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                read_some<float, 4>(part + (s0 + u < slices ? s0 + u : s0) * size + m * cols + n, some, x[u]);
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (s0 + u < slices) {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        sum[c] += x[u][c];
                }
        }
        finish<T, 4>(e, m, n, sum);
    }
}

// Up to 16 rows (a batch of queries, a single token): bound by reading B, which
// goes from memory to the matrix instructions' registers without a stop in LDS.
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

// ------------------------------------------------- operands of the gradient
//
// dX sums over the columns of dZ, dW over its rows, so W, dZ and X are also
// needed with their rows and columns exchanged.  One launch does that, 64 x 64
// elements a workgroup through LDS: reads and writes are whole cache lines.  dZ
// is computed on the way, rounded to its type, and its unrounded column sums
// per 64 rows kept for dbias.  Rows of the results are whole 16-byte pieces,
// zeros behind their end.
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

template <typename T>
__global__ __launch_bounds__(256) void k_turn(Turns a)
{
    constexpr int V = 16 / (int)sizeof(T), across = 64 / V, down = 256 / across, turns = 64 / down;
    __shared__ T tile[64][64 + 4 / sizeof(T) * 1];
    __shared__ float sums[down][64];
    const int tx = threadIdx.x % across, ty = threadIdx.x / across;
    for (int64_t id0 = blockIdx.x; id0 < a.tiles; id0 += gridDim.x) {
        int which = 0;
        int64_t id = id0;
        while (which < 2 && id >= a.job[which].tiles)
            id -= a.job[which++].tiles;
        const Turn& j = a.job[which];
        const int64_t wide = (j.cols + 63) / 64, tr = id / wide, r0 = tr * 64, c0 = (id - tr * wide) * 64;
        const int64_t c = c0 + tx * V;
        float sum[V];
#pragma unroll
        for (int i = 0; i < V; ++i)
            sum[i] = 0.0f;
#pragma unroll
        for (int u = 0; u < turns; ++u) {
            const int64_t r = r0 + ty + u * down;
            const int64_t some = r < j.rows ? j.cols - c : 0;
            const u32x4 raw = piece_at<T>((const T*)j.src + r * j.ld + c, some);
            Vec<T, V> x;
            __builtin_memcpy(&x, &raw, 16);
            if (which == 0) {
                if (a.act != kNone) {
                    const u32x4 rz = piece_at<T>((const T*)a.z + r * a.ldz + c, some);
                    Vec<T, V> z;
                    __builtin_memcpy(&z, &rz, 16);
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

// dbias from the column sums per 64 rows: 64 columns a workgroup, four parts of
// the tiles joined in order.
template <typename T>
__global__ __launch_bounds__(256) void k_dbias(const float* __restrict__ sums, int64_t tiles, int64_t cols,
                                               T* __restrict__ dbias)
{
    __shared__ float part[4][64];
    const int x = threadIdx.x & 63, y = threadIdx.x >> 6;
    const int64_t c = (int64_t)blockIdx.x * 64 + x, each = (tiles + 3) / 4;
    const int64_t from = y * each, to = from + each < tiles ? from + each : tiles;
    float sum = 0.0f;
    if (c < cols)
        for (int64_t t0 = from; t0 < to; t0 += 8) {
            float v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u)
                v[u] = t0 + u < to ? sums[(t0 + u) * cols + c] : 0.0f;
#pragma unroll
            for (int u = 0; u < 8; ++u)
                sum += v[u];
        }
    part[y][x] = sum;
    __syncthreads();
    if (y == 0 && c < cols)
        dbias[c] = T(((part[0][x] + part[1][x]) + part[2][x]) + part[3][x]);
}

// ------------------------------------------------------------------- host
constexpr uint32_t kMostWgs = 1 << 22;

int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to; }

// Which tile a product takes, and over how many slices of its depth.
struct Shape {
    int tile;   // 0: few rows; else rows of a tile
    int slices; // > 1: sums to the workspace, joined afterwards
    int steps;  // stages of a slice
};

Shape shape_of(int64_t rows, int64_t cols, int64_t depth, int dtype)
{
    const int64_t stages = up(depth * (int64_t)elem_bytes(dtype), kRow);
    Shape s{0, 1, (int)std::max<int64_t>(stages, 1)};
    if (rows <= 16 || cols == 0)
        return s;
    const int64_t big = up(rows, 256) * up(cols, 256), mid = up(rows, 128) * up(cols, 128);
    s.tile = big >= 200 && stages >= 8 ? 256 : rows > 64 ? 128 : 64;
    const int64_t tiles = s.tile == 256 ? big : s.tile == 128 ? mid : up(rows, 64) * up(cols, 128);
    // enough workgroups for every CU, each with at least 4 stages
    if (tiles < 256 && s.tile != 256) {
        const int64_t want = std::min<int64_t>(512 / tiles, stages / 4);
        if (want > 1) {
            s.steps = (int)up(stages, want);
            s.slices = (int)up(stages, s.steps);
        }
    }
    return s;
}

size_t part_bytes(int64_t rows, int64_t cols, int64_t depth, int dtype)
{
    const Shape s = shape_of(rows, cols, depth, dtype);
    return s.slices > 1 ? round256(sizeof(float) * (size_t)s.slices * (size_t)rows * (size_t)cols) : 0;
}

bool rows_aligned(const void* p, int64_t ld, int dtype)
{
    return ((uintptr_t)p & 15) == 0 && ld * (int64_t)elem_bytes(dtype) % 16 == 0;
}

template <typename T, int BM, int BN, int WM, int WN, bool DIRECT>
hipError_t gemm_launch(GemmArgs g, const Epilogue& e, int slices, hipStream_t st)
{
    g.tiles_m = (uint32_t)up(g.rows, BM);
    g.tiles_n = (uint32_t)up(g.cols, BN);
    const uint32_t all = g.tiles_m * g.tiles_n;
    for (g.tile0 = 0; g.tile0 < all; g.tile0 += kMostWgs) // a multiple of 8: the XCDs' turn goes on
        hipLaunchKernelGGL((k_gemm<T, BM, BN, WM, WN, DIRECT>), dim3(std::min(kMostWgs, all - g.tile0), slices),
                           dim3((BM / WM) * (BN / WN) * 64), 0, st, g, e);
    return hipGetLastError();
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
        // long rows: all four wavefronts on one tile
        const bool shared = g.depth * (int64_t)sizeof(T) >= 1024;
        const int64_t wgs = std::min<int64_t>(up(g.cols, shared ? 16 : 64), kMostWgs);
        if (shared)
            hipLaunchKernelGGL((k_gemm_few<T, 4>), dim3((unsigned)wgs), dim3(256), 0, st, g, e);
        else
            hipLaunchKernelGGL((k_gemm_few<T, 1>), dim3((unsigned)wgs), dim3(256), 0, st, g, e);
        return hipGetLastError();
    }
    const bool direct = rows_aligned(g.A, g.lda, dtype) && rows_aligned(g.B, g.ldb, dtype) &&
                        g.depth * (int64_t)sizeof(T) % 16 == 0;
    hipError_t err;
    if (s.tile == 256)
        err = direct ? gemm_launch<T, 256, 256, 128, 64, true>(g, e, 1, st)
                     : gemm_launch<T, 128, 128, 64, 64, false>(g, e, 1, st);
    else if (s.tile == 128)
        err = direct ? gemm_launch<T, 128, 128, 64, 64, true>(g, e, s.slices, st)
                     : gemm_launch<T, 128, 128, 64, 64, false>(g, e, s.slices, st);
    else
        err = direct ? gemm_launch<T, 64, 128, 32, 64, true>(g, e, s.slices, st)
                     : gemm_launch<T, 64, 128, 32, 64, false>(g, e, s.slices, st);
    if (err != hipSuccess || s.slices == 1)
        return err;
    const int64_t wgs = std::min<int64_t>(up(g.rows * up(g.cols, 4), 256), kMostWgs);
    hipLaunchKernelGGL((k_gemm_join<T>), dim3((unsigned)wgs), dim3(256), 0, st, (const float*)part, s.slices, g.rows,
                       g.cols, e);
    return hipGetLastError();
}

template <typename T>
hipError_t linear_typed(const LinearLaunch& a, hipStream_t st)
{
    GemmArgs g{a.x, a.w, a.ldx, a.ldw, a.M, a.N, a.K, 0, 0, 0, 0, nullptr};
    const Epilogue e{a.bias, a.residual, a.y, a.z, a.ldr, a.ldy, a.ldz, a.M, a.N, a.act};
    return gemm<T>(g, e, a.dtype, a.work, st);
}

struct GradWork {
    void *dz, *dz_t, *x_t, *w_t, *sums, *part;
    int64_t Mp, Np; // rows of whole pieces
    size_t bytes;
};

GradWork grad_work(int64_t M, int64_t N, int64_t K, int dtype, void* base)
{
    GradWork w;
    size_t at = 0;
    const size_t es = elem_bytes(dtype);
    auto take = [&](size_t bytes) {
        char* p = (char*)base + at;
        at += round256(bytes);
        return (void*)p;
    };
    const int64_t piece = 16 / (int64_t)es;
    w.Mp = up(M, piece) * piece;
    w.Np = up(N, piece) * piece;
    w.dz = take(es * (size_t)M * (size_t)w.Np);
    w.dz_t = take(es * (size_t)N * (size_t)w.Mp);
    w.x_t = take(es * (size_t)K * (size_t)w.Mp);
    w.w_t = take(es * (size_t)K * (size_t)w.Np);
    w.sums = take(sizeof(float) * (size_t)up(M, 64) * (size_t)N);
    w.part = take(std::max(part_bytes(M, K, N, dtype), part_bytes(N, K, M, dtype)));
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
    t.tiles = t.job[0].tiles + t.job[1].tiles + t.job[2].tiles;
    if (t.tiles)
        hipLaunchKernelGGL((k_turn<T>), dim3((unsigned)std::min<int64_t>(t.tiles, kMostWgs)), dim3(256), 0, st, t);
    hipError_t err = hipGetLastError();
    if (a.dx && err == hipSuccess) {
        GemmArgs g{as_is ? a.dy : w.dz, w.w_t, as_is ? a.lddy : w.Np, w.Np, a.M, a.K, a.N, 0, 0, 0, 0, nullptr};
        if (!as_is)
            g.depth = w.Np; // the zeros behind a row are part of it: whole pieces
        const Epilogue e{nullptr, nullptr, a.dx, nullptr, 0, a.lddx, 0, a.M, a.K, kNone};
        err = gemm<T>(g, e, a.dtype, w.part, st);
    }
    if (a.dw && err == hipSuccess) {
        GemmArgs g{w.dz_t, w.x_t, w.Mp, w.Mp, a.N, a.K, w.Mp, 0, 0, 0, 0, nullptr};
        const Epilogue e{nullptr, nullptr, a.dw, nullptr, 0, a.lddw, 0, a.N, a.K, kNone};
        err = gemm<T>(g, e, a.dtype, w.part, st);
    }
    if (a.dbias && a.N && err == hipSuccess) {
        hipLaunchKernelGGL((k_dbias<T>), dim3((unsigned)up(a.N, 64)), dim3(256), 0, st, (const float*)w.sums,
                           up(a.M, 64), a.N, (T*)a.dbias);
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
