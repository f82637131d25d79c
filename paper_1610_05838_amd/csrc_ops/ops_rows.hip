// ops_rows.hip -- rows of a table by id, and the gradient of that.
//
//   rows_get:   out[i, :] = s * T[ids[i], :]
//   rows_grad:  D[r, :] (+)= s * sum over the i with ids[i] = r of G[i, :]
//
// An id outside [0, rows) stands for no row: zeros come out of the lookup, and
// the gradient leaves its token out.
#include <algorithm>

#include "ops_common.hpp"

namespace mfsgd {
namespace ops {

namespace {

constexpr int kThreads = 256;
constexpr int64_t kMostWgs = 1 << 22; // of a launch; workgroups then take several parts

// ---------------------------------------------------------------- lookup
//
// Bound by memory: count * (2 k elements + one id).  A row is nv vectors of V
// elements (16 bytes where the row holds that many), the last one moved back to
// end with the row, so a row of any width is whole vectors and an overlapped
// element is written twice with one value.  A workgroup takes the vectors of
// as many whole rows as come nearest to kThreads * kAhead of them, and every
// thread has kAhead rows' loads in flight: the ids first, then the rows.  40,960
// rows of 1,000 bytes (68 MB with padding and repeated rows): 10.4 us; 50 rows of
// 256 bytes: 2.2 us, a launch and two trips to memory.
//
// ONCE: past the caches, where `out` is larger than the Infinity Cache and its
// rows are whole cache lines (1.4 M rows of 512 bytes: 202 us, 4.2 TB/s, against
// 225; 41 MB that stay in the caches: 11.7 us against 10.4).
constexpr int kAhead = 4;

template <typename T, int V, bool ONCE>
__global__ __launch_bounds__(kThreads) void k_rows_get(const T* __restrict__ table, int64_t rows, int64_t ld, int k,
                                                       const int32_t* __restrict__ ids, int64_t ids_stride,
                                                       int64_t count, float scale, T* __restrict__ out,
                                                       int64_t ld_out, int per_wg, FastDiv nv)
{
    for (int64_t row0 = (int64_t)blockIdx.x * per_wg; row0 < count; row0 += (int64_t)gridDim.x * per_wg) {
        const int here = (int)(count - row0 < per_wg ? count - row0 : per_wg);
        const uint32_t total = (uint32_t)here * nv.d;
        for (uint32_t f0 = threadIdx.x; f0 < total; f0 += kThreads * kAhead) {
            uint32_t row[kAhead];
            int col[kAhead];
            int32_t id[kAhead];
            Vec<T, V> x[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const uint32_t f = f0 + u * kThreads < total ? f0 + u * kThreads : f0;
                row[u] = div_by(f, nv);
                col[u] = (int)(f - row[u] * nv.d) * V;
                col[u] = col[u] < k - V ? col[u] : k - V;
                id[u] = ids[(row0 + row[u]) * ids_stride];
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const bool there = id[u] >= 0 && id[u] < rows;
                x[u] = load_vec<T, V>(table + (there ? id[u] : 0) * ld + col[u]);
                if (!there) {
#pragma unroll
                    for (int e = 0; e < V; ++e)
                        x[u].v[e] = T(0.0f);
                }
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
#pragma unroll
                for (int e = 0; e < V; ++e)
                    x[u].v[e] = T((float)x[u].v[e] * scale);
                if (f0 + u * kThreads < total) {
                    if (ONCE)
                        store_once<T, V>(out + (row0 + row[u]) * ld_out + col[u], x[u]);
                    else
                        store_vec<T, V>(out + (row0 + row[u]) * ld_out + col[u], x[u]);
                }
            }
        }
    }
}

template <typename T, int V>
hipError_t get_launch(const RowsLaunch& a, hipStream_t st)
{
    const int nv = (a.k + V - 1) / V;
    const int per_wg = std::max(1, kThreads * kAhead / nv);
    const int64_t wgs = std::min((a.count + per_wg - 1) / per_wg, kMostWgs);
    const int64_t row = (int64_t)a.k * (int64_t)sizeof(T), pitch = a.ld_out * (int64_t)sizeof(T);
    const bool once = V * sizeof(T) == 16 && ((uintptr_t)a.out & 127) == 0 && row % 128 == 0 && pitch % 128 == 0 &&
                      a.count * row > kInfinityCache;
    hipLaunchKernelGGL((once ? k_rows_get<T, V, V * sizeof(T) == 16> : k_rows_get<T, V, false>), dim3((unsigned)wgs),
                       dim3(kThreads), 0, st, (const T*)a.table, a.rows, a.ld, a.k, a.ids, a.ids_stride, a.count,
                       a.scale, (T*)a.out, a.ld_out, per_wg, fast_div((uint32_t)nv));
    return hipGetLastError();
}

template <typename T>
hipError_t get_typed(const RowsLaunch& a, hipStream_t st)
{
    constexpr int most = 16 / (int)sizeof(T);
    if (a.k >= most)
        return get_launch<T, most>(a, st);
    if (a.k >= most / 2)
        return get_launch<T, most / 2>(a, st);
    if (most == 8 && a.k >= 2)
        return get_launch<T, 2>(a, st);
    return get_launch<T, 1>(a, st);
}

// A value that every lane of the wavefront has, for the scalar unit: addresses
// and conditions made of it cost no vector registers and no masks.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// -------------------------------------------------------------- gradient
//
// The tokens of one row are added in their order, in binary32, by one of two
// paths; no float atomics, so the result is the same bits every time.
//
// A lane holds E consecutive columns, the last lane's moved back to end with
// the row (as in the lookup); a wavefront 64 E of them, the grid's y the rest.
struct Cols {
    int at;   // first column this lane reads
    int skip; // its first `skip` elements belong to the lane before (all: nothing to write)
};

template <int E>
__device__ __forceinline__ Cols my_cols(int k)
{
    const int col = ((int)blockIdx.y * 64 + (int)(threadIdx.x & 63)) * E;
    Cols c;
    c.at = col < k - E ? col : k - E;
    c.skip = col - c.at < E ? col - c.at : E;
    return c;
}

template <typename T, int E>
__device__ __forceinline__ void write_row(T* __restrict__ row, const Cols& c, const float (&sum)[E], float scale,
                                          int accumulate)
{
    if (c.skip >= E)
        return;
    Vec<T, E> x;
    if (accumulate) {
        x = load_vec<T, E>(row + c.at);
#pragma unroll
        for (int e = 0; e < E; ++e)
            x.v[e] = T((float)x.v[e] + scale * sum[e]);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            x.v[e] = T(scale * sum[e]);
    }
    // in place, an element shared with the lane before is that lane's alone
    if (accumulate && c.skip) {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (e >= c.skip)
                row[c.at + e] = x.v[e];
    } else {
        store_vec<T, E>(row + c.at, x);
    }
}

// Zeros in `rows` rows of k elements: the base of the scanned path.
template <typename T, int V>
__global__ __launch_bounds__(kThreads) void k_rows_zero(T* __restrict__ out, int64_t rows, int64_t ld, int k,
                                                        int per_wg, FastDiv nv)
{
    Vec<T, V> zero;
#pragma unroll
    for (int e = 0; e < V; ++e)
        zero.v[e] = T(0.0f);
    for (int64_t row0 = (int64_t)blockIdx.x * per_wg; row0 < rows; row0 += (int64_t)gridDim.x * per_wg) {
        const int here = (int)(rows - row0 < per_wg ? rows - row0 : per_wg);
        for (uint32_t f = threadIdx.x; f < (uint32_t)here * nv.d; f += kThreads) {
            const uint32_t row = div_by(f, nv);
            const int col = (int)(f - row * nv.d) * V;
            store_vec<T, V>(out + (row0 + row) * ld + (col < k - V ? col : k - V), zero);
        }
    }
}

// Few tokens: every id is compared with every other in LDS, one launch and no
// sort.  A wavefront takes one token; if no earlier one has its id it adds the
// rows of all that do.  Where these are more than kScanAlone the workgroup's
// four wavefronts add a consecutive part of the tokens each, and the four sums
// are joined in order.
//
// Bound by chains of dependent steps, not by its bytes: ids from memory to LDS,
// the comparisons, the most frequent row's sum.  4,001 Zipf tokens of 64 binary32:
// 13 us, sorting them 30; 8,192: 26 and 31 (512 bfloat16: 36 and 36); beyond that
// the comparisons, square in the number of tokens, outweigh the sort's launches.
// A row with much of the tokens is one workgroup's chain, 11 to 30 us per 1,000 of
// them, so a table whose rows have more than kScanAlone on average is sorted for
// from kScanSurely tokens on (8,192 of 512 binary32 for 10 rows: 22 us for 97; 4,000
// of 128 for 3 rows: 21 for 59, for 30 rows: 20 for 27).
constexpr int kScanMost = 8192;
constexpr int kScanSurely = 2048;
constexpr int kScanAlone = 64;
constexpr int kScanBlock = 256; // ids compared at a time: four a lane

template <typename T, int E>
__global__ __launch_bounds__(kThreads) void k_grad_scan(const T* __restrict__ dout, int64_t ld_dout,
                                                        const int32_t* __restrict__ ids, int64_t ids_stride, int count,
                                                        int k, float scale, T* __restrict__ dtable, int64_t rows,
                                                        int64_t ld, int accumulate)
{
    constexpr int ahead = (int)sizeof(T) * E >= 16 ? 8 : (int)sizeof(T) * E >= 4 ? 16 : 32; // rows in flight
    __shared__ __attribute__((aligned(16))) int32_t all[kScanMost];
    __shared__ float part[3][64 * E];
    __shared__ uint16_t list[4][kScanAlone + kScanBlock];
    __shared__ int more[4]; // the wavefronts' tokens with many rows, or -1
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const Cols c = my_cols<E>(k);
    const int blocks = (count + kScanBlock - 1) / kScanBlock;
    for (int j0 = threadIdx.x; j0 < blocks * kScanBlock; j0 += kThreads * 8) {
        int32_t id[8];
#pragma unroll
        for (int u = 0; u < 8; ++u)
            id[u] = ids[(j0 + u * kThreads < count ? j0 + u * kThreads : count - 1) * ids_stride];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int j = j0 + u * kThreads;
            if (j < blocks * kScanBlock)
                all[j] = j < count && id[u] >= 0 && id[u] < rows ? id[u] : -1;
        }
    }
    __syncthreads();

    float sum[E];
    // appends the tokens with id r of block b to this wavefront's list of n, in order
    auto look = [&](int32_t r, int b, int& n) {
        const int4 id = *(const int4*)&all[b * kScanBlock + lane * 4];
        const bool is[4] = {id.x == r, id.y == r, id.z == r, id.w == r};
        if (!__ballot(is[0] || is[1] || is[2] || is[3]))
            return;
        int at = n;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint64_t mask = __ballot(is[q]);
            at += __popcll(mask & ((uint64_t(1) << lane) - 1));
            n += __popcll(mask);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (is[q])
                list[wave][at++] = (uint16_t)(b * kScanBlock + lane * 4 + q);
    };
    // adds the rows of the listed tokens
    auto add = [&](int n) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
        for (int i0 = 0; i0 < n; i0 += ahead) {
            Vec<T, E> x[ahead];
#pragma unroll
            for (int u = 0; u < ahead; ++u) {
                const int token = uniform(list[wave][i0 + u < n ? i0 + u : n - 1]);
                x[u] = load_vec<T, E>(dout + (int64_t)token * ld_dout + c.at);
            }
#pragma unroll
            for (int u = 0; u < ahead; ++u)
                if (i0 + u < n) {
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        sum[e] += (float)x[u].v[e];
                }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    };
    auto clear = [&] {
#pragma unroll
        for (int e = 0; e < E; ++e)
            sum[e] = 0.0f;
    };

    const int i = (int)blockIdx.x * 4 + wave, home = i / kScanBlock;
    const int32_t r = i < count ? uniform(all[i]) : -1;
    int many = -1;
    if (r >= 0) {
        bool earlier = false;
        for (int b = 0; b < home && !earlier; ++b) {
            const int4 id = *(const int4*)&all[b * kScanBlock + lane * 4];
            earlier = __ballot(id.x == r || id.y == r || id.z == r || id.w == r) != 0;
        }
        int n = 0;
        if (!earlier) {
            look(r, home, n);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
            earlier = uniform(list[wave][0]) < i; // the first in its block
        }
        if (!earlier) {
            for (int b = home + 1; b < blocks && n <= kScanAlone; ++b)
                look(r, b, n);
            if (n > kScanAlone) {
                many = i;
            } else {
                clear();
                add(n);
                write_row<T, E>(dtable + (int64_t)r * ld, c, sum, scale, accumulate);
            }
        }
    }
    if (lane == 0)
        more[wave] = many;
    __syncthreads();
    for (int w = 0; w < 4; ++w) {
        const int first = uniform(more[w]);
        if (first < 0)
            continue;
        const int32_t id = uniform(all[first]);
        const int b0 = first / kScanBlock, each = (blocks - b0 + 3) / 4, from = b0 + wave * each;
        const int to = from + each < blocks ? from + each : blocks;
        clear();
        for (int b = from, n = 0; b < to; ++b) {
            look(id, b, n);
            if (n >= kScanAlone || b + 1 == to) {
                add(n);
                n = 0;
            }
        }
        if (wave) {
#pragma unroll
            for (int e = 0; e < E; ++e)
                part[wave - 1][e * 64 + lane] = sum[e];
        }
        __syncthreads();
        if (wave == 0) {
#pragma unroll
            for (int v = 0; v < 3; ++v)
#pragma unroll
                for (int e = 0; e < E; ++e)
                    sum[e] += part[v][e * 64 + lane];
            write_row<T, E>(dtable + (int64_t)id * ld, c, sum, scale, accumulate);
        }
        __syncthreads();
    }
}

// Many tokens: (row, token) pairs sorted by row, stably, so that a row's tokens
// stay in order; then tiles of the sorted tokens summed by one wavefront each.
//
// The sort is by digits of `bits` bits from the lowest: per chunk of
// tokens the count of every digit, the exclusive sums of these over the chunks,
// and every token to its place.  Tokens without a row have the key `rows` and
// end up last.
//
// 262,144 tokens of 17,770 rows, two passes: 4.0 + 2.7 + 7.4 and 3.5 + 2.6 + 6.3
// us.  They move 8 MB in all, which is 2 us: each is bound by a launch, one trip to
// memory and, where tokens are placed, a ballot per bit of the digit.
constexpr int kDigits = 256;

__device__ __forceinline__ uint32_t key_of(int32_t id, int64_t rows)
{
    return id >= 0 && id < rows ? (uint32_t)id : (uint32_t)rows;
}

template <int CHUNK>
__global__ __launch_bounds__(kThreads) void k_sort_count(const uint32_t* __restrict__ keys,
                                                         const int32_t* __restrict__ ids, int64_t ids_stride,
                                                         int64_t rows, int64_t count, int shift, uint32_t mask,
                                                         uint32_t* __restrict__ hist, uint32_t* __restrict__ crossing)
{
    __shared__ uint32_t n[kDigits];
    n[threadIdx.x] = 0;
    __syncthreads();
    const int64_t base = (int64_t)blockIdx.x * CHUNK;
#pragma unroll
    for (int s = 0; s < CHUNK / kThreads; ++s) {
        const int j = s * kThreads + (int)threadIdx.x;
        if (base + j < count) {
            const uint32_t key = keys ? keys[base + j] : key_of(ids[(base + j) * ids_stride], rows);
            atomicAdd(&n[key >> shift & mask], 1u);
        }
    }
    __syncthreads();
    if (threadIdx.x <= mask)
        hist[(int64_t)threadIdx.x * gridDim.x + blockIdx.x] = n[threadIdx.x];
    if (blockIdx.x == 0 && threadIdx.x == 0)
        *crossing = 0;
}

// Exclusive sum of x over the workgroup's 256 threads; `total` is its sum.
__device__ __forceinline__ uint32_t block_scan(uint32_t x, uint32_t* wave_sums, uint32_t& total)
{
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    uint32_t s = x;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t y = __shfl_up(s, d, 64);
        s += lane >= d ? y : 0;
    }
    if (lane == 63)
        wave_sums[wave] = s;
    __syncthreads();
    uint32_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        before += w < wave ? wave_sums[w] : 0;
        total += wave_sums[w];
    }
    __syncthreads();
    return before + s - x;
}

__global__ __launch_bounds__(kThreads) void k_sort_scan(uint32_t* __restrict__ hist, int chunks,
                                                        uint32_t* __restrict__ totals)
{
    __shared__ uint32_t sums[4];
    uint32_t* h = hist + (int64_t)blockIdx.x * chunks;
    uint32_t carry = 0;
    for (int b = 0; b < chunks; b += kThreads) {
        const int i = b + (int)threadIdx.x;
        const uint32_t x = i < chunks ? h[i] : 0;
        uint32_t total;
        const uint32_t before = block_scan(x, sums, total);
        if (i < chunks)
            h[i] = carry + before;
        carry += total;
    }
    if (threadIdx.x == 0)
        totals[blockIdx.x] = carry;
}

template <int CHUNK>
__global__ __launch_bounds__(kThreads) void k_sort_place(const uint32_t* __restrict__ keys,
                                                         const uint32_t* __restrict__ toks,
                                                         const int32_t* __restrict__ ids, int64_t ids_stride,
                                                         int64_t rows, int64_t count, int shift, int bits,
                                                         const uint32_t* __restrict__ hist,
                                                         const uint32_t* __restrict__ totals,
                                                         uint32_t* __restrict__ keys_out,
                                                         uint32_t* __restrict__ toks_out)
{
    constexpr int steps = CHUNK / kThreads; // 64 consecutive tokens a step, a wavefront's steps consecutive
    __shared__ uint32_t next[4][kDigits];
    __shared__ uint32_t sums[4];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const uint32_t mask = (1u << bits) - 1;
    const int64_t base = (int64_t)blockIdx.x * CHUNK + wave * (steps * 64) + lane;
    // all loads first: their latencies are most of this kernel
    const bool used = threadIdx.x <= mask;
    const uint32_t in_all = used ? totals[threadIdx.x] : 0;
    const uint32_t in_earlier = used ? hist[(int64_t)threadIdx.x * gridDim.x + blockIdx.x] : 0;
#pragma unroll
    for (int w = 0; w < 4; ++w)
        next[w][threadIdx.x] = 0;
    __syncthreads();
    uint32_t key[steps], tok[steps];
#pragma unroll
    for (int s = 0; s < steps; ++s) {
        const int64_t i = base + s * 64;
        key[s] = tok[s] = 0;
        if (i < count) {
            key[s] = keys ? keys[i] : key_of(ids[i * ids_stride], rows);
            tok[s] = keys ? toks[i] : (uint32_t)i;
        }
    }
#pragma unroll
    for (int s = 0; s < steps; ++s)
        if (base + s * 64 < count)
            atomicAdd(&next[wave][key[s] >> shift & mask], 1u);
    uint32_t total;
    uint32_t at = block_scan(in_all, sums, total) + in_earlier;
    if (used) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const uint32_t n = next[w][threadIdx.x];
            next[w][threadIdx.x] = at;
            at += n;
        }
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < steps; ++s) {
        const bool live = base + s * 64 < count;
        const uint32_t digit = key[s] >> shift & mask;
        uint64_t same = __ballot(live);
        for (int b = 0; b < bits; ++b) {
            const bool set = digit >> b & 1;
            const uint64_t m = __ballot(set);
            same &= set ? m : ~m;
        }
        if (live) {
            const int lead = __builtin_ctzll(same);
            uint32_t place = 0;
            if (lane == lead)
                place = atomicAdd(&next[wave][digit], (uint32_t)__popcll(same));
            place = (uint32_t)__shfl((int)place, lead, 64) + (uint32_t)__popcll(same & ((uint64_t(1) << lane) - 1));
            keys_out[place] = key[s];
            toks_out[place] = tok[s];
        }
    }
}

// The sums over the sorted tokens.  A wavefront adds the rows of one tile of
// `tile` tokens, several loads in flight.  A row whose tokens end in the tile
// they begin in, or in the next one, is added up and written by the tile where
// it begins.  Of a longer one that tile keeps its sum in `tails` and notes
// itself and the number of tiles in `begun`, every later tile its own in
// `heads`; k_grad_join adds those up in order.  The workgroups before the tiles
// write zeros to the rows that no token has (first, because they take longest from
// their start to their end).
//
// Bound by memory, in rows scattered over `dout`: 262,144 tokens of 128 binary16
// (67 MB, 4.5 of them written): 17.2 us, 4.2 TB/s; 131,072 of 512 bfloat16 in a
// table of 50,003 rows (172 MB): 30.8 us, 5.6 TB/s, some of it from the caches.

// Zeros in those of `here` rows whose bit of `taken` is clear, by one wavefront.
template <typename T, int V>
__device__ __forceinline__ void zero_rows(T* __restrict__ out, int64_t ld, int k, int here, uint64_t taken,
                                          const FastDiv& nv)
{
    Vec<T, V> zero;
#pragma unroll
    for (int e = 0; e < V; ++e)
        zero.v[e] = T(0.0f);
    for (uint32_t f = threadIdx.x & 63; f < (uint32_t)here * nv.d; f += 64) {
        const uint32_t row = div_by(f, nv);
        const int col = (int)(f - row * nv.d) * V;
        if (!(taken >> row & 1))
            store_vec<T, V>(out + row * ld + (col < k - V ? col : k - V), zero);
    }
}

// The first of the sorted keys that is not below `key` (count: none), found by
// a wavefront 64 places at a time.
__device__ __forceinline__ int64_t first_at_least(const uint32_t* __restrict__ keys, int64_t count, uint32_t key,
                                                  int lane)
{
    int64_t lo = 0, hi = count; // keys before lo are below it, keys from hi on are not
    while (hi > lo) {
        const int64_t step = (hi - lo + 63) / 64, p = lo + (lane + 1) * step - 1;
        const uint64_t not_below = __ballot(p >= hi || keys[p < hi ? p : lo] >= key);
        const int f = not_below ? __builtin_ctzll(not_below) : 64;
        const int64_t next = lo + f * step;
        hi = f < 64 && next + step - 1 < hi ? next + step - 1 : hi;
        lo = next < hi ? next : hi;
    }
    return lo;
}

// The sum of a row to its place, added to what was read from there if ACC.
template <typename T, int E, bool ACC>
__device__ __forceinline__ void put_row(T* row, const Cols& c, const float (&sum)[E], float scale, const Vec<T, E>& old)
{
    Vec<T, E> x;
#pragma unroll
    for (int e = 0; e < E; ++e)
        x.v[e] = ACC ? T((float)old.v[e] + scale * sum[e]) : T(scale * sum[e]);
    if (ACC && c.skip) { // a shared element is the other lane's to add to
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (e >= c.skip)
                row[c.at + e] = x.v[e];
    } else if (c.skip < E) {
        store_vec<T, E>(row + c.at, x);
    }
}

template <typename T, int E, bool ACC>
__global__ __launch_bounds__(kThreads) void k_grad_tiles(const T* __restrict__ dout, int64_t ld_dout,
                                                         const uint32_t* __restrict__ keys,
                                                         const uint32_t* __restrict__ toks, int64_t count, int k,
                                                         float scale, T* __restrict__ dtable, int64_t rows, int64_t ld,
                                                         int tile, int64_t tiles, int zero_wgs,
                                                         float* __restrict__ heads, float* __restrict__ tails,
                                                         uint2* __restrict__ begun, uint32_t* __restrict__ crossing,
                                                         FastDiv per_row)
{
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    if ((int)blockIdx.x < zero_wgs) {
        if (blockIdx.y)
            return;
        const int64_t stride = (int64_t)zero_wgs * 256;
        for (int64_t r0 = ((int64_t)blockIdx.x * 4 + wave) * 64; r0 < rows; r0 += stride) {
            // the tokens of these 64 rows, then a bit for every row that has one
            int64_t lo = first_at_least(keys, count, (uint32_t)r0, lane);
            const int64_t hi = first_at_least(keys, count, (uint32_t)(r0 + 64 < rows ? r0 + 64 : rows), lane);
            uint64_t taken = 0;
            if (hi - lo <= 1024) {
#pragma unroll 4
                for (; lo < hi; lo += 64)
                    taken |= uint64_t(lo + lane < hi) << (keys[lo + lane < hi ? lo + lane : lo] - (uint32_t)r0);
#pragma unroll
                for (int d = 32; d > 0; d >>= 1)
                    taken |= __shfl_xor((unsigned long long)taken, d, 64);
            } else {
                const uint32_t r = (uint32_t)r0 + lane;
                int64_t p = lo, q = hi; // first of them whose key is not below r
                while (p < q) {
                    const int64_t mid = (p + q) >> 1;
                    if (keys[mid] < r)
                        p = mid + 1;
                    else
                        q = mid;
                }
                taken = __ballot(p < hi && keys[p < hi ? p : lo] == r);
            }
            const int here = (int)(rows - r0 < 64 ? rows - r0 : 64);
            constexpr int most = 16 / (int)sizeof(T);
            if (k >= most)
                zero_rows<T, most>(dtable + r0 * ld, ld, k, here, taken, per_row);
            else if (k >= most / 2)
                zero_rows<T, most / 2>(dtable + r0 * ld, ld, k, here, taken, per_row);
            else if (most == 8 && k >= 2)
                zero_rows<T, 2>(dtable + r0 * ld, ld, k, here, taken, per_row);
            else
                zero_rows<T, 1>(dtable + r0 * ld, ld, k, here, taken, per_row);
        }
        return;
    }
    const int64_t t = (int64_t)(blockIdx.x - zero_wgs) * 4 + wave;
    if (t >= tiles)
        return;
    constexpr int batch = ACC || (int)sizeof(T) * E >= 16 ? 8 : 16;
    const Cols c = my_cols<E>(k);
    const int64_t start = t * tile;
    const int n = (int)(count - start < tile ? count - start : tile);
    const uint32_t none = 0xffffffffu;
    uint32_t key = keys[start + (lane < n ? lane : n - 1)], tok = toks[start + (lane < n ? lane : n - 1)];
    // the keys before the tile and behind it, before the previous tile and behind the next one
    const uint32_t prev = start > 0 ? keys[start - 1] : none;
    const uint32_t next = start + n < count ? keys[start + n] : none;
    const uint32_t before = start > tile ? keys[start - tile - 1] : none;
    const uint32_t beyond = start + 2 * tile < count ? keys[start + 2 * tile] : none;
    const int nv = __popcll(__ballot(lane < n && key < (uint32_t)rows)); // tokens with a row come first
    if (nv == 0)
        return;
    const uint32_t after = nv < n ? none : next;
    const uint32_t first = __builtin_amdgcn_readlane(key, 0), last = __builtin_amdgcn_readlane(key, nv - 1);
    // a bit for every token that begins a row, and one for every token (but the last) that ends one
    const uint32_t left = (uint32_t)__shfl_up((int)key, 1, 64);
    const uint64_t starts = __ballot(lane == 0 || key != left) & (~uint64_t(0) >> (64 - nv));
    const uint64_t ends = starts >> 1;
    float sum[E];
    // adds tokens [from, to) of those the lanes hold, writing every row that ends before the last token
    auto add = [&](int from, int to, uint64_t starts, uint64_t ends) {
        for (; from < to; from += batch) {
            Vec<T, E> x[batch], old[ACC ? batch : 1];
#pragma unroll
            for (int u = 0; u < batch; ++u) {
                const uint32_t row = __builtin_amdgcn_readlane(tok, from + u < to ? from + u : to - 1);
                x[u] = load_vec<T, E>(dout + (int64_t)row * ld_dout + c.at);
            }
            if (ACC) {
#pragma unroll
                for (int u = 0; u < batch; ++u) {
                    const uint32_t row = __builtin_amdgcn_readlane(key, from + u < to ? from + u : to - 1);
                    if (ends >> (from + u) & 1)
                        old[u] = load_vec<T, E>(dtable + (int64_t)row * ld + c.at);
                }
            }
#pragma unroll
            for (int u = 0; u < batch; ++u) {
                if (from + u < to) {
                    const bool fresh = starts >> (from + u) & 1;
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        sum[e] = (fresh ? 0.0f : sum[e]) + (float)x[u].v[e];
                    if (ends >> (from + u) & 1) {
                        const uint32_t row = __builtin_amdgcn_readlane(key, from + u);
                        put_row<T, E, ACC>(dtable + (int64_t)row * ld, c, sum, scale, old[ACC ? u : 0]);
                    }
                }
            }
        }
    };
    auto keep = [&](float* parts) {
        if (c.skip < E) {
            float* part = parts + t * k + c.at;
#pragma unroll
            for (int e = 0; e < E; ++e)
                part[e] = sum[e];
        }
    };
    int from = 0;
    if (prev == first) {
        const uint64_t more = starts & ~uint64_t(1);
        const int h = more ? __builtin_ctzll(more) : nv; // tokens of the row that began before
        if (h == nv && after == first) { // all of them, and it goes on
            add(0, nv, 1, 0);
            keep(heads);
            return;
        }
        if (before == first) { // the end of a row over several tiles (else the previous tile's, whose last row it is)
            add(0, h, 1, 0);
            keep(heads);
        }
        from = h;
        if (from == nv)
            return;
    }
    add(from, nv, starts, ends);
    if (after == last) {
        if (beyond == last) {
            keep(tails);
            if (blockIdx.y)
                return;
            // the last tile that begins with this key: tile `lo` does, tile `hi` does not; 64 places between them a
            // step
            int64_t lo = t + 1, hi = tiles;
            while (hi - lo > 1) {
                const int64_t step = (hi - lo + 63) / 64, p = lo + (lane + 1) * step;
                const int f = __builtin_ctzll(__ballot(p >= hi || keys[(p < hi ? p : lo) * tile] != last));
                const int64_t top = lo + (f + 1) * step;
                lo += f * step;
                hi = top < hi ? top : hi;
            }
            if (lane == 0)
                begun[atomicAdd(crossing, 1u)] = make_uint2((uint32_t)t, (uint32_t)(lo - t) + 1);
            return;
        }
        // it ends in the next tile: its tokens there
        const int64_t on = start + tile;
        const int m = (int)(count - on < tile ? count - on : tile);
        key = keys[on + (lane < m ? lane : m - 1)];
        tok = toks[on + (lane < m ? lane : m - 1)];
        add(0, __popcll(__ballot(lane < m && key == last)), 0, 0);
    }
    write_row<T, E>(dtable + (int64_t)last * ld, c, sum, scale, ACC);
}

// Joins the rows that go on over several tiles: tails[a], then the heads of the
// tiles after it.  A wavefront takes one such row a round and adds it alone up to
// kJoinAlone tiles; a longer one is then added by the whole workgroup, its
// wavefronts taking consecutive parts that are joined in order.
//
// Bound by the chain of its longest row (its place in `begun`, the parts, the
// workgroup's sum, the write): 8.2 us for 262,144 Zipf tokens of 128 binary16, 9.7
// for 131,072 of 512 bfloat16, a few MB each.
constexpr int kJoinThreads = 1024;
constexpr int kJoinAlone = 32;

template <int E>
__device__ __forceinline__ void add_parts(const float* __restrict__ heads, const float* __restrict__ tails, int64_t a,
                                          int from, int to, int k, const Cols& c, float (&sum)[E])
{
    constexpr int batch = E <= 2 ? 16 : 8;
    for (int i0 = from; i0 < to; i0 += batch) {
        Vec<float, E> x[batch];
#pragma unroll
        for (int u = 0; u < batch; ++u) {
            const int i = i0 + u < to ? i0 + u : to - 1;
            x[u] = load_vec<float, E>((i ? heads : tails) + (a + i) * k + c.at);
        }
#pragma unroll
        for (int u = 0; u < batch; ++u)
            if (i0 + u < to) {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    sum[e] += x[u].v[e];
            }
    }
}

template <typename T, int E>
__global__ __launch_bounds__(kJoinThreads) void k_grad_join(const uint32_t* __restrict__ keys, int k, float scale,
                                                            T* __restrict__ dtable, int64_t ld, int accumulate,
                                                            int tile, const float* __restrict__ heads,
                                                            const float* __restrict__ tails,
                                                            const uint2* __restrict__ begun,
                                                            const uint32_t* __restrict__ crossing)
{
    constexpr int waves = kJoinThreads / 64;
    __shared__ float part[waves][64 * E];
    __shared__ int long_at[waves], long_span[waves];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const Cols c = my_cols<E>(k);
    const int64_t n = *crossing;
    float sum[E];
    // the rows are dealt to the workgroups one at a time, so that a few rows meet many workgroups
    for (int64_t i0 = blockIdx.x; i0 < n; i0 += (int64_t)gridDim.x * waves) {
        int span = 0;
        const int64_t i = i0 + (int64_t)wave * gridDim.x;
        if (i < n) {
            const int64_t a = uniform((int)begun[i].x);
            span = uniform((int)begun[i].y);
            if (lane == 0)
                long_at[wave] = (int)a;
            if (span <= kJoinAlone) {
                const uint32_t key = uniform((int)keys[(a + 1) * tile]);
#pragma unroll
                for (int e = 0; e < E; ++e)
                    sum[e] = 0.0f;
                add_parts<E>(heads, tails, a, 0, span, k, c, sum);
                write_row<T, E>(dtable + (int64_t)key * ld, c, sum, scale, accumulate);
            }
        }
        if (lane == 0)
            long_span[wave] = span;
        __syncthreads();
        for (int w = 0; w < waves; ++w) {
            const int total = uniform(long_span[w]);
            if (total <= kJoinAlone)
                continue;
            const int64_t a = uniform(long_at[w]);
            const int each = (total + waves - 1) / waves, from = wave * each;
            const int to = from + each < total ? from + each : total;
#pragma unroll
            for (int e = 0; e < E; ++e)
                sum[e] = 0.0f;
            add_parts<E>(heads, tails, a, from, to, k, c, sum);
#pragma unroll
            for (int e = 0; e < E; ++e)
                part[wave][e * 64 + lane] = sum[e];
            __syncthreads();
            if (wave == 0) {
                for (int v = 1; v < waves; ++v)
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        sum[e] += part[v][e * 64 + lane];
                write_row<T, E>(dtable + (int64_t)keys[(a + 1) * tile] * ld, c, sum, scale, accumulate);
            }
            __syncthreads();
        }
        __syncthreads();
    }
}

// Elements of a 16-byte vector, or the largest power of two that a row holds.
template <typename T>
int vec_of(int k)
{
    int v = 16 / (int)sizeof(T);
    while (v > k)
        v /= 2;
    return v;
}

template <typename T, int V>
hipError_t zero_launch(const RowsGradLaunch& a, hipStream_t st)
{
    const int nv = (a.k + V - 1) / V, per_wg = std::max(1, kThreads * 8 / nv);
    const int64_t wgs = std::min((a.rows + per_wg - 1) / per_wg, kMostWgs);
    hipLaunchKernelGGL((k_rows_zero<T, V>), dim3((unsigned)wgs), dim3(kThreads), 0, st, (T*)a.dtable, a.rows, a.ld, a.k,
                       per_wg, fast_div((uint32_t)nv));
    return hipGetLastError();
}

template <typename T>
hipError_t zero_typed(const RowsGradLaunch& a, hipStream_t st)
{
    const int v = vec_of<T>(a.k);
    if (v == 8)
        return zero_launch<T, (sizeof(T) == 2 ? 8 : 4)>(a, st);
    return v == 4 ? zero_launch<T, 4>(a, st) : v == 2 ? zero_launch<T, 2>(a, st) : zero_launch<T, 1>(a, st);
}

bool scanned(int64_t count, int64_t rows)
{
    return count <= kScanSurely || (count <= kScanMost && count <= rows * kScanAlone);
}

// Tokens of a tile: 64 (a lane each), or fewer (at least 16) where that leaves
// the chip without 4096 wavefronts.  Half the tiles that it holds at once are as
// fast as all of them, and long rows then have half as many parts to join
// (262,144 Zipf tokens: 18 + 7 us with tiles of 64, 19 + 11 with tiles of 32).
int tile_of(int64_t count) { return (int)std::min<int64_t>(64, std::max<int64_t>(16, (count + 4095) / 4096)); }

// Tokens of a chunk of the sort: as few as still give every CU one (the sort's
// kernels are bound by their chains of dependent steps; 262,144 tokens, the whole
// gradient: 50 us with 1024, 71 with 4096), but not so many chunks that their
// counts outweigh the tokens (2,000,000: 207 and 203 us; 4,000,000: 365 and 349).
int chunk_of(int64_t count) { return count <= 1024 * 2048 ? 1024 : 4096; }

template <int CHUNK>
void sort_pass(const uint32_t* keys, const uint32_t* toks, const RowsGradLaunch& a, int shift, int bits, uint32_t* hist,
               uint32_t* totals, uint32_t* crossing, uint32_t* keys_out, uint32_t* toks_out, hipStream_t st)
{
    const unsigned chunks = (unsigned)((a.count + CHUNK - 1) / CHUNK);
    hipLaunchKernelGGL(k_sort_count<CHUNK>, dim3(chunks), dim3(kThreads), 0, st, keys, a.ids, a.ids_stride, a.rows,
                       a.count, shift, (1u << bits) - 1, hist, crossing);
    hipLaunchKernelGGL(k_sort_scan, dim3(1u << bits), dim3(kThreads), 0, st, hist, (int)chunks, totals);
    hipLaunchKernelGGL(k_sort_place<CHUNK>, dim3(chunks), dim3(kThreads), 0, st, keys, toks, a.ids, a.ids_stride,
                       a.rows, a.count, shift, bits, hist, totals, keys_out, toks_out);
}

struct GradWork {
    uint32_t *keys[2], *toks[2], *hist, *totals, *crossing;
    uint2* begun;
    float *heads, *tails;
    size_t bytes;
};

int key_bits(int64_t rows)
{
    int b = 1;
    while ((int64_t(1) << b) <= rows) // keys 0 .. rows
        ++b;
    return b;
}

GradWork grad_work(int64_t count, int k, void* base)
{
    GradWork w;
    size_t at = 0;
    auto part = [&](size_t bytes) {
        char* p = (char*)base + at;
        at += round256(bytes);
        return p;
    };
    const size_t chunks = (size_t)((count + chunk_of(count) - 1) / chunk_of(count));
    const size_t tiles = (size_t)((count + tile_of(count) - 1) / tile_of(count));
    for (int i = 0; i < 2; ++i) {
        w.keys[i] = (uint32_t*)part(4 * (size_t)count);
        w.toks[i] = (uint32_t*)part(4 * (size_t)count);
    }
    w.hist = (uint32_t*)part(4 * chunks * kDigits);
    w.totals = (uint32_t*)part(4 * kDigits);
    w.crossing = (uint32_t*)part(4);
    w.begun = (uint2*)part(8 * tiles);
    w.heads = (float*)part(4 * tiles * (size_t)k);
    w.tails = (float*)part(4 * tiles * (size_t)k);
    w.bytes = at;
    return w;
}

template <typename T, int E>
hipError_t grad_launch(const RowsGradLaunch& a, hipStream_t st)
{
    const unsigned ys = (unsigned)((a.k + 64 * E - 1) / (64 * E));
    if (scanned(a.count, a.rows)) {
        if (!a.accumulate && a.rows > 0) {
            const hipError_t e = zero_typed<T>(a, st);
            if (e != hipSuccess)
                return e;
        }
        if (a.count == 0)
            return hipSuccess;
        hipLaunchKernelGGL((k_grad_scan<T, E>), dim3((unsigned)((a.count + 3) / 4), ys), dim3(kThreads), 0,
                           st, (const T*)a.dout, a.ld_dout, a.ids, a.ids_stride, (int)a.count, a.k, a.scale,
                           (T*)a.dtable, a.rows, a.ld, a.accumulate);
        return hipGetLastError();
    }
    const GradWork w = grad_work(a.count, a.k, a.work);
    const int bits = key_bits(a.rows), passes = (bits + 7) / 8, width = (bits + passes - 1) / passes;
    const uint32_t *keys = nullptr, *toks = nullptr;
    for (int p = 0; p < passes; ++p) {
        const int shift = p * width, now = std::min(width, bits - shift);
        (chunk_of(a.count) == 1024 ? sort_pass<1024> : sort_pass<4096>)(keys, toks, a, shift, now, w.hist, w.totals,
                                                                       w.crossing, w.keys[p & 1], w.toks[p & 1], st);
        keys = w.keys[p & 1];
        toks = w.toks[p & 1];
    }
    const int tile = tile_of(a.count);
    const int64_t tiles = (a.count + tile - 1) / tile;
    const int tile_wgs = (int)((tiles + 3) / 4);
    const int zero_wgs = a.accumulate ? 0 : (int)std::min<int64_t>((a.rows + 255) / 256, 1 << 20);
    const int v = vec_of<T>(a.k);
    hipLaunchKernelGGL((a.accumulate ? k_grad_tiles<T, E, true> : k_grad_tiles<T, E, false>),
                       dim3((unsigned)(tile_wgs + zero_wgs), ys), dim3(kThreads), 0, st, (const T*)a.dout, a.ld_dout,
                       keys, toks, a.count, a.k, a.scale, (T*)a.dtable, a.rows, a.ld, tile, tiles, zero_wgs, w.heads,
                       w.tails, w.begun, w.crossing, fast_div((uint32_t)((a.k + v - 1) / v)));
    hipLaunchKernelGGL((k_grad_join<T, E>), dim3((unsigned)std::min<int64_t>((tiles + 15) / 16, 256), ys),
                       dim3(kJoinThreads), 0, st, keys, a.k, a.scale, (T*)a.dtable, a.ld, a.accumulate, tile,
                       w.heads, w.tails, w.begun, w.crossing);
    return hipGetLastError();
}

template <typename T>
hipError_t grad_typed(const RowsGradLaunch& a, hipStream_t st)
{
    if (a.k <= 64)
        return grad_launch<T, 1>(a, st);
    if (a.k <= 128)
        return grad_launch<T, 2>(a, st);
    if (a.k <= 256 || sizeof(T) == 4)
        return grad_launch<T, 4>(a, st);
    return grad_launch<T, (sizeof(T) == 2 ? 8 : 4)>(a, st);
}

} // namespace

hipError_t rows_get(const RowsLaunch& a, hipStream_t st)
{
    if (a.dtype == kF16)
        return get_typed<_Float16>(a, st);
    if (a.dtype == kBF16)
        return get_typed<__bf16>(a, st);
    return get_typed<float>(a, st);
}

size_t rows_grad_bytes(int64_t count, int k, int64_t rows)
{
    return scanned(count, rows) ? 0 : grad_work(count, k, nullptr).bytes;
}

hipError_t rows_grad(const RowsGradLaunch& a, hipStream_t st)
{
    if (a.dtype == kF16)
        return grad_typed<_Float16>(a, st);
    if (a.dtype == kBF16)
        return grad_typed<__bf16>(a, st);
    return grad_typed<float>(a, st);
}

} // namespace ops
} // namespace mfsgd
